// What a layer does to the rows of its projection before they can be probed, compressed or attended to: the RMS norm of every
// head's query and key and the rotation of their channel pairs by the token's position, each frequency on its own position axis
// (time, height, width), in one pass.
//   y = x / sqrt(mean_c x_c^2 + eps) * w          (no weights: y = x)
//   (a, b) -> (a cos - b sin, b cos + a sin) * s  angle = pos[axis of the frequency] * inv_freq
// All in float32 behind the storage type, one rounding at the end; the angle is a float64 product, whose whole turns are dropped
// before it becomes a float32 (a float32 product of a position of 10^6 would be off by 0.06 rad).
//
// Bound by memory traffic for prompts, by the chain load -> norm -> store for a few tokens.  D / 16 lanes share a (token, head) row:
// a lane holds eight channels of the first half of the rotating ones and the eight that pair with them, so that a warp's 16-byte
// loads cover whole 128-byte lines, a norm costs log2(D / 16) shuffles and a rotation none.  The lanes that hold the same channels
// of different rows share the token's sines: each computes its part of the eight and hands them on by shuffle.
#include <cmath>
#include <type_traits>

#include "fdkv_internal.h"

namespace fdkv {

namespace {

constexpr int kQkThreads = 256;

template <typename T>
struct Raw8;  // eight channels as they lie in memory
template <>
struct Raw8<__nv_bfloat16> {
    uint4 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint4*>(p) = v; }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            f[2 * i] = __uint_as_float(w[i] << 16);
            f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
    __device__ __forceinline__ void set(const float (&f)[8]) {
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
            w[i] = *reinterpret_cast<const uint32_t*>(&h);
        }
        v = make_uint4(w[0], w[1], w[2], w[3]);
    }
};
template <>
struct Raw8<float> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* p) { a = *reinterpret_cast<const float4*>(p); b = *reinterpret_cast<const float4*>(p + 4); }
    __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = a; *reinterpret_cast<float4*>(p + 4) = b; }
    __device__ __forceinline__ void get(float (&f)[8]) const {
        f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
    }
    __device__ __forceinline__ void set(const float (&f)[8]) { a = make_float4(f[0], f[1], f[2], f[3]); b = make_float4(f[4], f[5], f[6], f[7]); }
};

// A warp takes `steps` groups of 32 / LPR rows of one token; `parts` warps share a token.
template <typename T, int D>
__global__ void __launch_bounds__(kQkThreads) qk_prep_kernel(const __grid_constant__ QkPrepArgs a, int parts, int steps) {
    constexpr int LPR = D / 16, RPW = 32 / LPR, PER = 8 / RPW;  // lanes per row, rows at a time, sines per lane
    const int64_t w = ((int64_t)blockIdx.x * kQkThreads + threadIdx.x) >> 5;
    const int lane = threadIdx.x & 31, l = lane % LPR, rg = lane / LPR;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");  // (the rows belong to the kernels ahead, and the outputs may still be read by them)
    const int64_t t = w / parts;
    if (t >= a.n) return;
    const int first = (int)(w - t * parts) * steps * RPW;

    // this lane's channels: [ca, ca + 8) and [cb, cb + 8), pairs of each other where they rotate in halves
    const int half = a.rotary_dim >> 1;
    const bool turns = 8 * l < half;
    const int ca = turns ? 8 * l : a.rotary_dim + 16 * (l - half / 8), cb = turns ? half + 8 * l : ca + 8;

    const int rows = a.Hq + a.Hk + a.Hv;
    struct Row {
        const T* src;
        T* dst;
        int kind;  // 0 query, 1 key, 2 value, 3 none
    };
    auto row_at = [&](int i) {
        Row r;
        if (i < a.Hq) {
            r.src = reinterpret_cast<const T*>(a.q) + t * a.q_n + (int64_t)i * a.q_h;
            r.dst = reinterpret_cast<T*>(a.q_out) + t * a.qo_n + (int64_t)i * a.qo_h;
            r.kind = 0;
        } else if (i < a.Hq + a.Hk) {
            r.src = reinterpret_cast<const T*>(a.k) + t * a.k_n + (int64_t)(i - a.Hq) * a.k_h;
            r.dst = reinterpret_cast<T*>(a.k_out) + t * a.ko_n + (int64_t)(i - a.Hq) * a.ko_h;
            r.kind = 1;
        } else {
            r.src = reinterpret_cast<const T*>(a.v) + t * a.v_n + (int64_t)(i - a.Hq - a.Hk) * a.v_h;
            r.dst = reinterpret_cast<T*>(a.v_out) + t * a.vo_n + (int64_t)(i - a.Hq - a.Hk) * a.vo_h;
            r.kind = i < rows ? 2 : 3;
        }
        return r;
    };
    Raw8<T> xa, xb;
    Row r = row_at(first + rg);
    if (r.kind != 3) { xa.load(r.src + ca); xb.load(r.src + cb); }

    float cs[8], sn[8];
    if (a.rotary_dim) {
        float c[PER], s[PER];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int j = rg * PER + i;
            // halves: both channels of pair j have frequency 8 l + j; neighbours: pairs (0, 1), (2, 3), .. of [ca, ca + 8), then of [cb, cb + 8)
            const int f = a.interleaved ? (j < 4 ? 4 * l + j : a.rotary_dim / 4 + 4 * l + j - 4) : 8 * l + j;
            float turn = 0.f;
            if (turns) {
                const double x = (double)a.pos[a.axis[f] * a.pos_stride + t] * (double)a.inv_freq[f] * 0.15915494309189533577;  // 1 / (2 pi)
                turn = (float)(2.0 * (x - rint(x)));  // half turns, -1 to 1
            }
            sincospif(turn, &s[i], &c[i]);
            c[i] *= a.scale;
            s[i] *= a.scale;
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            cs[j] = __shfl_sync(0xFFFFFFFFu, c[j % PER], j / PER * LPR + l);
            sn[j] = __shfl_sync(0xFFFFFFFFu, s[j % PER], j / PER * LPR + l);
        }
    }

    for (int it = 0; it < steps; ++it) {
        // the next group's rows are on their way while this one is worked on
        Raw8<T> na, nb;
        Row nr = r;
        const bool more = it + 1 < steps;
        if (more) {
            nr = row_at(first + (it + 1) * RPW + rg);
            if (nr.kind != 3) { na.load(nr.src + ca); nb.load(nr.src + cb); }
        }
        float f[8], g[8];
        const void* const weight = r.kind == 0 ? a.q_weight : r.kind == 1 ? a.k_weight : nullptr;
        if (r.kind == 3) {
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = g[i] = 0.f;
        } else {
            xa.get(f);
            xb.get(g);
        }
        if (a.q_weight || a.k_weight) {  // (every lane takes part in the shuffles)
            float ss = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) ss = fmaf(f[i], f[i], fmaf(g[i], g[i], ss));
#pragma unroll
            for (int o = LPR / 2; o; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
            if (weight) {
                const float inv = rsqrtf(ss * (1.f / D) + a.eps);
                Raw8<T> wa, wb;
                float fa[8], fb[8];
                wa.load(reinterpret_cast<const T*>(weight) + ca);
                wb.load(reinterpret_cast<const T*>(weight) + cb);
                wa.get(fa);
                wb.get(fb);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    f[i] = f[i] * inv * fa[i];
                    g[i] = g[i] * inv * fb[i];
                }
            }
        }
        if (r.kind < 2) {
            if (turns) {
                if (a.interleaved) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        float x = f[2 * i], y = f[2 * i + 1];
                        f[2 * i] = x * cs[i] - y * sn[i];
                        f[2 * i + 1] = y * cs[i] + x * sn[i];
                        x = g[2 * i]; y = g[2 * i + 1];
                        g[2 * i] = x * cs[4 + i] - y * sn[4 + i];
                        g[2 * i + 1] = y * cs[4 + i] + x * sn[4 + i];
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float x = f[i], y = g[i];
                        f[i] = x * cs[i] - y * sn[i];
                        g[i] = y * cs[i] + x * sn[i];
                    }
                }
            }
            xa.set(f);
            xb.set(g);
        }
        if (r.kind != 3) { xa.store(r.dst + ca); xb.store(r.dst + cb); }
        xa = na;
        xb = nb;
        r = nr;
    }
}

// n rows [n][H][d] of one layer behind a sequence's tail rows: one thread per 16 bytes.
__global__ void __launch_bounds__(256) append_tail_kernel(const char* k, const char* v, int64_t stride_t, int64_t stride_h, char* tail_k, char* tail_v, int64_t head_bytes,
                                                          int n, int H, int chunks, int32_t* len, int new_len) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, per = (int64_t)n * H * chunks;
    if (i == 0) *len = new_len;
    if (i >= 2 * per) return;
    const bool is_v = i >= per;
    const int64_t j = is_v ? i - per : i;
    const int c = (int)(j % chunks), h = (int)(j / chunks % H);
    const int64_t t = j / chunks / H;
    const uint4 x = *reinterpret_cast<const uint4*>((is_v ? v : k) + t * stride_t + h * stride_h + c * 16);
    *reinterpret_cast<uint4*>((is_v ? tail_v : tail_k) + h * head_bytes + t * chunks * 16 + c * 16) = x;
}

}  // namespace

cudaError_t launch_qk_prep(const QkPrepArgs& a, int dtype, int d, cudaStream_t st) {
    static PerDevice once;
    int sms = 0;
    cudaError_t e = once.ensure([]() { return cudaSuccess; }, &sms);
    if (e != cudaSuccess) return e;
    const int rpw = 32 / (d / 16), groups = (a.Hq + a.Hk + a.Hv + rpw - 1) / rpw;
    // Warps per token: one walks all of a token's rows, which computes the sines once, where there are tokens enough to fill the
    // device (16 warps on every SM); else a token's rows are spread.
    const int64_t want = ((int64_t)16 * sms + a.n - 1) / a.n;
    const int steps = (int)((groups + (want < groups ? want : groups) - 1) / (want < groups ? want : groups));
    const int parts = (groups + steps - 1) / steps;
    const int64_t blocks = (a.n * parts * 32 + kQkThreads - 1) / kQkThreads;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)blocks);
    cfg.blockDim = dim3(kQkThreads);
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    if (dtype == FDKV_BF16)
        e = d == 128 ? cudaLaunchKernelEx(&cfg, qk_prep_kernel<__nv_bfloat16, 128>, a, parts, steps) : cudaLaunchKernelEx(&cfg, qk_prep_kernel<__nv_bfloat16, 64>, a, parts, steps);
    else
        e = d == 128 ? cudaLaunchKernelEx(&cfg, qk_prep_kernel<float, 128>, a, parts, steps) : cudaLaunchKernelEx(&cfg, qk_prep_kernel<float, 64>, a, parts, steps);
    if (e != cudaSuccess) return e;
    count_launch(1);
    return cudaGetLastError();
}

cudaError_t launch_append_tail(const void* k, const void* v, int64_t stride_t, int64_t stride_h, void* tail_k, void* tail_v, int64_t head_bytes, int n, int H, int row_bytes,
                               int32_t* len, int new_len, cudaStream_t st) {
    const int64_t work = (int64_t)2 * n * H * (row_bytes / 16);
    append_tail_kernel<<<(unsigned)((work + 255) / 256), 256, 0, st>>>((const char*)k, (const char*)v, stride_t, stride_h, (char*)tail_k, (char*)tail_v, head_bytes, n, H,
                                                                     row_bytes / 16, len, new_len);
    count_launch(1);
    return cudaGetLastError();
}

}  // namespace fdkv
