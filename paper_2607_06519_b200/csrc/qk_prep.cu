// What a layer does to the rows of its projection before they can be probed, compressed or attended to: the RMS norm of every
// head's query and key and the rotation of their channel pairs by the token's position, each frequency on its own position axis
// (time, height, width), in one pass.
//   y = x / sqrt(mean_c x_c^2 + eps) * w          (no weights: y = x)
//   (a, b) -> (a cos - b sin, b cos + a sin) * s  angle = pos[axis of the frequency] * inv_freq
// All in float32 behind the storage type, one rounding at the end; the angle is a float64 product, whose whole turns are dropped
// before it becomes a float32 (a float32 product of a position of 10^6 would be off by 0.06 rad).  What is left, up to half a turn, is rounded to float32 once: with
// float32 rows the outputs are off by 5.5e-8 (root mean square, relative), with float64 sines they would be by 4.2e-8; bf16 rows hide it.
//
// Bound by memory traffic for prompts, by the chain load -> norm -> store for a few tokens.  D / 8 lanes share a (token, head) row:
// a lane holds four channels of the first half of the rotating ones and the four that pair with them, so that a warp's loads
// cover whole 128-byte stretches, a norm costs log2(D / 8) shuffles and a rotation none.  The lanes that hold the same channels
// of different rows share the token's sines: each computes its part of the four and hands them on by shuffle.
// Measured: 32 768 tokens of 32 + 8 heads of 128 channels, out of and into strided rows, norm and rotation: 112 us for 671 MB, 6.0 TB/s; 16 383 tokens without
// norms 57 us, 5.9 TB/s; one token 2.5 us.  (71 or 72 registers, 26 one-warp blocks on an SM.)  Float32 with norms spills 52 bytes, 80 with neighbouring pairs; 16 384
// tokens of 32 + 8 heads of 128 channels take 111 us, without norms (and spills) 106, where the bytes need 102.7.
// A warp works on one token and a group of rows is of one tensor, so that with few heads most lanes have no row and the sines are the work: 16 384 bf16 tokens
// of 4 + 1 heads of 128 channels take 24 us without norms, of 1 + 1 heads 22.5, of 1 + 1 heads of 64 channels 18, where the bytes need 6.4, 2.6 and 1.3.
// (Eight channels a lane, in 16-byte loads, needed 118 registers with weights: 16 warps on an SM, two groups of rows in flight each, 3.9 TB/s for
// 32 768 tokens of 40 heads.)
#include <cmath>
#include <type_traits>

#include "fdkv_internal.h"

namespace fdkv {

namespace {

constexpr int kQkThreads = 32;  // (two warps, us for 32 768 tokens: 113 instead of 111, four 115, eight 126)

template <typename T>
struct Raw4;  // four channels as they lie in memory
template <>
struct Raw4<__nv_bfloat16> {
    uint2 v;
    __device__ __forceinline__ void load(const __nv_bfloat16* p) { v = *reinterpret_cast<const uint2*>(p); }
    __device__ __forceinline__ void store(__nv_bfloat16* p) const { *reinterpret_cast<uint2*>(p) = v; }
    __device__ __forceinline__ void get(float (&f)[4]) const {
        f[0] = __uint_as_float(v.x << 16); f[1] = __uint_as_float(v.x & 0xFFFF0000u);
        f[2] = __uint_as_float(v.y << 16); f[3] = __uint_as_float(v.y & 0xFFFF0000u);
    }
    __device__ __forceinline__ void set(const float (&f)[4]) {
        const __nv_bfloat162 x = __floats2bfloat162_rn(f[0], f[1]), y = __floats2bfloat162_rn(f[2], f[3]);
        v = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
    }
};
template <>
struct Raw4<float> {
    float4 v;
    __device__ __forceinline__ void load(const float* p) { v = *reinterpret_cast<const float4*>(p); }
    __device__ __forceinline__ void store(float* p) const { *reinterpret_cast<float4*>(p) = v; }
    __device__ __forceinline__ void get(float (&f)[4]) const { f[0] = v.x; f[1] = v.y; f[2] = v.z; f[3] = v.w; }
    __device__ __forceinline__ void set(const float (&f)[4]) { v = make_float4(f[0], f[1], f[2], f[3]); }
};

// two float32 operations in one instruction
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 p, q;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tmul.rn.f32x2 p, p, q;\n\tmov.b64 {%0, %1}, p;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 p, q, r;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %5};\n\tmov.b64 r, {%6, %7};\n\tfma.rn.f32x2 p, p, q, r;\n\tmov.b64 {%0, %1}, p;\n\t}"
        : "=f"(d.x), "=f"(d.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}

// A warp takes up to `steps` groups of one token; `parts` warps share a token.  A group is 32 / LPR rows of one tensor (the queries' groups come
// first, then the keys', then the values'); U groups are on their way at a time.
// The weights are folded into the sines: a pair (u, v) becomes r (u (w_u cos) - v (w_v sin), v (w_v cos) + u (w_u sin)), r the inverse root.
template <typename T, int D, bool NORM, bool INTER>
__global__ void __launch_bounds__(kQkThreads, 26) qk_prep_kernel(const __grid_constant__ QkPrepArgs a, int parts, int steps) {
    constexpr int LPR = D / 8, RPW = 32 / LPR, PER = 4 / RPW;  // lanes per row, rows of a group, sines per lane
    constexpr int U = 4;
    const int64_t w = (int64_t)blockIdx.x * (kQkThreads / 32) + __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0);  // (uniform to the compiler, which saves registers)
    const int lane = threadIdx.x & 31, l = lane % LPR, rg = lane / LPR;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    asm volatile("griddepcontrol.wait;" ::: "memory");  // (the rows belong to the kernels ahead, and the outputs may still be read by them)
    const int64_t t = w / parts;
    if (t >= a.n) return;
    const int first = (int)(w - t * parts) * steps;

    // this lane's channels: [ca, ca + 4) and [cb, cb + 4), pairs of each other where they rotate in halves
    const int half = a.rotary_dim >> 1;
    const bool turns = 4 * l < half;
    const int ca = turns ? 4 * l : a.rotary_dim + 8 * (l - half / 4), cb = turns ? half + 4 * l : ca + 4;
    // sines and cosines of this lane's four pairs; halves: (channel ca + j, channel cb + j), frequency 4 l + j; neighbours: pairs (0, 1), (2, 3)
    // of [ca, ca + 4), then of [cb, cb + 4)
    float2 cs[2] = {make_float2(1.f, 1.f), make_float2(1.f, 1.f)}, sn[2] = {};
    if (a.rotary_dim) {
        float c[PER], s[PER], cj[4], sj[4];
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int j = rg * PER + i;
            const int f = INTER ? (j < 2 ? 2 * l + j : a.rotary_dim / 4 + 2 * l + j - 2) : 4 * l + j;
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
        for (int j = 0; j < 4; ++j) {
            cj[j] = __shfl_sync(0xFFFFFFFFu, c[j % PER], j / PER * LPR + l);
            sj[j] = __shfl_sync(0xFFFFFFFFu, s[j % PER], j / PER * LPR + l);
        }
        if (turns) {
            cs[0] = make_float2(cj[0], cj[1]); cs[1] = make_float2(cj[2], cj[3]);
            sn[0] = make_float2(sj[0], sj[1]); sn[1] = make_float2(sj[2], sj[3]);
        }
    }

    // the warp's groups [lo, hi) of one tensor of `rows` rows; `skip`: it is copied as it is
    auto tensor = [&](const void* from, int64_t in_n, int64_t in_h, void* to, int64_t out_n, int64_t out_h, int rows, const void* wt, int lo, int hi, bool skip) {
        if (lo >= hi) return;
        const T* src = reinterpret_cast<const T*>(from) + t * in_n + (lo * RPW + rg) * in_h + ca;
        T* dst = reinterpret_cast<T*>(to) + t * out_n + (lo * RPW + rg) * out_h + ca;
        const int64_t src_step = RPW * in_h, dst_step = RPW * out_h;
        const int ab = cb - ca;
        int left = rows - (lo * RPW + rg);  // rows from this lane's on
        float2 cu[2], cv[2], sv[2], su[2];  // pairs 2 i and 2 i + 1: w_u cos, w_v cos, w_v sin, w_u sin
        const bool normed = NORM && wt != nullptr;
        float fa[4] = {1.f, 1.f, 1.f, 1.f}, fb[4] = {1.f, 1.f, 1.f, 1.f};
        if (normed) {
            Raw4<T> ra, rb;
            ra.load(reinterpret_cast<const T*>(wt) + ca);
            rb.load(reinterpret_cast<const T*>(wt) + cb);
            ra.get(fa);
            rb.get(fb);
        }
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float* const x = i == 0 ? fa : fb;
            const float2 u = INTER ? make_float2(x[0], x[2]) : make_float2(fa[2 * i], fa[2 * i + 1]), v = INTER ? make_float2(x[1], x[3]) : make_float2(fb[2 * i], fb[2 * i + 1]);
            cu[i] = NORM ? mul2(u, cs[i]) : cs[i];
            cv[i] = NORM ? mul2(v, cs[i]) : cs[i];
            sv[i] = NORM ? mul2(v, sn[i]) : sn[i];
            su[i] = NORM ? mul2(u, sn[i]) : sn[i];
        }
#pragma unroll 1
        for (int gr = lo; gr < hi; gr += U) {
            Raw4<T> xa[U], xb[U];
#pragma unroll
            for (int i = 0; i < U; ++i) {
                if (gr + i < hi && i * RPW < left) {
                    xa[i].load(src);
                    xb[i].load(src + ab);
                }
                src += src_step;
            }
#pragma unroll
            for (int i = 0; i < U; ++i) {
                if (gr + i >= hi) break;
                const bool live = i * RPW < left;
                if (!skip) {
                    float f[4] = {}, g[4] = {};
                    if (live) { xa[i].get(f); xb[i].get(g); }
                    float2 r = make_float2(1.f, 1.f);
                    if (normed) {
                        float2 s2 = mul2(make_float2(f[0], f[1]), make_float2(f[0], f[1]));
                        s2 = fma2(make_float2(f[2], f[3]), make_float2(f[2], f[3]), s2);
                        s2 = fma2(make_float2(g[0], g[1]), make_float2(g[0], g[1]), s2);
                        s2 = fma2(make_float2(g[2], g[3]), make_float2(g[2], g[3]), s2);
                        float ss = s2.x + s2.y;
#pragma unroll
                        for (int o = LPR / 2; o; o >>= 1) ss += __shfl_xor_sync(0xFFFFFFFFu, ss, o);
                        r.x = r.y = rsqrtf(ss * (1.f / D) + a.eps);
                    }
#pragma unroll
                    for (int p = 0; p < 2; ++p) {  // pairs 2 p and 2 p + 1
                        float* const x = p == 0 ? f : g;
                        const float2 u = INTER ? make_float2(x[0], x[2]) : make_float2(f[2 * p], f[2 * p + 1]), v = INTER ? make_float2(x[1], x[3]) : make_float2(g[2 * p], g[2 * p + 1]);
                        float2 y = mul2(u, cu[p]), z = mul2(v, cv[p]);
                        if (turns) {  // (the others' sines are zero, which an infinite value would turn into NaN)
                            y = fma2(make_float2(-v.x, -v.y), sv[p], y);
                            z = fma2(u, su[p], z);
                        }
                        if (NORM) {
                            y = mul2(y, r);
                            z = mul2(z, r);
                        }
                        if (INTER) {
                            x[0] = y.x; x[2] = y.y; x[1] = z.x; x[3] = z.y;
                        } else {
                            f[2 * p] = y.x; f[2 * p + 1] = y.y; g[2 * p] = z.x; g[2 * p + 1] = z.y;
                        }
                    }
                    xa[i].set(f);
                    xb[i].set(g);
                }
                if (live) {
                    xa[i].store(dst);
                    xb[i].store(dst + ab);
                }
                dst += dst_step;
            }
            left -= U * RPW;
        }
    };
    const int gq = (a.Hq + RPW - 1) / RPW, gk = (a.Hk + RPW - 1) / RPW, gv = (a.Hv + RPW - 1) / RPW;
    tensor(a.q, a.q_n, a.q_h, a.q_out, a.qo_n, a.qo_h, a.Hq, a.q_weight, first, min(gq, first + steps), false);
    tensor(a.k, a.k_n, a.k_h, a.k_out, a.ko_n, a.ko_h, a.Hk, a.k_weight, max(0, first - gq), min(gk, first + steps - gq), false);
    if (a.Hv) tensor(a.v, a.v_n, a.v_h, a.v_out, a.vo_n, a.vo_h, a.Hv, nullptr, max(0, first - gq - gk), min(gv, first + steps - gq - gk), true);
}

// n rows [n][H][d] of one layer behind a sequence's tail rows: one thread per 16 bytes, a plain copy (once per sequence and layer, a few microseconds; memory
// bounds it from some ten thousand rows on, more than tails have).
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

template <typename T, int D>
cudaError_t launch_qk(const cudaLaunchConfig_t& cfg, const QkPrepArgs& a, int parts, int steps) {
    const bool norm = a.q_weight || a.k_weight;
    if (a.interleaved) return norm ? cudaLaunchKernelEx(&cfg, qk_prep_kernel<T, D, true, true>, a, parts, steps) : cudaLaunchKernelEx(&cfg, qk_prep_kernel<T, D, false, true>, a, parts, steps);
    return norm ? cudaLaunchKernelEx(&cfg, qk_prep_kernel<T, D, true, false>, a, parts, steps) : cudaLaunchKernelEx(&cfg, qk_prep_kernel<T, D, false, false>, a, parts, steps);
}

}  // namespace

cudaError_t launch_qk_prep(const QkPrepArgs& a, int dtype, int d, cudaStream_t st) {
    static PerDevice once;
    int sms = 0;
    cudaError_t e = once.ensure([]() { return cudaSuccess; }, &sms);
    if (e != cudaSuccess) return e;
    const int rpw = 32 / (d / 8), groups = (a.Hq + rpw - 1) / rpw + (a.Hk + rpw - 1) / rpw + (a.Hv + rpw - 1) / rpw;
    // Warps per token: one walks all of a token's rows, which computes the sines once, where there are tokens enough to fill the
    // device (eight warps on every SM; with sixteen, us for 64 tokens of 40 heads 5.3 instead of 3.6, for 2 048 13.0 instead of 13.8); else a token's
    // rows are spread.
    const int64_t want = ((int64_t)8 * sms + a.n - 1) / a.n;
    const int steps = (int)((groups + (want < groups ? want : groups) - 1) / (want < groups ? want : groups));
    const int parts = (groups + steps - 1) / steps;
    const int64_t blocks = (a.n * parts + kQkThreads / 32 - 1) / (kQkThreads / 32);
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
        e = d == 128 ? launch_qk<__nv_bfloat16, 128>(cfg, a, parts, steps) : launch_qk<__nv_bfloat16, 64>(cfg, a, parts, steps);
    else
        e = d == 128 ? launch_qk<float, 128>(cfg, a, parts, steps) : launch_qk<float, 64>(cfg, a, parts, steps);
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
