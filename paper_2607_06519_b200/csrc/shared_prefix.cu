// Decode attention of a batch whose sequences share one committed prompt and have generated tokens of their own: the prompt's
// compressed rows are read and reconstructed once for all query rows of a KV head.
//   out[b, g] = softmax over (the prompt's T rows, then the tail of sequence b) of khat . q / sqrt(d), times vhat
// Two kernels: the prompt part (here for float32 storage or head_dim 64, in shared_tc.cu for bf16 / head_dim 128) leaves split-K
// parts (maximum, sum, unnormalised output per query row); shared_join_kernel attends to each sequence's tail, joins it with the
// parts of its rows and writes the outputs.
#include <algorithm>
#include <type_traits>

#include "fdkv_internal.h"

namespace fdkv {

cudaError_t launch_shared_tc(const SharedArgs& a, const SharedSched& sch, cudaStream_t st);

namespace {

template <typename T>
__device__ __forceinline__ float ldf(const T* p);
template <>
__device__ __forceinline__ float ldf<float>(const float* p) { return *p; }
template <>
__device__ __forceinline__ float ldf<__nv_bfloat16>(const __nv_bfloat16* p) { return __bfloat162float(*p); }

// eight consecutive channels of a row
__device__ __forceinline__ void load8(const float* p, float (&f)[8]) {
    const float4 a = __ldcg(reinterpret_cast<const float4*>(p)), b = __ldcg(reinterpret_cast<const float4*>(p + 4));
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w; f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void load8(const __nv_bfloat16* p, float (&f)[8]) {
    const uint4 v = __ldcg(reinterpret_cast<const uint4*>(p));
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
    }
}

// ------------------------------------------------------------------------------------------------ prompt part, portable
constexpr int kRows = 32;      // query rows of a group
constexpr int kTok = 32;       // tokens at a time: a tile of the schedule
constexpr int kThreads = 256;

template <int D>
constexpr int part_smem() { return (kRows * (D + 4) + 2 * kTok * (D + 4) + kRows * (kTok + 1) + 2 * kRows) * 4; }

// Tiles of kTok tokens are reconstructed into shared memory as float32 (rows, plus the sign times the scattered residual entries;
// the unit's scale is applied to the logits and the outputs) and multiplied with the group's query rows: a thread has two rows x
// two tokens of the logits and 2 x D / 16 of the outputs.  float32 FMA; for float32 storage eight channels' products at a time
// are added up in float64, since the exponential magnifies the rounding of logits of a few tens.
// Short prompts are bound by latency: the correctness workload's 4 099 tokens, 2 KV heads, 6 sequences make two tiles for each of 148 blocks, and a call of
// 13.9 us is two dependent kernels, of which the bytes need 0.7.  From some thousand tokens on the loads from shared memory bound it, one of 16 bytes for every four products of
// a thread: 8 to 10 TFLOP/s whatever the type.  8 KV heads x 4, 8 and 64 sequences, us (and what the bytes need): float32 of 128 channels, 8 192 tokens 116 and 898 (10.6),
// 32 768 tokens 445 and 3 541 (42.5); of 64 channels 71 and 539 (5.3), 268 and 2 105 (21.3); bf16 of 64 channels 89 and 500 (2.7), 349 and 2 075 (10.7).
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) shared_part_kernel(SharedArgs a, const __grid_constant__ SharedSched sch) {
    using ACC = typename std::conditional<sizeof(T) == 4, double, float>::type;
    extern __shared__ __align__(16) float smem[];
    constexpr int P = D + 4;  // row pitch: neighbouring rows lie four banks apart
    float* const sq = smem;
    float* const sk = sq + kRows * P;
    float* const sv = sk + kTok * P;
    float* const sp = sv + kTok * P;             // [kRows][kTok + 1]
    float* const sm = sp + kRows * (kTok + 1);   // maxima, sums
    float* const sl = sm + kRows;
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;  // rows ty, ty + 16; tokens tx, tx + 16; channels 4 tx + 64 i
    const int R = a.batch * a.G;
    const int range = blockIdx.x / sch.groups, group = blockIdx.x % sch.groups, row0 = group * kRows, rows = min(kRows, R - row0);
    int g0 = sch.start[range];
    const int g1 = sch.start[range + 1];
    bool waited = false;
    auto put8 = [&](float* to, const float (&f)[8]) {
        *reinterpret_cast<float4*>(to) = make_float4(f[0], f[1], f[2], f[3]);
        *reinterpret_cast<float4*>(to + 4) = make_float4(f[4], f[5], f[6], f[7]);
    };
    while (g0 < g1) {
        const int h = g0 / sch.tiles, t_first = g0 % sch.tiles, t_last = min(sch.tiles, t_first + g1 - g0);
        g0 += t_last - t_first;
        const UnitDesc ud = a.desc[h];
        const bool resid = ud.mode == FDKV_MODE_RESIDUAL;
        const float kscale = ud.scale * rsqrtf((float)D), sign = ud.sign;
        float o[2][D / 16];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[i][j] = 0.f;
        const int tok_end = min(ud.T, t_last * kTok);
        constexpr int kPF = 2;
        int next0[2] = {}, next1[2] = {};  // a tile's entries in either list
        auto bounds = [&](int tok) {
            const int s0 = tok / kResTile, s1 = (min(tok + kTok, tok_end) + kResTile - 1) / kResTile;
            next0[0] = ud.k_off[s0];
            next1[0] = ud.k_off[s1];
            next0[1] = ud.v_off ? ud.v_off[s0] : next0[0];
            next1[1] = ud.v_off ? ud.v_off[s1] : next1[0];
        };
        if (resid) bounds(t_first * kTok);
        for (int tok = t_first * kTok; tok < tok_end; tok += kTok) {
            const int n = min(kTok, tok_end - tok);
            // the first entries of either list travel with the rows; the next tile's bounds are on their way meanwhile
            int e0[2] = {next0[0], next0[1]}, e1[2] = {next1[0], next1[1]}, pi[2][kPF];
            float pv[2][kPF];
            if (resid) {
                if (tok + kTok < tok_end) bounds(tok + kTok);
                if (ud.res_kind != 1)
#pragma unroll
                    for (int l = 0; l < 2; ++l)
#pragma unroll
                        for (int k = 0; k < kPF; ++k) {
                            const int e = e0[l] + tid + k * kThreads;
                            if (e < e1[l]) {
                                pi[l][k] = (l && ud.v_idx ? ud.v_idx : ud.k_idx)[e];
                                pv[l][k] = ldf<T>(reinterpret_cast<const T*>(l ? ud.v_val : ud.k_val) + e);
                            }
                        }
            }
            __syncthreads();
#pragma unroll
            for (int i = tid; i < 2 * kTok * D / 8; i += kThreads) {
                const bool is_v = i >= kTok * D / 8;
                const int j = is_v ? i - kTok * D / 8 : i, t = j / (D / 8), c = j % (D / 8) * 8;
                float f[8] = {};
                if (t < n) load8(reinterpret_cast<const T*>(is_v ? ud.v_rows : ud.k_rows) + (int64_t)(tok + t) * D + c, f);
                put8((is_v ? sv : sk) + t * P + c, f);
            }
            __syncthreads();
            if (resid) {  // (every position is in a list once: no two threads add to the same place)
#pragma unroll
                for (int is_v = 0; is_v < 2; ++is_v) {
                    const int32_t* const idx = is_v && ud.v_idx ? ud.v_idx : ud.k_idx;
                    const T* const val = reinterpret_cast<const T*>(is_v ? ud.v_val : ud.k_val);
                    float* const to = is_v ? sv : sk;
                    if (ud.res_kind == 1) {  // whole rows of selected tokens
                        for (int i = e0[is_v] * D + tid; i < e1[is_v] * D; i += kThreads) to[(idx[i / D] - tok) * P + i % D] += sign * ldf<T>(val + i);
                    } else {
#pragma unroll
                        for (int k = 0; k < kPF; ++k)
                            if (e0[is_v] + tid + k * kThreads < e1[is_v]) {
                                const int at = pi[is_v][k] - tok * D;
                                to[at / D * P + at % D] += sign * pv[is_v][k];
                            }
                        for (int e = e0[is_v] + tid + kPF * kThreads; e < e1[is_v]; e += kThreads) {
                            const int at = idx[e] - tok * D;
                            to[at / D * P + at % D] += sign * ldf<T>(val + e);
                        }
                    }
                }
            }
            if (!waited) {  // (all so far is static since commit)
                asm volatile("griddepcontrol.wait;" ::: "memory");               // q belongs to the kernels ahead
                asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (behind the wait: the join reads the tails before its own)
                waited = true;
            }
            if (tok == t_first * kTok) {
                for (int i = tid; i < kRows * D / 8; i += kThreads) {
                    const int r = i / (D / 8), c = i % (D / 8) * 8;
                    float f[8] = {};
                    if (r < rows) {
                        const int row = row0 + r, b = row / a.G, g = row % a.G;
                        load8(reinterpret_cast<const T*>(a.q) + ((int64_t)b * a.Hq + h * a.G + g) * D + c, f);
                    }
                    put8(sq + r * P + c, f);
                }
                if (tid < kRows) { sm[tid] = -INFINITY; sl[tid] = 0.f; }
            }
            __syncthreads();
            // logits
            ACC s[2][2] = {};
#pragma unroll 2
            for (int c = 0; c < D; c += 8) {
                float q[2][8], k[2][8];
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int x = 0; x < 8; x += 4) {
                        *reinterpret_cast<float4*>(&q[i][x]) = *reinterpret_cast<const float4*>(sq + (ty + 16 * i) * P + c + x);
                        *reinterpret_cast<float4*>(&k[i][x]) = *reinterpret_cast<const float4*>(sk + (tx + 16 * i) * P + c + x);
                    }
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) {
                        float d = q[i][0] * k[j][0];
#pragma unroll
                        for (int x = 1; x < 8; ++x) d = fmaf(q[i][x], k[j][x], d);
                        s[i][j] += (ACC)d;
                    }
            }
            // softmax over this step's tokens; the sixteen lanes with the same ty hold a row
            float f[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = ty + 16 * i;
                float x[2], mx = -INFINITY;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    x[j] = tx + 16 * j < n ? (float)(s[i][j] * (ACC)kscale) : -INFINITY;
                    mx = fmaxf(mx, x[j]);
                }
#pragma unroll
                for (int w = 8; w; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xFFFFFFFFu, mx, w));
                const float m_old = sm[r], m = fmaxf(m_old, mx);
                f[i] = m_old == -INFINITY ? 0.f : __expf(m_old - m);
                float sum = 0.f;
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const float p = x[j] == -INFINITY ? 0.f : __expf(x[j] - m);
                    sp[r * (kTok + 1) + tx + 16 * j] = p;
                    sum += p;
                }
#pragma unroll
                for (int w = 8; w; w >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, w);
                __syncwarp();  // (the row's maximum has been read by its lanes)
                if (tx == 0) { sm[r] = m; sl[r] = sl[r] * f[i] + sum; }
            }
            __syncwarp();  // (a row's probabilities are written and read by one warp)
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < D / 16; ++j) o[i][j] *= f[i];
#pragma unroll 4
            for (int t = 0; t < kTok; ++t) {
                const float p0 = sp[ty * (kTok + 1) + t], p1 = sp[(ty + 16) * (kTok + 1) + t];
#pragma unroll
                for (int j = 0; j < D / 16; j += 4) {
                    const float4 v = *reinterpret_cast<const float4*>(sv + t * P + 16 * j + 4 * tx);
                    o[0][j] = fmaf(p0, v.x, o[0][j]); o[0][j + 1] = fmaf(p0, v.y, o[0][j + 1]); o[0][j + 2] = fmaf(p0, v.z, o[0][j + 2]); o[0][j + 3] = fmaf(p0, v.w, o[0][j + 3]);
                    o[1][j] = fmaf(p1, v.x, o[1][j]); o[1][j + 1] = fmaf(p1, v.y, o[1][j + 1]); o[1][j + 2] = fmaf(p1, v.z, o[1][j + 2]); o[1][j + 3] = fmaf(p1, v.w, o[1][j + 3]);
                }
            }
        }
        __syncthreads();
        float* const part = a.partials + ((int64_t)(range + h) * sch.groups + group) * shared_part_floats(sch.row_tile, D);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int r = ty + 16 * i;
            if (r >= rows) continue;
#pragma unroll
            for (int j = 0; j < D / 16; j += 4) {
                const int c4 = (16 * j + 4 * tx) >> 2;
                *reinterpret_cast<float4*>(part + ((int64_t)c4 * sch.row_tile + r) * 4) =
                    make_float4(o[i][j] * ud.scale, o[i][j + 1] * ud.scale, o[i][j + 2] * ud.scale, o[i][j + 3] * ud.scale);
            }
            if (tx == 0) {
                part[(int64_t)sch.row_tile * D + r] = sm[r];
                part[(int64_t)sch.row_tile * (D + 1) + r] = sl[r];
            }
        }
    }
}

// ------------------------------------------------------------------------------------------------ tails and the join
template <int NB>
struct SharedSeqs {
    int32_t slot[NB], len[NB];  // len counts this call's append
};

// Ranges [lo, hi] that meet head h.
__device__ __forceinline__ void ranges_of_head(const SharedSched& sch, int h, int& lo, int& hi) {
    lo = 0;
    for (int step = 128; step; step >>= 1)
        if (lo + step < sch.ranges && sch.start[lo + step] <= h * sch.tiles) lo += step;
    hi = lo;
    for (int step = 128; step; step >>= 1)
        if (hi + step < sch.ranges && sch.start[hi + step] < (h + 1) * sch.tiles) hi += step;
}

// A softmax state: what the exponents are relative to (natural logarithm), their sum, four channels of the weighted sum.
struct State4 {
    float m = -INFINITY, l = 0.f;
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    __device__ __forceinline__ void add(float pm, float pl, const float4& o) {
        const float mn = fmaxf(m, pm), ref = mn == -INFINITY ? 0.f : mn, f0 = __expf(m - ref), f1 = __expf(pm - ref);
        l = l * f0 + pl * f1;
        a.x = a.x * f0 + o.x * f1; a.y = a.y * f0 + o.y * f1; a.z = a.z * f0 + o.z * f1; a.w = a.w * f0 + o.w * f1;
        m = mn;
    }
    // parts c, c + step, .. up to hi of the row r of a group (p0: that of range 0; `stride` floats on: that of the next), BATCH of them on their way
    template <int D, int BATCH>
    __device__ __forceinline__ void add_parts(const float* p0, int64_t stride, int row_tile, int r, int c4, int c, int hi, int step) {
        for (; c <= hi; c += BATCH * step) {
            float pm[BATCH], pl[BATCH];
            float4 po[BATCH];
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const int cc = c + k * step;
                pm[k] = -INFINITY;
                pl[k] = 0.f;
                po[k] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (cc <= hi) {
                    const float* const part = p0 + cc * stride;
                    pm[k] = __ldcg(part + (int64_t)row_tile * D + r);
                    pl[k] = __ldcg(part + (int64_t)row_tile * (D + 1) + r);
                    po[k] = __ldcg(reinterpret_cast<const float4*>(part + ((int64_t)c4 * row_tile + r) * 4));
                }
            }
            float mn = m;
#pragma unroll
            for (int k = 0; k < BATCH; ++k) mn = fmaxf(mn, pm[k]);
            const float ref = mn == -INFINITY ? 0.f : mn, f0 = __expf(m - ref);
            l *= f0;
            a.x *= f0; a.y *= f0; a.z *= f0; a.w *= f0;
#pragma unroll
            for (int k = 0; k < BATCH; ++k) {
                const float f = __expf(pm[k] - ref);
                l = fmaf(pl[k], f, l);
                a.x = fmaf(po[k].x, f, a.x); a.y = fmaf(po[k].y, f, a.y); a.z = fmaf(po[k].z, f, a.z); a.w = fmaf(po[k].w, f, a.w);
            }
            m = mn;
        }
    }
    __device__ __forceinline__ void store(void* out, int out_dtype, int64_t at) const {
        const float inv = l > 0.f ? 1.f / l : 0.f;
        if (out_dtype == FDKV_BF16) {
            const __nv_bfloat162 x = __floats2bfloat162_rn(a.x * inv, a.y * inv), y = __floats2bfloat162_rn(a.z * inv, a.w * inv);
            *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(out) + at) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
        } else {
            *reinterpret_cast<float4*>(reinterpret_cast<float*>(out) + at) = make_float4(a.x * inv, a.y * inv, a.z * inv, a.w * inv);
        }
    }
};

constexpr int kJoinWarps = 8;

// Portable join.  grid (Hkv, batch).  D / 8 lanes share a tail token, eight channels each; every such lane group keeps a softmax state of its own,
// joined through shared memory with the prompt's parts.  The tails, q and the new rows are read before the dependency wait: the
// prompt kernel lets this one start only behind its own, when all they come from is complete.  Bound by the chain of its loads.  (Eight float32 heads a group need more than
// 255 registers: 280 bytes spilled.)
template <typename T, int D, int G, int NB>
__global__ void __launch_bounds__(kJoinWarps * 32) shared_join_kernel(SharedArgs a, const __grid_constant__ SharedSched sch, const __grid_constant__ SharedSeqs<NB> sq) {
    using ACC = typename std::conditional<sizeof(T) == 4, double, float>::type;
    constexpr int LPT = D / 8, TPI = 32 / LPT, U = sizeof(T) == 4 || G == 8 ? 2 : 4;
    // outputs in fours; threads that share one, each with its share of the parts
    constexpr int ITEMS = G * D / 4, WAYS = kJoinWarps * 32 / ITEMS;
    static_assert(WAYS >= 1 && WAYS * ITEMS == kJoinWarps * 32, "one four of outputs per thread");
    __shared__ __align__(16) float s_acc[kJoinWarps][G][D];
    __shared__ float s_m[kJoinWarps][G], s_l[kJoinWarps][G];
    __shared__ float4 j_acc[WAYS][ITEMS];
    __shared__ float2 j_ml[WAYS][ITEMS];
    const int h = blockIdx.x, b = blockIdx.y;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, grp = lane / LPT, c0 = lane % LPT * 8;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int n = sq.len[b], slot = sq.slot[b];
    const int64_t tail0 = ((int64_t)slot * a.Hkv + h) * a.tail_rows * D;
    T* const tk = reinterpret_cast<T*>(a.tail_k) + tail0;
    T* const tv = reinterpret_cast<T*>(a.tail_v) + tail0;
    const T* const kn = a.k_new ? reinterpret_cast<const T*>(a.k_new) + ((int64_t)b * a.Hkv + h) * D : nullptr;
    const T* const vn = a.k_new ? reinterpret_cast<const T*>(a.v_new) + ((int64_t)b * a.Hkv + h) * D : nullptr;
    const float kscale = rsqrtf((float)D);
    float q[G][8], acc[G][8], m[G], l[G];
#pragma unroll
    for (int g = 0; g < G; ++g) {
        load8(reinterpret_cast<const T*>(a.q) + ((int64_t)b * a.Hq + h * G + g) * D + c0, q[g]);
        m[g] = -INFINITY;
        l[g] = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[g][i] = 0.f;
    }
    for (int t0 = warp * TPI * U; t0 < n; t0 += kJoinWarps * TPI * U) {
        float k[U][8], v[U][8], p[G][U];
#pragma unroll
        for (int s = 0; s < U; ++s) {  // (rows behind the last are read as the last and masked; the appended one comes from the caller)
            const int t = min(t0 + s * TPI + grp, n - 1);
            const bool fresh = kn && t == n - 1;
            load8((fresh ? kn : tk + (int64_t)t * D) + c0, k[s]);
            load8((fresh ? vn : tv + (int64_t)t * D) + c0, v[s]);
        }
#pragma unroll
        for (int g = 0; g < G; ++g) {
            float mx = m[g];
#pragma unroll
            for (int s = 0; s < U; ++s) {
                ACC d = 0;
#pragma unroll
                for (int i = 0; i < 8; ++i) d = fma((ACC)q[g][i], (ACC)k[s][i], d);
#pragma unroll
                for (int o = LPT / 2; o; o >>= 1) d += __shfl_xor_sync(0xFFFFFFFFu, d, o);
                p[g][s] = t0 + s * TPI + grp < n ? (float)d * kscale : -INFINITY;
                mx = fmaxf(mx, p[g][s]);
            }
            const float ref = mx == -INFINITY ? 0.f : mx;  // (this lane group may have met no token yet)
            const float f = __expf(m[g] - ref);
            l[g] *= f;
#pragma unroll
            for (int i = 0; i < 8; ++i) acc[g][i] *= f;
            m[g] = mx;
#pragma unroll
            for (int s = 0; s < U; ++s) {
                const float w = __expf(p[g][s] - ref);
                l[g] += w;
#pragma unroll
                for (int i = 0; i < 8; ++i) acc[g][i] = fmaf(w, v[s][i], acc[g][i]);
            }
        }
    }
    if (kn && warp == 0 && lane < LPT) {  // the new row joins the tail for later calls
        float f[8];
        const int64_t at = (int64_t)(n - 1) * D + c0;
        if constexpr (sizeof(T) == 2) {
            *reinterpret_cast<uint4*>(tk + at) = *reinterpret_cast<const uint4*>(kn + c0);
            *reinterpret_cast<uint4*>(tv + at) = *reinterpret_cast<const uint4*>(vn + c0);
        } else {
            load8(kn + c0, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) tk[at + i] = f[i];
            load8(vn + c0, f);
#pragma unroll
            for (int i = 0; i < 8; ++i) tv[at + i] = f[i];
        }
        if (lane == 0 && h == 0) a.tail_len[slot] = n;
    }
    // ---- the lane groups of a warp, then the warps ----
#pragma unroll
    for (int g = 0; g < G; ++g) {
        float M = m[g];
#pragma unroll
        for (int o = LPT; o < 32; o <<= 1) M = fmaxf(M, __shfl_xor_sync(0xFFFFFFFFu, M, o));
        const float f = m[g] == -INFINITY ? 0.f : __expf(m[g] - M);
        l[g] *= f;
#pragma unroll
        for (int o = LPT; o < 32; o <<= 1) l[g] += __shfl_xor_sync(0xFFFFFFFFu, l[g], o);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            acc[g][i] *= f;
#pragma unroll
            for (int o = LPT; o < 32; o <<= 1) acc[g][i] += __shfl_xor_sync(0xFFFFFFFFu, acc[g][i], o);
        }
        if (grp == 0) {
            *reinterpret_cast<float4*>(&s_acc[warp][g][c0]) = make_float4(acc[g][0], acc[g][1], acc[g][2], acc[g][3]);
            *reinterpret_cast<float4*>(&s_acc[warp][g][c0 + 4]) = make_float4(acc[g][4], acc[g][5], acc[g][6], acc[g][7]);
            if (lane == 0) { s_m[warp][g] = M; s_l[warp][g] = l[g]; }
        }
    }
    const int group = b * G / sch.row_tile, r0 = b * G - group * sch.row_tile;  // (row tiles hold whole sequences)
    int c_lo, c_hi;
    ranges_of_head(sch, h, c_lo, c_hi);
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");  // the prompt's parts
    const int i = threadIdx.x % ITEMS, way = threadIdx.x / ITEMS, g = i % G, c4 = i / G;
    const int64_t part = shared_part_floats(sch.row_tile, D), stride = sch.groups * part;
    State4 s;
    s.add_parts<D, 6>(a.partials + h * stride + group * part, stride, sch.row_tile, r0 + g, c4, c_lo + way, c_hi, WAYS);
    if constexpr (WAYS > 1) {
        j_acc[way][i] = s.a;
        j_ml[way][i] = make_float2(s.m, s.l);
        __syncthreads();
        if (way > 0) return;
#pragma unroll
        for (int w = 1; w < WAYS; ++w) s.add(j_ml[w][i].x, j_ml[w][i].y, j_acc[w][i]);
    }
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) s.add(s_m[w][g], s_l[w][g], *reinterpret_cast<const float4*>(&s_acc[w][g][c4 * 4]));
    s.store(a.out, a.out_dtype, ((int64_t)b * a.Hq + h * G + g) * D + c4 * 4);
}

// ------------------------------------------------------------------------------------------------ the join for bf16, 128 channels
constexpr int kTcWarps = 4;
constexpr int kMaxJoin = 8;  // thread blocks of a cluster

__device__ __forceinline__ void mma_bf16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t a) {  // an 8 x 8 matrix of 16-bit elements held by the warp
    uint32_t d;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
    return d;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 x = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&x);
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t peer_addr(const void* p, int rank) {
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ float4 peer_load4(uint32_t addr) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ float peer_load(uint32_t addr) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}

// grid (blocks of a cluster, Hkv, batch).  The tail on mma.sync, fragments straight from memory, sixteen tokens per warp and step:
//   S[token][head] = K q^T     the sums over channels are in an order of the fragments' own, the same for K and q, so that a lane's 16
//                              bytes of a row are two steps' fragments
//   O^T[channel][head] += V^T P^T   a lane has eight channels of four tokens; a product's rows are channels eight apart
// Up to four heads per group fill columns 0-3, columns 4-7 carry the remainder of P's rounding to bf16; eight heads take a second
// product for it, so that P acts with 16 bits.  Blocks of a cluster share a unit's tail and parts (small batches, long tails).
// Bound by memory and the loads on their way: 64 sequences of 200 tokens are 52 MB of tails, 10 us of a call (8 at the copy rate), of 1 000 262 MB, 50 us; for small
// batches by the chain parts -> sums -> outputs behind the prompt kernel, with ten parts on their way at a time.
// A prompt block fills its SM, so that where there is one on every SM no block of this kernel runs before a prompt block has left: the tails' bytes come behind the prompt's.
// BLOCKS: on an SM at least.  Three keep all of a warp's registers; four (128 registers, 28 to 44 bytes spilled), for more blocks than three have room for, keep more tail rows on their way
// (32 768 and 2 048 tokens, 64 sequences of 200 tail tokens: 67.1 -> 64.8 and 27.3 -> 22.8 us; 32 sequences, which three hold, 17.3 and 19.7).
template <int G, int NB, int BLOCKS>
__global__ void __launch_bounds__(kTcWarps * 32, BLOCKS) shared_join_tc_kernel(SharedArgs a, const __grid_constant__ SharedSched sch, const __grid_constant__ SharedSeqs<NB> sq) {
    constexpr int D = 128, ITEMS = G * D / 4, THREADS = kTcWarps * 32;
    constexpr bool SPLIT = G <= 4;
    __shared__ __align__(16) float s_acc[kTcWarps][G][D];
    __shared__ float s_m[kTcWarps][G], s_l[kTcWarps][G];
    __shared__ float4 j_acc[THREADS];
    __shared__ float2 j_ml[THREADS];
    const int rank = blockIdx.x, ranks = (int)gridDim.x, h = blockIdx.y, b = blockIdx.z;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, gid = lane >> 2, tig = lane & 3;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int n = sq.len[b], slot = sq.slot[b];
    const int64_t tail0 = ((int64_t)slot * a.Hkv + h) * a.tail_rows * D;
    __nv_bfloat16* const tk = reinterpret_cast<__nv_bfloat16*>(a.tail_k) + tail0;
    __nv_bfloat16* const tv = reinterpret_cast<__nv_bfloat16*>(a.tail_v) + tail0;
    const int64_t new0 = ((int64_t)b * a.Hkv + h) * D;
    const __nv_bfloat16* const kn = a.k_new ? reinterpret_cast<const __nv_bfloat16*>(a.k_new) + new0 : nullptr;
    const __nv_bfloat16* const vn = a.k_new ? reinterpret_cast<const __nv_bfloat16*>(a.v_new) + new0 : nullptr;

    const int group = b * G / sch.row_tile, r0 = b * G - group * sch.row_tile;  // (row tiles hold whole sequences)
    int c_lo, c_hi;
    ranges_of_head(sch, h, c_lo, c_hi);

    float o[8][4], m[2] = {-INFINITY, -INFINITY}, l[2] = {0.f, 0.f};
#pragma unroll
    for (int j = 0; j < 8; ++j) o[j][0] = o[j][1] = o[j][2] = o[j][3] = 0.f;
    const int first = (rank * kTcWarps + warp) * 16, step = ranks * kTcWarps * 16;
    if (first < n) {
        const int qcol = SPLIT ? gid & 3 : gid;
        uint4 q[4];
#pragma unroll
        for (int k = 0; k < 4; ++k)
            q[k] = qcol < G ? __ldcg(reinterpret_cast<const uint4*>(reinterpret_cast<const __nv_bfloat16*>(a.q) + ((int64_t)b * a.Hq + h * G + qcol) * D + 32 * k + 8 * tig))
                            : make_uint4(0u, 0u, 0u, 0u);
        const float ks = 0.08838834764831845f * 1.4426950408889634f;  // / sqrt(128), in powers of two
#pragma unroll 1
        for (int t0 = first; t0 < n; t0 += step) {
            // (rows behind the last are read as the last and masked; the appended one comes from the caller)
            uint4 k[2][4], v[4][2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int t = min(t0 + gid + 8 * i, n - 1);
                const __nv_bfloat16* const p = (kn && t == n - 1 ? kn : tk + (int64_t)t * D) + 8 * tig;
#pragma unroll
                for (int c = 0; c < 4; ++c) k[i][c] = __ldcg(reinterpret_cast<const uint4*>(p + 32 * c));
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int t = min(t0 + 2 * tig + (i & 1) + 8 * (i >> 1), n - 1);
                const __nv_bfloat16* const p = (kn && t == n - 1 ? vn : tv + (int64_t)t * D) + 8 * gid;
                v[i][0] = __ldcg(reinterpret_cast<const uint4*>(p));
                v[i][1] = __ldcg(reinterpret_cast<const uint4*>(p + 64));
            }
            // The next step's rows, one a lane, on their way to L2 (64 sequences of 1 000 own tokens: 82.9 -> 62.0 us; two steps ahead 67.5, both
            // 69.8; of 200, 22.6 -> 23.5 behind 2 048 tokens and 64.6 -> 62.4 behind 32 768: asked for in either case, since the tail's length does not tell these apart).
            if (t0 + step < n) {
                const int t = t0 + step + (lane & 15);
                if (t < n) {
                    const __nv_bfloat16* const p = (lane < 16 ? tk : tv) + (int64_t)t * D;
                    asm volatile("prefetch.global.L2 [%0];\n\tprefetch.global.L2 [%0 + 128];" ::"l"(p));
                }
            }
            float s[2][4] = {};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                mma_bf16(s[0], k[0][c].x, k[1][c].x, k[0][c].y, k[1][c].y, q[c].x, q[c].y);
                mma_bf16(s[1], k[0][c].z, k[1][c].z, k[0][c].w, k[1][c].w, q[c].z, q[c].w);
            }
            float p[2][2], mt[2];
#pragma unroll
            for (int e = 0; e < 2; ++e) {
#pragma unroll
                for (int i = 0; i < 2; ++i) p[i][e] = t0 + gid + 8 * i < n ? __fmul_rn(s[0][2 * i + e] + s[1][2 * i + e], ks) : -INFINITY;
                mt[e] = fmaxf(p[0][e], p[1][e]);
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) mt[e] = fmaxf(mt[e], __shfl_xor_sync(0xFFFFFFFFu, mt[e], x));
                const float mn = fmaxf(fmaxf(m[e], mt[e]), -1e38f), f = ex2(m[e] - mn);  // (finite where every key so far is infinitely far off, and below all finite scores)
                m[e] = mn;
                l[e] *= f;
#pragma unroll
                for (int j = 0; j < 8; ++j) { o[j][e] *= f; o[j][2 + e] *= f; }
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    p[i][e] = ex2(p[i][e] - mn);
                    l[e] += p[i][e];
                }
            }
            uint32_t ph[2], pl[2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const float h0 = __bfloat162float(__float2bfloat16_rn(p[i][0])), h1 = __bfloat162float(__float2bfloat16_rn(p[i][1]));
                const uint32_t lo = pack2(p[i][0] - h0, p[i][1] - h1), hi = pack2(h0, h1);
                ph[i] = transposed(SPLIT && tig >= 2 ? lo : hi);
                if constexpr (!SPLIT) pl[i] = transposed(lo);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                uint32_t x[4][2];
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int c = 0; c < 2; ++c) x[i][c] = j < 2 ? v[i][c].x : j < 4 ? v[i][c].y : j < 6 ? v[i][c].z : v[i][c].w;
                const uint32_t sel = j & 1 ? 0x7632 : 0x5410;
                const uint32_t a0 = __byte_perm(x[0][0], x[1][0], sel), a1 = __byte_perm(x[0][1], x[1][1], sel), a2 = __byte_perm(x[2][0], x[3][0], sel),
                               a3 = __byte_perm(x[2][1], x[3][1], sel);
                mma_bf16(o[j], a0, a1, a2, a3, ph[0], ph[1]);
                if constexpr (!SPLIT) mma_bf16(o[j], a0, a1, a2, a3, pl[0], pl[1]);
            }
        }
    }
    if (kn && rank == 0 && warp == 0) {  // the new row joins the tail for later calls: lanes 0-15 K, lanes 16-31 V
        const int c = lane & 15;
        reinterpret_cast<uint4*>((lane < 16 ? tk : tv) + (int64_t)(n - 1) * D)[c] = __ldcg(reinterpret_cast<const uint4*>(lane < 16 ? kn : vn) + c);
        if (lane == 0 && h == 0) a.tail_len[slot] = n;
    }
    // ---- the warps' states: lane (gid, tig) has channels 8 gid .. and 64 + 8 gid .. of columns 2 tig and 2 tig + 1 ----
#pragma unroll
    for (int e = 0; e < 2; ++e) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[e] += __shfl_xor_sync(0xFFFFFFFFu, l[e], x);
        float w[16];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            w[j] = o[j][e];
            w[8 + j] = o[j][2 + e];
            if (SPLIT) {
                w[j] += __shfl_xor_sync(0xFFFFFFFFu, w[j], 2);
                w[8 + j] += __shfl_xor_sync(0xFFFFFFFFu, w[8 + j], 2);
            }
        }
        const int g = 2 * tig + e;
        if (g < G) {
#pragma unroll
            for (int j = 0; j < 16; j += 4) *reinterpret_cast<float4*>(&s_acc[warp][g][(j >> 3) * 64 + 8 * gid + (j & 7)]) = make_float4(w[j], w[j + 1], w[j + 2], w[j + 3]);
            if (gid == 0) {
                s_m[warp][g] = m[e] * 0.6931471805599453f;  // natural logarithms from here on
                s_l[warp][g] = l[e];
            }
        }
    }
    // ---- fours of outputs: this block's share of the unit's, each over as many threads as there are; first the tail's states, those of the
    // cluster's other blocks among them, then, when it is there, the prompt ----
    const int share = ITEMS / ranks, ways = share < THREADS ? THREADS / share : 1;
    if (ranks > 1) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    else __syncthreads();
    const int64_t part = shared_part_floats(sch.row_tile, D), stride = sch.groups * part;
    const float* const p0 = a.partials + h * stride + group * part;
    constexpr int ROUNDS = ITEMS > THREADS ? ITEMS / THREADS : 1;  // (more than one: ranks == 1 or a share that still is one)
    State4 s[ROUNDS];
    const int way = threadIdx.x / share;
#pragma unroll
    for (int round = 0; round < ROUNDS; ++round) {
        const int k = (int)threadIdx.x % share + round * THREADS, i = rank * share + k, g = i % G, c4 = i / G;
        if (k < share)
            for (int e = way; e < kTcWarps * ranks; e += ways) {
                const int w = e % kTcWarps, c = e / kTcWarps;
                if (ranks == 1) {
                    s[round].add(s_m[w][g], s_l[w][g], *reinterpret_cast<const float4*>(&s_acc[w][g][c4 * 4]));
                } else {
                    s[round].add(peer_load(peer_addr(&s_m[w][g], c)), peer_load(peer_addr(&s_l[w][g], c)), peer_load4(peer_addr(&s_acc[w][g][c4 * 4], c)));
                }
            }
    }
    if (ranks > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");  // (the peers' states have been read; awaited at the end)
    asm volatile("griddepcontrol.wait;" ::: "memory");  // the prompt's parts
#pragma unroll
    for (int round = 0; round < ROUNDS; ++round) {
        if (round > 0 && share <= THREADS) break;
        const int k = (int)threadIdx.x % share + round * THREADS, i = rank * share + k, g = i % G, c4 = i / G;
        if (k < share) s[round].add_parts<D, 10>(p0, stride, sch.row_tile, r0 + g, c4, c_lo + way, c_hi, ways);
        if (ways > 1) {  // (one round)
            j_acc[threadIdx.x] = s[round].a;
            j_ml[threadIdx.x] = make_float2(s[round].m, s[round].l);
            __syncthreads();
            if (way == 0)
                for (int w = 1; w < ways; ++w) s[round].add(j_ml[w * share + k].x, j_ml[w * share + k].y, j_acc[w * share + k]);
        }
        if (way == 0 && k < share) s[round].store(a.out, a.out_dtype, ((int64_t)b * a.Hq + h * G + g) * D + c4 * 4);
    }
    if (ranks > 1) asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}

cudaLaunchConfig_t config(dim3 grid, int threads, size_t smem, cudaStream_t st, cudaLaunchAttribute* attr) {
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cfg;
}

template <int NB>
SharedSeqs<NB> seqs_of(const SharedArgs& a) {
    SharedSeqs<NB> sq;
    for (int b = 0; b < a.batch; ++b) {
        sq.slot[b] = a.seqs[b];
        sq.len[b] = a.lens[b];
    }
    return sq;
}
template <typename T, int D, int NB>
cudaError_t launch_join(const SharedArgs& a, const SharedSched& sch, cudaStream_t st) {
    cudaLaunchAttribute attr[1];
    cudaLaunchConfig_t cfg = config(dim3(a.Hkv, a.batch), kJoinWarps * 32, 0, st, attr);
    const SharedSeqs<NB> sq = seqs_of<NB>(a);
    switch (a.G) {
        case 1: return cudaLaunchKernelEx(&cfg, shared_join_kernel<T, D, 1, NB>, a, sch, sq);
        case 2: return cudaLaunchKernelEx(&cfg, shared_join_kernel<T, D, 2, NB>, a, sch, sq);
        case 4: return cudaLaunchKernelEx(&cfg, shared_join_kernel<T, D, 4, NB>, a, sch, sq);
        case 8: return cudaLaunchKernelEx(&cfg, shared_join_kernel<T, D, 8, NB>, a, sch, sq);
        default: return cudaErrorInvalidValue;
    }
}
template <typename T, int D>
cudaError_t launch_join(const SharedArgs& a, const SharedSched& sch, cudaStream_t st) {
    return a.batch <= kSharedFew ? launch_join<T, D, kSharedFew>(a, sch, st) : launch_join<T, D, kMaxShared>(a, sch, st);
}
template <int NB, int BLOCKS>
cudaError_t launch_join_tc(const cudaLaunchConfig_t& cfg, const SharedArgs& a, const SharedSched& sch, const SharedSeqs<NB>& sq) {
    switch (a.G) {
        case 1: return cudaLaunchKernelEx(&cfg, shared_join_tc_kernel<1, NB, BLOCKS>, a, sch, sq);
        case 2: return cudaLaunchKernelEx(&cfg, shared_join_tc_kernel<2, NB, BLOCKS>, a, sch, sq);
        case 4: return cudaLaunchKernelEx(&cfg, shared_join_tc_kernel<4, NB, BLOCKS>, a, sch, sq);
        case 8: return cudaLaunchKernelEx(&cfg, shared_join_tc_kernel<8, NB, BLOCKS>, a, sch, sq);
        default: return cudaErrorInvalidValue;
    }
}
template <int NB>
cudaError_t launch_join_tc(const SharedArgs& a, const SharedSched& sch, int sms, cudaStream_t st) {
    // blocks per unit: more than one while they leave half of the device idle and have parts or tail tokens for each
    int longest = 0;
    for (int b = 0; b < a.batch; ++b) longest = std::max(longest, a.lens[b]);
    const int parts = std::max(1, sch.ranges / a.Hkv);
    int ranks = 1;
    while (ranks < kMaxJoin && a.Hkv * a.batch * ranks <= sms && (parts >= 8 * ranks || longest >= 128 * ranks)) ranks *= 2;
    cudaLaunchAttribute attr[2];
    cudaLaunchConfig_t cfg = config(dim3(ranks, a.Hkv, a.batch), kTcWarps * 32, 0, st, attr);
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = ranks;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cfg.numAttrs = ranks > 1 ? 2 : 1;
    const SharedSeqs<NB> sq = seqs_of<NB>(a);
    return a.Hkv * a.batch * ranks > 3 * sms ? launch_join_tc<NB, 4>(cfg, a, sch, sq) : launch_join_tc<NB, 3>(cfg, a, sch, sq);
}

template <typename T, int D>
cudaError_t launch_part(const SharedArgs& a, const SharedSched& sch, cudaStream_t st) {
    static PerDevice once;
    const cudaError_t e = once.ensure([]() { return cudaFuncSetAttribute(shared_part_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, part_smem<D>()); });
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr[1];
    cudaLaunchConfig_t cfg = config(dim3(sch.ranges * sch.groups), kThreads, part_smem<D>(), st, attr);
    return cudaLaunchKernelEx(&cfg, shared_part_kernel<T, D>, a, sch);
}

}  // namespace

// us per tile of 128 tokens: with entries (one or more row groups, and per kept fraction), without them when memory bounds all blocks (one or more row groups), and when it does
// not.  Swept with half of the heads' tiles and more in each mode; us a call for equal tiles, 1.75, 1.9 and 2.1: 128k (1/32 kept, 16 sequences) 119.9, 108.1, 101.7 and 100.7, 32k
// (1/16, eight) 38.1, 33.4, 32.9 and 32.1, (1/8) 45.6, 37.6, 36.1 and 35.6; two row groups, 32k: 69.1, 62.0, 63.3 and 65.8.
static constexpr double kSlowTile = 2.1, kSlowGroupTile = 1.75, kSlowKept = 4.4, kMeanTile = 1.62, kGroupTile = 1.15, kFastTile = 1.0;
// Whole tiles to the ranges, as evenly as their costs go.
cudaError_t plan_shared_decode(const SharedArgs& a, int row_tile, int tile, int sms, SharedSched& sch) {
    const int R = a.batch * a.G;
    sms = std::min(sms, kMaxSplits);  // (what the partial sums have room for)
    sch.row_tile = std::min(row_tile, R);
    sch.groups = (R + row_tile - 1) / row_tile;
    sch.tiles = (a.T + tile - 1) / tile;
    const int64_t total = (int64_t)a.Hkv * sch.tiles;
    if (total >= (int64_t)1 << 31) return cudaErrorInvalidValue;
    // as many ranges as make one round of blocks, or, where one would leave SMs idle (more than 37 groups), two or three
    int ranges = 1;
    double best = 0.0;
    for (int rounds = 1; rounds <= 3; ++rounds) {
        const int n = std::min(rounds * sms / sch.groups, kMaxSplits);
        const double used = n ? (double)n * sch.groups / (((n * sch.groups + sms - 1) / sms) * sms) : 0.0;
        if (used > best + 0.1) {
            best = used;
            ranges = n;
        }
    }
    sch.ranges = (int)std::min<int64_t>(ranges, total);
    // A block takes `slow` us for a tile with entries, whatever the others do, and for one without as long as the memory needs on average, or
    // less where blocks that are slower leave it room: that share of the time is what the others then take.
    int n_slow = 0;
    for (int h = 0; h < a.Hkv; ++h) n_slow += a.modes[h] == FDKV_MODE_RESIDUAL;
    const double f = (double)n_slow / a.Hkv, slow = (sch.groups > 1 ? kSlowGroupTile : kSlowTile) + kSlowKept * a.keep, mean = sch.groups > 1 ? kGroupTile : kMeanTile;
    const double plain = n_slow < a.Hkv ? std::max(kFastTile, (mean - f * slow) / (1.0 - f)) : mean;
    const double resid = tile == kSharedTile ? slow / plain : 1.0;  // (the portable kernel's blocks have a tile or two)
    double cost = 0.0;
    for (int h = 0; h < a.Hkv; ++h) cost += sch.tiles * (a.modes[h] == FDKV_MODE_RESIDUAL ? resid : 1.0);
    int h = 0;
    double before = 0.0;  // cost of the heads before h
    sch.start[0] = 0;
    for (int c = 1; c < sch.ranges; ++c) {
        const double at = cost * c / sch.ranges;
        double w = a.modes[h] == FDKV_MODE_RESIDUAL ? resid : 1.0;
        while (h + 1 < a.Hkv && at >= before + sch.tiles * w) {
            before += sch.tiles * w;
            w = a.modes[++h] == FDKV_MODE_RESIDUAL ? resid : 1.0;
        }
        const int64_t cut = (int64_t)h * sch.tiles + std::min<int64_t>(sch.tiles, (int64_t)((at - before) / w + 0.5));
        sch.start[c] = (int)std::min<int64_t>(std::max<int64_t>(cut, sch.start[c - 1] + 1), total - (sch.ranges - c));
    }
    sch.start[sch.ranges] = (int)total;
    const int64_t parts = ((int64_t)sch.ranges + a.Hkv - 1) * sch.groups;
    return parts * shared_part_floats(sch.row_tile, a.d) <= a.partial_floats ? cudaSuccess : cudaErrorInvalidValue;
}

cudaError_t launch_shared_decode(const SharedArgs& a, int dtype, cudaStream_t st) {
    static PerDevice once;
    int sms = 0;
    cudaError_t e = once.ensure([]() { return cudaSuccess; }, &sms);
    if (e != cudaSuccess) return e;
    SharedSched sch;
    const bool tc = a.tmap != nullptr;
    if ((e = (tc ? plan_shared_decode(a, kSharedRows, kSharedTile, sms, sch) : plan_shared_decode(a, kRows, kTok, sms, sch))) != cudaSuccess) return e;
    if (tc) {
        e = launch_shared_tc(a, sch, st);
        if (e == cudaSuccess) e = a.batch <= kSharedFew ? launch_join_tc<kSharedFew>(a, sch, sms, st) : launch_join_tc<kMaxShared>(a, sch, sms, st);
    } else if (dtype == FDKV_BF16) {
        if (a.d == 128) return cudaErrorNotSupported;  // (no tensor map of the arena)
        e = launch_part<__nv_bfloat16, 64>(a, sch, st);
        if (e == cudaSuccess) e = launch_join<__nv_bfloat16, 64>(a, sch, st);
    } else {
        e = a.d == 128 ? launch_part<float, 128>(a, sch, st) : launch_part<float, 64>(a, sch, st);
        if (e == cudaSuccess) e = a.d == 128 ? launch_join<float, 128>(a, sch, st) : launch_join<float, 64>(a, sch, st);
    }
    if (e != cudaSuccess) return e;
    count_launch(2);
    count_kernel(tc ? FDKV_KERNEL_SHARED_TC : FDKV_KERNEL_SHARED_PORTABLE);
    return cudaGetLastError();
}

}  // namespace fdkv
