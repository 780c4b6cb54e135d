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
constexpr int kTok = 32;       // tokens at a time
constexpr int kThreads = 256;

template <int D>
constexpr int part_smem() { return (kRows * (D + 4) + 2 * kTok * (D + 4) + kRows * (kTok + 1) + 3 * kRows) * 4; }

// Tiles of kTok tokens are reconstructed into shared memory as float32 (rows, plus the sign times the scattered residual entries;
// the unit's scale is applied to the logits and the outputs) and multiplied with the group's query rows: a thread has two rows x
// two tokens of the logits and 2 x D / 16 of the outputs.  float32 FMA; for float32 storage eight channels' products at a time
// are added up in float64, since the exponential magnifies the rounding of logits of a few tens.
template <typename T, int D>
__global__ void __launch_bounds__(kThreads) shared_part_kernel(SharedArgs a, const __grid_constant__ SharedSched sch) {
    using ACC = typename std::conditional<sizeof(T) == 4, double, float>::type;
    extern __shared__ __align__(16) float smem[];
    constexpr int P = D + 4;  // row pitch: neighbouring rows lie four banks apart
    float* const sq = smem;
    float* const sk = sq + kRows * P;
    float* const sv = sk + kTok * P;
    float* const sp = sv + kTok * P;             // [kRows][kTok + 1]
    float* const sm = sp + kRows * (kTok + 1);   // maxima, sums, factors
    float* const sl = sm + kRows;
    float* const sf = sl + kRows;
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;  // rows ty, ty + 16; tokens tx, tx + 16; channels 4 tx + 64 i
    asm volatile("griddepcontrol.wait;" ::: "memory");  // q belongs to the kernels ahead
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (behind the wait: the join reads the tails before its own)
    const int R = a.batch * a.G;
    int g0 = sch.start[blockIdx.x];
    const int g1 = sch.start[blockIdx.x + 1];
    while (g0 < g1) {
        const int u = g0 / sch.tiles, t_first = g0 % sch.tiles, t_last = min(sch.tiles, t_first + g1 - g0);
        g0 += t_last - t_first;
        const int h = u / sch.groups, row0 = (u % sch.groups) * kRows, rows = min(kRows, R - row0);
        const UnitDesc ud = a.desc[h];
        const bool resid = ud.mode == FDKV_MODE_RESIDUAL;
        const float kscale = ud.scale * rsqrtf((float)D), sign = ud.sign;
        __syncthreads();
        for (int i = tid; i < kRows * D / 8; i += kThreads) {
            const int r = i / (D / 8), c = i % (D / 8) * 8;
            float f[8] = {};
            if (r < rows) {
                const int row = row0 + r, b = row / a.G, g = row % a.G;
                load8(reinterpret_cast<const T*>(a.q) + ((int64_t)b * a.Hq + h * a.G + g) * D + c, f);
            }
#pragma unroll
            for (int j = 0; j < 8; ++j) sq[r * P + c + j] = f[j];
        }
        if (tid < kRows) { sm[tid] = -INFINITY; sl[tid] = 0.f; }
        float o[2][D / 16];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < D / 16; ++j) o[i][j] = 0.f;
        const int tok_end = min(ud.T, t_last * kSharedTile);
        for (int tok = t_first * kSharedTile; tok < tok_end; tok += kTok) {
            const int n = min(kTok, tok_end - tok);
            __syncthreads();
            for (int i = tid; i < 2 * kTok * D / 8; i += kThreads) {
                const bool is_v = i >= kTok * D / 8;
                const int j = is_v ? i - kTok * D / 8 : i, t = j / (D / 8), c = j % (D / 8) * 8;
                float f[8] = {};
                if (t < n) load8(reinterpret_cast<const T*>(is_v ? ud.v_rows : ud.k_rows) + (int64_t)(tok + t) * D + c, f);
                float* const to = (is_v ? sv : sk) + t * P + c;
#pragma unroll
                for (int x = 0; x < 8; ++x) to[x] = f[x];
            }
            __syncthreads();
            if (resid) {  // (every position is in a list once: no two threads add to the same place)
                const int s0 = tok / kResTile, s1 = (tok + n + kResTile - 1) / kResTile;
                for (int is_v = 0; is_v < 2; ++is_v) {
                    const int32_t* const off = is_v && ud.v_off ? ud.v_off : ud.k_off;
                    const int32_t* const idx = is_v && ud.v_idx ? ud.v_idx : ud.k_idx;
                    const T* const val = reinterpret_cast<const T*>(is_v ? ud.v_val : ud.k_val);
                    float* const to = is_v ? sv : sk;
                    const int e0 = off[s0], e1 = off[s1];
                    if (ud.res_kind == 1) {  // whole rows of selected tokens
                        for (int i = e0 * D + tid; i < e1 * D; i += kThreads) to[(idx[i / D] - tok) * P + i % D] += sign * ldf<T>(val + i);
                    } else {
                        for (int e = e0 + tid; e < e1; e += kThreads) {
                            const int at = idx[e] - tok * D;
                            to[at / D * P + at % D] += sign * ldf<T>(val + e);
                        }
                    }
                }
                __syncthreads();
            }
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
        float* const part = a.partials + (int64_t)(blockIdx.x + u) * shared_part_floats(sch.row_tile, D);
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

constexpr int kJoinWarps = 8;

// grid (Hkv, batch).  D / 8 lanes share a tail token, eight channels each; every such lane group keeps a softmax state of its own,
// joined through shared memory with the prompt's parts.  The tails, q and the new rows are read before the dependency wait: the
// prompt kernel lets this one start only behind its own, when all they come from is complete.
template <typename T, int D, int G, int NB>
__global__ void __launch_bounds__(kJoinWarps * 32) shared_join_kernel(SharedArgs a, const __grid_constant__ SharedSched sch, const __grid_constant__ SharedSeqs<NB> sq) {
    using ACC = typename std::conditional<sizeof(T) == 4, double, float>::type;
    constexpr int LPT = D / 8, TPI = 32 / LPT, U = sizeof(T) == 4 || G == 8 ? 2 : 4;
    __shared__ __align__(16) float s_acc[kJoinWarps][G][D];
    __shared__ float s_m[kJoinWarps][G], s_l[kJoinWarps][G];
    constexpr int JW = kJoinWarps * 32 / (G * D / 4) > 1 ? kJoinWarps * 32 / (G * D / 4) - 1 : 1;
    __shared__ float4 j_acc[JW][G * D / 4];
    __shared__ float2 j_ml[JW][G * D / 4];
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
    // ---- the blocks whose ranges meet the item of the unit's rows (row tiles hold whole sequences) ----
    const int row0 = b * G, u = h * sch.groups + row0 / sch.row_tile, r0 = row0 % sch.row_tile;
    int c_lo = 0;
    for (int step = 128; step; step >>= 1)
        if (c_lo + step < sch.ncta && sch.start[c_lo + step] <= u * sch.tiles) c_lo += step;
    int c_hi = c_lo;  // the last block that starts before the item's end
    for (int step = 128; step; step >>= 1)
        if (c_hi + step < sch.ncta && sch.start[c_hi + step] < (u + 1) * sch.tiles) c_hi += step;
    __syncthreads();
    asm volatile("griddepcontrol.wait;" ::: "memory");  // the prompt's parts
    // ---- four channels of a head per thread, the parts spread over as many threads as there are: six at a time on their way ----
    constexpr int ITEMS = G * D / 4, WAYS = kJoinWarps * 32 / ITEMS > 0 ? kJoinWarps * 32 / ITEMS : 1, BATCH = 6;
    for (int i0 = 0; i0 < ITEMS * WAYS; i0 += kJoinWarps * 32) {
        const int i = (i0 + (int)threadIdx.x) % ITEMS, way = (i0 + (int)threadIdx.x) / ITEMS, g = i % G, c4 = i / G;
        float M = -INFINITY, L = 0.f;
        float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i0 + (int)threadIdx.x < ITEMS * WAYS) {
            const int64_t stride = shared_part_floats(sch.row_tile, D);
            const float* const p0 = a.partials + u * stride;
            for (int c = c_lo + way; c <= c_hi; c += BATCH * WAYS) {
                float pm[BATCH], pl[BATCH];
                float4 po[BATCH];
#pragma unroll
                for (int k = 0; k < BATCH; ++k) {
                    const int cc = c + k * WAYS;
                    const float* const part = p0 + (cc <= c_hi ? cc : c) * stride;
                    pm[k] = cc <= c_hi ? __ldcg(part + (int64_t)sch.row_tile * D + r0 + g) : -INFINITY;
                    pl[k] = __ldcg(part + (int64_t)sch.row_tile * (D + 1) + r0 + g);
                    po[k] = __ldcg(reinterpret_cast<const float4*>(part + ((int64_t)c4 * sch.row_tile + r0 + g) * 4));
                }
                float mn = M;
#pragma unroll
                for (int k = 0; k < BATCH; ++k) mn = fmaxf(mn, pm[k]);
                const float ref = mn == -INFINITY ? 0.f : mn, f0 = __expf(M - ref);
                L *= f0;
                A.x *= f0; A.y *= f0; A.z *= f0; A.w *= f0;
#pragma unroll
                for (int k = 0; k < BATCH; ++k) {
                    const float f = __expf(pm[k] - ref);
                    L = fmaf(pl[k], f, L);
                    A.x = fmaf(po[k].x, f, A.x); A.y = fmaf(po[k].y, f, A.y); A.z = fmaf(po[k].z, f, A.z); A.w = fmaf(po[k].w, f, A.w);
                }
                M = mn;
            }
        }
        auto add = [&](float pm, float pl, const float4& o) {
            const float mn = fmaxf(M, pm), ref = mn == -INFINITY ? 0.f : mn, f0 = __expf(M - ref), f1 = __expf(pm - ref);
            L = L * f0 + pl * f1;
            A.x = A.x * f0 + o.x * f1; A.y = A.y * f0 + o.y * f1; A.z = A.z * f0 + o.z * f1; A.w = A.w * f0 + o.w * f1;
            M = mn;
        };
        if constexpr (WAYS > 1) {  // (one round: every thread has at most one item)
            if (way > 0 && way < WAYS) {
                j_acc[way - 1][i] = A;
                j_ml[way - 1][i] = make_float2(M, L);
            }
            __syncthreads();
            if (way > 0) return;
#pragma unroll
            for (int w = 1; w < WAYS; ++w) add(j_ml[w - 1][i].x, j_ml[w - 1][i].y, j_acc[w - 1][i]);
        }
        if (i0 + (int)threadIdx.x >= ITEMS * WAYS) return;
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) add(s_m[w][g], s_l[w][g], *reinterpret_cast<const float4*>(&s_acc[w][g][c4 * 4]));
        const float inv = L > 0.f ? 1.f / L : 0.f;
        const int64_t o = ((int64_t)b * a.Hq + h * G + g) * D + c4 * 4;
        if (a.out_dtype == FDKV_BF16) {
            const __nv_bfloat162 x = __floats2bfloat162_rn(A.x * inv, A.y * inv), y = __floats2bfloat162_rn(A.z * inv, A.w * inv);
            *reinterpret_cast<uint2*>(reinterpret_cast<__nv_bfloat16*>(a.out) + o) = make_uint2(*reinterpret_cast<const uint32_t*>(&x), *reinterpret_cast<const uint32_t*>(&y));
        } else {
            *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + o) = make_float4(A.x * inv, A.y * inv, A.z * inv, A.w * inv);
        }
    }
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

template <typename T, int D, int NB>
cudaError_t launch_join(const SharedArgs& a, const SharedSched& sch, cudaStream_t st) {
    cudaLaunchAttribute attr[1];
    cudaLaunchConfig_t cfg = config(dim3(a.Hkv, a.batch), kJoinWarps * 32, 0, st, attr);
    SharedSeqs<NB> sq;
    for (int b = 0; b < a.batch; ++b) {
        sq.slot[b] = a.seqs[b];
        sq.len[b] = a.lens[b];
    }
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

template <typename T, int D>
cudaError_t launch_part(const SharedArgs& a, const SharedSched& sch, cudaStream_t st) {
    static PerDevice once;
    const cudaError_t e = once.ensure([]() { return cudaFuncSetAttribute(shared_part_kernel<T, D>, cudaFuncAttributeMaxDynamicSharedMemorySize, part_smem<D>()); });
    if (e != cudaSuccess) return e;
    cudaLaunchAttribute attr[1];
    cudaLaunchConfig_t cfg = config(dim3(sch.ncta), kThreads, part_smem<D>(), st, attr);
    return cudaLaunchKernelEx(&cfg, shared_part_kernel<T, D>, a, sch);
}

// Whole tiles to the blocks, as evenly as they go.
cudaError_t plan_shared(const SharedArgs& a, int row_tile, int sms, SharedSched& sch) {
    const int R = a.batch * a.G;
    sch.row_tile = std::min(row_tile, R);
    sch.groups = (R + row_tile - 1) / row_tile;
    sch.tiles = (a.T + kSharedTile - 1) / kSharedTile;
    const int64_t total = (int64_t)a.Hkv * sch.groups * sch.tiles;
    if (total >= (int64_t)1 << 31) return cudaErrorInvalidValue;
    sch.ncta = (int)std::min<int64_t>(std::min(sms, kMaxSplits), total);
    for (int c = 0; c <= sch.ncta; ++c) sch.start[c] = (int)(total * c / sch.ncta);
    const int64_t parts = sch.ncta + (int64_t)a.Hkv * sch.groups - 1;
    return parts * shared_part_floats(sch.row_tile, a.d) <= a.partial_floats ? cudaSuccess : cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_shared_decode(const SharedArgs& a, int dtype, cudaStream_t st) {
    static PerDevice once;
    int sms = 0;
    cudaError_t e = once.ensure([]() { return cudaSuccess; }, &sms);
    if (e != cudaSuccess) return e;
    SharedSched sch;
    const bool tc = a.tmap != nullptr;
    if ((e = plan_shared(a, tc ? 128 : kRows, sms, sch)) != cudaSuccess) return e;
    if (tc) {
        e = launch_shared_tc(a, sch, st);
        if (e == cudaSuccess) e = launch_join<__nv_bfloat16, 128>(a, sch, st);
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
