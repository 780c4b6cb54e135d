// The prompt part of decode attention on one shared prompt, bf16 / head_dim 128 (see shared_prefix.cu): the query rows of all
// sequences of a KV head fill the rows of tcgen05 products, so that a tile of the compressed prompt is read once and used by up to 128 rows.
//
// A persistent block of ten warps per SM walks a range of the flat (KV head, row group, 128-token tile) list:
//   warp 8     TMA producer: the tile's K and V rows (2 x 64 channels x 128 tokens, 128-byte swizzle)
//   warps 4-7  residual units: the tile's kept entries, scattered into a zeroed tile of the same layout (32 tokens per warp)
//   warp 9     issues S = Q K^T (Q from tensor memory, K-major K) and O += P V (P from tensor memory, MN-major V).  Residual units add
//              the products with the entries' tiles into the same accumulators, so that the correction is exact in float32
//   warps 0-3  softmax: thread = query row.  S is read from tensor memory, P = exp2(S - max) rounded to bf16 takes its place; the
//              running maximum only moves, and O is only rescaled, where a score passes it by more than 2^8
// All tiles, rows and entries alike, go through one ring of 32 KiB slots in the order in which the products use them: K of the next
// tile lies before V of this one, so that the next S is formed while the softmax of this one runs (S has two accumulators).
// P in bf16: a probability is off by 2^-8 at most, each its own way; the sums l are those of the unrounded ones.
#include <cuda.h>

#include "fdkv_internal.h"
#include "umma.cuh"

namespace fdkv {

namespace {

constexpr int kThreads = 320;
constexpr int kSlots = 7, kSlotBytes = 32768, kHalf = 16384;
constexpr int kHeader = 1024;
constexpr int kSmem = kHeader + kSlots * kSlotBytes;
static_assert(kSmem <= 227 * 1024, "shared memory budget");
// header
constexpr int oFull = 0, oEmpty = 64, oS = 128, oP = 144, oO = 160, oQ = 176, oAbort = 184, oTmem = 188;
// tensor memory columns
constexpr uint32_t cS = 0, cO = 256, cQ = 384;
constexpr uint32_t kIdescS = umma_idesc(128, 128, false), kIdescO = umma_idesc(128, 128, false) | (1u << 16);  // (B of the second product is MN-major)

// D[tmem] (+)= A[tmem] * B[smem]
template <uint32_t IDESC>
__device__ __forceinline__ void umma_ts(uint32_t tmem_d, uint32_t tmem_a, uint64_t db, uint32_t acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(tmem_d),
        "r"(tmem_a), "l"(db), "n"(IDESC), "r"(acc)
        : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t x;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(x));
    return x != 0;
}
// All lanes wait for a barrier's phase; false when the block has given up.
__device__ __forceinline__ bool wait_warp(uint32_t bar, uint32_t parity, volatile uint32_t* abort_flag, int32_t* status) {
    if (__all_sync(0xFFFFFFFFu, mbar_try_wait(bar, parity) != 0)) return true;
    mb_wait(bar, parity, abort_flag, status);
    __syncwarp();
    return !__any_sync(0xFFFFFFFFu, *abort_flag != 0);
}
// 32 bytes past the L1 cache, in one request where the address allows it (the caller's tensors are aligned to 16 bytes)
__device__ __forceinline__ void ldcg32(const void* p, uint32_t* x) {
    if (reinterpret_cast<uint64_t>(p) & 16) {
        const uint4 a = __ldcg(reinterpret_cast<const uint4*>(p)), b = __ldcg(reinterpret_cast<const uint4*>(p) + 1);
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
        return;
    }
    asm volatile("ld.global.cg.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7])
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void st_u16(uint32_t addr, uint32_t v) { asm volatile("st.shared.u16 [%0], %1;" ::"r"(addr), "h"((uint16_t)v) : "memory"); }
__device__ __forceinline__ void st_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// What of a block's range every role walks: runs of tiles of one item.
struct Run {
    int u, h, row0, t0, n;
};
__device__ __forceinline__ bool next_run(const SharedSched& sch, int& g, int g_end, Run& r) {
    if (g >= g_end) return false;
    r.u = g / sch.tiles;
    r.t0 = g - r.u * sch.tiles;
    r.n = min(sch.tiles - r.t0, g_end - g);
    r.h = r.u / sch.groups;
    r.row0 = (r.u - r.h * sch.groups) * 128;
    g += r.n;
    return true;
}

__global__ void __launch_bounds__(kThreads, 1)
shared_tc_kernel(const __grid_constant__ CUtensorMap tmap, SharedArgs a, const __grid_constant__ SharedSched sch) {
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sm0 = s_u32(smem), slot0 = sm0 + kHeader;
    volatile uint32_t* const abort_flag = reinterpret_cast<volatile uint32_t*>(smem + oAbort);
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;  // (uniform to the compiler)
    if (sm0 & 1023u) {  // the swizzled tiles need 1024-byte alignment; report instead of computing garbage
        if (threadIdx.x == 0) atomicMax(a.status, (int32_t)kFlagCountMismatch);
        return;
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < kSlots; ++s) {
            mb_init(sm0 + oFull + 8 * s, 5);  // the producer and the entries' warps: both pass every slot, so that no role is a round ahead of or behind another
            mb_init(sm0 + oEmpty + 8 * s, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mb_init(sm0 + oS + 8 * i, 1);
            mb_init(sm0 + oP + 8 * i, 4);
            // (two: the S that a warp has seen says that the product with P two tiles back is done, not the one before)
            mb_init(sm0 + oO + 8 * i, 1);
        }
        mb_init(sm0 + oQ, 4);
        *abort_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 9) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(sm0 + oTmem), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem + oTmem);
    int g = sch.start[blockIdx.x];
    const int g_end = sch.start[blockIdx.x + 1];
    Run r;
    // Slots in ring order: K (and its entries) of tile 0, then for every tile j: K of tile j + 1, V of tile j.
    int sl = 0;
    uint32_t ph = 0;  // this pass over the ring
    auto advance = [&]() {
        if (++sl == kSlots) { sl = 0; ph ^= 1u; }
    };

    if (warp == 8) {
        if (lane == 0) {
            while (next_run(sch, g, g_end, r)) {
                const UnitDesc* const ud = a.desc + r.h;
                const bool resid = ud->mode == FDKV_MODE_RESIDUAL;
                const uint64_t arena = reinterpret_cast<uint64_t>(a.arena_base);
                const int krow = (int)((reinterpret_cast<uint64_t>(ud->k_rows) - arena) >> 8), vrow = (int)((reinterpret_cast<uint64_t>(ud->v_rows) - arena) >> 8);
                auto load = [&](int row) {
                    const uint32_t full = sm0 + oFull + 8 * sl, dst = slot0 + sl * kSlotBytes;
                    mb_wait(sm0 + oEmpty + 8 * sl, ph ^ 1u, abort_flag, a.status);
                    if (!*abort_flag) {
                        mb_expect_tx(full, kSlotBytes);
                        tma_2d(dst, &tmap, 0, row, full);
                        tma_2d(dst + kHalf, &tmap, 64, row, full);
                    }
                    advance();
                    if (resid) {
                        mb_wait(sm0 + oEmpty + 8 * sl, ph ^ 1u, abort_flag, a.status);
                        mb_arrive(sm0 + oFull + 8 * sl);
                        advance();
                    }
                };
                for (int j = -1; j < r.n; ++j) {
                    if (j + 1 < r.n) load(krow + (r.t0 + j + 1) * kSharedTile);
                    if (j >= 0) load(vrow + (r.t0 + j) * kSharedTile);
                }
            }
        }
    } else if (warp == 9) {
        // The whole warp walks the loop and one lane issues, so that descriptors and addresses stay in uniform registers: with
        // the loop behind `if (lane == 0)` issuing a tile's products took 2 700 cycles, more than the softmax.
        const bool leader = elect_one();
        int it = 0;
        uint32_t qph = 0;
        bool ok = true;
        while (ok && next_run(sch, g, g_end, r)) {
            const int parts = a.desc[r.h].mode == FDKV_MODE_RESIDUAL ? 2 : 1;  // a tile's rows, then its entries
            ok = wait_warp(sm0 + oQ, qph, abort_flag, a.status);
            qph ^= 1u;
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            auto scores = [&](int b) {
                for (int e = 0; e < parts && ok; ++e) {
                    ok = wait_warp(sm0 + oFull + 8 * sl, ph, abort_flag, a.status);
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t d = smem_desc(slot0 + sl * kSlotBytes);
                    const uint32_t ts = tmem + cS + b * 128;
                    if (leader && ok) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) umma_ts<kIdescS>(ts, tmem + cQ + 8 * k, d + (k >> 2) * (kHalf >> 4) + (k & 3) * 2, e > 0 || k > 0);
                        umma_commit(sm0 + oEmpty + 8 * sl);
                        if (e + 1 == parts) umma_commit(sm0 + oS + 8 * b);
                    }
                    __syncwarp();
                    advance();
                }
            };
            if (ok) scores(it & 1);
            for (int j = 0; j < r.n && ok; ++j, ++it) {
                if (j + 1 < r.n) scores((it + 1) & 1);
                ok = ok && wait_warp(sm0 + oP + 8 * (it & 1), (uint32_t)(it >> 1) & 1u, abort_flag, a.status);
                for (int e = 0; e < parts && ok; ++e) {
                    ok = wait_warp(sm0 + oFull + 8 * sl, ph, abort_flag, a.status);
                    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                    const uint64_t d = smem_desc_sw128(slot0 + sl * kSlotBytes, kHalf, 1024);
                    const uint32_t tp = tmem + cS + (it & 1) * 128;
                    if (leader && ok) {
#pragma unroll
                        for (int k = 0; k < 8; ++k) umma_ts<kIdescO>(tmem + cO, tp + 8 * k, d + k * (2048 >> 4), j > 0 || e > 0 || k > 0);
                        umma_commit(sm0 + oEmpty + 8 * sl);
                        if (e + 1 == parts) umma_commit(sm0 + oO + 8 * (it & 1));
                    }
                    __syncwarp();
                    advance();
                }
            }
        }
    } else if (warp >= 4) {
        // ---- the residual's tiles: this warp has tokens [32 w, 32 w + 32) of them, two 16-token slices ----
        const int w = warp - 4;
        while (next_run(sch, g, g_end, r)) {
            const UnitDesc ud = a.desc[r.h];
            auto pass_rows = [&]() {
                mb_wait(sm0 + oEmpty + 8 * sl, ph ^ 1u, abort_flag, a.status);
                __syncwarp();
                if (lane == 0) mb_arrive(sm0 + oFull + 8 * sl);
                advance();
            };
            if (ud.mode != FDKV_MODE_RESIDUAL) {
                for (int i = 0; i < 2 * r.n; ++i) pass_rows();
                continue;
            }
            const int slices = (ud.T + kResTile - 1) / kResTile;
            const int k_end = ud.k_off[slices], v_end = ud.v_off ? ud.v_off[slices] : k_end;
            const uint32_t flip = ud.sign < 0.f ? 0x8000u : 0u;
            const bool tokens = ud.res_kind == 1, packed = !tokens && !ud.k_val, twice = ud.sign == 2.f && !a.twice;
            // The fills of the run in ring order: K of tile 0, then K of tile j + 1 and V of tile j in turn.  A fill's entries are requested
            // when the one before is done and land while the ring makes room, out of L2, where a request two tiles ahead has put them.
            constexpr int kPF = 12;  // entries a lane requests ahead (the rest are loaded when they are used)
            int rk[3] = {}, rv[3] = {};  // bounds of this warp's two slices in either list, one tile per lane
            auto ranges = [&](bool is_v, int j, int& e0, int& mid, int& e1) {
                int(&x)[3] = is_v ? rv : rk;
                if ((j & 31) == 0) {
                    const int32_t* const off = is_v && ud.v_off ? ud.v_off : ud.k_off;
                    const int s0 = min(slices, (r.t0 + j + lane) * 8 + 2 * w);
#pragma unroll
                    for (int i = 0; i < 3; ++i) x[i] = off[min(slices, s0 + i)];
                }
                e0 = __shfl_sync(0xFFFFFFFFu, x[0], j & 31);
                mid = __shfl_sync(0xFFFFFFFFu, x[1], j & 31);
                e1 = __shfl_sync(0xFFFFFFFFu, x[2], j & 31);
            };
            uint32_t pe[kPF];
            int e0 = 0, mid = 0, e1 = 0;
            auto entry = [&](const int32_t* idx, const void* val, int e) {  // value in the low half, place in a slice's tile (in elements) in the high one
                const uint32_t x = (uint32_t)idx[e];
                if (packed) return x;
                uint32_t v = reinterpret_cast<const uint16_t*>(val)[e];
                if (twice) v = __bfloat16_as_ushort(__float2bfloat16_rn(2.f * __uint_as_float(v << 16)));
                const uint32_t row = x >> 7 & 15, ch = x & 127;  // (flat index token * 128 + channel)
                return v | ((ch >> 6) * 1024 + row * 64 + (((ch >> 3 & 7) ^ (row & 7)) << 3) + (ch & 7)) << 16;
            };
            auto is_v_of = [&](int f) { return f > 0 && ((f & 1) == 0 || f == 2 * r.n - 1); };
            auto tile_of = [&](int f) { return f == 2 * r.n - 1 ? r.n - 1 : f & 1 ? (f + 1) >> 1 : f == 0 ? 0 : (f >> 1) - 1; };
            auto request = [&](int f) {
                if (f >= 2 * r.n) return;
                const bool is_v = is_v_of(f);
                ranges(is_v, tile_of(f), e0, mid, e1);
                if (tokens) return;
                const int32_t* const idx = is_v && ud.v_idx ? ud.v_idx : ud.k_idx;
                const void* const val = is_v ? ud.v_val : ud.k_val;
#pragma unroll
                for (int i = 0; i < kPF; ++i)
                    if (e0 + lane + 32 * i < e1) pe[i] = entry(idx, val, e0 + lane + 32 * i);
                // (about where the list is two tiles on: the slices' counts are much alike)
                const int ahead = e0 + (e1 - e0) * 8 + lane * 32;
                const int last = is_v ? v_end : k_end;
                if (lane * 32 < (e1 - e0) + 64 && ahead < last) asm volatile("prefetch.global.L2 [%0];" ::"l"(idx + ahead));
            };
            request(0);
            for (int f = 0; f < 2 * r.n; ++f) {
                const bool is_v = is_v_of(f);
                const int32_t* const idx = is_v && ud.v_idx ? ud.v_idx : ud.k_idx;
                const void* const val = is_v ? ud.v_val : ud.k_val;
                pass_rows();
                const uint32_t base = slot0 + sl * kSlotBytes + w * 4096;
                mb_wait(sm0 + oEmpty + 8 * sl, ph ^ 1u, abort_flag, a.status);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    st_v4(base + (lane + 32 * i) * 16, 0u, 0u, 0u, 0u);
                    st_v4(base + kHalf + (lane + 32 * i) * 16, 0u, 0u, 0u, 0u);
                }
                __syncwarp();
                if (tokens) {  // whole rows, half a warp each
                    for (int e = e0 + (lane >> 4); e < e1; e += 2) {
                        const int c = lane & 15, row = idx[e] & 15;
                        uint4 x = reinterpret_cast<const uint4*>(val)[(int64_t)e * 16 + c];
                        const uint32_t f2 = flip | flip << 16;
                        st_v4(base + (c >> 3) * kHalf + (e >= mid ? 2048 : 0) + row * 128 + (((c & 7) ^ (row & 7)) << 4), x.x ^ f2, x.y ^ f2, x.z ^ f2, x.w ^ f2);
                    }
                } else {
                    auto put = [&](int e, uint32_t x) {
                        const uint32_t o = x >> 16 << 1;
                        st_u16(base + (o >> 11) * kHalf + (o & 2047) + (e >= mid ? 2048 : 0), x ^ flip);
                    };
#pragma unroll
                    for (int i = 0; i < kPF; ++i)
                        if (e0 + lane + 32 * i < e1) put(e0 + lane + 32 * i, pe[i]);
                    for (int eb = e0 + 32 * kPF; eb < e1; eb += 128) {  // dense slices: four in flight
                        uint32_t x[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (eb + lane + 32 * i < e1) x[i] = entry(idx, val, eb + lane + 32 * i);
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            if (eb + lane + 32 * i < e1) put(eb + lane + 32 * i, x[i]);
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mb_arrive(sm0 + oFull + 8 * sl);
                advance();
                request(f + 1);
            }
        }
    } else {
        // ---- softmax: thread = query row = tensor memory lane ----
        const uint32_t tq = tmem + ((uint32_t)(warp * 32) << 16);
        asm volatile("griddepcontrol.wait;" ::: "memory");  // q and the parts belong to the kernels ahead
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (behind the wait: the join reads the tails before its own)
        int it = 0;
        while (next_run(sch, g, g_end, r)) {
            const int rows = min(128, a.batch * a.G - r.row0);
            const float uscale = a.desc[r.h].scale;
            const float ks = uscale * (0.08838834764831845f * 1.4426950408889634f);  // / sqrt(128), in powers of two
            {
                const int row = r.row0 + (int)threadIdx.x, b = row / a.G;
                const char* const src = reinterpret_cast<const char*>(a.q) + (((int64_t)b * a.Hq + r.h * a.G + (row - b * a.G)) << 8);
                uint32_t x[2][32];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    if ((int)threadIdx.x < rows) ldcg32(src + 32 * i, &x[i >> 2][8 * (i & 3)]);
                    else
#pragma unroll
                        for (int k = 0; k < 8; ++k) x[i >> 2][8 * (i & 3) + k] = 0u;
                }
                tmem_st32(tq + cQ, x[0]);
                tmem_st32(tq + cQ + 32, x[1]);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mb_arrive(sm0 + oQ);
            }
            float m = -INFINITY, l = 0.f;
            for (int j = 0; j < r.n; ++j, ++it) {
                const uint32_t ts = tq + cS + (it & 1) * 128;
                mb_wait(sm0 + oS + 8 * (it & 1), (uint32_t)(it >> 1) & 1u, abort_flag, a.status);
                __syncwarp();
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                uint32_t s[4][32];
#pragma unroll
                for (int c = 0; c < 4; ++c) tmem_ld32(ts + 32 * c, s[c]);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                const int left = a.T - (r.t0 + j) * kSharedTile;
                if (left < kSharedTile) {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (32 * c + i >= left) s[c][i] = 0xFF800000u;
                }
                float mx[4];
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    mx[c] = __uint_as_float(s[c][0]);
#pragma unroll
                    for (int i = 1; i < 32; ++i) mx[c] = fmaxf(mx[c], __uint_as_float(s[c][i]));
                }
                const float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * ks;
                if (__any_sync(0xFFFFFFFFu, top > m + 8.f)) {  // (always at the first tile)
                    const float m_new = fmaxf(m, top), f = ex2(m - m_new);
                    if (j > 0) {
                        mb_wait(sm0 + oO + 8 * ((it - 1) & 1), (uint32_t)((it - 1) >> 1) & 1u, abort_flag, a.status);
                        __syncwarp();
                        asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
                        for (int c = 0; c < 4; ++c) {
                            uint32_t o[32];
                            tmem_ld32(tq + cO + 32 * c, o);
                            asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                            tmem_st32(tq + cO + 32 * c, o);
                        }
                        l *= f;
                    }
                    m = m_new;
                }
                float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int c = 0; c < 4; c += 2) {
                    uint32_t p[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int k = 2 * i & 31;
                        const float x = ex2(fmaf(__uint_as_float(s[c + (i >> 4)][k]), ks, -m)), y = ex2(fmaf(__uint_as_float(s[c + (i >> 4)][k + 1]), ks, -m));
                        sum[(i & 1) * 2] += x;
                        sum[(i & 1) * 2 + 1] += y;
                        p[i] = pack2(x, y);
                    }
                    tmem_st32(ts + 16 * c, p);
                }
                l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mb_arrive(sm0 + oP + 8 * (it & 1));
            }
            mb_wait(sm0 + oO + 8 * ((it - 1) & 1), (uint32_t)((it - 1) >> 1) & 1u, abort_flag, a.status);
            __syncwarp();
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            float* const part = a.partials + (int64_t)(blockIdx.x + r.u) * shared_part_floats(sch.row_tile, 128);
#pragma unroll 1
            for (int c = 0; c < 4; ++c) {
                uint32_t o[32];
                tmem_ld32(tq + cO + 32 * c, o);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                if ((int)threadIdx.x < rows)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        *reinterpret_cast<float4*>(part + ((int64_t)(8 * c + i) * sch.row_tile + threadIdx.x) * 4) =
                            make_float4(__uint_as_float(o[4 * i]) * uscale, __uint_as_float(o[4 * i + 1]) * uscale, __uint_as_float(o[4 * i + 2]) * uscale,
                                        __uint_as_float(o[4 * i + 3]) * uscale);
            }
            if ((int)threadIdx.x < rows) {
                part[(int64_t)sch.row_tile * 128 + threadIdx.x] = m * 0.6931471805599453f;  // the join works in natural-log units
                part[(int64_t)sch.row_tile * 129 + threadIdx.x] = l;
            }
            asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
        }
    }
    // after a timed-out wait: give copies and products that may still be in flight time to land before the block retires
    if (*abort_flag)
        for (int i = 0; i < 200; ++i) __nanosleep(1000);
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    if (warp == 9) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

}  // namespace

cudaError_t launch_shared_tc(const SharedArgs& a, const SharedSched& sch, cudaStream_t st) {
    static PerDevice once;
    const cudaError_t e = once.ensure([]() { return cudaFuncSetAttribute(shared_tc_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem); });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(sch.ncta);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, shared_tc_kernel, *reinterpret_cast<const CUtensorMap*>(a.tmap), a, sch);
}

}  // namespace fdkv
