// The prompt part of decode attention on one shared prompt, bf16 / head_dim 128 (see shared_prefix.cu): the query rows of all
// sequences of a KV head fill the rows of tcgen05 products, so that a tile of the compressed prompt is read once and used by up to 128 rows.
//
// A persistent block per SM walks a range of the flat (KV head, 128-token tile) list for one group of 128 query rows:
//   warp 16    TMA producer: the tile's K and V rows (2 x 64 channels x 128 tokens, 128-byte swizzle)
//   warps 8-15 residual units: the tile's kept entries of K (8-11) and V (12-15), scattered into a zeroed tile of the same layout (32
//              tokens per warp)
//   warp 17    issues S = Q K^T (Q from tensor memory, K-major K) and O += P V (P from tensor memory, MN-major V).  Residual units add
//              the products with the entries' tiles into the same accumulators, so that the correction is exact in float32
//   warps 0-7  softmax: thread = query row and half of the tile's tokens.  S is read from tensor memory, P = exp2(S - m) rounded to bf16
//              takes its place; the reference m only moves, and O is only rescaled, where a score passes it by more than 2^16.  (One
//              warp per scheduler, four in all, took 2 900 cycles for a tile, its chains of maxima and exponentials in the open.)
// All tiles, rows and entries alike, go through one ring of 32 KiB slots in the order in which the products use them: K of the next
// tile lies before V of this one, so that the next S is formed while the softmax of this one runs (S has two accumulators).
// P in bf16: a probability is off by 2^-8 at most, each its own way.  Its sum is that of the rounded ones, a third product with a column
// of ones: what is wrong with a probability then shifts the mean instead of scaling it (a row with one large probability is not
// off at all), and the softmax has no additions to do.  (Sums of the unrounded ones: outputs off by 2.3e-3 instead of 1.7e-3, of which 1.7e-3 is the
// rounding of the outputs.)
// For float32 outputs, whose rounding does not hide it, what bf16 leaves of P goes through the same products: P of 16 bits, 24 products a tile more with
// entries, 16 without (us a call with bf16 and with float32 outputs: 8 191 tokens, 16 sequences 19.3 and 21.1; 32 768 tokens, 8 sequences 31.9 and 38.7, 64
// sequences 58.9 and 74.7; 131 072 tokens, 16 sequences 95.2 and 123.5).
//
// What bounds it.  One row group (a batch of up to 128 query rows per KV head): memory, as long as few heads are residual.  32 768 tokens, 8 KV heads x 4, 8 sequences, a
// sixteenth kept in three heads: 141 MB, 22 us of the call's 31 with nothing in L2, the rest its start, first copies and the join (131 072
// tokens: 96 us for 556 MB, 5.8 TB/s).  A tile with entries needs 32 + 8 products instead of 16 + 8, 3 460 cycles of the tensor pipe, twice what its
// rows need from memory; ranges are cut by cost, so that blocks without such tiles do more of the rest.
// What a tile takes a block, from the difference of 65 536 and 32 768 tokens with all heads in one mode: one row group 1.37 us without entries (7.1 TB/s of reads), 1.78
// with them (3 500 cycles); two row groups (64 sequences) 1.20 and 1.92 us.  With two groups the rows come once from memory for both, at a third of its rate, the tensor pipe is
// busy for 54 % of the time, and the exponentials (16 384 a tile) take 1 024 of the 2 350 cycles of a tile without entries: no one unit bounds it, and what makes up the
// rest of those cycles has not been measured.  32 768 tokens, three of eight heads with entries: 27.7 tiles a block, 41 us.
#include <cuda.h>

#include "fdkv_internal.h"
#include "umma.cuh"

namespace fdkv {

namespace {

constexpr int kThreads = 640;  // five warpgroups; the last one's warps 18 and 19 have nothing to do
constexpr int kSlots = 7, kSlotBytes = 32768, kHalf = 16384;
constexpr float kLazy = 16.f;  // (powers of two)
// The exponents' reference while a row has met no finite score: below all of those (float32's lowest / sqrt(128), in powers of two, is -4.4e37) and finite itself,
// so that the exponential of a score of minus infinity is zero, not that of a NaN.
constexpr float kFloor = -1e38f;
// s * ks - m in one rounding differs from the rounded products, of which m is one, by up to 2^-24 |m|.  Beyond this reference, where neighbouring scores are
// 16 powers of two apart, a power of two takes the place of ks, so that the largest score's difference is zero.
constexpr float kFar = 134217728.f;
constexpr int kHeader = 1024, kOnes = 2048;  // (16 rows of 128 bytes, bf16 ones)
constexpr int kSmem = kHeader + kOnes + kSlots * kSlotBytes;
static_assert(kSmem <= 227 * 1024, "shared memory budget");
// header
constexpr int oFull = 0, oEmpty = 64, oS = 128, oP = 144, oO = 160, oQ = 176, oAbort = 184, oTmem = 188, oRun = 192;
// tensor memory columns
constexpr uint32_t cS = 0, cO = 256, cQ = 384, cL = 448, cX = 464;
constexpr uint32_t kIdescS = umma_idesc(128, 128, false), kIdescO = umma_idesc(128, 128, false) | (1u << 16);  // (B of the second product is MN-major)
constexpr uint32_t kIdescL = umma_idesc(128, 16, false);

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
// (x, y) = (a, b) * s + t, two at a time
__device__ __forceinline__ void scaled2(uint32_t a, uint32_t b, float s, float t, float& x, float& y) {
    asm("{\n\t.reg .b64 p, q, r;\n\tmov.b64 p, {%2, %3};\n\tmov.b64 q, {%4, %4};\n\tmov.b64 r, {%5, %5};\n\tfma.rn.f32x2 p, p, q, r;\n\tmov.b64 {%0, %1}, p;\n\t}"
        : "=f"(x), "=f"(y)
        : "r"(a), "r"(b), "f"(s), "f"(t));
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&r)[16]) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]),
                   "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(taddr));
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                 "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
                 : "memory");
}
__device__ __forceinline__ uint32_t tmem_ld1(uint32_t taddr) {
    uint32_t x;
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x1.b32 {%0}, [%1];\n\ttcgen05.wait::ld.sync.aligned;" : "=r"(x) : "r"(taddr) : "memory");
    return x;
}
__device__ __forceinline__ void tmem_st1(uint32_t taddr, uint32_t x) { asm volatile("tcgen05.st.sync.aligned.32x32b.x1.b32 [%0], {%1};" ::"r"(taddr), "r"(x) : "memory"); }
// the two warps of a pair (hardware barriers 1 to 4): whether some thread's x holds; or only meet
__device__ __forceinline__ bool pair_any(int pair, bool x) {
    uint32_t r;
    asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 q, %2, 0;\n\tbarrier.cta.red.or.pred p, %1, 64, q;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(r) : "r"(pair + 1), "r"((uint32_t)x) : "memory");
    return r != 0;
}
__device__ __forceinline__ void pair_sync(int pair) { asm volatile("barrier.cta.sync %0, 64;" ::"r"(pair + 1) : "memory"); }
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ void st_u16(uint32_t addr, uint32_t v) { asm volatile("st.shared.u16 [%0], %1;" ::"r"(addr), "h"((uint16_t)v) : "memory"); }
__device__ __forceinline__ void st_v4(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// What of a block's range every role walks: runs of tiles of one head.
struct Run {
    int h, t0, n;
};
__device__ __forceinline__ bool next_run(const SharedSched& sch, int& g, int g_end, Run& r) {
    if (g >= g_end) return false;
    r.h = g / sch.tiles;
    r.t0 = g - r.h * sch.tiles;
    r.n = min(sch.tiles - r.t0, g_end - g);
    g += r.n;
    return true;
}

// 640 threads x 96 registers at launch; the softmax's two warpgroups take 112, the others keep 80 (together 464 of the 480 per thread of a warpgroup; 72 spilled, which cost 3 %).
// FINE: what bf16 leaves of P takes the score columns that P does not, and both products with P once more (see above).
template <bool FINE>
__global__ void __launch_bounds__(kThreads, 1)
shared_tc_kernel(const __grid_constant__ CUtensorMap tmap, SharedArgs a, const __grid_constant__ SharedSched sch) {
    extern __shared__ __align__(1024) uint8_t smem[];
    const uint32_t sm0 = s_u32(smem), ones = sm0 + kHeader, slot0 = ones + kOnes;
    volatile uint32_t* const abort_flag = reinterpret_cast<volatile uint32_t*>(smem + oAbort);
    volatile uint32_t* const run_no = reinterpret_cast<volatile uint32_t*>(smem + oRun);  // runs that the producer has begun
    const int warp = __shfl_sync(0xFFFFFFFFu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;  // (uniform to the compiler)
    if (sm0 & 1023u) {  // the swizzled tiles need 1024-byte alignment; report instead of computing garbage
        if (threadIdx.x == 0) atomicMax(a.status, (int32_t)kFlagCountMismatch);
        return;
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < kSlots; ++s) {
            mb_init(sm0 + oFull + 8 * s, 4);  // the four warps that fill a tile of entries, or as many arrivals of the producer
            mb_init(sm0 + oEmpty + 8 * s, 1);
        }
        for (int i = 0; i < 2; ++i) {
            mb_init(sm0 + oS + 8 * i, 1);
            mb_init(sm0 + oP + 8 * i, 8);
            // (two: the S that a warp has seen says that the product with P two tiles back is done, not the one before)
            mb_init(sm0 + oO + 8 * i, 1);
        }
        mb_init(sm0 + oQ, 8);
        *abort_flag = 0;
        *run_no = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (threadIdx.x < kOnes / 16) {
        st_v4(ones + threadIdx.x * 16, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 17) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(sm0 + oTmem), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
    __syncthreads();
    asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
    const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(smem + oTmem);
    const int range = blockIdx.x / sch.groups, group = blockIdx.x - range * sch.groups, row0 = group * 128;
    int g = sch.start[range];
    const int g_end = sch.start[range + 1];
    Run r;
    // Slots in ring order: K (and its entries) of tile 0, then for every tile j: K of tile j + 1, V of tile j.
    int sl = 0;
    uint32_t ph = 0;  // this pass over the ring
    auto advance = [&]() {
        if (++sl == kSlots) { sl = 0; ph ^= 1u; }
    };

    if (warp >= 16) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        if (warp == 16) {
            if (lane == 0) {
                uint32_t runs = 0;
                while (next_run(sch, g, g_end, r)) {
                    *run_no = ++runs;
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
                            for (int i = 0; i < 3; ++i) mb_arrive(full);
                        }
                        advance();
                        if (resid) advance();
                    };
                    for (int j = -1; j < r.n; ++j) {
                        if (j + 1 < r.n) load(krow + (r.t0 + j + 1) * kSharedTile);
                        if (j >= 0) load(vrow + (r.t0 + j) * kSharedTile);
                    }
                }
            }
        } else if (warp == 17) {
            // The whole warp walks the loop and one lane issues, so that descriptors and addresses stay in uniform registers: with
            // the loop behind `if (lane == 0)` issuing a tile's products took 2 700 cycles, more than the softmax.
            const bool leader = elect_one();
            const uint64_t one = smem_desc(ones);
            constexpr int kParts = FINE ? 16 : 8;  // slices of 16 tokens of P, then of what is left of it
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
                            for (int k = 0; k < kParts; ++k) umma_ts<kIdescO>(tmem + cO, tp + 8 * k, d + (k & 7) * (2048 >> 4), j > 0 || e > 0 || k > 0);
                            if (e == 0)
#pragma unroll
                                for (int k = 0; k < kParts; ++k) umma_ts<kIdescL>(tmem + cL, tp + 8 * k, one, j > 0 || k > 0);
                            umma_commit(sm0 + oEmpty + 8 * sl);
                            if (e + 1 == parts) umma_commit(sm0 + oO + 8 * (it & 1));
                        }
                        __syncwarp();
                        advance();
                    }
                }
            }
        }
    } else if (warp >= 8) {
        // ---- the residual's tiles of K or of V: this warp has tokens [32 w, 32 w + 32) of them, two 16-token slices ----
        asm volatile("setmaxnreg.dec.sync.aligned.u32 80;");
        const int w = warp & 3;
        const bool is_v = warp >= 12;
        uint32_t runs = 0;
        while (next_run(sch, g, g_end, r)) {
            const UnitDesc ud = a.desc[r.h];
            const bool resid = ud.mode == FDKV_MODE_RESIDUAL;
            ++runs;
            if (!resid) {
                for (int i = 0; i < 2 * r.n; ++i) advance();
                continue;
            }
            // A phase of the ring can be told from the one before, not from the one before that.  Within a run every fourth slot is this
            // warp's; runs without entries it passes at once, so that it waits until the producer, which has waited for slots all along, is here.
            count_wait_bounded(run_no, runs, abort_flag, a.status);
            const int slices = (ud.T + kResTile - 1) / kResTile;
            const uint32_t flip = ud.sign < 0.f ? 0x8000u : 0u;
            const bool tokens = ud.res_kind == 1, packed = !tokens && !ud.k_val, twice = ud.sign == 2.f && !a.twice;
            const int32_t* const off = is_v && ud.v_off ? ud.v_off : ud.k_off;
            const int32_t* const idx = is_v && ud.v_idx ? ud.v_idx : ud.k_idx;
            const void* const val = is_v ? ud.v_val : ud.k_val;
            const int list_end = off[slices];
            // A tile's entries are requested when the one before is done and land while the ring makes room, out of L2, where a request
            // two tiles ahead has put them.
            constexpr int kPF = 12;  // entries a lane requests ahead (the rest are loaded when they are used)
            int bounds[3] = {};      // of this warp's two slices, one tile per lane
            uint32_t pe[kPF];
            int e0 = 0, mid = 0, e1 = 0;
            auto request = [&](int j) {
                if (j >= r.n) return;
                if ((j & 31) == 0) {
                    const int s0 = min(slices, (r.t0 + j + lane) * 8 + 2 * w);
#pragma unroll
                    for (int i = 0; i < 3; ++i) bounds[i] = off[min(slices, s0 + i)];
                }
                e0 = __shfl_sync(0xFFFFFFFFu, bounds[0], j & 31);
                mid = __shfl_sync(0xFFFFFFFFu, bounds[1], j & 31);
                e1 = __shfl_sync(0xFFFFFFFFu, bounds[2], j & 31);
                if (!packed) return;
#pragma unroll
                for (int i = 0; i < kPF; ++i)
                    if (e0 + lane + 32 * i < e1) pe[i] = (uint32_t)idx[e0 + lane + 32 * i];
                // (about where the list is two tiles on: the slices' counts are much alike)
                const int64_t ahead = (int64_t)e0 + (e1 - e0) * 8 + lane * 32;
                if (lane * 32 < (e1 - e0) + 64 && ahead < list_end) asm volatile("prefetch.global.L2 [%0];" ::"l"(idx + ahead));
            };
            auto fill = [&](int j) {
                const uint32_t base = slot0 + sl * kSlotBytes + w * 4096;
                if (lane == 0) mb_wait(sm0 + oEmpty + 8 * sl, ph ^ 1u, abort_flag, a.status);
                __syncwarp();
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    st_v4(base + (lane + 32 * i) * 16, 0u, 0u, 0u, 0u);
                    st_v4(base + kHalf + (lane + 32 * i) * 16, 0u, 0u, 0u, 0u);
                }
                __syncwarp();
                if (tokens) {  // whole rows, half a warp each
                    for (int e = e0 + (lane >> 4); e < e1; e += 2) {
                        const int c = lane & 15, row = idx[e] & 15;
                        const uint4 x = reinterpret_cast<const uint4*>(val)[(int64_t)e * 16 + c];
                        const uint32_t f2 = flip | flip << 16;
                        st_v4(base + (c >> 3) * kHalf + (e >= mid ? 2048 : 0) + row * 128 + (((c & 7) ^ (row & 7)) << 4), x.x ^ f2, x.y ^ f2, x.z ^ f2, x.w ^ f2);
                    }
                } else {
                    auto put = [&](int e, uint32_t x) {  // value in the low half, place in the slice's tile (in elements) in the high one
                        const uint32_t o = x >> 16 << 1;
                        st_u16(base + (e >= mid ? 2048u : 0u) + o + (o & 2048u) * 7u, x ^ flip);  // (the second 64 channels: kHalf on)
                    };
                    if (packed) {
#pragma unroll
                        for (int i = 0; i < kPF; ++i)
                            if (e0 + lane + 32 * i < e1) put(e0 + lane + 32 * i, pe[i]);
#pragma unroll 1
                        for (int eb = e0 + 32 * kPF; eb < e1; eb += 128) {  // dense slices: four in flight
                            uint32_t x[4];
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (eb + lane + 32 * i < e1) x[i] = (uint32_t)idx[eb + lane + 32 * i];
#pragma unroll
                            for (int i = 0; i < 4; ++i)
                                if (eb + lane + 32 * i < e1) put(eb + lane + 32 * i, x[i]);
                        }
                    } else {  // flat indices token * 128 + channel, and values
#pragma unroll 1
                        for (int e = e0 + lane; e < e1; e += 32) {
                            const uint32_t x = (uint32_t)idx[e], row = x >> 7 & 15, ch = x & 127;
                            uint32_t v = reinterpret_cast<const uint16_t*>(val)[e];
                            if (twice) v = __bfloat16_as_ushort(__float2bfloat16_rn(2.f * __uint_as_float(v << 16)));
                            put(e, v | ((ch >> 6) * 1024 + row * 64 + (((ch >> 3 & 7) ^ (row & 7)) << 3) + (ch & 7)) << 16);
                        }
                    }
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
                if (lane == 0) mb_arrive(sm0 + oFull + 8 * sl);
                advance();
                request(j + 1);
            };
            request(0);
            for (int j = -1; j < r.n; ++j) {
                if (j + 1 < r.n) {
                    advance();
                    if (is_v) advance(); else fill(j + 1);
                }
                if (j >= 0) {
                    advance();
                    if (is_v) fill(j); else advance();
                }
            }
        }
    } else {
        // ---- softmax: thread = query row = tensor memory lane ----
        asm volatile("setmaxnreg.inc.sync.aligned.u32 112;");
        const int pair = warp & 3, half = warp >> 2, row = pair * 32 + lane;
        const uint32_t tq = tmem + ((uint32_t)(pair * 32) << 16);
        asm volatile("griddepcontrol.wait;" ::: "memory");  // q and the parts belong to the kernels ahead
        asm volatile("griddepcontrol.launch_dependents;" ::: "memory");  // (behind the wait: the join reads the tails before its own)
        int it = 0;
        while (next_run(sch, g, g_end, r)) {
            const int rows = min(128, a.batch * a.G - row0);
            const float uscale = a.desc[r.h].scale;
            const float ks = uscale * (0.08838834764831845f * 1.4426950408889634f);  // / sqrt(128), in powers of two
            {
                const int i = row0 + row, b = i / a.G;
                const char* const src = reinterpret_cast<const char*>(a.q) + (((int64_t)b * a.Hq + r.h * a.G + (i - b * a.G)) << 8) + 128 * half;
                uint32_t x[32];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    if (row < rows) ldcg32(src + 32 * k, &x[8 * k]);
                    else
#pragma unroll
                        for (int e = 0; e < 8; ++e) x[8 * k + e] = 0u;
                }
                tmem_st32(tq + cQ + 32 * half, x);
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mb_arrive(sm0 + oQ);
            }
            // A score's exponent is score * scale + shift: ks and minus the reference m (in powers of two, the same for both halves), or, far off, the
            // power of two below ks and what makes the reference's exponent zero.
            const float two = __uint_as_float(__float_as_uint(ks) & 0x7F800000u);
            float scale = two, shift = -kFloor;
            auto reference = [&]() { return scale == ks ? -shift : fmaxf(-shift / scale * ks, kFloor); };
            auto set_reference = [&](float raw) {
                const float m = fmaxf(raw * ks, kFloor);
                scale = fabsf(m) > kFar ? two : ks;
                shift = fabsf(m) > kFar ? fminf(-raw * two, -kFloor) : -m;
            };
            // A score of the warps' rows passes the reference by more than 2^kLazy (or there is none yet): both halves take the larger of their
            // maxima, and each scales its half of the accumulators down, by a power of two.  From or to a reference far off (rows whose scores so far were
            // the lowest values) the steps would be rounded, and it is set anew.
            auto move_reference = [&](float raw, int j) {
                tmem_st1(tq + cX + half, __float_as_uint(raw));
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                pair_sync(pair);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                raw = fmaxf(raw, __uint_as_float(tmem_ld1(tq + cX + (half ^ 1))));
                // (the other half has read this one's before either comes here again: the barrier of the next tile lies between)
                if (j == 0) {
                    set_reference(raw);
                    return;
                }
                const float m = reference(), up = fmaxf(0.f, ceilf(raw * ks - m));
                float f = 1.f;
                if (up < 200.f && scale == ks) {
                    f = ex2((shift - up) - shift);  // (the step as it is rounded)
                    shift -= up;
                } else if (up > 0.f) {
                    f = ex2(m - raw * ks);
                    set_reference(raw);
                }
                mb_wait(sm0 + oO + 8 * ((it - 1) & 1), (uint32_t)((it - 1) >> 1) & 1u, abort_flag, a.status);
                __syncwarp();
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
#pragma unroll 1
                for (int k = 0; k < 4 + half; ++k) {  // (the second half also has the sums)
                    uint32_t o[16];
                    const uint32_t at = tq + (k < 4 ? cO + 64 * half + 16 * k : cL);
                    tmem_ld16(at, o);
                    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                    tmem_st16(at, o);
                }
            };
            for (int j = 0; j < r.n; ++j, ++it) {
                const uint32_t ts = tq + cS + (it & 1) * 128;
                mb_wait(sm0 + oS + 8 * (it & 1), (uint32_t)(it >> 1) & 1u, abort_flag, a.status);
                __syncwarp();
                if (pair * 32 >= rows) {  // (no query has these rows: their scores, all zero, may stand for P)
                    if (lane == 0) mb_arrive(sm0 + oP + 8 * (it & 1));
                    continue;
                }
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                uint32_t s[2][32];
                tmem_ld32(ts + 64 * half, s[0]);
                tmem_ld32(ts + 64 * half + 32, s[1]);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                const int left = a.T - (r.t0 + j) * kSharedTile - 64 * half;  // this half's tokens
                if (left < 64) {
#pragma unroll
                    for (int c = 0; c < 2; ++c)
#pragma unroll
                        for (int i = 0; i < 32; ++i)
                            if (32 * c + i >= left) s[c][i] = 0xFF800000u;
                }
                float mx[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    mx[k] = fmaxf(__uint_as_float(s[k & 1][16 * (k >> 1)]), __uint_as_float(s[k & 1][16 * (k >> 1) + 1]));
#pragma unroll
                    for (int i = 2; i < 16; i += 2)
                        mx[k] = fmaxf(fmaxf(mx[k], __uint_as_float(s[k & 1][16 * (k >> 1) + i])), __uint_as_float(s[k & 1][16 * (k >> 1) + i + 1]));
                }
                const float raw = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
                // (also says that the other half has read its scores: P of this one lies where they were)
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                if (pair_any(pair, fmaf(raw, scale, shift) > kLazy)) move_reference(raw, j);
                asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
                if constexpr (FINE) {
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        uint32_t p[16], rest[16];
#pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            float x, y;
                            scaled2(s[c][2 * i], s[c][2 * i + 1], scale, shift, x, y);
                            x = ex2(x);
                            y = ex2(y);
                            p[i] = pack2(x, y);
                            rest[i] = pack2(x - __uint_as_float(p[i] << 16), y - __uint_as_float(p[i] & 0xFFFF0000u));
                        }
                        tmem_st16(ts + 32 * half + 16 * c, p);
                        tmem_st16(ts + 64 + 32 * half + 16 * c, rest);
                    }
                } else {
                    uint32_t p[32];
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        const int k = 2 * i & 31;
                        float x, y;
                        scaled2(s[i >> 4][k], s[i >> 4][k + 1], scale, shift, x, y);
                        p[i] = pack2(ex2(x), ex2(y));
                    }
                    tmem_st32(ts + 32 * half, p);
                }
                asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
                asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
                __syncwarp();
                if (lane == 0) mb_arrive(sm0 + oP + 8 * (it & 1));
            }
            mb_wait(sm0 + oO + 8 * ((it - 1) & 1), (uint32_t)((it - 1) >> 1) & 1u, abort_flag, a.status);
            __syncwarp();
            asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
            float* const part = a.partials + ((int64_t)(range + r.h) * sch.groups + group) * shared_part_floats(sch.row_tile, 128);
#pragma unroll 1
            for (int c = 2 * half; c < 2 * half + 2; ++c) {
                uint32_t o[32];
                tmem_ld32(tq + cO + 32 * c, o);
                asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
                if (row < rows)
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        *reinterpret_cast<float4*>(part + ((int64_t)(8 * c + i) * sch.row_tile + row) * 4) =
                            make_float4(__uint_as_float(o[4 * i]) * uscale, __uint_as_float(o[4 * i + 1]) * uscale, __uint_as_float(o[4 * i + 2]) * uscale,
                                        __uint_as_float(o[4 * i + 3]) * uscale);
            }
            const uint32_t sum = tmem_ld1(tq + cL);
            if (half == 0 && row < rows) {
                part[(int64_t)sch.row_tile * 128 + row] = reference() * 0.6931471805599453f;  // the join works in natural-log units
                part[(int64_t)sch.row_tile * 129 + row] = __uint_as_float(sum);
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
    if (warp == 17) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

}  // namespace

cudaError_t launch_shared_tc(const SharedArgs& a, const SharedSched& sch, cudaStream_t st) {
    static PerDevice once;
    const cudaError_t e = once.ensure([]() {
        const cudaError_t e = cudaFuncSetAttribute(shared_tc_kernel<false>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
        return e != cudaSuccess ? e : cudaFuncSetAttribute(shared_tc_kernel<true>, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    });
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3(sch.ranges * sch.groups);
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = kSmem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, a.out_dtype == FDKV_F32 ? shared_tc_kernel<true> : shared_tc_kernel<false>, *reinterpret_cast<const CUtensorMap*>(a.tmap), a, sch);
}

}  // namespace fdkv
