// Product of 8-bit activations with 8-bit weights, scaled by blocks of 128:
//     out[m, n] = sum_b  sx[m, b] sw[n / 128, b]  sum_{k in block b} x[m, k] w[n, k]
// The inner sums run on the fifth-generation tensor cores (tcgen05.mma, kind f8f6f4, e4m3 operands, fp32 accumulators in tensor
// memory): a block of K is four instructions of 32.  The scales differ from block to block, so an accumulator holds
// one block only; eight warps read it, multiply it by the two scales and add it to fp32 registers while the tensor cores fill the
// next accumulator.  (The tensor cores' sum over a block of 128 is exact to fp32 rounding here: measured error 0 against 64 bits.)
//
// Roles: warps 0-7 scale and add, a row per thread and half of the tile's columns per warpgroup; warp 8 loads (a box of x and one
// of w per block of K, 128-byte rows, swizzled); warp 9 issues the products; warps 10 and 11 stage the scales' products, some blocks ahead (loaded
// by the adding warps themselves, a line per row, they cost those 140 of 870 cycles per block).
#include "w8.cuh"

namespace plora {
namespace w8 {
namespace {

using paged::mbar_arrive;
using paged::mbar_arrive_expect_tx;
using paged::mbar_init;
using paged::mbar_init_fence;
using paged::mbar_try_wait;
using paged::pack16;
using paged::smem_u32;

constexpr int kMaxWeights = 4;
constexpr int kThreads = 384, kAddWarps = 8, kLoadWarp = 8, kMmaWarp = 9, kScaleWarp = 10;      // (two of the last)
constexpr int kRows = 128;                // rows of x per CTA
constexpr int kRowBytes = 128;            // one block of K
constexpr int kScaleRun = 4;              // blocks of K whose scales are staged together
constexpr int kScaleBytes = kScaleRun * 2 * kRows * 4;
constexpr long long kWaitCycles = 4000000000ll;      // limit of a wait: about two seconds of SM clock

// CG: CTAs that share a tile (cta_group); BN: columns of the tile.
template <int CG, int BN>
struct Cfg {
    static constexpr int kABytes = kRows * kRowBytes, kBBytes = BN / CG * kRowBytes, kStageBytes = kABytes + kBBytes;
    // one CTA per SM in pairs, two otherwise
    static constexpr int kStages = CG == 2 ? (BN == 256 ? 6 : 8) : (BN == 128 ? 3 : 4);
    static constexpr int kAccs = CG == 2 ? 512 / BN : 256 / BN, kTmemCols = kAccs * BN;
    static constexpr int kScaleSlots = CG == 2 ? 4 : 2;       // such runs
    static constexpr int kBars = 2 * kStages + 2 * kAccs + 2 * kScaleSlots + 1;
    static constexpr int kSmemBytes = 1024 + kStages * kStageBytes + kScaleSlots * kScaleBytes + kBars * 8 + 16;
    static constexpr int kCols = BN / 2;  // columns of a thread
    static constexpr int kRead = BN == 256 ? 16 : 32;     // columns read at a time (two such buffers beside the sums)
    static constexpr int kPitch = BN + 1; // floats between the rows of a partial tile in shared memory
    static_assert(CG == 2 || kRows * kPitch * 4 <= kStages * kStageBytes, "a partial tile fits into the ring");
};

struct Params {
    const float* x_scale;
    const float* w_scale[kMaxWeights];
    void* out[kMaxWeights];
    long long out_stride[kMaxWeights];
    int32_t n[kMaxWeights], tile_end[kMaxWeights];     // columns; tiles of columns up to and with this weight's
    int32_t m, blocks, m_tiles, n_tiles, tiles, splits, x_rows;   // blocks of K; x_rows: rows of a box of x
    int32_t wide;                                      // every row of every output is 32-byte aligned
    int32_t* status;
};
struct Maps {
    CUtensorMap x, w[kMaxWeights];
};

// ---- PTX ------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// K-major operand of 128-byte rows, 128-byte swizzle: groups of 8 rows lie 1024 bytes apart.
__device__ __forceinline__ constexpr uint64_t smem_desc(uint32_t saddr) {
    return (uint64_t)((saddr >> 4) & 0x3fffu) | ((uint64_t)1 << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// fp32 accumulate, e4m3 operands, both K-major.
__device__ __forceinline__ constexpr uint32_t instr_desc(int m, int n) {
    return (1u << 4) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}
template <int CG>
__device__ __forceinline__ void umma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool acc) {
    if (CG == 2)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc)
            : "memory");
}
// Arrives when the products issued so far are complete; BOTH: at this place in both CTAs of a pair.
template <int CG, bool BOTH>
__device__ __forceinline__ void umma_commit(uint32_t bar) {
    if (CG == 2 && BOTH)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
                     "h"((uint16_t)3)
                     : "memory");
    else if (CG == 2)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t a, uint32_t* r) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]),
          "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]),
          "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(a));
}
__device__ __forceinline__ void tmem_ld16(uint32_t a, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(a));
}
template <int N>
__device__ __forceinline__ void tmem_ld(uint32_t a, uint32_t* r) {
    if (N == 32) tmem_ld32(a, r);
    else tmem_ld16(a, r);
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// A box of rows of 128 bytes.  In a pair the barrier may be the other CTA's.
template <int CG>
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap* tm, int k, int row, uint32_t bar) {
    if (CG == 2)
        asm volatile(
            "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(tm)), "r"(k), "r"(row), "r"(bar)
            : "memory");
    else
        asm volatile(
            "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
            "l"(reinterpret_cast<uint64_t>(tm)), "r"(k), "r"(row), "r"(bar)
            : "memory");
}
__device__ __forceinline__ void prefetch_map(const CUtensorMap* tm) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(reinterpret_cast<uint64_t>(tm)) : "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t in_cta(uint32_t addr, uint32_t rank) {     // the same place in another CTA of the cluster
    uint32_t r;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
// (Hands nothing over in memory, only the right to tensor memory, whose reads are complete: a release at cluster scope cost the
// warps that add some 800 cycles per block of K.)
__device__ __forceinline__ void arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ float ld_cluster(uint32_t a) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ uint64_t desc_of(uint32_t lo, uint32_t hi) { return (uint64_t)lo | ((uint64_t)hi << 32); }
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ void st_global32(void* p, const uint32_t* w) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                 "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}
// Every wait is bounded.  When one runs out, the CTA's abort flag goes up, the status word gets PLORA_ERR_TIMEOUT, and every
// role leaves its loop.
struct WaitCtl {
    volatile int* abort_flag;
    int32_t* status;
};
__device__ __forceinline__ bool wait_slow(uint32_t bar, uint32_t parity, WaitCtl w) {
    const long long t0 = clock64();
#pragma unroll 1
    for (uint32_t n = 1;; ++n) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((n & 63) == 0 && (*w.abort_flag || clock64() - t0 > kWaitCycles)) break;
    }
    if (!*w.abort_flag && w.status) atomicCAS(w.status, 0, PLORA_ERR_TIMEOUT);
    *w.abort_flag = 1;
    return false;
}
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, const WaitCtl& w) {
    return mbar_try_wait(bar, parity) || wait_slow(bar, parity, w);
}

// ---- the tiles ----------------------------------------------------------------------------------------------------
// Tiles are numbered so that those under way at one time (some 74) form a near-square of x and w: runs of kGroup tiles of rows by all
// tiles of columns.
constexpr int kGroup = 8;
struct Tile {
    int32_t mt, w, nt;      // tile of rows; weight, and tile of its columns
};
__device__ __forceinline__ Tile tile_of(const Params& p, int i) {
    const int per = kGroup * p.n_tiles, g = i / per, rest = i - g * per, rows = min(kGroup, p.m_tiles - g * kGroup);
    Tile t;
    t.nt = rest / rows;
    t.mt = g * kGroup + rest - t.nt * rows;
    t.w = 0;
    int first = 0;
#pragma unroll
    for (int j = 0; j < kMaxWeights - 1; ++j)
        if (t.nt >= p.tile_end[j]) {
            t.w = j + 1;
            first = p.tile_end[j];
        }
    t.nt -= first;
    return t;
}
// What a cluster does: tiles first, first + step, ...; blocks of K [b0, b1).
struct Share {
    int32_t first, step, b0, b1;
};
template <int CG>
__device__ __forceinline__ Share share_of(const Params& p, uint32_t rank) {
    if (CG == 2) return {(int)(blockIdx.x >> 1), (int)(gridDim.x >> 1), 0, p.blocks};
    const int per = (p.blocks + p.splits - 1) / p.splits, b0 = min((int)rank * per, p.blocks);
    return {(int)blockIdx.x / p.splits, p.tiles, b0, min(b0 + per, p.blocks)};
}

struct Smem {
    uint32_t ring, full, empty, acc_full, acc_empty, scale_full, scale_empty, done;
    float* scales;       // [run][block][half of the columns][row]
    uint32_t* tmem_slot;
    WaitCtl wc;
};

// Warps 8 and 9 stay together and an elected lane issues: copies and products take uniform registers, and in a branch of a single
// lane each of them costs 100 cycles and more (the first form of this kernel: 1900 cycles per block of K instead of 512).
template <int CG, int BN>
__device__ __forceinline__ void load_warp(const Params& p, const Maps& maps, const Smem& sm, uint32_t rank) {
    using C = Cfg<CG, BN>;
    const unsigned all = 0xffffffffu;
    const Share sh = share_of<CG>(p, rank);
    const uint32_t bytes = CG * (uint32_t)(p.x_rows * kRowBytes + C::kBBytes);
    const uint32_t ring = uniform(sm.ring), full = uniform(sm.full), counts = uniform(CG == 2 ? in_cta(sm.full, 0) : sm.full);
    uint32_t it = 0, early = 0;
    bool stopped = false;
    // The weights of the first stages are fetched before the kernel in front has completed: no kernel of the library that lets
    // the next one start early writes weights.
    auto begin = [&](uint32_t s, const Tile& t, int b) {
        if (elect_one()) {
            if (CG == 1 || rank == 0) mbar_arrive_expect_tx(full + s * 8, bytes);
            tma_box<CG>(ring + s * C::kStageBytes + C::kABytes, &maps.w[t.w], b * kRowBytes, t.nt * BN + (CG == 2 ? (int)rank * (BN / 2) : 0),
                        counts + s * 8);
        }
    };
    auto finish = [&](uint32_t s, const Tile& t, int b) {
        if (elect_one())
            tma_box<CG>(ring + s * C::kStageBytes, &maps.x, b * kRowBytes, (t.mt * CG + (CG == 2 ? (int)rank : 0)) * kRows, counts + s * 8);
    };
    if (sh.first < p.tiles) {
        const Tile t = tile_of(p, sh.first);
        for (; early < C::kStages && sh.b0 + (int)early < sh.b1; ++early) begin(early, t, sh.b0 + early);
    }
    paged::grid_wait();
#pragma unroll 1
    for (int i = sh.first; i < p.tiles && !stopped; i += sh.step) {
        const Tile t = tile_of(p, i);
#pragma unroll 1
        for (int b = sh.b0; b < sh.b1; ++b, ++it) {
            const uint32_t s = it % C::kStages;
            if (it >= early) {
                if (!__all_sync(all, wait(sm.empty + s * 8, ((it / C::kStages) & 1) ^ 1, sm.wc))) {
                    stopped = true;
                    break;
                }
                begin(s, t, b);
            }
            finish(s, t, b);
        }
    }
    const uint32_t n = max(it, early);
    if (!stopped) {
        // the products' last signals come from the pair's first CTA: they must have come before the second one leaves
        if (CG == 2)
            for (uint32_t j = n > C::kStages ? n - C::kStages : 0; j < n; ++j) wait(sm.empty + j % C::kStages * 8, (j / C::kStages) & 1, sm.wc);
    } else if (CG == 1 || rank == 0) {
        // copies in flight must land before the CTA leaves (in a pair they are counted by the first CTA's barriers)
        for (uint32_t j = n > C::kStages ? n - C::kStages : 0; j < n; ++j)
            paged::mbar_drain(sm.full + j % C::kStages * 8, (j / C::kStages) & 1, kWaitCycles);
    }
}

template <int CG, int BN>
__device__ __forceinline__ void mma_warp(const Params& p, const Smem& sm, uint32_t tmem, uint32_t rank) {
    using C = Cfg<CG, BN>;
    const unsigned all = 0xffffffffu;
    const Share sh = share_of<CG>(p, rank);
    constexpr uint32_t idesc = instr_desc(CG * kRows, BN);
    constexpr uint32_t kHi = (uint32_t)(smem_desc(0) >> 32), kLo = (uint32_t)smem_desc(0);
    const uint32_t ring = uniform(sm.ring >> 4), empty = uniform(sm.empty), acc_full = uniform(sm.acc_full);
    tmem = uniform(tmem);
    uint32_t it = 0;
    bool stopped = false;
#pragma unroll 1
    for (int i = sh.first; i < p.tiles && !stopped; i += sh.step) {
#pragma unroll 1
        for (int b = sh.b0; b < sh.b1; ++b, ++it) {
            const uint32_t s = it % C::kStages, a = it % C::kAccs;
            if (!__all_sync(all, wait(sm.acc_empty + a * 8, ((it / C::kAccs) & 1) ^ 1, sm.wc)) ||
                !__all_sync(all, wait(sm.full + s * 8, (it / C::kStages) & 1, sm.wc))) {
                stopped = true;
                break;
            }
            tc_fence_after();
            const uint32_t da = (ring + s * (C::kStageBytes >> 4)) | kLo, db = da + (C::kABytes >> 4);
            if (elect_one()) {
#pragma unroll
                for (int k = 0; k < 4; ++k) umma<CG>(tmem + a * BN, desc_of(da + 2 * k, kHi), desc_of(db + 2 * k, kHi), idesc, k > 0);
                umma_commit<CG, true>(empty + s * 8);
                umma_commit<CG, true>(acc_full + a * 8);
            }
        }
    }
    // no product is under way when tensor memory is given back
    if (elect_one()) umma_commit<CG, false>(sm.done);
    if (!paged::mbar_drain(sm.done, 0, kWaitCycles) && p.status) atomicCAS(p.status, 0, PLORA_ERR_TIMEOUT);
}

template <int KIND>
__device__ __forceinline__ void store_one(void* out, long long at, float v) {
    if (KIND == PLORA_INPUT_FP32) static_cast<float*>(out)[at] = v;
    else static_cast<uint16_t*>(out)[at] = (uint16_t)pack16<KIND == PLORA_INPUT_FP16>(v, 0.f);
}

// Warps 10 and 11: sx sw of each row, block and half of the tile's columns (a half lies in one block of w's rows).
template <int CG, int BN>
__device__ __forceinline__ void scale_warps(const Params& p, const Smem& sm, uint32_t rank) {
    using C = Cfg<CG, BN>;
    const Share sh = share_of<CG>(p, rank);
    const int lane = threadIdx.x & 31, r0 = threadIdx.x - kScaleWarp * 32;
    uint32_t it = 0;
    paged::grid_wait();
#pragma unroll 1
    for (int i = sh.first; i < p.tiles; i += sh.step) {
        const Tile t = tile_of(p, i);
        const int row0 = (t.mt * CG + (CG == 2 ? (int)rank : 0)) * kRows, last = (p.n[t.w] - 1) / kBlock;
        const float *x0 = p.x_scale + (size_t)min(row0 + r0, p.m - 1) * p.blocks, *x1 = p.x_scale + (size_t)min(row0 + r0 + 64, p.m - 1) * p.blocks;
        const float *w0 = p.w_scale[t.w] + (size_t)min(t.nt * BN / kBlock, last) * p.blocks;
        const float *w1 = p.w_scale[t.w] + (size_t)min((t.nt * BN + C::kCols) / kBlock, last) * p.blocks;
#pragma unroll 1
        for (int b = sh.b0; b < sh.b1; b += kScaleRun, ++it) {
            const uint32_t slot = it % C::kScaleSlots;
            float x[2][kScaleRun], w[2][kScaleRun];
#pragma unroll
            for (int j = 0; j < kScaleRun; ++j) {
                const int at = min(b + j, sh.b1 - 1);
                x[0][j] = x0[at]; x[1][j] = x1[at];
                w[0][j] = w0[at]; w[1][j] = w1[at];
            }
            if (!__all_sync(0xffffffffu, wait(sm.scale_empty + slot * 8, ((it / C::kScaleSlots) & 1) ^ 1, sm.wc))) return;
            float* s = sm.scales + slot * (kScaleBytes / 4) + r0;
#pragma unroll
            for (int j = 0; j < kScaleRun; ++j)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    s[(j * 2 + h) * kRows] = x[0][j] * w[h][j];
                    s[(j * 2 + h) * kRows + 64] = x[1][j] * w[h][j];
                }
            __syncwarp();
            if (lane == 0) mbar_arrive(sm.scale_full + slot * 8);
        }
    }
}

// Scales and adds the accumulators of one tile: row (warp & 3) * 32 + lane of the CTA's, half warp >> 2 of the columns.
template <int CG, int BN>
__device__ __forceinline__ bool add_tile(const Smem& sm, uint32_t tmem, const Share& sh, bool any, int warp, int lane, uint32_t& it, uint32_t& run,
                                         float2 (&acc)[Cfg<CG, BN>::kCols / 2]) {
    using C = Cfg<CG, BN>;
    const uint32_t from = tmem + ((uint32_t)(warp & 3) << 21) + (warp >> 2) * C::kCols;
    const float* scales = sm.scales + (warp >> 2) * kRows + (warp & 3) * 32 + lane;
#pragma unroll
    for (int i = 0; i < C::kCols / 2; ++i) acc[i] = make_float2(0.f, 0.f);
#pragma unroll 1
    for (int left = sh.b1 - sh.b0; left > 0; left -= kScaleRun, ++run) {
        const uint32_t slot = run % C::kScaleSlots;
        if (!__all_sync(0xffffffffu, wait(sm.scale_full + slot * 8, (run / C::kScaleSlots) & 1, sm.wc))) return false;
#pragma unroll 1
        for (int j = 0; j < min(left, kScaleRun); ++j, ++it) {
            const uint32_t a = it % C::kAccs;
            const float f = scales[slot * (kScaleBytes / 4) + j * 2 * kRows];
            if (!__all_sync(0xffffffffu, wait(sm.acc_full + a * 8, (it / C::kAccs) & 1, sm.wc))) return false;
            tc_fence_after();
            if (any) {        // (a row of this warp exists)
                const float2 f2 = make_float2(f, f);
                uint32_t buf[2][C::kRead];
                tmem_ld<C::kRead>(from + a * BN, buf[0]);
#pragma unroll
                for (int c = 0; c < C::kCols / C::kRead; ++c) {
                    tmem_ld_wait();
                    if (c + 1 < C::kCols / C::kRead) tmem_ld<C::kRead>(from + a * BN + (c + 1) * C::kRead, buf[(c + 1) & 1]);
                    const float* v = reinterpret_cast<const float*>(buf[c & 1]);
#pragma unroll
                    for (int i = 0; i < C::kRead / 2; ++i) {
                        float2& o = acc[c * (C::kRead / 2) + i];
                        o = __ffma2_rn(make_float2(v[2 * i], v[2 * i + 1]), f2, o);
                    }
                }
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0) {
                if (CG == 2) arrive_cluster(in_cta(sm.acc_empty + a * 8, 0));
                else mbar_arrive(sm.acc_empty + a * 8);
            }
        }
        if (lane == 0) mbar_arrive(sm.scale_empty + slot * 8);
    }
    return true;
}

template <int CG, int BN, int KIND>
__device__ __forceinline__ void store_tile(const Params& p, const Tile& t, int row, int col, const float2 (&acc)[Cfg<CG, BN>::kCols / 2]) {
    using C = Cfg<CG, BN>;
    if (row >= p.m) return;
    const int n = p.n[t.w];
    const long long at = row * p.out_stride[t.w] + col;
    constexpr int kStep = KIND == PLORA_INPUT_FP32 ? 8 : 16;       // columns of a 32-byte store
#pragma unroll
    for (int c = 0; c < C::kCols; c += kStep) {
        const float* v = reinterpret_cast<const float*>(acc) + c;
        if (p.wide && col + c + kStep <= n) {
            uint32_t w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i)
                w[i] = KIND == PLORA_INPUT_FP32 ? __float_as_uint(v[i]) : pack16<KIND == PLORA_INPUT_FP16>(v[(2 * i) % kStep], v[(2 * i + 1) % kStep]);
            st_global32(static_cast<char*>(p.out[t.w]) + (at + c) * (KIND == PLORA_INPUT_FP32 ? 4 : 2), w);
        } else {
#pragma unroll
            for (int i = 0; i < kStep; ++i)
                if (col + c + i < n) store_one<KIND>(p.out[t.w], at + c + i, v[i]);
        }
    }
}

template <int CG, int BN, int KIND>
__global__ void __launch_bounds__(kThreads, CG == 2 ? 1 : 2) gemm_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Params p) {
    using C = Cfg<CG, BN>;
    extern __shared__ uint8_t raw[];
    uint8_t* base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    uint8_t* bars = base + C::kStages * C::kStageBytes + C::kScaleSlots * kScaleBytes;
    Smem sm;
    sm.ring = smem_u32(base);
    sm.full = smem_u32(bars);
    sm.empty = sm.full + C::kStages * 8;
    sm.acc_full = sm.empty + C::kStages * 8;
    sm.acc_empty = sm.acc_full + C::kAccs * 8;
    sm.scale_full = sm.acc_empty + C::kAccs * 8;
    sm.scale_empty = sm.scale_full + C::kScaleSlots * 8;
    sm.done = sm.scale_empty + C::kScaleSlots * 8;
    sm.scales = reinterpret_cast<float*>(base + C::kStages * C::kStageBytes);
    sm.tmem_slot = reinterpret_cast<uint32_t*>(bars + C::kBars * 8);
    sm.wc.abort_flag = reinterpret_cast<volatile int*>(bars + C::kBars * 8 + 8);
    sm.wc.status = p.status;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(sm.full + s * 8, 1);
            mbar_init(sm.empty + s * 8, 1);
        }
        for (int a = 0; a < C::kAccs; ++a) {
            mbar_init(sm.acc_full + a * 8, 1);
            mbar_init(sm.acc_empty + a * 8, kAddWarps * CG);
        }
        for (int r = 0; r < C::kScaleSlots; ++r) {
            mbar_init(sm.scale_full + r * 8, 2);
            mbar_init(sm.scale_empty + r * 8, kAddWarps);
        }
        mbar_init(sm.done, 1);
        sm.wc.abort_flag[0] = 0;
        mbar_init_fence();
    }
    if (warp == kLoadWarp && lane == 0) {
        prefetch_map(&maps.x);
        prefetch_map(&maps.w[0]);
    }
    if (warp == kMmaWarp) {
        if (CG == 2) {
            asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(sm.tmem_slot)), "n"(C::kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
        } else {
            asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(sm.tmem_slot)), "n"(C::kTmemCols) : "memory");
            asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        }
        tc_fence_before();
    }
    __syncthreads();
    if (CG == 2) cluster_sync();        // the other CTA's barriers exist
    tc_fence_after();
    const uint32_t tmem = *sm.tmem_slot;
    const Share sh = share_of<CG>(p, rank);
    if (warp < kAddWarps) {
        if (CG == 2 && BN == 256) asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        paged::grid_wait();
        if (threadIdx.x == 0) paged::grid_launch_dependents();     // (what the kernel in front wrote is complete by now)
        const int r = (CG == 2 ? (int)rank * kRows : 0) + (warp & 3) * 32 + lane, c = (warp >> 2) * C::kCols;
        uint32_t it = 0, run = 0;
        float2 acc[C::kCols / 2];
#pragma unroll 1
        for (int i = sh.first; i < p.tiles; i += sh.step) {
            const Tile t = tile_of(p, i);
            const int row = t.mt * CG * kRows + r, col = t.nt * BN + c;
            if (!add_tile<CG, BN>(sm, tmem, sh, row - lane < p.m, warp, lane, it, run, acc)) break;
            if (CG == 2 || p.splits == 1) {
                store_tile<CG, BN, KIND>(p, t, row, col, acc);
            } else if (row < p.m) {       // all products are complete: the ring is free for the partial tile
                float* part = reinterpret_cast<float*>(base) + r * C::kPitch + c;
#pragma unroll
                for (int e = 0; e < C::kCols / 2; ++e) {
                    part[2 * e] = acc[e].x;
                    part[2 * e + 1] = acc[e].y;
                }
            }
        }
    } else {
        if (CG == 2 && BN == 256) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == kLoadWarp) load_warp<CG, BN>(p, maps, sm, rank);
        else if (warp == kMmaWarp && (CG == 1 || rank == 0)) mma_warp<CG, BN>(p, sm, tmem, rank);
        else if (warp >= kScaleWarp) scale_warps<CG, BN>(p, sm, rank);
        __syncwarp();
    }
    tc_fence_before();
    __syncthreads();
    if (CG == 2) {
        cluster_sync();                 // products read both CTAs' memory
    } else if (p.splits > 1) {
        // the partial tiles of the cluster, added in the order of K; each CTA has its share of the elements
        cluster_sync();
        const Tile t = tile_of(p, sh.first);
        const int rows = min(kRows, p.m - t.mt * kRows), cols = min(BN, p.n[t.w] - t.nt * BN);
#pragma unroll 1
        for (int e = (int)rank * kThreads + threadIdx.x; e < rows * BN; e += p.splits * kThreads) {
            const int r = e / BN, c = e % BN;
            if (c >= cols) continue;
            const uint32_t at = sm.ring + (r * C::kPitch + c) * 4;
            float v = 0.f;
#pragma unroll 4
            for (int s = 0; s < p.splits; ++s) v += ld_cluster(in_cta(at, s));
            store_one<KIND>(p.out[t.w], (t.mt * kRows + r) * p.out_stride[t.w] + t.nt * BN + c, v);
        }
        cluster_sync();
    }
    tc_fence_after();
    if (warp == kMmaWarp) {
        if (CG == 2) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(C::kTmemCols) : "memory");
        else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(C::kTmemCols) : "memory");
    }
}

// ---- host side --------------------------------------------------------------------------------------------------
template <int CG, int BN, int KIND>
cudaError_t go(const Maps& maps, Params p, paged::Device dev, cudaStream_t st) {
    auto kern = gemm_kernel<CG, BN, KIND>;
    static paged::Configured configured;
    const cudaError_t e = configured.ensure(reinterpret_cast<const void*>(kern), Cfg<CG, BN>::kSmemBytes, dev.id);
    if (e != cudaSuccess) return e;
    const int cluster = CG == 2 ? 2 : p.splits, most = CG == 2 ? dev.sms / 2 : p.tiles;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((p.tiles < most ? p.tiles : most) * cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = Cfg<CG, BN>::kSmemBytes;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 2;
    void* args[] = {const_cast<Maps*>(&maps), &p};
    return cudaLaunchKernelExC(&cfg, reinterpret_cast<const void*>(kern), args);
}
template <int CG, int BN>
cudaError_t go_kind(int kind, const Maps& maps, const Params& p, paged::Device dev, cudaStream_t st) {
    if (kind == PLORA_INPUT_FP32) return go<CG, BN, PLORA_INPUT_FP32>(maps, p, dev, st);
    if (kind == PLORA_INPUT_BF16) return go<CG, BN, PLORA_INPUT_BF16>(maps, p, dev, st);
    return go<CG, BN, PLORA_INPUT_FP16>(maps, p, dev, st);
}
bool aligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
bool map_bytes(CUtensorMap* tm, const void* base, long long cols, long long rows, long long stride, int box_rows) {
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)stride};
    const cuuint32_t box[2] = {kRowBytes, (cuuint32_t)box_rows}, es[2] = {1, 1};
    return paged::encode_tiled()(tm, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void*>(base), dims, strides, box, es,
                                 CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                                 CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace

cudaError_t device(paged::Device& dev) {
    static std::atomic<int> sms_of[64];
    dev = {0, 0};
    cudaError_t e = cudaGetDevice(&dev.id);
    if (e == cudaSuccess && dev.id < 64) dev.sms = sms_of[dev.id].load(std::memory_order_relaxed);
    if (e == cudaSuccess && dev.sms == 0) {
        e = cudaDeviceGetAttribute(&dev.sms, cudaDevAttrMultiProcessorCount, dev.id);
        if (e == cudaSuccess && dev.id < 64) sms_of[dev.id].store(dev.sms, std::memory_order_relaxed);
    }
    if (e != cudaSuccess) (void)cudaGetLastError();
    return e;
}

}  // namespace w8
}  // namespace plora

using namespace plora::w8;

extern "C" PLORA_API plora_status plora_gemm_fp8(const plora_gemm_fp8_args* a, void* stream) {
    if (!a || a->m < 0 || a->k < 1 || a->n_weights < 1 || a->n_weights > kMaxWeights) return PLORA_ERR_INVALID_ARG;
    if (a->out_type != PLORA_INPUT_FP32 && a->out_type != PLORA_INPUT_BF16 && a->out_type != PLORA_INPUT_FP16) return PLORA_ERR_INVALID_ARG;
    for (int i = 0; i < a->n_weights; ++i)
        if (a->n[i] < 1) return PLORA_ERR_INVALID_ARG;
    if (a->m == 0) return PLORA_OK;
    const long long packed = ((long long)a->k + 15) & ~15ll, es = a->out_type == PLORA_INPUT_FP32 ? 4 : 2;
    auto matrix = [&](const void* p, long long& stride) {
        if (!stride) stride = packed;
        return p && aligned(p, 16) && stride >= a->k && stride % 16 == 0 && stride < (1ll << 40);
    };
    long long x_stride = a->x_stride, w_stride[kMaxWeights];
    if (!matrix(a->x, x_stride) || !a->x_scale || !aligned(a->x_scale, 4) || (a->status && !aligned(a->status, 4))) return PLORA_ERR_INVALID_ARG;
    Params p{};
    p.wide = 1;
    for (int i = 0; i < a->n_weights; ++i) {
        w_stride[i] = a->w_stride[i];
        if (!matrix(a->w[i], w_stride[i]) || !a->w_scale[i] || !aligned(a->w_scale[i], 4) || !a->out[i] || !aligned(a->out[i], es))
            return PLORA_ERR_INVALID_ARG;
        p.out_stride[i] = a->out_stride[i] ? a->out_stride[i] : a->n[i];
        if (p.out_stride[i] < a->n[i]) return PLORA_ERR_INVALID_ARG;
        p.wide = p.wide && aligned(a->out[i], 32) && p.out_stride[i] * es % 32 == 0;
        p.w_scale[i] = a->w_scale[i];
        p.out[i] = a->out[i];
        p.n[i] = a->n[i];
    }
    plora::paged::Device dev;
    if (device(dev) != cudaSuccess) return PLORA_ERR_CUDA;
    if (!plora::paged::encode_tiled()) return PLORA_ERR_UNSUPPORTED;
    p.x_scale = a->x_scale;
    p.m = a->m;
    p.blocks = (int)(((long long)a->k + kBlock - 1) / kBlock);
    p.status = a->status;
    auto tiles_of = [&](int bn) {
        long long t = 0;
        for (int i = 0; i < a->n_weights; ++i) t += ((long long)a->n[i] + bn - 1) / bn;
        return t;
    };
    const bool pair = a->m > kRows;
    int bn = 64;
    p.splits = 1;
    if (pair) {
        const long long m_tiles = (a->m + 2 * kRows - 1) / (2 * kRows);
        bn = m_tiles * tiles_of(256) >= dev.sms / 2 ? 256 : 128;
    } else {
        const long long t = tiles_of(64);
        while (p.splits < 8 && t * p.splits * 2 <= 2 * dev.sms && p.blocks >= 4 * p.splits) p.splits *= 2;
    }
    const int cg = pair ? 2 : 1;
    const long long m_tiles = ((long long)a->m + cg * kRows - 1) / (cg * kRows), n_tiles = tiles_of(bn);
    if (m_tiles * n_tiles * 8 > INT32_MAX) return PLORA_ERR_UNSUPPORTED;
    p.m_tiles = (int)m_tiles;
    p.n_tiles = (int)n_tiles;
    p.tiles = (int)(m_tiles * n_tiles);
    for (int i = 0, t = 0; i < kMaxWeights; ++i) {
        if (i < a->n_weights) t += (a->n[i] + bn - 1) / bn;
        p.tile_end[i] = t;
    }
    p.x_rows = pair || a->m >= kRows ? kRows : (a->m + 7) / 8 * 8;
    Maps maps;
    if (!map_bytes(&maps.x, a->x, a->k, a->m, x_stride, p.x_rows)) return PLORA_ERR_INVALID_ARG;
    for (int i = 0; i < a->n_weights; ++i)
        if (!map_bytes(&maps.w[i], a->w[i], a->k, a->n[i], w_stride[i], bn / cg)) return PLORA_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (pair) e = bn == 256 ? go_kind<2, 256>(a->out_type, maps, p, dev, st) : go_kind<2, 128>(a->out_type, maps, p, dev, st);
    else e = go_kind<1, 64>(a->out_type, maps, p, dev, st);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();      // reported here; a later call must not find it
        return PLORA_ERR_CUDA;
    }
    return PLORA_OK;
}
