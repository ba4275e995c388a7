// Product of 8-bit activations with 8-bit weights, scaled by blocks of 128:
//     out[m, n] = sum_b  sx[m, b] sw[n / 128, b]  sum_{k in block b} x[m, k] w[n, k]
// The inner sums run on the fifth-generation tensor cores (tcgen05.mma, kind f8f6f4, e4m3 operands, fp32 accumulators in tensor
// memory): a block of K is four instructions of 32.  The scales differ from block to block, so an accumulator holds
// one block only; eight warps read it, multiply it by the two scales and add it to fp32 registers while the tensor cores fill the
// next accumulator.  (The tensor cores align a sum's 32 products and the accumulator to the largest of them and cut what lies more
// than some 24 bits below it.  Measured over single blocks of 128, against 64 bits: of normally distributed values 97 % are exact, the worst
// off by 2^-24.5 of the sum of the magnitudes; of values of all exponents the worst by 2^-21.6 of that sum, 2^-19.6 of the largest product.)
//
// Roles: warps 0-7 scale and add, a row per thread and half of the tile's columns per warpgroup; warp 8 loads (a box of x and one
// of w per block of K, 128-byte rows, swizzled); warp 9 issues the products; warps 10 and 11 stage the scales, some blocks ahead
// (loaded by the adding warps themselves, a line per row, they cost those 140 of 870 cycles per block).
//
// Forms: pairs of CTAs share tiles of 256 rows (cta_group::2: each holds half of w's rows, so that a tile needs two thirds of the copies);
// single CTAs take tiles of 128 rows, and clusters of them split K where tiles are few, each leaving its sums in shared memory for
// the others to add in the order of K.  Tiles have 64 to 256 columns; choose() estimates what is fastest.
//
// What bounds it (launches behind one another, graph replay).  Few rows: HBM (64 rows by 27648 x 5120 28.1 us, 5.3 TB/s, in a burst; 31.8 in
// a long run at the power limit), a launch's start and the first copies (12288 x 4096 by one row 12.7 us, of which 7.7 are the weights;
// 11.3 where the caller says that they are ready).  Many rows: 4096 x 8192 x 8192 takes 300 us, 1.8 PFLOP/s at the power limit of 1000 W and
// 1.5 to 1.6 GHz.  Without its reads and additions it takes 241, with the reads alone 262: tensor memory serves the products and the
// reads, and energy goes into both.  (The library's product of the same operands with one scale for all takes 228 for long, 185 in a burst.)
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
constexpr long long kMaxTiles = 1 << 28;  // of 128 rows and 64 columns (no form has more): tile numbers times kGroup are counted in 32 bits
constexpr int kThreads = 384, kAddWarps = 8, kLoadWarp = 8, kMmaWarp = 9, kScaleWarp = 10;      // (two of the last)
constexpr int kRows = 128;                // rows of x per CTA
constexpr int kRowBytes = 128;            // one block of K
constexpr int kScaleRun = 8, kScaleSlots = 2;          // blocks of K whose scales are staged together; such runs
constexpr int kScaleBytes = kScaleRun * (kRows + 4) * 4;    // of a run: sx [block][row], then sw [block][half of the columns][2]
constexpr int kMaxStages = 16, kPairBytes = 200 * 1024;
constexpr int kRingOffset = (kScaleSlots * kScaleBytes + 512 + 1023) / 1024 * 1024;        // scales, barriers and words lie in front of the ring
constexpr long long kWaitCycles = 4000000000ll;      // limit of a wait unless the caller sets one: about two seconds of SM clock

// CG: CTAs that share a tile (cta_group); BN: columns of the tile, a multiple of 32.
// Narrow tiles of single CTAs leave room for a second CTA on the SM, so that one starts or ends while the other streams (7.6 against
// 11 us for 16 rows by 4096 x 4096, a launch behind another); the others have the SM to themselves.
template <int CG, int BN>
struct Cfg {
    static constexpr int kCtas = CG == 1 && BN == 64 ? 2 : 1;
    static constexpr int kTmemCols = 512 / kCtas, kSmemMost = kCtas == 2 ? 112 * 1024 : 227 * 1024;
    static constexpr int kBBytes = BN / CG * kRowBytes;
    // Blocks of K per stage and accumulator: two where tensor memory holds two such accumulators (a block's hand-overs cost some 600
    // cycles whatever its size: one row by 12288 x 4096 weights in tiles of 64 columns 14.2 us with one, 12.1 with two).
    static constexpr int kRun = BN <= 128 ? 2 : 1;
    static constexpr int kAccs = kTmemCols / (BN * kRun) > 4 ? 4 : kTmemCols / (BN * kRun);
    static constexpr int kCols = BN / 2;                  // columns of a thread
    static constexpr bool kCrosses = kBlock % kCols != 0; // a half may lie in two blocks of w's rows
    // Columns read from tensor memory at a time: 32 (4 % faster in tiles of 160 columns), but 16 where the halves are multiples of 32,
    // for reads of 32 take far longer there (tiles of 256 columns 359 against 294 us for 4096 x 8192 x 8192, of 128 367 against 329).
    static constexpr int kRead = kCols % 32 == 0 ? 16 : 32;
    static constexpr int kPitch = BN + 4; // floats between the rows of a partial tile in shared memory (4 banks apart, accesses of 16 bytes)
    static_assert(BN % 32 == 0 && kBBytes % 1024 == 0, "");
};

// The sticky status word of calls that bring none.
__device__ int32_t default_status;

struct Params {
    const float* x_scale;
    const float* w_scale[kMaxWeights];
    void* out[kMaxWeights];
    long long out_stride[kMaxWeights];
    int32_t n[kMaxWeights], tile_end[kMaxWeights];     // columns; tiles of columns up to and with this weight's
    int32_t m, blocks, m_tiles, n_tiles, tiles, splits, x_rows;   // blocks of K; x_rows: rows of a box of x
    int32_t stages, x_bytes;                           // of the ring; bytes of a stage's box of x, a multiple of 1024
    int32_t quads;                                     // groups of 32 rows of a tile that have rows (4 if any tile is full)
    int32_t test_hook;                                 // PLORA_HOOK_*: tests make a wait run out with it
    long long wait_cycles;                             // limit of a wait
    int32_t weights_ready;                             // the caller's word that w was complete before the kernel in front began
    int32_t vec;                                       // bytes that every row of every output is aligned to: 32, 16, or fewer
    int32_t* status;                                   // nullptr: default_status
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
__device__ __forceinline__ float lds32(uint32_t a) {
    float v;
    asm volatile("ld.shared.f32 %0, [%1];" : "=f"(v) : "r"(a));
    return v;
}
__device__ __forceinline__ float2 lds64(uint32_t a) {
    float2 v;
    asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(a));
    return v;
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
__device__ __forceinline__ int opaque(int v) {     // the same value, but the compiler does not know
    asm volatile("" : "+r"(v));
    return v;
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
// An arrival by the lanes that say so, without a branch.  REMOTE: at a barrier of the cluster; it hands nothing over in memory, only the
// right to tensor memory, whose reads are complete (a release at cluster scope cost the warps that add some 800 cycles per block of K).
template <bool REMOTE>
__device__ __forceinline__ void arrive_if(uint32_t bar, bool yes) {
    if (REMOTE)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %1, 0;\n\t@p mbarrier.arrive.relaxed.cluster.shared::cluster.b64 _, [%0];\n\t}" ::"r"(bar),
            "r"((uint32_t)yes)
            : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %1, 0;\n\t@p mbarrier.arrive.shared::cta.b64 _, [%0];\n\t}" ::"r"(bar), "r"((uint32_t)yes)
                     : "memory");
}
__device__ __forceinline__ float4 ld_cluster(uint32_t a) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
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
    long long limit;
};
__device__ __forceinline__ bool wait_slow(uint32_t bar, uint32_t parity, WaitCtl w) {
    const long long t0 = clock64();
#pragma unroll 1
    for (uint32_t n = 1;; ++n) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((n & 63) == 0 && (*w.abort_flag || clock64() - t0 > w.limit)) break;
    }
    if (!*w.abort_flag) atomicCAS(w.status, 0, PLORA_ERR_TIMEOUT);
    *w.abort_flag = 1;
    return false;
}
__device__ __forceinline__ bool wait(uint32_t bar, uint32_t parity, const WaitCtl& w) {
    return mbar_try_wait(bar, parity) || wait_slow(bar, parity, w);
}

// A place in a ring of N, and the parity of the turn.
template <uint32_t N>
struct Turn {
    uint32_t at = 0, parity = 0;
    __device__ __forceinline__ void next(uint32_t n = N) {
        if (++at == n) {
            at = 0;
            parity ^= 1;
        }
    }
};

// ---- the tiles ----------------------------------------------------------------------------------------------------
// Tiles are numbered so that those under way at one time (some 74) form a near-square of x and w: runs of kGroup tiles of rows by all
// tiles of columns.
constexpr int kGroup = 8;
static_assert(kMaxTiles * kGroup <= (1ll << 31), "");
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
template <int CG, int RUN>
__device__ __forceinline__ Share share_of(const Params& p, uint32_t rank) {
    if (CG == 2 || p.splits == 1) return {(int)blockIdx.x / CG, (int)gridDim.x / CG, 0, p.blocks};
    const int per = ((p.blocks + p.splits - 1) / p.splits + RUN - 1) / RUN * RUN, b0 = min((int)rank * per, p.blocks);
    return {(int)blockIdx.x / p.splits, p.tiles, b0, min(b0 + per, p.blocks)};
}

struct Smem {
    uint32_t ring, full, empty, acc_full, acc_empty, scale_full, scale_empty, done, peer;
    float* scales;       // [run]: sx [block][row], then sw [block][half of the columns][2]
    uint32_t* tmem_slot;
    WaitCtl wc;
};

// Warps 8 and 9 stay together and an elected lane issues: copies and products take uniform registers, and in a branch of a single
// lane each of them costs 100 cycles and more (the first form of this kernel: 1900 cycles per block of K instead of 512).
template <int CG, int BN>
__device__ __forceinline__ void load_warp(const Params& p, const Maps& maps, const Smem& sm, uint32_t rank) {
    using C = Cfg<CG, BN>;
    const unsigned all = 0xffffffffu;
    const Share sh = share_of<CG, Cfg<CG, BN>::kRun>(p, rank);
    const uint32_t bytes = CG * C::kRun * (uint32_t)(p.x_rows * kRowBytes + C::kBBytes);
    const uint32_t ring = uniform(sm.ring), full = uniform(sm.full), counts = uniform(CG == 2 ? in_cta(sm.full, 0) : sm.full);
    uint32_t it = 0, early = 0;
    Turn<0> turn;
    const uint32_t stages = p.stages, stage_bytes = C::kRun * (p.x_bytes + C::kBBytes);
    bool stopped = false;
    // Where the caller says that they were complete before the kernel in front began, the weights of the first stages are fetched
    // before that kernel has completed (one row by 12288 x 4096 11.3 us so, 12.7 behind it).  Nothing here shows whether that kernel
    // writes them: it may let this one start before it has, and even if it does not, its writes are visible only behind the wait.
    auto begin = [&](uint32_t s, const Tile& t, int b) {
        if (elect_one()) {
            if (CG == 1 || rank == 0) mbar_arrive_expect_tx(full + s * 8, bytes);
#pragma unroll
            for (int j = 0; j < C::kRun; ++j)        // (what lies beyond K reads as zeros)
                tma_box<CG>(ring + s * stage_bytes + C::kRun * p.x_bytes + j * C::kBBytes, &maps.w[t.w], (b + j) * kRowBytes,
                            t.nt * BN + (CG == 2 ? (int)rank * (BN / 2) : 0), counts + s * 8);
        }
    };
    auto finish = [&](uint32_t s, const Tile& t, int b) {
        if (elect_one())
#pragma unroll
            for (int j = 0; j < C::kRun; ++j)
                tma_box<CG>(ring + s * stage_bytes + j * p.x_bytes, &maps.x, (b + j) * kRowBytes, (t.mt * CG + (CG == 2 ? (int)rank : 0)) * kRows,
                            counts + s * 8);
    };
    if (!p.weights_ready) paged::grid_wait();
    if (sh.first < p.tiles) {
        const Tile t = tile_of(p, sh.first);
        for (int b = sh.b0; early < stages && b < sh.b1; ++early, b += C::kRun) begin(early, t, b);
    }
    paged::grid_wait();
#pragma unroll 1
    for (int i = sh.first; i < p.tiles && !stopped; i += sh.step) {
        const Tile t = tile_of(p, i);
#pragma unroll 1
        for (int b = sh.b0; b < sh.b1; b += C::kRun, ++it, turn.next(stages)) {
            if (it >= early) {
                if (!__all_sync(all, wait(sm.empty + turn.at * 8, turn.parity ^ 1, sm.wc))) {
                    stopped = true;
                    break;
                }
                begin(turn.at, t, b);
            }
            finish(turn.at, t, b);
        }
    }
    const uint32_t n = max(it, early);
    if (!stopped) {
        // the products' last signals come from the pair's first CTA: they must have come before the second one leaves
        if (CG == 2)
            for (uint32_t j = n > stages ? n - stages : 0; j < n; ++j) wait(sm.empty + j % stages * 8, (j / stages) & 1, sm.wc);
    } else if (CG == 1 || rank == 0) {
        // copies in flight must land before the CTA leaves (in a pair they are counted by the first CTA's barriers): one limit for all
        // of them, for a stage that the pair's other CTA never asked for does not fill
        const long long t0 = clock64();
        for (uint32_t j = n > stages ? n - stages : 0; j < n; ++j)
            paged::mbar_drain(sm.full + j % stages * 8, (j / stages) & 1, sm.wc.limit - (clock64() - t0));
    }
}

template <int CG, int BN>
__device__ __forceinline__ void mma_warp(const Params& p, const Smem& sm, uint32_t tmem, uint32_t rank) {
    using C = Cfg<CG, BN>;
    const unsigned all = 0xffffffffu;
    const Share sh = share_of<CG, Cfg<CG, BN>::kRun>(p, rank);
    constexpr uint32_t idesc = instr_desc(CG * kRows, BN);
    constexpr uint32_t kHi = (uint32_t)(smem_desc(0) >> 32), kLo = (uint32_t)smem_desc(0);
    const uint32_t ring = uniform(sm.ring >> 4), empty = uniform(sm.empty), acc_full = uniform(sm.acc_full);
    tmem = uniform(tmem);
    Turn<0> turn;
    const uint32_t stages = p.stages, stage_step = C::kRun * (p.x_bytes + C::kBBytes) >> 4, x_step = p.x_bytes >> 4;
    Turn<C::kAccs> acc;
    bool stopped = false;
    // Both barriers of a block are tried at once, right behind the block before: a try's answer takes some 100 cycles, and
    // with one after the other this warp took longer than the products.
    bool go_acc = mbar_try_wait(sm.acc_empty, 1), go_full = false;
    if (sh.first < p.tiles && sh.b0 < sh.b1) go_full = mbar_try_wait(sm.full, 0);
#pragma unroll 1
    for (int i = sh.first; i < p.tiles && !stopped; i += sh.step) {
#pragma unroll 1
        for (int b = sh.b0; b < sh.b1; b += C::kRun) {
            if (!__all_sync(all, go_acc && go_full)) {
                if (!__all_sync(all, wait(sm.acc_empty + acc.at * 8, acc.parity ^ 1, sm.wc) && wait(sm.full + turn.at * 8, turn.parity, sm.wc))) {
                    stopped = true;
                    break;
                }
            }
            tc_fence_after();
            const uint32_t da = (ring + turn.at * stage_step) | kLo, db = da + C::kRun * x_step;
            if (elect_one()) {
#pragma unroll
                for (int j = 0; j < C::kRun; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k)
                        umma<CG>(tmem + (acc.at * C::kRun + j) * BN, desc_of(da + j * x_step + 2 * k, kHi),
                                 desc_of(db + j * (C::kBBytes >> 4) + 2 * k, kHi), idesc, k > 0);
                umma_commit<CG, true>(acc_full + acc.at * 8);
                umma_commit<CG, true>(empty + turn.at * 8);
            }
            turn.next(stages);
            acc.next();
            // (not behind the last block: a try sleeps for microseconds if nothing comes)
            if (b + C::kRun < sh.b1 || i + sh.step < p.tiles) {
                go_acc = mbar_try_wait(sm.acc_empty + acc.at * 8, acc.parity ^ 1);
                go_full = mbar_try_wait(sm.full + turn.at * 8, turn.parity);
            }
        }
    }
    // no product is under way when tensor memory is given back
    if (elect_one()) umma_commit<CG, false>(sm.done);
    if (!paged::mbar_drain(sm.done, 0, sm.wc.limit)) atomicCAS(sm.wc.status, 0, PLORA_ERR_TIMEOUT);
}

template <int KIND>
__device__ __forceinline__ void store_one(void* out, long long at, float v) {
    if (KIND == PLORA_INPUT_FP32) static_cast<float*>(out)[at] = v;
    else static_cast<uint16_t*>(out)[at] = (uint16_t)pack16<KIND == PLORA_INPUT_FP16>(v, 0.f);
}

// Four columns of a row, of which `left` exist.
template <int KIND>
__device__ __forceinline__ void store_four(void* out, long long at, float4 v, int left, int vec) {
    if (left >= 4 && vec >= (KIND == PLORA_INPUT_FP32 ? 16 : 8)) {
        if (KIND == PLORA_INPUT_FP32) *reinterpret_cast<float4*>(static_cast<float*>(out) + at) = v;
        else *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + at) = make_uint2(pack16<KIND == PLORA_INPUT_FP16>(v.x, v.y), pack16<KIND == PLORA_INPUT_FP16>(v.z, v.w));
        return;
    }
    const float f[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i)
        if (i < left) store_one<KIND>(out, at + i, f[i]);
}

// First of the (at most two) blocks of w's rows that columns [col, ..) lie in, and the columns up to the next one.
__device__ __forceinline__ int block_of(int col) { return col / kBlock; }
__device__ __forceinline__ int left_in_block(int col) { return kBlock - col % kBlock; }

// Warps 10 and 11: the scales of the rows, two rows per thread, and of the halves' columns.
template <int CG, int BN>
__device__ __forceinline__ void scale_warps(const Params& p, const Smem& sm, uint32_t rank) {
    using C = Cfg<CG, BN>;
    const Share sh = share_of<CG, Cfg<CG, BN>::kRun>(p, rank);
    const int lane = threadIdx.x & 31, r0 = threadIdx.x - kScaleWarp * 32;
    Turn<kScaleSlots> turn;
    paged::grid_wait();
#pragma unroll 1
    for (int i = sh.first; i < p.tiles; i += sh.step) {
        const Tile t = tile_of(p, i);
        const int row0 = (t.mt * CG + (CG == 2 ? (int)rank : 0)) * kRows;
        const float *x0 = p.x_scale + (size_t)min(row0 + r0, p.m - 1) * p.blocks, *x1 = p.x_scale + (size_t)min(row0 + r0 + 64, p.m - 1) * p.blocks;
        // thread 4 j + 2 h + i of the first 32: block j of the run, half h, i-th of its blocks
        const int j4 = r0 >> 2, wb = block_of(t.nt * BN + (r0 >> 1 & 1) * C::kCols) + (r0 & 1);
        const float* w0 = p.w_scale[t.w] + (size_t)min(wb, block_of(p.n[t.w] - 1)) * p.blocks;
#pragma unroll 1
        for (int b = sh.b0; b < sh.b1; b += kScaleRun, turn.next()) {
            float x[2][kScaleRun], w = 0.f;
#pragma unroll
            for (int j = 0; j < kScaleRun; ++j) {
                const bool there = b + j < sh.b1;        // (a block beyond the last one counts nothing)
                x[0][j] = there ? x0[b + j] : 0.f;
                x[1][j] = there ? x1[b + j] : 0.f;
            }
            if (r0 < 4 * kScaleRun && b + j4 < sh.b1) w = w0[b + j4];
            if (!__all_sync(0xffffffffu, wait(sm.scale_empty + turn.at * 8, turn.parity ^ 1, sm.wc))) return;
            float* s = sm.scales + turn.at * (kScaleBytes / 4);
#pragma unroll
            for (int j = 0; j < kScaleRun; ++j) {
                s[j * kRows + r0] = x[0][j];
                s[j * kRows + r0 + 64] = x[1][j];
            }
            if (r0 < 4 * kScaleRun) s[kScaleRun * kRows + r0] = w;
            __syncwarp();
            if (lane == 0) mbar_arrive(sm.scale_full + turn.at * 8);
        }
    }
}

// Scales and adds the accumulators of one tile: row (warp & 3) * 32 + lane of the CTA's, half warp >> 2 of the columns, of which the
// first `first` lie in the half's first block.  These warps bound the kernel (a block took them 1010 cycles in tiles of 256 columns, 520
// of them to read and add), so a block's scales are fetched while the one before it is read, and places and addresses are kept.
template <int CG, int BN>
__device__ __forceinline__ bool add_tile(const Smem& sm, uint32_t from, uint32_t hand_back, bool hands_back, int blocks, bool any, int first, Turn<Cfg<CG, BN>::kAccs>& in,
                                         Turn<kScaleSlots>& run, float2 (&acc)[Cfg<CG, BN>::kCols / 2]) {
    using C = Cfg<CG, BN>;
    const unsigned all = 0xffffffffu;
    const int lane = threadIdx.x & 31;
    const uint32_t sx = smem_u32(sm.scales) + (threadIdx.x & 127) * 4, sw = smem_u32(sm.scales) + kScaleRun * kRows * 4 + (threadIdx.x >> 7) * 8;
#pragma unroll
    for (int i = 0; i < C::kCols / 2; ++i) acc[i] = make_float2(0.f, 0.f);
#pragma unroll 1
    for (; blocks > 0; blocks -= kScaleRun, run.next()) {
        if (!__all_sync(all, wait(sm.scale_full + run.at * 8, run.parity, sm.wc))) return false;
        float x[C::kRun];
        float2 w[C::kRun];
        auto fetch = [&](int j) {
#pragma unroll
            for (int r = 0; r < C::kRun; ++r) {
                x[r] = lds32(sx + run.at * kScaleBytes + (j + r) * kRows * 4);
                w[r] = lds64(sw + run.at * kScaleBytes + (j + r) * 16);
            }
        };
        fetch(0);
        const int here = min(blocks, kScaleRun);
#pragma unroll 1
        for (int j = 0; j < here; j += C::kRun, in.next()) {
            const uint32_t a = in.at;
            if (!__all_sync(all, wait(sm.acc_full + a * 8, in.parity, sm.wc))) return false;
            tc_fence_after();
            if (any) {        // (a row of this warp exists)
                uint32_t buf[C::kRead];
                tmem_ld<C::kRead>(from + a * C::kRun * BN, buf);
                float2 f[C::kRun], g[C::kRun];        // the scales in the half's first and second block
#pragma unroll
                for (int r = 0; r < C::kRun; ++r) {
                    f[r] = make_float2(x[r] * w[r].x, x[r] * w[r].x);
                    g[r] = C::kCrosses ? make_float2(x[r] * w[r].y, x[r] * w[r].y) : f[r];
                }
                if (j + C::kRun < here) fetch(j + C::kRun);
#pragma unroll
                for (int r = 0; r < C::kRun; ++r)
#pragma unroll
                    for (int c = 0; c < C::kCols; c += C::kRead) {
                        const bool whole = c + C::kRead <= C::kCols;        // (or the last 16 columns)
                        if (r > 0 || c > 0) {
                            if (whole) tmem_ld<C::kRead>(from + (a * C::kRun + r) * BN + c, buf);
                            else tmem_ld<16>(from + (a * C::kRun + r) * BN + c, buf);
                        }
                        tmem_ld_wait();
                        const float* v = reinterpret_cast<const float*>(buf);
#pragma unroll
                        for (int e = 0; e < (whole ? C::kRead / 2 : 8); ++e) {
                            float2& o = acc[c / 2 + e];
                            o = __ffma2_rn(make_float2(v[2 * e], v[2 * e + 1]), C::kCrosses && c + e / 8 * 16 >= first ? g[r] : f[r], o);
                        }
                    }
            }
            tc_fence_before();
            arrive_if<CG == 2>(hand_back + a * 8, hands_back);        // (the warp's reads are complete: it reads as one)
        }
        __syncwarp();
        arrive_if<false>(sm.scale_empty + run.at * 8, lane == 0);
    }
    return true;
}

// 32 bytes of a row.
template <int KIND>
__device__ __forceinline__ void words_of(const float* v, uint32_t (&w)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i)
        w[i] = KIND == PLORA_INPUT_FP32 ? __float_as_uint(v[i]) : pack16<KIND == PLORA_INPUT_FP16>(v[KIND == PLORA_INPUT_FP32 ? 0 : 2 * i], v[KIND == PLORA_INPUT_FP32 ? 0 : 2 * i + 1]);
}
// Row `row` of the tile's half, kCols columns from `col` on: each lane writes its row in pieces of 32 bytes.  (Four lanes to a piece of 64
// bytes through shared memory took as long: what a tile's end waits for is the write itself, 128 KB per CTA.)
template <int CG, int BN, int KIND>
__device__ __forceinline__ void store_tile(const Params& p, const Tile& t, int row, int col, const float2 (&acc)[Cfg<CG, BN>::kCols / 2]) {
    using C = Cfg<CG, BN>;
    if (row >= p.m) return;
    const int n = p.n[t.w];
    const long long at = row * p.out_stride[t.w] + col;
    constexpr int kSize = KIND == PLORA_INPUT_FP32 ? 4 : 2, kStep = 32 / kSize;       // columns of a 32-byte store
#pragma unroll
    for (int c = 0; c < C::kCols; c += kStep) {
        const float* v = reinterpret_cast<const float*>(acc) + c;
        if (p.vec >= 16 && col + c + kStep <= n) {
            uint32_t w[8];
            words_of<KIND>(v, w);
            char* o = static_cast<char*>(p.out[t.w]) + (at + c) * kSize;
            if (p.vec == 32) {
                st_global32(o, w);
            } else {
                *reinterpret_cast<uint4*>(o) = make_uint4(w[0], w[1], w[2], w[3]);
                *reinterpret_cast<uint4*>(o + 16) = make_uint4(w[4], w[5], w[6], w[7]);
            }
        } else {
#pragma unroll
            for (int i = 0; i < kStep; ++i)
                if (col + c + i < n) store_one<KIND>(p.out[t.w], at + c + i, v[i]);
        }
    }
}

template <int CG, int BN, int KIND>
__global__ void __launch_bounds__(kThreads, Cfg<CG, BN>::kCtas) gemm_kernel(const __grid_constant__ Maps maps, const __grid_constant__ Params p) {
    using C = Cfg<CG, BN>;
    extern __shared__ uint8_t raw[];
    uint8_t* base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    uint8_t* bars = base + kScaleSlots * kScaleBytes;
    Smem sm;
    // scales, barriers and words first: products read 128 rows of x from a stage whatever its box has, and what they read behind
    // it has to be this CTA's (the host leaves room behind the last stage); it goes into rows that nobody takes
    sm.ring = smem_u32(base) + kRingOffset;
    sm.full = smem_u32(bars);
    sm.empty = sm.full + kMaxStages * 8;
    sm.acc_full = sm.empty + kMaxStages * 8;
    sm.acc_empty = sm.acc_full + C::kAccs * 8;
    sm.scale_full = sm.acc_empty + C::kAccs * 8;
    sm.scale_empty = sm.scale_full + kScaleSlots * 8;
    sm.done = sm.scale_empty + kScaleSlots * 8;
    sm.peer = sm.done + 8;
    sm.scales = reinterpret_cast<float*>(base);
    constexpr int kBars = 2 * kMaxStages + 2 * C::kAccs + 2 * kScaleSlots + 2;
    static_assert(kScaleSlots * kScaleBytes + kBars * 8 + 16 <= kRingOffset, "");
    sm.tmem_slot = reinterpret_cast<uint32_t*>(bars + kBars * 8);
    sm.wc.abort_flag = reinterpret_cast<volatile int*>(bars + kBars * 8 + 8);
    sm.wc.status = p.status ? p.status : &default_status;
    sm.wc.limit = p.wait_cycles;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) {
            mbar_init(sm.full + s * 8, 1);
            mbar_init(sm.empty + s * 8, 1);
        }
        for (int a = 0; a < C::kAccs; ++a) {
            mbar_init(sm.acc_full + a * 8, 1);
            mbar_init(sm.acc_empty + a * 8, kAddWarps / 4 * p.quads * CG);
        }
        for (int r = 0; r < kScaleSlots; ++r) {
            mbar_init(sm.scale_full + r * 8, 2);
            mbar_init(sm.scale_empty + r * 8, kAddWarps / 4 * p.quads);
        }
        mbar_init(sm.done, 1);
        mbar_init(sm.peer, 1);
        sm.wc.abort_flag[0] = 0;
        mbar_init_fence();
    }
    if (warp == kLoadWarp && lane == 0) {
        prefetch_map(&maps.x);
        prefetch_map(&maps.w[0]);
    }
    __syncthreads();
    if (CG == 2) cluster_sync();        // the other CTA's barriers exist
    // Tensor memory is taken when the kernel in front has completed, not before: it may have let this one start before it took
    // its own.  The next kernel may start when this one has its tensor memory.
    uint32_t tmem = 0;
    auto tmem_taken = [&] {
        asm volatile("bar.sync 1, %0;" ::"n"((kAddWarps + 1) * 32) : "memory");
        tc_fence_after();
        tmem = *sm.tmem_slot;
    };
    const Share sh = share_of<CG, Cfg<CG, BN>::kRun>(p, rank);
    if (warp < kAddWarps) {
        if (BN > 192) asm volatile("setmaxnreg.inc.sync.aligned.u32 224;");
        paged::grid_wait();
        tmem_taken();
        if (threadIdx.x == 0) paged::grid_launch_dependents();
        const int r = (CG == 2 ? (int)rank * kRows : 0) + (warp & 3) * 32 + lane, c = (warp >> 2) * C::kCols;
        const uint32_t from = tmem + ((uint32_t)(warp & 3) << 21) + c, hand_back = CG == 2 ? in_cta(sm.acc_empty, 0) : sm.acc_empty;
        const bool hands_back = lane == 0 && !(p.test_hook == PLORA_HOOK_WITHHOLD_RELEASE && warp == 0);
        Turn<C::kAccs> in;
        Turn<kScaleSlots> run;
        float2 acc[C::kCols / 2];
        // (warps whose rows no tile has leave at once: one row by 12288 x 4096, weights ready, 11.5 -> 11.35 us)
#pragma unroll 1
        for (int i = (warp & 3) < p.quads ? sh.first : p.tiles; i < p.tiles; i += sh.step) {
            const Tile u = tile_of(p, i);
            if (!add_tile<CG, BN>(sm, from, hand_back, hands_back, sh.b1 - sh.b0, u.mt * CG * kRows + r - lane < p.m, left_in_block(u.nt * BN + c), in, run, acc)) break;
            const Tile t = tile_of(p, opaque(i));       // (made again rather than kept beside the sums)
            const int row = t.mt * CG * kRows + r, col = t.nt * BN + c;
            if (CG == 2 || p.splits == 1) {
                store_tile<CG, BN, KIND>(p, t, row, col, acc);
            } else if (row < p.m) {       // all products are complete: the ring is free for the partial tile
                float4* part = reinterpret_cast<float4*>(base + kRingOffset) + (r * C::kPitch + c) / 4;
#pragma unroll
                for (int e = 0; e < C::kCols / 4; ++e) part[e] = make_float4(acc[2 * e].x, acc[2 * e].y, acc[2 * e + 1].x, acc[2 * e + 1].y);
            }
        }
    } else {
        if (BN > 192) asm volatile("setmaxnreg.dec.sync.aligned.u32 56;");
        if (warp == kLoadWarp) load_warp<CG, BN>(p, maps, sm, rank);
        if (warp == kMmaWarp) {
            paged::grid_wait();
            if (CG == 2) {
                asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(sm.tmem_slot)), "n"(C::kTmemCols) : "memory");
                asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
            } else {
                asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(sm.tmem_slot)), "n"(C::kTmemCols) : "memory");
                asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
            }
            tc_fence_before();
            tmem_taken();
            if (CG == 2 && rank == 1) arrive_if<true>(in_cta(sm.peer, 0), lane == 0);        // products write into this CTA's, too
            else if (CG == 1 || __all_sync(0xffffffffu, wait(sm.peer, 0, sm.wc))) mma_warp<CG, BN>(p, sm, tmem, rank);
        }
        if (warp >= kScaleWarp) scale_warps<CG, BN>(p, sm, rank);
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
        for (int e = (int)rank * kThreads + threadIdx.x; e < rows * (BN / 4); e += p.splits * kThreads) {
            const int r = e / (BN / 4), c = e % (BN / 4) * 4;
            if (c >= cols) continue;
            const uint32_t at = sm.ring + (r * C::kPitch + c) * 4;
            float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
            for (int s = 0; s < p.splits; ++s) {
                const float4 o = ld_cluster(in_cta(at, s));
                v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
            }
            store_four<KIND>(p.out[t.w], (t.mt * kRows + r) * p.out_stride[t.w] + t.nt * BN + c, v, cols - c, p.vec);
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
    using C = Cfg<CG, BN>;
    auto kern = gemm_kernel<CG, BN, KIND>;
    static paged::Configured configured;
    const cudaError_t e = configured.ensure(reinterpret_cast<const void*>(kern), C::kSmemMost, dev.id);
    if (e != cudaSuccess) return e;
    const int cluster = CG == 2 ? 2 : p.splits, most = p.splits > 1 ? p.tiles : dev.sms * C::kCtas / CG;
    // As deep a ring as fits, with 128 rows of x (or the rows of a partial tile) behind the start of its last stage.
    const int stage = C::kRun * (p.x_bytes + C::kBBytes), room = C::kSmemMost - 1024 - kRingOffset;
    const int last_x = stage - (C::kRun - 1) * p.x_bytes, behind = kRows * kRowBytes > last_x ? kRows * kRowBytes - last_x : 0;
    p.stages = (room - behind) / stage;
    if (p.stages > kMaxStages) p.stages = kMaxStages;
    const int stages_of_k = (p.blocks + C::kRun - 1) / C::kRun;
    if (p.tiles <= most && p.stages > stages_of_k) p.stages = stages_of_k;        // (a CTA has one tile)
    int ring = p.stages * stage + behind;
    const int rows = p.m < kRows ? p.m : kRows, part = p.splits > 1 ? rows * C::kPitch * 4 : 0;
    if (ring < part) ring = part;
    // (A pair takes tensor memory on two SMs: it has both to itself, so that it never holds one half while a kernel of another stream
    // that holds the other waits for a CTA of its own.)
    int smem = 1024 + kRingOffset + ring;
    if (CG == 2 && smem < kPairBytes) smem = kPairBytes;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3((unsigned)((p.tiles < most ? p.tiles : most) * cluster));
    cfg.blockDim = dim3(kThreads);
    cfg.dynamicSmemBytes = smem;
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
template <int CG>
cudaError_t go_bn(int bn, int kind, const Maps& maps, const Params& p, paged::Device dev, cudaStream_t st) {
    switch (bn) {
        case 64: return go_kind<CG, 64>(kind, maps, p, dev, st);
        case 96: return go_kind<CG, 96>(kind, maps, p, dev, st);
        case 128: return go_kind<CG, 128>(kind, maps, p, dev, st);
        case 160: return go_kind<CG, 160>(kind, maps, p, dev, st);
        case 192: return go_kind<CG, 192>(kind, maps, p, dev, st);
        case 224: return go_kind<CG, 224>(kind, maps, p, dev, st);
        default: return go_kind<CG, 256>(kind, maps, p, dev, st);
    }
}
bool aligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

// How a call is cut: single CTAs or pairs, columns of a tile, and parts that a tile's K is split into (a cluster of single CTAs).
// Taken is the form whose estimate is least; the estimate is the time of a block of K in a CTA times the blocks that a CTA has, and
// what a tile costs besides.  Its constants are measured: 60 bytes per ns and SM of what comes from HBM (one tile of rows), 75 of what
// mostly comes from L2, 6500 from HBM in all; 1600 cycles per us under load; the hand-over of accumulators, which bounds wide tiles.
// Of 37 calls of 1 to 4096 rows, 320 to 27648 columns and K up to 13824 it chose the fastest form, or one within 13 %, for all but one
// (28 % behind, 5.4 against 4.2 us).
struct Form {
    int cg, bn, splits;
};
Form choose(const plora_gemm_fp8_args* a, int blocks, int sms) {
    Form best{1, 64, 1};
    double least = 1e30;
    const int size = a->out_type == PLORA_INPUT_FP32 ? 4 : 2, x_rows = a->m < kRows ? a->m : kRows;
    for (int cg = 1; cg <= (a->m > kRows ? 2 : 1); ++cg) {
        const long long rows = ((long long)a->m + cg * kRows - 1) / (cg * kRows);
        for (int bn = 64; bn <= 256; bn += 32) {
            long long cols = 0;
            for (int i = 0; i < a->n_weights; ++i) cols += ((long long)a->n[i] + bn - 1) / bn;
            const double hand_over = bn <= 128 ? 0.17 : bn == 160 ? 0.37 : 0.12 + 0.0017 * bn;
            const bool two = cg == 1 && bn == 64;        // CTAs on an SM
            for (int s = 1; s <= (cg == 1 ? 8 : 1) && (s == 1 || blocks >= 2 * s); ++s) {
                if (s > 1 && rows * cols * (s - 1) >= sms * (two ? 2 : 1)) break;        // (one part less fills the SMs already)
                // (clusters do not fill the processing clusters of 16 to 20 SMs that they have to lie in: percent of the CTAs that
                // fit at one time, by the size of a cluster, as the occupancy query gives them on a B200)
                static const int fit[2][9] = {{0, 100, 100, 91, 89, 87, 89, 70, 81}, {0, 100, 100, 94, 95, 94, 91, 87, 89}};
                const long long slots = (long long)sms * (two ? 2 : 1) * fit[two][s] / 100;
                const long long ctas = rows * cols * s * cg, rounds = (ctas + slots - 1) / slots, active = ctas < slots ? ctas : slots;
                const double on_sm = active > sms ? 2 : 1;
                double t = (x_rows + bn / cg) * kRowBytes * on_sm / (rows == 1 ? 60e3 : 75e3);
                const double products = bn * 2 * on_sm / 1600, hbm = (double)active * (bn / cg) * kRowBytes / rows / 6.5e6;
                t = products > t ? products : t;
                t = hand_over > t ? hand_over : t;
                t = hbm > t ? hbm : t;
                const double us = 3 + rounds * ((blocks + s - 1) / s * t + (double)x_rows * bn * size / 28e3) + (s > 1 ? 2 + 3 * (rounds - 1) + (double)x_rows * bn / 10e3 : 0);
                if (us < least) {
                    least = us;
                    best = Form{cg, bn, s};
                }
            }
        }
    }
    return best;
}
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
    if (a->weights_ready != 0 && a->weights_ready != 1) return PLORA_ERR_INVALID_ARG;
    if (a->wait_cycles < 0 || (a->test_hook != PLORA_HOOK_NONE && a->test_hook != PLORA_HOOK_WITHHOLD_RELEASE)) return PLORA_ERR_INVALID_ARG;
    if (a->test_hook != PLORA_HOOK_NONE && (a->wait_cycles < 1 || a->wait_cycles > PLORA_HOOK_MAX_CYCLES)) return PLORA_ERR_INVALID_ARG;
    if (a->m == 0) return PLORA_OK;
    const long long packed = ((long long)a->k + 15) & ~15ll, es = a->out_type == PLORA_INPUT_FP32 ? 4 : 2;
    auto matrix = [&](const void* p, long long& stride) {
        if (!stride) stride = packed;
        return p && aligned(p, 16) && stride >= a->k && stride % 16 == 0 && stride < (1ll << 40);
    };
    long long x_stride = a->x_stride, w_stride[kMaxWeights];
    if (!matrix(a->x, x_stride) || !a->x_scale || !aligned(a->x_scale, 4) || (a->status && !aligned(a->status, 4))) return PLORA_ERR_INVALID_ARG;
    Params p{};
    p.vec = 32;
    for (int i = 0; i < a->n_weights; ++i) {
        w_stride[i] = a->w_stride[i];
        if (!matrix(a->w[i], w_stride[i]) || !a->w_scale[i] || !aligned(a->w_scale[i], 4) || !a->out[i] || !aligned(a->out[i], es))
            return PLORA_ERR_INVALID_ARG;
        p.out_stride[i] = a->out_stride[i] ? a->out_stride[i] : a->n[i];
        if (p.out_stride[i] < a->n[i]) return PLORA_ERR_INVALID_ARG;
        while (p.vec > es && (!aligned(a->out[i], p.vec) || p.out_stride[i] * es % p.vec)) p.vec /= 2;
        p.w_scale[i] = a->w_scale[i];
        p.out[i] = a->out[i];
        p.n[i] = a->n[i];
    }
    // (rows and columns are counted in 32 bits, too)
    constexpr int kMost = 1 << 30;
    if (a->m > kMost || a->k > kMost) return PLORA_ERR_UNSUPPORTED;
    auto tiles_of = [&](int bn) {
        long long t = 0;
        for (int i = 0; i < a->n_weights; ++i) t += ((long long)a->n[i] + bn - 1) / bn;
        return t;
    };
    for (int i = 0; i < a->n_weights; ++i)
        if (a->n[i] > kMost) return PLORA_ERR_UNSUPPORTED;
    if (((long long)a->m + kRows - 1) / kRows * tiles_of(64) >= kMaxTiles) return PLORA_ERR_UNSUPPORTED;
    plora::paged::Device dev;
    if (device(dev) != cudaSuccess) return PLORA_ERR_CUDA;
    if (!plora::paged::encode_tiled()) return PLORA_ERR_UNSUPPORTED;
    p.x_scale = a->x_scale;
    p.m = a->m;
    p.blocks = (int)(((long long)a->k + kBlock - 1) / kBlock);
    p.status = a->status;
    p.weights_ready = a->weights_ready;
    p.wait_cycles = a->wait_cycles ? a->wait_cycles : kWaitCycles;
    p.test_hook = a->test_hook;
    const Form form = choose(a, p.blocks, dev.sms);
    const int cg = form.cg, bn = form.bn;
    p.splits = form.splits;
    const long long m_tiles = ((long long)a->m + cg * kRows - 1) / (cg * kRows), n_tiles = tiles_of(bn);
    p.m_tiles = (int)m_tiles;
    p.n_tiles = (int)n_tiles;
    p.tiles = (int)(m_tiles * n_tiles);
    for (int i = 0, t = 0; i < kMaxWeights; ++i) {
        if (i < a->n_weights) t += (a->n[i] + bn - 1) / bn;
        p.tile_end[i] = t;
    }
    p.x_rows = a->m >= kRows ? kRows : (a->m + 7) / 8 * 8;
    p.x_bytes = p.x_rows * kRowBytes;
    p.quads = a->m >= kRows ? 4 : (a->m + 31) / 32;
    Maps maps;
    if (!map_bytes(&maps.x, a->x, a->k, a->m, x_stride, p.x_rows)) return PLORA_ERR_INVALID_ARG;
    for (int i = 0; i < a->n_weights; ++i)
        if (!map_bytes(&maps.w[i], a->w[i], a->k, a->n[i], w_stride[i], bn / cg)) return PLORA_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    e = cg == 2 ? go_bn<2>(bn, a->out_type, maps, p, dev, st) : go_bn<1>(bn, a->out_type, maps, p, dev, st);
    if (e != cudaSuccess) {
        (void)cudaGetLastError();      // reported here; a later call must not find it
        return PLORA_ERR_CUDA;
    }
    return PLORA_OK;
}

extern "C" PLORA_API plora_status plora_gemm_fp8_status(void* stream, int32_t* host_out) {
    if (!host_out) return PLORA_ERR_INVALID_ARG;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    void* word = nullptr;
    const bool done = cudaGetSymbolAddress(&word, default_status) == cudaSuccess &&
                      cudaMemcpyAsync(host_out, word, 4, cudaMemcpyDeviceToHost, st) == cudaSuccess &&
                      cudaMemsetAsync(word, 0, 4, st) == cudaSuccess && cudaStreamSynchronize(st) == cudaSuccess;
    if (!done) (void)cudaGetLastError();      // reported here; a later call must not find it
    return done ? PLORA_OK : PLORA_ERR_CUDA;
}
