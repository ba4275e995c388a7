// Attention over a paged KV cache, units of up to 256 rows: prompts, and groups of requests against a shared prefix.
//
// Both products run on the fifth-generation tensor cores (tcgen05.mma, M = 128, accumulators in tensor memory):
//     S[128 rows, 128 keys] = Q K^T        operands in shared memory
//     O[128 rows, D]       += P V          P from tensor memory, where it replaces the S it was made of
// A unit has two tiles of 128 rows (query tokens times the G heads of a KV head); they share every tile of
// K and V, and while one tile's scores are in the softmax the tensor cores work for the other.
// Roles: warps 0-3 and 4-7 are the softmax of the two tiles, a row per thread (no shuffles); warp 8 issues the MMAs;
// warps 9 and 13 keep K and V coming through a ring (tensor-map boxes, one per page piece); warp 10 clears the rows of V
// behind an item's last key; warp 11 fetches items from a counter, an item ahead, and their queries.  Tensor memory (all
// 512 columns): S of the two tiles, O of the two tiles.
//
// The running maximum is followed lazily: O and l are rescaled only when a row's maximum has grown by more than
// 2^8 over the one in use (P then stays below 2^8, far inside both 16-bit types, and fp32 sums do not care), so the
// accumulator in tensor memory is hardly ever touched between the products.
// P is rounded to the input type for the second product (unlike the small units' weights, which keep what is left, too); l sums
// the unrounded weights in fp32.  The rests would need a second P V: that alone, without making them, costs 11 % on the long
// prompts below and 7 % on prompts of 512 tokens, and P's rests need columns that the scores still hold.  What it leaves of an
// error is that of the output's own rounding again: 0.0021 of the norm in bf16 (the output's 0.0016), 0.00025 in half (0.0002).
//
// A tile's step is: scores (512 cycles of the tensor pipe at D = 128), softmax, O += P V (512).  Measured by the clock inside the
// kernel on 16 prompts of 2048 to 4096 tokens: the two tiles' steps take 3700 cycles together, 2050 of them with the tensor
// pipe busy (46 %; 0.9 PFLOP/s at the 1.7 GHz the part holds under it, 1.09 ms; 1.22 ms once the power limit sets in).  A
// step is a chain, softmax (2000) - hand-over (250) - products (1350) - hand-over (250), and tensor memory holds the scores
// of two tiles, so at most two chains run.  What the instructions cost hardly shows: a third of the exponentials on the FMA
// pipe, two threads to a row, an MMA warp per tile, 64 keys with two sets of scores per tile all took as long or longer.
// What did show is code size (instruction fetch bounds five roles that run different code): hence the rolled loops below.
#include <limits.h>

#include "paged.cuh"

namespace plora {
namespace paged {
namespace {

constexpr int kTileKeys = 128;
constexpr int kSoftmaxWarps = 8, kMmaWarp = 8, kKeyWarp = 9, kTailWarp = 10, kItemWarp = 11, kValueWarp = 13;
constexpr int kThreads = 16 * 32;       // four warpgroups (three warps only give their registers away)
constexpr int kSoftmaxRegs = 184, kOtherRegs = 72;       // of 128 a thread at launch: 2 * 184 + 2 * 72 = 4 * 128
constexpr int kSched = 2;
constexpr float kWideCap = 256.f;   // caps above take the form of their own in scores_of()
constexpr float kLazy = 8.f;        // base-2 logarithm of the growth a row's maximum may have before O is rescaled

template <int D>
struct Cfg {
    static constexpr int kPanels = D / 64;
    static constexpr int kPanelBytes = 128 * 128;            // 128 rows of 64 values, 128-byte swizzled
    static constexpr int kTileBytes = kPanels * kPanelBytes;
    static constexpr int kStages = D == 128 ? 5 : 8;
    static constexpr int kBars = 2 * kStages + 2 + 8 + 2 * kSched + 3;
    static constexpr int kSmemBytes = 1024 + 2 * kTileBytes + kStages * kTileBytes + kBars * 8 + kSched * 48 + 32;
};
constexpr uint32_t kTmemS = 0, kTmemO = 256, kTmemTile = 128;    // column of tile t: base + t * 128

struct Item {       // 48 bytes
    int32_t head, tok0, ntok, req;
    int32_t kf, n_tiles, k0, k1;     // first key of the first tile; keys [k0, k1)
    int32_t part, more;              // more = 0: nothing follows
    int32_t range[2];                // of each tile of rows: the tiles of keys it looks at, first | (one past the last) << 16
};
__device__ __forceinline__ int range_first(int r) { return r & 0xffff; }
__device__ __forceinline__ int range_end(int r) { return (int)((unsigned)r >> 16); }

// ---- tcgen05 ------------------------------------------------------------------------------------------
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Shared-memory matrix descriptor: start address, leading and stride byte offsets (16-byte units), version 1, 128-byte swizzle.
__device__ __forceinline__ constexpr uint64_t smem_desc(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
    return (uint64_t)((saddr >> 4) & 0x3fffu) | ((uint64_t)((lbo >> 4) & 0x3fffu) << 16) | ((uint64_t)((sbo >> 4) & 0x3fffu) << 32) |
           ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
// Instruction descriptor: fp32 accumulate, bf16 (1) or half (0) operands, A K-major, B K- or MN-major, M = 128.
__device__ __forceinline__ constexpr uint32_t instr_desc(int n, bool b_mn_major, bool fp16) {
    return (1u << 4) | ((fp16 ? 0u : 1u) << 7) | ((fp16 ? 0u : 1u) << 10) | (b_mn_major ? (1u << 16) : 0u) | ((uint32_t)(n >> 3) << 17) |
           ((128u >> 4) << 24);
}
__device__ __forceinline__ void umma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc)
        : "memory");
}
__device__ __forceinline__ void umma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool acc) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
        "r"(a), "l"(b), "r"(idesc), "r"((uint32_t)acc)
        : "memory");
}
__device__ __forceinline__ void umma_commit(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// 32 consecutive columns of this thread's lane
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
__device__ __forceinline__ void tmem_st32(uint32_t a, const uint32_t* r) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};" ::"r"(r[0]),
        "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
        "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]),
        "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]), "r"(a)
        : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t a, uint32_t* r) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
                   "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(a));
}
__device__ __forceinline__ void tmem_st16(uint32_t a, const uint32_t* r) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15};" ::"r"(r[0]),
                 "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
                 "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(a)
                 : "memory");
}
__device__ __forceinline__ void tmem_ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void st_global32(void* p, const uint32_t* w) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                 "r"(w[5]), "r"(w[6]), "r"(w[7])
                 : "memory");
}
// Box of the 3-D query tensor [token][head][dim]: 64 dims of the G heads of a KV head, of the tokens of a tile.
__device__ __forceinline__ void tma_box3(uint32_t dst, const CUtensorMap* tm, int dim, int head, int tok, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tm)), "r"(dim), "r"(head), "r"(tok), "r"(bar)
        : "memory");
}

__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ uint64_t desc_of(uint32_t lo, uint32_t hi) { return (uint64_t)lo | ((uint64_t)hi << 32); }
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }


struct Smem {
    uint32_t q, ring;
    uint32_t kv_full, kv_empty, q_full, q_empty, s_full, p_ready, o_full, sched_full, sched_empty, wind_down, tail_go, tail_done;
    Item* items;
    uint32_t* tmem_slot;
    uint32_t* filled;        // [2]: how far each loader got
    WaitCtl wc;
};
template <int D>
__device__ __forceinline__ Smem carve(uint8_t* raw, const Params& p) {
    using C = Cfg<D>;
    uint8_t* base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    uint8_t* items = base + (2 + C::kStages) * C::kTileBytes;
    uint8_t* bars = items + kSched * sizeof(Item);
    uint8_t* words = bars + C::kBars * 8;
    Smem s;
    s.q = smem_u32(base);
    s.ring = s.q + 2 * C::kTileBytes;
    s.items = reinterpret_cast<Item*>(items);
    s.kv_full = smem_u32(bars);
    s.kv_empty = s.kv_full + C::kStages * 8;
    s.q_full = s.kv_empty + C::kStages * 8;
    s.q_empty = s.q_full + 8;
    s.s_full = s.q_empty + 8;
    s.p_ready = s.s_full + 16;
    s.o_full = s.p_ready + 32;
    s.sched_full = s.o_full + 16;
    s.sched_empty = s.sched_full + kSched * 8;
    s.wind_down = s.sched_empty + kSched * 8;
    s.tail_go = s.wind_down + 8;
    s.tail_done = s.tail_go + 8;
    s.wc.abort_flag = reinterpret_cast<volatile int*>(words);
    s.wc.header = p.header;
    s.tmem_slot = reinterpret_cast<uint32_t*>(words + 8);
    s.filled = reinterpret_cast<uint32_t*>(words + 16);
    return s;
}

// ---- warp 11: items and their queries --------------------------------------------------------------------------
// It runs an item ahead of the others: the chain from the counter to a token's interval is some thousand cycles long.
template <int D>
__device__ __forceinline__ void item_warp(const Params& p, const Smem& sm, const CUtensorMap* tm_q, int n_items, int lane) {
    using C = Cfg<D>;
    const unsigned all = 0xffffffffu;
    const int bp = min(p.page_size, 64), TT = p.big_tile_tok;
    uint32_t ic = 0, qn = 0;
    int next = 0;
    if (lane == 0) next = atomicAdd(p.header + kBigNextWord, 1);
#pragma unroll 1
    for (;; ++ic) {
        const int item = __shfl_sync(all, next, 0);
        const bool more = item < n_items;
        Item d{};
        if (more) {
            if (lane == 0) next = atomicAdd(p.header + kBigNextWord, 1);
            const int un = item / p.n_kv_heads;
            const Unit u = checked(p, p.big_units[un]);
            d.head = item - un * p.n_kv_heads;
            d.tok0 = u.tok0; d.ntok = u.ntok; d.req = u.req; d.part = u.part;
            // the keys that one of the tokens sees, for each tile of rows
            int lo[2] = {INT_MAX, INT_MAX}, hi[2] = {0, 0};
            TokInfo ti[8];                       // (a unit has at most 256 tokens: all loads at once)
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (lane + 32 * i < u.ntok) ti[i] = p.tok_info[u.tok0 + lane + 32 * i];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int t = lane + 32 * i;
                if (t < u.ntok) {
                    const int a = max(ti[i].lo, u.k0), b = min(ti[i].hi, u.k1), w = t < TT ? 0 : 1;
                    if (a < b) {
                        if (w == 0) {
                            lo[0] = min(lo[0], a);
                            hi[0] = max(hi[0], b);
                        } else {
                            lo[1] = min(lo[1], a);
                            hi[1] = max(hi[1], b);
                        }
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < 2; ++t) {
                lo[t] = __reduce_min_sync(all, lo[t]);
                hi[t] = __reduce_max_sync(all, hi[t]);
            }
            d.k0 = min(lo[0], lo[1]);
            d.k1 = max(hi[0], hi[1]);
            if (d.k0 >= d.k1) d.k0 = d.k1 = 0;
            d.kf = d.k0 / bp * bp;
            d.n_tiles = (d.k1 - d.kf + kTileKeys - 1) / kTileKeys;
#pragma unroll
            for (int t = 0; t < 2; ++t)
                d.range[t] = hi[t] > 0 ? (lo[t] - d.kf) / kTileKeys | ((hi[t] - d.kf + kTileKeys - 1) / kTileKeys) << 16 : 0;
            d.more = 1;
        }
        const uint32_t ss = ic % kSched;
        int ok = 1;
        if (lane == 0) {
            ok = mbar_wait(sm.sched_empty + ss * 8, ((ic / kSched) & 1) ^ 1, sm.wc);
            if (ok) {
                sm.items[ss] = d;
                mbar_arrive(sm.sched_full + ss * 8);
                if (d.n_tiles > 0) {
                    ok = mbar_wait(sm.q_empty, (qn & 1) ^ 1, sm.wc);
                    if (ok) {
                        const int tiles_q = d.ntok > TT ? 2 : 1;
                        mbar_arrive_expect_tx(sm.q_full, (uint32_t)tiles_q * TT * p.G * D * 2);
#pragma unroll 1
                        for (int t = 0; t < tiles_q; ++t)
                            for (int c = 0; c < C::kPanels; ++c)
                                tma_box3(sm.q + t * C::kTileBytes + c * C::kPanelBytes, tm_q, c * 64, d.head * p.G, d.tok0 + t * TT, sm.q_full);
                        ++qn;
                    }
                }
            }
        }
        if (!__shfl_sync(all, ok, 0) || !more) break;
    }
    // a copy in flight must land before the CTA leaves
    if (lane == 0 && qn > 0 && !mbar_drain(sm.q_full, (qn - 1) & 1, wait_limit(p.header))) atomicCAS(p.header, 0, PLORA_ERR_TIMEOUT);
    __syncwarp();
}

// When both loaders have stopped: the copies still in flight must land before the CTA leaves (after a wait that ran out, up to
// all of a ring may be).  A lane per stage looks at what was sent there last; only then does a phase tell the copy, for
// the two loaders share the ring, and the one that stops first does not know which stages the other has filled again.
template <int D>
__device__ __forceinline__ void drain_ring(const Params& p, const Smem& sm, int lane) {
    constexpr uint32_t kStages = Cfg<D>::kStages;
    int last = -1;                           // (stages are numbered through, K even, V odd; a loader has filled all of its below filled[])
#pragma unroll 1
    for (int i = 0; i < 2 * (int)kStages; ++i) {
        const int x = (int)sm.filled[i & 1] - 2 - (i & ~1);
        if (lane < (int)kStages && x >= 0 && x % (int)kStages == lane) last = max(last, x);
    }
    if (last >= 0 && !mbar_drain(sm.kv_full + lane * 8, (last / (int)kStages) & 1, wait_limit(p.header))) atomicCAS(p.header, 0, PLORA_ERR_TIMEOUT);
    __syncwarp();
}

// ---- warps 9 and 13: keys, values ------------------------------------------------------------------------------------
// A warp each: with pages of 16 tokens a tile is 16 boxes.  As with the MMAs, the warp stays together and an elected lane
// issues (a copy that every lane issues for itself cost 100 to 200 cycles).
template <int D>
__device__ __forceinline__ void load_warp(const Params& p, const Smem& sm, const CUtensorMap* tm, uint32_t kv, int lane) {
    using C = Cfg<D>;
    const unsigned all = 0xffffffffu;
    const int bp = min(p.page_size, 64);
    uint32_t it = kv, ic = 0;                // stages kv, kv + 2, ...
    bool stopped = false;
#pragma unroll 1
    for (; !stopped; ++ic) {
        const uint32_t ss = ic % kSched;
        if (!__all_sync(all, mbar_wait(sm.sched_full + ss * 8, (ic / kSched) & 1, sm.wc))) break;
        const Item& src = sm.items[ss];
        const int more = (int)uniform(src.more), n_tiles = (int)uniform(src.n_tiles), kf = (int)uniform(src.kf), k1 = (int)uniform(src.k1);
        const int head = (int)uniform(src.head), req = (int)uniform(src.req);
        __syncwarp();
        if (lane == 0) mbar_arrive(sm.sched_empty + ss * 8);
        if (!more) break;
        const int32_t* table = p.block_table + (size_t)req * p.max_blocks;
        auto page_of = [&](int j) {              // the page of this lane's piece of key tile j
            const int key = kf + j * kTileKeys + lane * bp;
            int page = 0;
            if (lane < kTileKeys / bp && key < k1) PLORA_CHECKED(key < p.max_kv, p.header) page = table[key >> p.page_shift];
            return page;
        };
        int page_next = page_of(0);
#pragma unroll 1
        for (int j = 0; j < n_tiles; ++j, it += 2) {
            const int key = kf + j * kTileKeys, nb = (min(kTileKeys, k1 - key) + bp - 1) / bp;
            int page = page_next;
            if (j + 1 < n_tiles) page_next = page_of(j + 1);
            if (lane < nb && (unsigned)page >= (unsigned)p.n_pages) {   // such a page reads as zeros
                atomicCAS(p.header, 0, PLORA_ERR_INVALID_ARG);
                page = p.n_pages;
            }
            const uint32_t slot = it % C::kStages, dst = sm.ring + slot * C::kTileBytes, bar = sm.kv_full + slot * 8;
            if (!__all_sync(all, mbar_wait(sm.kv_empty + slot * 8, ((it / C::kStages) & 1) ^ 1, sm.wc))) {
                stopped = true;
                break;
            }
            if (elect_one()) mbar_arrive_expect_tx(bar, (uint32_t)nb * bp * D * 2);
#pragma unroll 1
            for (int i = 0; i < nb; ++i) {
                const int pg = __shfl_sync(all, page, i), so = (key + i * bp) & (p.page_size - 1);
                if (elect_one()) {
#pragma unroll
                    for (int c = 0; c < C::kPanels; ++c)
                        tma_box4(dst + c * C::kPanelBytes + i * bp * 128, tm, c * 64, so, head, pg, bar);
                }
            }
        }
    }
    if (lane == 0) sm.filled[kv] = it;
    __syncwarp();
    asm volatile("bar.sync 1, 64;" ::: "memory");       // (the two loaders; their waits are bounded, so both get here)
    if (kv == 0) drain_ring<D>(p, sm, lane);
}
// ---- warp 8: the products ---------------------------------------------------------------------------------------
// The warp stays together and one elected lane issues: the MMA's operands are uniform registers, and under a plain
// `lane == 0` the compiler cannot know that a single lane is active (an MMA then cost the issuer about 100 cycles, more
// than the 64 it takes).  The upper half of a matrix descriptor is the same for all operands of a kind, and the lower half
// is an address that advances by constants.
template <int D, bool FP16>
__device__ __forceinline__ void mma_warp(const Params& p, const Smem& sm, uint32_t tmem) {
    using C = Cfg<D>;
    const unsigned all = 0xffffffffu;
    constexpr uint32_t idesc_s = instr_desc(kTileKeys, false, FP16), idesc_o = instr_desc(D, true, FP16);
    constexpr uint32_t kHi = (uint32_t)(smem_desc(0, 0, 1024) >> 32);
    constexpr uint32_t kLoK = 1u << 16, kLoV = (uint32_t)(C::kPanelBytes >> 4) << 16;     // leading offsets: unused; the next panel
    const bool withhold = p.header[kHookWord] == PLORA_HOOK_WITHHOLD_RELEASE;   // test hook: stages are never handed back
    uint32_t it = 0, ic = 0, qn = 0, tails = 0, np = 0;       // np: a phase bit for each tile
    const uint32_t q_lo = uniform((sm.q >> 4) | kLoK), ring_lo = uniform(sm.ring >> 4);
    tmem = uniform(tmem);
    bool ok = true;
    auto wait_for = [&](uint32_t bar, uint32_t parity) {
        ok = __all_sync(all, mbar_wait(bar, parity, sm.wc));
        return ok;
    };
#pragma unroll 1
    for (;; ++ic) {
        const uint32_t ss = ic % kSched;
        if (!wait_for(sm.sched_full + ss * 8, (ic / kSched) & 1)) break;
        const Item& src = sm.items[ss];
        const int n_tiles = (int)uniform(src.n_tiles), more = (int)uniform(src.more), last = (int)uniform(src.k1 - src.kf);
        const int range0 = (int)uniform(src.range[0]), range1 = (int)uniform(src.range[1]);
        if (elect_one()) mbar_arrive(sm.sched_empty + ss * 8);
        if (!more) break;
        if (n_tiles == 0) continue;
        if (!wait_for(sm.q_full, qn & 1)) break;
        ++qn;
        // step j: O += P V of key tile j - 1, then S = Q K^T of key tile j, for each tile of rows that looks at them.  What the
        // step needs of K and V is waited for first, so that nothing stands between a tile's weights and its next scores:
        // the two tiles then settle into turns, one in the softmax while the other has the tensor cores.
#pragma unroll 1
        for (int j = 0; j <= n_tiles; ++j) {
            uint32_t v_slot = 0, k_slot = 0;
            int steps = kTileKeys / 16;
            if (j > 0) {
                v_slot = it % C::kStages;
                if (!wait_for(sm.kv_full + v_slot * 8, (it / C::kStages) & 1)) break;
                ++it;
                const int left = last - (j - 1) * kTileKeys;                   // keys of tile j - 1 that count
                if (left < kTileKeys) {
                    steps = (left + 15) / 16;
                    if (left & 15) {
                        if (elect_one()) mbar_arrive(sm.tail_go);
                        if (!wait_for(sm.tail_done, tails & 1)) break;
                        ++tails;
                    }
                }
            }
            if (j < n_tiles) {
                k_slot = it % C::kStages;
                if (!wait_for(sm.kv_full + k_slot * 8, (it / C::kStages) & 1)) break;
                ++it;
            }
            const uint32_t v = (ring_lo + v_slot * (C::kTileBytes >> 4)) | kLoV, k = (ring_lo + k_slot * (C::kTileBytes >> 4)) | kLoK;
#pragma unroll 1
            for (int t = 0; t < 2; ++t) {
                const int range = t ? range1 : range0, first = range_first(range), end = range_end(range);
                const uint32_t o = tmem + kTmemO + t * kTmemTile, ts = tmem + kTmemS + t * kTmemTile, q = q_lo + t * (C::kTileBytes >> 4);
                const bool pv = j > first && j <= end, qk = j >= first && j < end;
                if (pv) {
                    if (!wait_for(sm.p_ready + t * 16, (np >> t) & 1)) break;
                    tc_fence_after();
                    if (elect_one()) {
#pragma unroll
                        for (int s = 0; s < 4; ++s)
                            if (s < steps) umma_ts(o, ts + s * 8, desc_of(v + s * 128, kHi), idesc_o, j - 1 > first || s > 0);
                    }
                    if (!wait_for(sm.p_ready + t * 16 + 8, (np >> t) & 1)) break;
                    np ^= 1u << t;
                }
                tc_fence_after();
                if (elect_one()) {
                    if (pv) {
#pragma unroll
                        for (int s = 4; s < 8; ++s)
                            if (s < steps) umma_ts(o, ts + s * 8, desc_of(v + s * 128, kHi), idesc_o, true);
                    }
                    if (qk) {
#pragma unroll
                        for (int s = 0; s < D / 16; ++s) {
                            const uint32_t off = ((s >> 2) * C::kPanelBytes + (s & 3) * 32) >> 4;
                            umma_ss(ts, desc_of(q + off, kHi), desc_of(k + off, kHi), idesc_s, s > 0);
                        }
                        umma_commit(sm.s_full + t * 8);
                    }
                    if (pv && j == end) umma_commit(sm.o_full + t * 8);
                }
            }
            if (!ok) break;
            if (elect_one()) {
                if (j > 0 && !withhold) umma_commit(sm.kv_empty + v_slot * 8);
                if (j < n_tiles && !withhold) umma_commit(sm.kv_empty + k_slot * 8);
                if (j + 1 == n_tiles) umma_commit(sm.q_empty);
            }
        }
        if (!ok) break;
    }
    // nothing of the tensor pipe may be under way when the tensor memory is freed
    if (elect_one()) {
        umma_commit(sm.wind_down);
        if (!mbar_drain(sm.wind_down, 0, wait_limit(p.header))) atomicCAS(p.header, 0, PLORA_ERR_TIMEOUT);
    }
    __syncwarp();
}

// ---- warp 10: rows of V behind an item's last key may hold anything, and 0 * NaN must not reach the sum ----------------
template <int D>
__device__ __forceinline__ void tail_warp(const Params& p, const Smem& sm, int lane) {
    using C = Cfg<D>;
    const unsigned all = 0xffffffffu;
    uint32_t it = 0, ic = 0, tails = 0;
#pragma unroll 1
    for (;; ++ic) {
        const uint32_t ss = ic % kSched;
        if (!__all_sync(all, mbar_wait(sm.sched_full + ss * 8, (ic / kSched) & 1, sm.wc))) return;
        const Item d = sm.items[ss];
        __syncwarp();
        if (lane == 0) mbar_arrive(sm.sched_empty + ss * 8);
        if (!d.more) return;
        it += 2 * d.n_tiles;
        const int left = d.k1 - (d.kf + (d.n_tiles - 1) * kTileKeys);
        if (d.n_tiles == 0 || left == kTileKeys || !(left & 15)) continue;      // (the product takes 16 keys at a time)
        if (!__all_sync(all, mbar_wait(sm.tail_go, tails & 1, sm.wc))) return;
        ++tails;
        const uint32_t v = sm.ring + (it - 1) % C::kStages * C::kTileBytes;
        const int n = (16 - (left & 15)) * (D / 8);
#pragma unroll 1
        for (int i = lane; i < n; i += 32) {
            const int r = left + i / (D / 8), c = i % (D / 8);
            sts128(v + (c >> 3) * C::kPanelBytes + r * 128 + ((c & 7) << 4), 0u, 0u, 0u, 0u);
        }
        fence_async_smem();
        __syncwarp();
        if (lane == 0) mbar_arrive(sm.tail_done);
    }
}

// 32 raw products of a row -> scores in the base-2 domain (cap, bias by distance); dist0: distance of the first one's key.
// CAP 1, caps of up to kWideCap: a row whose 32 products are all small takes the cap's polynomial, two at a time on the FMA pipe;
// one with a larger product (a hidden one may be anything) takes the other form for all, which is off by 1.5e-7 of the cap, 4e-5
// at most.  CAP 2, larger caps: chosen product by product (see capped()).  That form for all caps costs packed documents 8 %
// (331 -> 358 us), most of it by the loop's code size: choosing in the rare branch alone costs as much.
template <int CAP, bool BIAS>
__device__ __forceinline__ void scores_of(const Params& p, float* s, float slope, float dist0) {
    if (CAP == 2) {
#pragma unroll
        for (int i = 0; i < 32; ++i) s[i] = capped(p, s[i]);
    }
    if (CAP == 1) {
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < 32; i += 2) most = fmaxf(fmaxf(most, fabsf(s[i])), fabsf(s[i + 1]));
        if (most <= p.cap_poly_below) {
#pragma unroll
            for (int i = 0; i < 32; i += 2) {
                const float2 x = make_float2(s[i], s[i + 1]), u = __fmul2_rn(x, x);
                float2 q = __ffma2_rn(u, make_float2(p.cap_d[4], p.cap_d[4]), make_float2(p.cap_d[3], p.cap_d[3]));
                q = __ffma2_rn(q, u, make_float2(p.cap_d[2], p.cap_d[2]));
                q = __ffma2_rn(q, u, make_float2(p.cap_d[1], p.cap_d[1]));
                q = __ffma2_rn(q, u, make_float2(p.cap_d[0], p.cap_d[0]));
                q = __fmul2_rn(q, x);
                s[i] = q.x;
                s[i + 1] = q.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < 32; ++i) s[i] = capped_far(p, s[i]);
        }
        __syncwarp();
    }
    if (BIAS) {
        // |distance| as a float, counted down from the first key's (an integer conversion per score would go to the
        // special-function unit)
#pragma unroll
        for (int i = 0; i < 32; ++i) s[i] = fmaf(-slope, fabsf(dist0 - (float)i), CAP ? s[i] : s[i] * p.scale_log2e);
    }
}

// ---- warps 0-7: softmax and output ------------------------------------------------------------------------------
template <int D, bool FP16, int CAP, bool BIAS>
__device__ __forceinline__ void softmax_warp(const Params& p, const Smem& sm, uint32_t tmem, int warp, int lane) {
    const unsigned all = 0xffffffffu;
    const int t = warp >> 2, row = (warp & 3) * 32 + lane, TT = p.big_tile_tok;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + lanes + kTmemS + t * kTmemTile, to = tmem + lanes + kTmemO + t * kTmemTile;
    const int tr = row / p.G, g = row - tr * p.G;
    uint32_t ic = 0, ns = 0, no = 0;
#pragma unroll 1
    for (;; ++ic) {
        const uint32_t ss = ic % kSched;
        if (!__all_sync(all, mbar_wait(sm.sched_full + ss * 8, (ic / kSched) & 1, sm.wc))) return;
        const Item d = sm.items[ss];
        __syncwarp();
        if (lane == 0) mbar_arrive(sm.sched_empty + ss * 8);
        if (!d.more) return;
        if (t == 1 && d.ntok <= TT) continue;
        const int rel = t * TT + tr;                  // the row's token, counted from the unit's first
        const bool mine = tr < TT && rel < d.ntok;
        const int hq = d.head * p.G + g;
        int lo = 0, hi = 0, pos = 0;
        float slope = 0.f;
        if (mine) {
            const TokInfo ti = p.tok_info[d.tok0 + rel];
            lo = max(ti.lo, d.k0);
            hi = min(ti.hi, d.k1);
            pos = ti.pos;
            if (BIAS && p.slopes) slope = p.slopes[hq] * 1.4426950408889634f;
        }
        float m = -INFINITY, l = 0.f;
        const int first = range_first(d.range[t]), end = range_end(d.range[t]);
#pragma unroll 1
        for (int j = first; j < end; ++j) {
            const int key = d.kf + j * kTileKeys;
            if (!__all_sync(all, mbar_wait(sm.s_full + t * 8, ns & 1, sm.wc))) return;
            ++ns;
            tc_fence_after();
            // The row is read twice from tensor memory, 32 columns at a time, rather than held in 128 registers: the room is
            // worth more to the scheduler of the second pass.  What the first pass changes it writes back.
            uint32_t buf[2][32];                 // (one is loaded while the other is worked on)
            const float mul = CAP || BIAS ? 1.f : p.scale_log2e;
            const bool mask = __any_sync(all, lo > key || hi < key + kTileKeys), changed = CAP || BIAS || mask;
            float mx[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) mx[i] = -INFINITY;
            tmem_ld32(ts, buf[0]);
#pragma unroll 1
            for (int c2 = 0; c2 < 4; c2 += 2)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int c = c2 + h;
                    float* s = reinterpret_cast<float*>(buf[h]);
                    tmem_ld_wait();
                    tmem_ld32(ts + ((c + 1) & 3) * 32, buf[h ^ 1]);        // (after the last one the first, for the second pass)
                    if (CAP || BIAS) scores_of<CAP, BIAS>(p, s, slope, (float)(pos - key - c * 32));
                    if (mask) {
                        const int a = min(max(lo - key - c * 32, 0), 32), b = min(max(hi - key - c * 32, 0), 32);
                        // bits [a, b) of the 32 (a shift by 32 gives 0)
                        const uint32_t see = a < b ? __funnelshift_lc(0u, 0xffffffffu, a) & ~__funnelshift_lc(0u, 0xffffffffu, b) : 0u;
#pragma unroll
                        for (int i = 0; i < 32; ++i) s[i] = see & (1u << i) ? s[i] : -INFINITY;
                    }
                    if (changed) tmem_st32(ts + c * 32, buf[h]);
#pragma unroll
                    for (int i = 0; i < 32; i += 16)
#pragma unroll
                        for (int e = 0; e < 8; ++e) mx[e] = fmaxf(fmaxf(mx[e], s[i + e]), s[i + 8 + e]);
                }
            if (changed) {
                tmem_ld_wait();
                tmem_st_wait();
                tmem_ld32(ts, buf[0]);
            }
            const float tile_max = fmaxf(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), fmaxf(fmaxf(mx[4], mx[5]), fmaxf(mx[6], mx[7]))) * mul;
            if (j == first) {
                m = tile_max;
            } else if (__any_sync(all, tile_max > m + kLazy)) {
                // (the products of the tiles before are complete: this tile's scores were issued behind them)
                const float mn = fmaxf(m, tile_max);
                const float f = mn == -INFINITY ? 1.f : ex2(m - mn);
                l *= f;
                m = mn;
#pragma unroll 1
                for (int c = 0; c < D / 16; ++c) {
                    uint32_t o[16];
                    tmem_ld16(to + c * 16, o);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
                    tmem_st16(to + c * 16, o);
                }
            }
            const float me = m == -INFINITY ? 0.f : m;
            float2 sum[4] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
            const float2 mul2 = make_float2(mul, mul), me2 = make_float2(-me, -me);
#pragma unroll 1
            for (int c2 = 0; c2 < 4; c2 += 2) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float* s = reinterpret_cast<const float*>(buf[h]);
                    tmem_ld_wait();
                    if (h == 0) tmem_ld32(ts + (c2 + 1) * 32, buf[1]);
                    else if (c2 == 0) tmem_ld32(ts + 64, buf[0]);
                    uint32_t w[16];
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        const float2 x = __ffma2_rn(make_float2(s[2 * i], s[2 * i + 1]), mul2, me2);
                        const float2 e = make_float2(ex2(x.x), ex2(x.y));
                        sum[i & 3] = __fadd2_rn(sum[i & 3], e);
                        w[i] = pack16<FP16>(e.x, e.y);
                    }
                    tmem_st16(ts + (c2 + h) * 16, w);
                }
                tmem_st_wait();                           // half of the keys: the second product may start
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(sm.p_ready + t * 16 + (c2 >> 1) * 8);
            }
            const float2 all2 = __fadd2_rn(__fadd2_rn(sum[0], sum[1]), __fadd2_rn(sum[2], sum[3]));
            l += all2.x + all2.y;
        }
        // output
        if (end > first) {
            if (!__all_sync(all, mbar_wait(sm.o_full + t * 8, no & 1, sm.wc))) return;
            ++no;
            tc_fence_after();
        }
        const float inv = m == -INFINITY ? 0.f : 1.f / l;              // nothing visible: a zero row
        const size_t at = (size_t)((d.part < 0 ? d.tok0 : d.part) + rel) * p.n_q_heads + hq;
        const bool writes = mine && row_exists(p, (d.part < 0 ? d.tok0 : d.part) + rel, d.part >= 0);
        if (writes && d.part >= 0) p.part_ml[at] = make_float2(m, l);
#pragma unroll 1
        for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            if (end > first) {
                tmem_ld32(to + c * 32, o);
                tmem_ld_wait();
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = 0u;
            }
            if (!writes) continue;
            // (32 bytes per lane and store: the rows lie far apart, and the store unit is paced by the lines it touches)
            if (d.part < 0) {
                uint16_t* dst = p.out + at * D + c * 32;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    uint32_t w[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e)
                        w[e] = pack16<FP16>(__uint_as_float(o[16 * i + 2 * e]) * inv, __uint_as_float(o[16 * i + 2 * e + 1]) * inv);
                    st_global32(dst + 16 * i, w);
                }
            } else {
                float* dst = p.part_o + at * D + c * 32;
#pragma unroll
                for (int i = 0; i < 4; ++i) st_global32(dst + 8 * i, o + 8 * i);
            }
        }
        tc_fence_before();
    }
}

template <int D, bool FP16, int CAP, bool BIAS>
__global__ void __launch_bounds__(kThreads, 1)
big_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v,
           const Params p) {
    using C = Cfg<D>;
    extern __shared__ uint8_t raw[];
    const Smem sm = carve<D>(raw, p);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(sm.kv_full + s * 8, 1);
            mbar_init(sm.kv_empty + s * 8, 1);
        }
        mbar_init(sm.q_full, 1);
        mbar_init(sm.q_empty, 1);
        for (int t = 0; t < 2; ++t) {
            mbar_init(sm.s_full + t * 8, 1);
            mbar_init(sm.p_ready + t * 16, 4);
            mbar_init(sm.p_ready + t * 16 + 8, 4);
            mbar_init(sm.o_full + t * 8, 1);
        }
        for (int s = 0; s < kSched; ++s) {
            mbar_init(sm.sched_full + s * 8, 1);
            mbar_init(sm.sched_empty + s * 8, kSoftmaxWarps + 4);
        }
        mbar_init(sm.wind_down, 1);
        mbar_init(sm.tail_go, 1);
        mbar_init(sm.tail_done, 1);
        sm.wc.abort_flag[0] = 0;
        mbar_init_fence();
    }
    grid_wait();                 // the units come from the plan kernel
    grid_launch_dependents();
    const int n_items = p.header[kBigUnitsWord] * p.n_kv_heads;
    if (n_items == 0) return;
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;" ::"r"(smem_u32(sm.tmem_slot)) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
        tc_fence_before();
    }
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *sm.tmem_slot;
    if (warp < kSoftmaxWarps) {
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
        softmax_warp<D, FP16, CAP, BIAS>(p, sm, tmem, warp, lane);
    } else {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
        if (warp == kMmaWarp) mma_warp<D, FP16>(p, sm, tmem);
        else if (warp == kTailWarp) tail_warp<D>(p, sm, lane);
        else if (warp == kItemWarp) item_warp<D>(p, sm, &tm_q, n_items, lane);
        else if (warp == kKeyWarp) load_warp<D>(p, sm, &tm_k, 0, lane);
        else if (warp == kValueWarp) load_warp<D>(p, sm, &tm_v, 1, lane);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

template <int D, bool FP16, int CAP, bool BIAS>
cudaError_t go(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const Params& p, Device dev, cudaStream_t st) {
    auto kern = big_kernel<D, FP16, CAP, BIAS>;
    static Configured configured;
    const cudaError_t e = configured.ensure(reinterpret_cast<const void*>(kern), Cfg<D>::kSmemBytes, dev.id);
    if (e != cudaSuccess) return e;
    const long long items = (long long)p.cap_big * p.n_kv_heads;
    const int grid = (int)(items < dev.sms ? items : dev.sms);
    void* args[] = {const_cast<CUtensorMap*>(&q), const_cast<CUtensorMap*>(&k), const_cast<CUtensorMap*>(&v), const_cast<Params*>(&p)};
    return launch_pdl(reinterpret_cast<const void*>(kern), dim3(grid), dim3(kThreads), Cfg<D>::kSmemBytes, st, args);
}
template <int D, bool FP16>
cudaError_t go2(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const Params& p, Device dev, cudaStream_t st) {
    // (a scale that is not positive takes the form that scales before it masks and looks for the maximum)
    const bool bias = p.slopes || !(p.scale_log2e > 0.f);
    if (p.cap_log2e > kWideCap * 1.4426950408889634f)
        return bias ? go<D, FP16, 2, true>(q, k, v, p, dev, st) : go<D, FP16, 2, false>(q, k, v, p, dev, st);
    if (p.cap_log2e > 0.f) return bias ? go<D, FP16, 1, true>(q, k, v, p, dev, st) : go<D, FP16, 1, false>(q, k, v, p, dev, st);
    return bias ? go<D, FP16, 0, true>(q, k, v, p, dev, st) : go<D, FP16, 0, false>(q, k, v, p, dev, st);
}

}  // namespace

cudaError_t launch_big(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const Params& p, int head_dim, bool fp16,
                       Device dev, cudaStream_t st) {
    if (head_dim == 128) return fp16 ? go2<128, true>(q, k, v, p, dev, st) : go2<128, false>(q, k, v, p, dev, st);
    return fp16 ? go2<64, true>(q, k, v, p, dev, st) : go2<64, false>(q, k, v, p, dev, st);
}

}  // namespace paged
}  // namespace plora
