// Attention over a paged KV cache, units of up to 256 rows: prompts, and groups of requests against a shared prefix.
//
// Both products run on the fifth-generation tensor cores (tcgen05.mma, M = 128, accumulators in tensor memory):
//     S[128 rows, 128 keys] = Q K^T        operands in shared memory
//     O[128 rows, D]       += P V          P from tensor memory, where it replaces the S it was made of
// A unit has two tiles of 128 rows (query tokens times the G heads of a KV head); they share every tile of
// K and V, and while one tile's scores are in the softmax the tensor cores work for the other.
// Roles: warps 0-3 and 4-7 are the softmax of the two tiles, a row per thread (no shuffles); warp 8 issues the
// MMAs; warp 9 fetches items from a counter and keeps K and V coming through a ring (tensor-map boxes, one per page
// piece).  Tensor memory (all 512 columns): S of the two tiles, O of the two tiles.
//
// The running maximum is followed lazily: O and l are rescaled only when a row's maximum has grown by more than
// 2^8 over the one in use (P then stays below 2^8, far inside both 16-bit types, and fp32 sums do not care), so the
// accumulator in tensor memory is hardly ever touched between the products.
// P is rounded to the input type for the second product; l sums the unrounded weights in fp32.
#include <limits.h>

#include "paged.cuh"

namespace plora {
namespace paged {
namespace {

constexpr int kTileKeys = 128;
constexpr int kSoftmaxWarps = 8, kMmaWarp = 8, kLoadWarp = 9;
constexpr int kThreads = 12 * 32;       // three warpgroups; the last one's two other warps only give their registers away
constexpr int kSoftmaxRegs = 208, kOtherRegs = 88;      // of 168 a thread at launch: 2 * 208 + 88 = 3 * 168
constexpr int kSched = 2;
constexpr float kLazy = 8.f;        // base-2 logarithm of the growth a row's maximum may have before O is rescaled

template <int D>
struct Cfg {
    static constexpr int kPanels = D / 64;
    static constexpr int kPanelBytes = 128 * 128;            // 128 rows of 64 values, 128-byte swizzled
    static constexpr int kTileBytes = kPanels * kPanelBytes;
    static constexpr int kStages = D == 128 ? 5 : 8;
    static constexpr int kBars = 2 * kStages + 2 + 6 + 2 * kSched + 1;
    static constexpr int kSmemBytes = 1024 + 2 * kTileBytes + kStages * kTileBytes + kBars * 8 + kSched * 48 + 32;
};
constexpr uint32_t kTmemS = 0, kTmemO = 256, kTmemTile = 128;    // column of tile t: base + t * 128

struct Item {       // 48 bytes
    int32_t head, tok0, ntok, req;
    int32_t kf, n_tiles, k0, k1;     // first key of the first tile; keys [k0, k1)
    int32_t part, more, pad_[2];     // more = 0: nothing follows
};

// ---- tcgen05 ------------------------------------------------------------------------------------------
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Shared-memory matrix descriptor: start address, leading and stride byte offsets (16-byte units), version 1, 128-byte swizzle.
__device__ __forceinline__ uint64_t smem_desc(uint32_t saddr, uint32_t lbo, uint32_t sbo) {
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
// Box of the 3-D query tensor [token][head][dim]: 64 dims of the G heads of a KV head, of the tokens of a tile.
__device__ __forceinline__ void tma_box3(uint32_t dst, const CUtensorMap* tm, int dim, int head, int tok, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4}], [%5];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tm)), "r"(dim), "r"(head), "r"(tok), "r"(bar)
        : "memory");
}

struct Smem {
    uint32_t q, ring;
    uint32_t kv_full, kv_empty, q_full, q_empty, s_full, p_ready, o_full, sched_full, sched_empty, wind_down;
    Item* items;
    uint32_t* tmem_slot;
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
    s.o_full = s.p_ready + 16;
    s.sched_full = s.o_full + 16;
    s.sched_empty = s.sched_full + kSched * 8;
    s.wind_down = s.sched_empty + kSched * 8;
    s.wc.abort_flag = reinterpret_cast<volatile int*>(words);
    s.wc.header = p.header;
    s.tmem_slot = reinterpret_cast<uint32_t*>(words + 8);
    return s;
}

// ---- warp 9: items, queries, keys and values -----------------------------------------------------------------
template <int D>
__device__ __forceinline__ void load_warp(const Params& p, const Smem& sm, const CUtensorMap* tm_q, const CUtensorMap* tm_k,
                                          const CUtensorMap* tm_v, int n_items, int lane) {
    using C = Cfg<D>;
    const unsigned all = 0xffffffffu;
    const int bp = min(p.page_size, 64), TT = p.big_tile_tok;
    uint32_t it = 0, ic = 0, qn = 0;     // stages, items, query loads so far
    bool stopped = false;
    int next = 0;
    if (lane == 0) next = atomicAdd(p.header + kBigNextWord, 1);
    for (;; ++ic) {
        const int item = __shfl_sync(all, next, 0);
        const bool more = item < n_items;
        Item d{};
        if (more) {
            if (lane == 0) next = atomicAdd(p.header + kBigNextWord, 1);
            const int un = item / p.n_kv_heads;
            const Unit u = p.big_units[un];
            d.head = item - un * p.n_kv_heads;
            d.tok0 = u.tok0; d.ntok = u.ntok; d.req = u.req; d.part = u.part;
            // the keys that one of the tokens sees
            int lo = INT_MAX, hi = 0;
            for (int t = lane; t < u.ntok; t += 32) {
                const TokInfo ti = p.tok_info[u.tok0 + t];
                if (ti.lo < ti.hi) {
                    lo = min(lo, ti.lo);
                    hi = max(hi, ti.hi);
                }
            }
            lo = __reduce_min_sync(all, lo);
            hi = __reduce_max_sync(all, hi);
            d.k0 = max(lo, u.k0);
            d.k1 = min(hi, u.k1);
            if (d.k0 >= d.k1) d.k0 = d.k1 = 0;
            d.kf = d.k0 / bp * bp;
            d.n_tiles = (d.k1 - d.kf + kTileKeys - 1) / kTileKeys;
            d.more = 1;
        }
        const uint32_t ss = ic % kSched;
        int ok = 1;
        if (lane == 0) {
            ok = mbar_wait(sm.sched_empty + ss * 8, ((ic / kSched) & 1) ^ 1, sm.wc);
            if (ok) {
                sm.items[ss] = d;
                mbar_arrive(sm.sched_full + ss * 8);
            }
        }
        if (!__shfl_sync(all, ok, 0)) {
            stopped = true;
            break;
        }
        if (!more) break;
        if (d.n_tiles == 0) continue;
        const int tiles_q = d.ntok > TT ? 2 : 1;
        if (lane == 0) {
            ok = mbar_wait(sm.q_empty, (qn & 1) ^ 1, sm.wc);
            if (ok) {
                mbar_arrive_expect_tx(sm.q_full, (uint32_t)tiles_q * TT * p.G * D * 2);
                for (int t = 0; t < tiles_q; ++t)
                    for (int c = 0; c < C::kPanels; ++c)
                        tma_box3(sm.q + t * C::kTileBytes + c * C::kPanelBytes, tm_q, c * 64, d.head * p.G, d.tok0 + t * TT, sm.q_full);
            }
        }
        if (!__shfl_sync(all, ok, 0)) {
            stopped = true;
            break;
        }
        ++qn;
        const int32_t* table = p.block_table + (size_t)d.req * p.max_blocks;
        for (int j = 0; j < d.n_tiles && !stopped; ++j) {
            const int key = d.kf + j * kTileKeys, nb = (min(kTileKeys, d.k1 - key) + bp - 1) / bp;
            const int my_key = key + lane * bp, so = my_key & (p.page_size - 1);
            int page = 0;
            if (lane < nb) {
                page = table[my_key >> p.page_shift];
                if ((unsigned)page >= (unsigned)p.n_pages) {   // such a page reads as zeros
                    atomicCAS(p.header, 0, PLORA_ERR_INVALID_ARG);
                    page = p.n_pages;
                }
            }
            for (int kv = 0; kv < 2; ++kv, ++it) {
                const uint32_t slot = it % C::kStages, dst = sm.ring + slot * C::kTileBytes, bar = sm.kv_full + slot * 8;
                if (lane == 0) {
                    ok = mbar_wait(sm.kv_empty + slot * 8, ((it / C::kStages) & 1) ^ 1, sm.wc);
                    if (ok) mbar_arrive_expect_tx(bar, (uint32_t)nb * bp * D * 2);
                }
                if (!__shfl_sync(all, ok, 0)) {
                    stopped = true;
                    break;
                }
                if (lane < nb) {
#pragma unroll
                    for (int c = 0; c < C::kPanels; ++c)
                        tma_box4(dst + c * C::kPanelBytes + lane * bp * 128, kv ? tm_v : tm_k, c * 64, so, d.head, page, bar);
                }
            }
        }
        if (stopped) break;
    }
    // copies in flight must land before the CTA leaves
    if (lane == 0) {
        const long long limit = wait_limit(p.header);
        for (uint32_t k = 1; k <= (uint32_t)C::kStages && k <= it; ++k) {
            const uint32_t j = it - k;
            if (!mbar_drain(sm.kv_full + (j % C::kStages) * 8, (j / C::kStages) & 1, limit)) atomicCAS(p.header, 0, PLORA_ERR_TIMEOUT);
        }
        if (qn > 0 && !mbar_drain(sm.q_full, (qn - 1) & 1, limit)) atomicCAS(p.header, 0, PLORA_ERR_TIMEOUT);
    }
    __syncwarp();
}

// ---- warp 8: the products -------------------------------------------------------------------------------------
template <int D, bool FP16>
__device__ __forceinline__ void mma_warp(const Params& p, const Smem& sm, uint32_t tmem, int lane) {
    using C = Cfg<D>;
    const unsigned all = 0xffffffffu;
    constexpr uint32_t idesc_s = instr_desc(kTileKeys, false, FP16), idesc_o = instr_desc(D, true, FP16);
    const bool withhold = p.header[kHookWord] == PLORA_HOOK_WITHHOLD_RELEASE;   // test hook: stages are never handed back
    const int TT = p.big_tile_tok;
    uint32_t it = 0, ic = 0, qn = 0, np[2] = {0, 0};
    bool ok = true;
    auto wait_for = [&](uint32_t bar, uint32_t parity) {
        ok = __all_sync(all, mbar_wait(bar, parity, sm.wc));
        return ok;
    };
    auto scores = [&](int t, uint32_t slot) {        // S of tile t = Q K^T over the stage's keys
        const uint32_t q = sm.q + t * C::kTileBytes, k = sm.ring + slot * C::kTileBytes, d = tmem + kTmemS + t * kTmemTile;
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
            const uint32_t off = (s >> 2) * C::kPanelBytes + (s & 3) * 32;
            umma_ss(d, smem_desc(q + off, 16, 1024), smem_desc(k + off, 16, 1024), idesc_s, s > 0);
        }
        umma_commit(sm.s_full + t * 8);
    };
    for (;; ++ic) {
        const uint32_t ss = ic % kSched;
        if (!wait_for(sm.sched_full + ss * 8, (ic / kSched) & 1)) break;
        const Item d = sm.items[ss];
        __syncwarp();
        if (lane == 0) mbar_arrive(sm.sched_empty + ss * 8);
        if (!d.more) break;
        if (d.n_tiles == 0) continue;
        const int tiles_q = d.ntok > TT ? 2 : 1;
        if (!wait_for(sm.q_full, qn & 1)) break;
        ++qn;
        // first scores
        uint32_t slot = it % C::kStages;
        if (!wait_for(sm.kv_full + slot * 8, (it / C::kStages) & 1)) break;
        tc_fence_after();
        if (lane == 0) {
            for (int t = 0; t < tiles_q; ++t) scores(t, slot);
            if (!withhold) umma_commit(sm.kv_empty + slot * 8);
            if (d.n_tiles == 1) umma_commit(sm.q_empty);
        }
        ++it;
        for (int j = 0; j < d.n_tiles && ok; ++j) {
            const uint32_t vs = it % C::kStages, v = sm.ring + vs * C::kTileBytes;
            if (!wait_for(sm.kv_full + vs * 8, (it / C::kStages) & 1)) break;
            ++it;
            const int left = d.k1 - (d.kf + j * kTileKeys);          // keys of this tile that count
            const int steps = left >= kTileKeys ? kTileKeys / 16 : (left + 15) / 16;
            if (left < steps * 16) {
                // rows of V behind the last key may hold anything: 0 * NaN must not reach the sum
                const int n = (steps * 16 - left) * (D / 8);
                for (int i = lane; i < n; i += 32) {
                    const int r = left + i / (D / 8), c = i % (D / 8);
                    sts128(v + (c >> 3) * C::kPanelBytes + r * 128 + ((c & 7) << 4), 0u, 0u, 0u, 0u);
                }
                fence_async_smem();
                __syncwarp();
            }
            const uint32_t ks = it % C::kStages;
            const bool again = j + 1 < d.n_tiles;
            for (int t = 0; t < tiles_q; ++t) {
                if (!wait_for(sm.p_ready + t * 8, np[t] & 1)) break;
                ++np[t];
                if (t == 0 && again && !wait_for(sm.kv_full + ks * 8, (it / C::kStages) & 1)) break;
                tc_fence_after();
                if (lane == 0) {
                    const uint32_t o = tmem + kTmemO + t * kTmemTile, pa = tmem + kTmemS + t * kTmemTile;
                    for (int s = 0; s < steps; ++s)
                        umma_ts(o, pa + s * 8, smem_desc(v + s * 2048, C::kPanelBytes, 1024), idesc_o, j > 0 || s > 0);
                    if (again) scores(t, ks);
                    else umma_commit(sm.o_full + t * 8);
                }
            }
            if (!ok) break;
            if (lane == 0) {
                if (!withhold) umma_commit(sm.kv_empty + vs * 8);
                if (again) {
                    if (!withhold) umma_commit(sm.kv_empty + ks * 8);
                    if (j + 2 == d.n_tiles) umma_commit(sm.q_empty);
                }
            }
            if (again) ++it;
        }
        if (!ok) break;
    }
    // nothing of the tensor pipe may be under way when the tensor memory is freed
    if (lane == 0) {
        umma_commit(sm.wind_down);
        if (!mbar_drain(sm.wind_down, 0, wait_limit(p.header))) atomicCAS(p.header, 0, PLORA_ERR_TIMEOUT);
    }
    __syncwarp();
}

// ---- warps 0-7: softmax and output ------------------------------------------------------------------------------
template <int D, bool FP16, bool CAP, bool BIAS>
__device__ __forceinline__ void softmax_warp(const Params& p, const Smem& sm, uint32_t tmem, int warp, int lane) {
    const unsigned all = 0xffffffffu;
    const int t = warp >> 2, row = (warp & 3) * 32 + lane, TT = p.big_tile_tok;
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t ts = tmem + lanes + kTmemS + t * kTmemTile, to = tmem + lanes + kTmemO + t * kTmemTile;
    const int tr = row / p.G, g = row - tr * p.G;
    uint32_t ic = 0, ns = 0, no = 0;
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
        for (int j = 0; j < d.n_tiles; ++j) {
            const int key = d.kf + j * kTileKeys;
            if (!__all_sync(all, mbar_wait(sm.s_full + t * 8, ns & 1, sm.wc))) return;
            ++ns;
            tc_fence_after();
            uint32_t r[128];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld32(ts + c * 32, r + c * 32);
            tmem_ld_wait();
            float* s = reinterpret_cast<float*>(r);
            const float mul = CAP || BIAS ? 1.f : p.scale_log2e;
            if (CAP || BIAS) {
#pragma unroll
                for (int i = 0; i < 128; ++i) s[i] = score<CAP, BIAS>(p, s[i], slope, pos - (key + i));
            }
            if (__any_sync(all, lo > key || hi < key + kTileKeys)) {
                const int a = lo - key, b = hi - key;
#pragma unroll
                for (int i = 0; i < 128; ++i) s[i] = i >= a && i < b ? s[i] : -INFINITY;
            }
            float mx[4] = {s[0], s[1], s[2], s[3]};
#pragma unroll
            for (int i = 4; i < 128; ++i) mx[i & 3] = fmaxf(mx[i & 3], s[i]);
            const float tile_max = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])) * mul;
            if (j == 0) {
                m = tile_max;
            } else if (__any_sync(all, tile_max > m + kLazy)) {
                // (the products of the tiles before are complete: this tile's scores were issued behind them)
                const float mn = fmaxf(m, tile_max);
                const float f = mn == -INFINITY ? 1.f : ex2(m - mn);
                l *= f;
                m = mn;
#pragma unroll
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
            float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t w[16];
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const float a = ex2(fmaf(s[c * 32 + 2 * i], mul, -me)), b = ex2(fmaf(s[c * 32 + 2 * i + 1], mul, -me));
                    sum[(2 * i) & 3] += a;
                    sum[(2 * i + 1) & 3] += b;
                    w[i] = pack16<FP16>(a, b);
                }
                tmem_st16(ts + c * 16, w);
            }
            l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(sm.p_ready + t * 8);
        }
        // output
        if (d.n_tiles > 0) {
            if (!__all_sync(all, mbar_wait(sm.o_full + t * 8, no & 1, sm.wc))) return;
            ++no;
            tc_fence_after();
        }
        const float inv = l > 0.f ? 1.f / l : (l == 0.f ? 0.f : l);    // nothing visible: a zero row
        const size_t at = (size_t)((d.part < 0 ? d.tok0 : d.part) + rel) * p.n_q_heads + hq;
        if (mine && d.part >= 0) p.part_ml[at] = make_float2(m, l);
#pragma unroll
        for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            if (d.n_tiles > 0) {
                tmem_ld32(to + c * 32, o);
                tmem_ld_wait();
            } else {
#pragma unroll
                for (int i = 0; i < 32; ++i) o[i] = 0u;
            }
            if (!mine) continue;
            if (d.part < 0) {
                uint4* dst = reinterpret_cast<uint4*>(p.out + at * D + c * 32);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    uint32_t w[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        w[e] = pack16<FP16>(__uint_as_float(o[8 * i + 2 * e]) * inv, __uint_as_float(o[8 * i + 2 * e + 1]) * inv);
                    dst[i] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            } else {
                uint4* dst = reinterpret_cast<uint4*>(p.part_o + at * D + c * 32);
#pragma unroll
                for (int i = 0; i < 8; ++i) dst[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
            }
        }
        tc_fence_before();
    }
}

template <int D, bool FP16, bool CAP, bool BIAS>
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
            mbar_init(sm.p_ready + t * 8, 4);
            mbar_init(sm.o_full + t * 8, 1);
        }
        for (int s = 0; s < kSched; ++s) {
            mbar_init(sm.sched_full + s * 8, 1);
            mbar_init(sm.sched_empty + s * 8, kSoftmaxWarps + 1);
        }
        mbar_init(sm.wind_down, 1);
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
        if (warp == kMmaWarp) mma_warp<D, FP16>(p, sm, tmem, lane);
        else if (warp == kLoadWarp) load_warp<D>(p, sm, &tm_q, &tm_k, &tm_v, n_items, lane);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;" ::"r"(tmem) : "memory");
}

template <int D, bool FP16, bool CAP, bool BIAS>
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
    const bool cap = p.cap_log2e > 0.f, bias = p.slopes || !(p.scale_log2e > 0.f);
    if (cap) return bias ? go<D, FP16, true, true>(q, k, v, p, dev, st) : go<D, FP16, true, false>(q, k, v, p, dev, st);
    return bias ? go<D, FP16, false, true>(q, k, v, p, dev, st) : go<D, FP16, false, false>(q, k, v, p, dev, st);
}

}  // namespace

cudaError_t launch_big(const CUtensorMap& q, const CUtensorMap& k, const CUtensorMap& v, const Params& p, int head_dim, bool fp16,
                       Device dev, cudaStream_t st) {
    if (head_dim == 128) return fp16 ? go2<128, true>(q, k, v, p, dev, st) : go2<128, false>(q, k, v, p, dev, st);
    return fp16 ? go2<64, true>(q, k, v, p, dev, st) : go2<64, false>(q, k, v, p, dev, st);
}

}  // namespace paged
}  // namespace plora
