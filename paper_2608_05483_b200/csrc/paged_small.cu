// Attention over a paged KV cache, units of at most 16 rows: single tokens (the query heads of one KV head),
// a few tokens, or a small group of requests against its prefix.
//
// Bound by HBM: every key and value is read once per item and meets 16 rows, so what counts is the
// copies in flight.  A producer warp brings tiles of 64 tokens of K and V (tensor-map boxes, one per page
// piece, into 128-byte-swizzled rows) through a ring; four consumer warps take 16 tokens of every
// tile each: S = Q K^T and O += P V by mma.sync with the unit's rows as the 16-row operand, an online
// softmax per warp in 32 bits.  (The legacy tensor instruction fits: its operands stay in registers, and at
// 16 rows the tensor pipe is idle four fifths of the time anyway.)  At the end of an item the warps' (m, l, o)
// meet in shared memory.
// The weights P enter the second product in two parts of the input type, the rounded value and the rest (16 bits of a bf16
// weight, 22 of a half one, so that the output's own rounding is what is left of the error, as in plora_attn_decode).  With at
// most 8 rows the rests are rows 8 to 15 of the same instruction and cost nothing there; with more the product runs twice.
// Half-precision weights are held times 2^15, so that those of distant keys do not sink below its range (their row's
// maximum then counts 15 less).
#include <limits.h>

#include <type_traits>

#include "paged.cuh"

namespace plora {
namespace paged {
namespace {

constexpr int kTile = 64;
constexpr int kConsumers = 4;
constexpr int kThreads = (kConsumers + 1) * 32;
constexpr int kFlagFirst = 1, kFlagLast = 2, kFlagEnd = 4;

template <int D>
struct Cfg {
    static constexpr int kPanels = D / 64;
    static constexpr int kPanelBytes = kTile * 128;
    static constexpr int kKBytes = kPanels * kPanelBytes;
    static constexpr int kQPitch = D * 2 + 16;             // 16 bytes more than a row: eight rows in distinct banks
    static constexpr int kQOff = 2 * kKBytes;
    static constexpr int kRowOff = kQOff + kSmallRows * kQPitch;      // {lo, hi, pos, slope} of every row
    static constexpr int kHdrOff = kRowOff + kSmallRows * 16;
    static constexpr int kSlotBytes = (kHdrOff + 32 + 1023) / 1024 * 1024;
    static constexpr int kStages = D == 128 ? 3 : 5;
    static constexpr int kMeetPitch = D + 4;               // floats: o[D], m, l
    static constexpr int kSmemBytes = 1024 + kStages * kSlotBytes + (2 * kStages + 1) * 8 + 16 + 2 * kSelfRequests;
    static_assert(kConsumers * kSmallRows * kMeetPitch * 4 <= kRowOff, "the meeting place fits in a stage");
};

__device__ __forceinline__ void ldsm4(uint32_t a, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t a, uint32_t (&r)[4]) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
// D[16 x 8] += A[16 x 16] B[16 x 8], fp32 accumulate
template <bool FP16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    if (FP16)
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                     : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// two weights -> their values in the input type, and what is left of them
template <bool FP16>
__device__ __forceinline__ void split16(float x, float y, uint32_t& hi, uint32_t& lo) {
    hi = pack16<FP16>(x, y);
    float2 h;
    if (FP16) {
        h = __half22float2(*reinterpret_cast<const __half2*>(&hi));
    } else {
        h.x = __uint_as_float(hi << 16);
        h.y = __uint_as_float(hi & 0xffff0000u);
    }
    lo = pack16<FP16>(x - h.x, y - h.y);
}

// SELF: single tokens of at most kSelfRequests requests that are read one by one.  Each CTA's producer then finds its items
// from the lengths itself, and no plan kernel runs before (5 us, as much as a short decode's reads take); CTA 0 lists the
// tokens to merge.
template <int D, bool FP16, bool CAP, bool BIAS, bool SELF>
__global__ void __launch_bounds__(kThreads, 2)
small_kernel(const __grid_constant__ CUtensorMap tm_k, const __grid_constant__ CUtensorMap tm_v, const Params p) {
    using C = Cfg<D>;
    extern __shared__ uint8_t raw[];
    uint8_t* base = raw + ((1024u - (smem_u32(raw) & 1023u)) & 1023u);
    const uint32_t slots = smem_u32(base);
    uint8_t* bars = base + C::kStages * C::kSlotBytes;
    const uint32_t full = smem_u32(bars), empty = full + C::kStages * 8, meet = empty + C::kStages * 8;
    volatile int* abort_flag = reinterpret_cast<volatile int*>(bars + (2 * C::kStages + 1) * 8);
    uint16_t* first_unit = reinterpret_cast<uint16_t*>(bars + (2 * C::kStages + 1) * 8 + 16);    // SELF: of every request
    const WaitCtl wc{abort_flag, p.header};
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    if (tid == 0) {
        for (int s = 0; s < C::kStages; ++s) {
            mbar_init(full + s * 8, 1);
            mbar_init(empty + s * 8, kConsumers);
        }
        mbar_init(meet, kConsumers);
        abort_flag[0] = 0;
        mbar_init_fence();
    }
    // The units come from the plan kernel.  Behind the tensor-core kernel of the same call the plan is complete when this kernel
    // starts (that kernel waits for it before it lets this one start), and the two have nothing to do with each other: this one
    // takes the SMs that the other leaves, and waits for it only when it is done, so that its end is the end of both.  What the
    // plan wrote is read from L2 throughout, for no wait has passed over this SM's L1.
    if (!p.after_big) grid_wait();
    grid_launch_dependents();
    if (tid == 0) abort_flag[1] = __ldcg(p.header + kHookWord) == PLORA_HOOK_WITHHOLD_RELEASE;   // test hook: warp 0 never hands a stage back
    __syncthreads();
    int n_items = SELF ? 0 : __ldcg(p.header + kSmallUnitsWord) * p.n_kv_heads;
    const unsigned all = 0xffffffffu;

    if (warp == kConsumers) {
        // ------------------------------- producer warp -------------------------------
        const int bp = min(p.page_size, kTile);     // tokens of a box
        uint32_t it = 0;
        bool stopped = false;
        int next = 0, chunk = 0;
        auto keys_of = [&](int r, int& lo, int& hi) {
            const int kv = min(max(p.kv_len[r], 0), p.max_kv);
            lo = p.key_lo ? max(p.key_lo[r], 0) : 0;
            hi = max(lo, p.key_hi ? min(p.key_hi[r], kv) : kv);
            return kv;
        };
        if (SELF) {
            constexpr int kPer = kSelfRequests / 32;
            int len[kPer];
            long long keys = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = i * 32 + lane;
                len[i] = 0;
                if (r < p.n_req) {
                    int lo, hi;
                    keys_of(r, lo, hi);
                    len[i] = hi - lo;
                }
                keys += len[i];
            }
            for (int d = 16; d > 0; d >>= 1) keys += __shfl_xor_sync(all, keys, d);
            chunk = small_chunk(keys, p.n_kv_heads);
            int before = 0, listed = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int r = i * 32 + lane, n = (len[i] + chunk - 1) / chunk;
                int sum = n;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int v = __shfl_up_sync(all, sum, d);
                    if (lane >= d) sum += v;
                }
                const int first = before + sum - n;
                if (r < kSelfRequests) first_unit[r] = (uint16_t)first;
                before += __shfl_sync(all, sum, 31);
                if (blockIdx.x == 0) {      // (the partial results of a request are numbered as its units)
                    const unsigned merges = __ballot_sync(all, r < p.n_req && n != 1);
                    if (r < p.n_req && n != 1)
                        p.tok_merge[listed + __popc(merges & ((1u << lane) - 1u))] = TokMerge{r, {first, 0}, {n, 0}, {1, 0}, 0};
                    listed += __popc(merges);
                }
            }
            n_items = before * p.n_kv_heads;
            if (blockIdx.x == 0 && lane == 0) p.header[kMergeWord] = listed;
            __syncwarp();
            next = blockIdx.x;
        } else if (lane == 0) {
            next = atomicAdd(p.header + kSmallNextWord, 1);
        }
        while (!stopped) {
            const int item = __shfl_sync(all, next, 0);
            if (item >= n_items) break;
            if (SELF) next += gridDim.x;
            else if (lane == 0) next = atomicAdd(p.header + kSmallNextWord, 1);
            const int un = item / p.n_kv_heads, head = item - un * p.n_kv_heads;
            Unit u;
            TokInfo ti{0, 0, 0, 0};
            if (SELF) {
                int r = 0;                      // the last request whose first unit is not behind un (of empty ones: the next)
                for (int step = kSelfRequests / 2; step > 0; step >>= 1)
                    if (r + step < p.n_req && first_unit[r + step] <= un) r += step;
                int lo, hi;
                const int kv = keys_of(r, lo, hi), i = un - first_unit[r];
                u = Unit{r, 1, r, lo + i * chunk, min(hi, lo + (i + 1) * chunk), hi - lo > chunk ? un : -1, {0, 0}};
                ti = TokInfo{lo, hi, kv - 1, 0};
            } else {
                const int4 a = __ldcg(reinterpret_cast<const int4*>(p.small_units + un)), b = __ldcg(reinterpret_cast<const int4*>(p.small_units + un) + 1);
                u = Unit{a.x, a.y, a.z, a.w, b.x, b.y, {0, 0}};
            }
            u = checked(p, u);
            const int rows = u.ntok * p.G;
            // this lane's row: what it may see, and where its query lies
            float slope = 0.f;
            const uint16_t* qsrc = nullptr;
            if (lane < rows) {
                const int t = u.tok0 + lane / p.G, hq = head * p.G + lane % p.G;
                if (!SELF) {
                    const int4 a = __ldcg(reinterpret_cast<const int4*>(p.tok_info + t));
                    ti = TokInfo{a.x, a.y, a.z, 0};
                }
                if (BIAS) slope = __ldcg(p.slopes + hq) * 1.4426950408889634f;
                qsrc = p.q + t * p.q_stride + (size_t)hq * D;
            } else {
                ti.lo = ti.hi = 0;
            }
            ti.lo = max(ti.lo, u.k0);
            ti.hi = min(ti.hi, u.k1);
            if (!SELF && (p.key_lo || p.key_hi)) {
                // Of its keys a unit reads those that a token sees (pages of a prefix that lie before every window may be gone).
                // With none there is still a tile, without a page, for the result that says so.  (Without intervals the plan's
                // ranges are right as they are, and the pages need not wait for the tokens' intervals.)
                const bool sees = ti.lo < ti.hi;
                u.k0 = __reduce_min_sync(all, sees ? ti.lo : INT_MAX);
                u.k1 = __reduce_max_sync(all, sees ? ti.hi : 0);
                if (u.k0 >= u.k1) u.k0 = u.k1 = 0;
            }
            const int kf = u.k0 / bp * bp;
            const int n_tiles = max(1, (u.k1 - kf + kTile - 1) / kTile);
            const int32_t* table = p.block_table + (size_t)u.req * p.max_blocks;
            for (int t = 0; t < n_tiles; ++t, ++it) {
                const uint32_t slot = it % C::kStages, dst = slots + slot * C::kSlotBytes, bar = full + slot * 8;
                const int key = kf + t * kTile, nb = (min(kTile, u.k1 - key) + bp - 1) / bp;
                int page = 0;
                const int my_key = key + lane * bp;
                if (lane < nb) {
                    PLORA_CHECKED(my_key < p.max_kv, p.header) page = __ldcg(table + (my_key >> p.page_shift));
                    if ((unsigned)page >= (unsigned)p.n_pages) {   // such a page reads as zeros
                        atomicCAS(p.header, 0, PLORA_ERR_INVALID_ARG);
                        page = p.n_pages;
                    }
                }
                int ok = 1;
                if (lane == 0) ok = mbar_wait(empty + slot * 8, ((it / C::kStages) & 1) ^ 1, wc);
                if (!__shfl_sync(all, ok, 0)) {
                    stopped = true;
                    break;
                }
                if (t == 0 && lane < kSmallRows)
                    sts128(dst + C::kRowOff + lane * 16, (uint32_t)ti.lo, (uint32_t)ti.hi, (uint32_t)ti.pos, __float_as_uint(slope));
                if (lane == 0) {
                    const int flags = (t == 0 ? kFlagFirst : 0) | (t == n_tiles - 1 ? kFlagLast : 0);
                    sts128(dst + C::kHdrOff, (uint32_t)flags, (uint32_t)head, (uint32_t)key, 0u);
                    sts128(dst + C::kHdrOff + 16, (uint32_t)u.k1, (uint32_t)rows, (uint32_t)u.tok0, (uint32_t)u.part);
                }
                __syncwarp();
                if (lane == 0) mbar_arrive_expect_tx(bar, (uint32_t)nb * bp * D * 4 + (t == 0 ? (uint32_t)rows * D * 2 : 0u));
                __syncwarp();
                if (lane < nb) {
                    const int so = my_key & (p.page_size - 1);
#pragma unroll
                    for (int c = 0; c < C::kPanels; ++c) {
                        tma_box4(dst + c * C::kPanelBytes + lane * bp * 128, &tm_k, c * 64, so, head, page, bar);
                        tma_box4(dst + C::kKBytes + c * C::kPanelBytes + lane * bp * 128, &tm_v, c * 64, so, head, page, bar);
                    }
                }
                if (t == 0 && lane < rows) bulk_g2s(dst + C::kQOff + lane * C::kQPitch, qsrc, D * 2, bar);
            }
        }
        const uint32_t slot = it % C::kStages;   // tell the consumers that nothing follows
        int ok = 0;
        if (lane == 0) {
            ok = !stopped && mbar_wait(empty + slot * 8, ((it / C::kStages) & 1) ^ 1, wc);
            if (ok) {
                sts128(slots + slot * C::kSlotBytes + C::kHdrOff, (uint32_t)kFlagEnd, 0u, 0u, 0u);
                mbar_arrive(full + slot * 8);
                ++it;
            }
            // the copies of the stages armed last must have landed before the CTA's shared memory goes to another
            const long long limit = wait_limit(p.header);
            for (uint32_t k = 1; k <= (uint32_t)C::kStages && k <= it; ++k) {
                const uint32_t j = it - k;
                if (!mbar_drain(full + (j % C::kStages) * 8, (j / C::kStages) & 1, limit)) atomicCAS(p.header, 0, PLORA_ERR_TIMEOUT);
            }
        }
        __syncwarp();
        if (p.after_big) grid_wait();
        return;
    }

    // ------------------------------- consumer warps -------------------------------
    const int r0 = lane >> 2, c0 = (lane & 3) * 2;      // rows r0 and r0 + 8, columns c0, c0 + 1 of every 8-column block
    const int mi = lane >> 3, mr = lane & 7;            // ldmatrix: which 8 x 8 matrix this lane addresses, and which row of it
    constexpr float kLift = FP16 ? 15.f : 0.f;
    uint32_t qf[D / 16][4];
    float o[D / 8][4];
    float m[2], l[2], slope[2];
    int lo[2], hi[2], pos[2];
    uint32_t meetings = 0;
    bool alive = true;
    auto consumer_meet = [&]() {
        __syncwarp();
        if (lane == 0) mbar_arrive(meet);
        alive = __all_sync(all, alive && mbar_wait(meet, meetings & 1, wc));
        ++meetings;
    };
    for (uint32_t it = 0; alive; ++it) {
        const uint32_t slot = it % C::kStages;
        if (!__all_sync(all, mbar_wait(full + slot * 8, (it / C::kStages) & 1, wc))) break;
        const uint32_t st = slots + slot * C::kSlotBytes;
        const uint4 h = lds128(st + C::kHdrOff);
        const int flags = (int)h.x;
        if (flags & kFlagEnd) break;
        const uint4 h2 = lds128(st + C::kHdrOff + 16);
        const int key0 = (int)h.z + warp * 16, k1 = (int)h2.x, rows = (int)h2.y;
        if (flags & kFlagFirst) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const uint4 ri = lds128(st + C::kRowOff + (r0 + 8 * i) * 16);
                lo[i] = (int)ri.x; hi[i] = (int)ri.y; pos[i] = (int)ri.z;
                slope[i] = __uint_as_float(ri.w);
                m[i] = -INFINITY;
                l[i] = 0.f;
            }
#pragma unroll
            for (int n = 0; n < D / 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
            // rows beyond the unit's are whatever the stage held: their scores are masked, their results never leave
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks)
                ldsm4(st + C::kQOff + ((mi & 1) * 8 + mr) * C::kQPitch + (2 * ks + (mi >> 1)) * 16, qf[ks]);
        }
        const int row0 = warp * 16;
        if (key0 + 16 > k1) {
            // rows of V beyond the unit's keys may hold anything: 0 * NaN must not reach the sum (this warp alone reads them)
            for (int i = lane; i < 16 * (D / 8); i += 32) {
                const int r = i / (D / 8), c = i % (D / 8);
                if (key0 + r >= k1)
                    sts128(st + C::kKBytes + (c >> 3) * C::kPanelBytes + (row0 + r) * 128 + (((c & 7) ^ (r & 7)) << 4), 0u, 0u, 0u, 0u);
            }
            __syncwarp();
        }
        // S[16 rows][16 tokens]
        float s[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
        {
            const int r = row0 + (mi >> 1) * 8 + mr;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                const int ch = 2 * ks + (mi & 1);
                uint32_t b[4];
                ldsm4(st + (ch >> 3) * C::kPanelBytes + r * 128 + (((ch & 7) ^ (r & 7)) << 4), b);
                mma<FP16>(s[0], qf[ks], b[0], b[1]);
                mma<FP16>(s[1], qf[ks], b[2], b[3]);
            }
        }
        // weights of the first `n_rows` of this lane's two rows
        float al[2];
        auto softmax = [&](auto n_rows) {
            constexpr int R = decltype(n_rows)::value;
            float mx[2] = {-INFINITY, -INFINITY}, me[2];
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 2 * R; ++e) {
                    const int i = e >> 1, key = key0 + n * 8 + c0 + (e & 1);
                    const float v = score<CAP, BIAS>(p, s[n][e], slope[i], pos[i] - key);
                    s[n][e] = key >= lo[i] && key < hi[i] ? v : -INFINITY;
                    mx[i] = fmaxf(mx[i], s[n][e]);
                }
#pragma unroll
            for (int i = 0; i < R; ++i) {
                mx[i] = fmaxf(mx[i], __shfl_xor_sync(all, mx[i], 1));
                mx[i] = fmaxf(mx[i], __shfl_xor_sync(all, mx[i], 2));
                const float mn = fmaxf(m[i], mx[i]);
                me[i] = mn == -INFINITY ? 0.f : mn;      // a row that has seen nothing yet: all its weights are 2^-inf
                al[i] = ex2(m[i] - me[i]);
                me[i] -= kLift;
                m[i] = mn;
            }
#pragma unroll
            for (int n = 0; n < 2; ++n)
#pragma unroll
                for (int e = 0; e < 2 * R; ++e) s[n][e] = ex2(s[n][e] - me[e >> 1]);
#pragma unroll
            for (int i = 0; i < R; ++i) l[i] = l[i] * al[i] + ((s[0][2 * i] + s[0][2 * i + 1]) + (s[1][2 * i] + s[1][2 * i + 1]));
        };
        const bool halves = rows <= 8;               // rows 8 to 15 are the rests of rows 0 to 7
        uint32_t pf[4], pl[4];
        if (halves) {
            softmax(std::integral_constant<int, 1>{});
            al[1] = al[0];
            split16<FP16>(s[0][0], s[0][1], pf[0], pf[1]);
            split16<FP16>(s[1][0], s[1][1], pf[2], pf[3]);
        } else {
            softmax(std::integral_constant<int, 2>{});
#pragma unroll
            for (int e = 0; e < 4; ++e) split16<FP16>(s[e >> 1][2 * (e & 1)], s[e >> 1][2 * (e & 1) + 1], pf[e], pl[e]);
        }
        if (__any_sync(all, al[0] != 1.f || al[1] != 1.f)) {
#pragma unroll
            for (int n = 0; n < D / 8; ++n) {
                o[n][0] *= al[0]; o[n][1] *= al[0];
                o[n][2] *= al[1]; o[n][3] *= al[1];
            }
        }
        // (a form each: with the second product under a condition inside the loop the tensor pipe was busy even where it is left
        // out, 27 % instead of 18, and 64 long caches took 146 us instead of 144)
        auto product = [&](auto two) {
            const int r = row0 + (mi & 1) * 8 + mr;
#pragma unroll
            for (int j = 0; j < D / 16; ++j) {
                const int ch = 2 * j + (mi >> 1);
                uint32_t b[4];
                ldsm4_t(st + C::kKBytes + (ch >> 3) * C::kPanelBytes + r * 128 + (((ch & 7) ^ (r & 7)) << 4), b);
                mma<FP16>(o[2 * j], pf, b[0], b[1]);
                mma<FP16>(o[2 * j + 1], pf, b[2], b[3]);
                if (decltype(two)::value) {
                    mma<FP16>(o[2 * j], pl, b[0], b[1]);
                    mma<FP16>(o[2 * j + 1], pl, b[2], b[3]);
                }
            }
        };
        if (halves) product(std::false_type{});
        else product(std::true_type{});
        if (flags & kFlagLast) {
            // the four warps' shares meet in the stage whose tile has just been used
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                l[i] += __shfl_xor_sync(all, l[i], 1);
                l[i] += __shfl_xor_sync(all, l[i], 2);
            }
            if (halves) {
#pragma unroll
                for (int n = 0; n < D / 8; ++n) {
                    o[n][0] += o[n][2];
                    o[n][1] += o[n][3];
                }
            }
            consumer_meet();      // nobody reads the tile any more
            float* scr = reinterpret_cast<float*>(base + slot * C::kSlotBytes);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = r0 + 8 * i;
                if (r < rows) {
                    float* mine = scr + (warp * kSmallRows + r) * C::kMeetPitch;
#pragma unroll
                    for (int n = 0; n < D / 8; ++n) *reinterpret_cast<float2*>(mine + 8 * n + c0) = make_float2(o[n][2 * i], o[n][2 * i + 1]);
                    if (c0 == 0) *reinterpret_cast<float2*>(mine + D) = make_float2(m[i], l[i]);
                }
            }
            consumer_meet();
            if (alive) {
                const int tok0 = (int)h2.z, part = (int)h2.w;
                // four dims of a row per thread
                for (int i = tid; i < rows * (D / 4); i += kConsumers * 32) {
                    const int r = i / (D / 4), d = i % (D / 4) * 4;
                    float2 ml[kConsumers];
                    float M = -INFINITY;
#pragma unroll
                    for (int w = 0; w < kConsumers; ++w) {
                        ml[w] = *reinterpret_cast<const float2*>(scr + (w * kSmallRows + r) * C::kMeetPitch + D);
                        M = fmaxf(M, ml[w].x);
                    }
                    const float Me = M == -INFINITY ? 0.f : M;
                    float L = 0.f;
                    float4 O = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
                    for (int w = 0; w < kConsumers; ++w) {
                        const float f = ex2(ml[w].x - Me);
                        const float4 ow = *reinterpret_cast<const float4*>(scr + (w * kSmallRows + r) * C::kMeetPitch + d);
                        L = fmaf(f, ml[w].y, L);
                        O.x = fmaf(f, ow.x, O.x); O.y = fmaf(f, ow.y, O.y); O.z = fmaf(f, ow.z, O.z); O.w = fmaf(f, ow.w, O.w);
                    }
                    const int tr = r / p.G, hq = (int)h.y * p.G + r % p.G;
                    if (!row_exists(p, part < 0 ? tok0 + tr : part + tr, part >= 0)) continue;
                    if (part < 0) {
                        const float inv = L > 0.f ? 1.f / L : (L == 0.f ? 0.f : L);   // nothing visible: a zero row
                        uint2 w2 = make_uint2(pack16<FP16>(O.x * inv, O.y * inv), pack16<FP16>(O.z * inv, O.w * inv));
                        *reinterpret_cast<uint2*>(p.out + ((size_t)(tok0 + tr) * p.n_q_heads + hq) * D + d) = w2;
                    } else {
                        const size_t at = (size_t)(part + tr) * p.n_q_heads + hq;
                        *reinterpret_cast<float4*>(p.part_o + at * D + d) = O;
                        if (d == 0) p.part_ml[at] = make_float2(M - kLift, L);
                    }
                }
            }
            fence_async_smem();      // the stage goes back to the copy engine
        } else if (key0 + 16 > k1) {
            fence_async_smem();
        }
        __syncwarp();
        if (lane == 0 && !(warp == 0 && abort_flag[1])) mbar_arrive(empty + slot * 8);
    }
}

template <int D, bool FP16, bool CAP, bool BIAS, bool SELF>
cudaError_t go(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const Params& p, Device dev, cudaStream_t st) {
    auto kern = small_kernel<D, FP16, CAP, BIAS, SELF>;
    static Configured configured;
    const cudaError_t e = configured.ensure(reinterpret_cast<const void*>(kern), Cfg<D>::kSmemBytes, dev.id);
    if (e != cudaSuccess) return e;
    const long long items = (long long)p.cap_small * p.n_kv_heads;
    const int grid = (int)(items < 2 * dev.sms ? items : 2 * dev.sms);
    void* args[] = {const_cast<CUtensorMap*>(&tm_k), const_cast<CUtensorMap*>(&tm_v), const_cast<Params*>(&p)};
    return launch_pdl(reinterpret_cast<const void*>(kern), dim3(grid), dim3(kThreads), Cfg<D>::kSmemBytes, st, args);
}
template <int D, bool FP16, bool SELF>
cudaError_t go2(const CUtensorMap& k, const CUtensorMap& v, const Params& p, Device dev, cudaStream_t st) {
    if (p.cap_log2e > 0.f)
        return p.slopes ? go<D, FP16, true, true, SELF>(k, v, p, dev, st) : go<D, FP16, true, false, SELF>(k, v, p, dev, st);
    return p.slopes ? go<D, FP16, false, true, SELF>(k, v, p, dev, st) : go<D, FP16, false, false, SELF>(k, v, p, dev, st);
}
template <int D, bool FP16>
cudaError_t go3(const CUtensorMap& k, const CUtensorMap& v, const Params& p, bool self, Device dev, cudaStream_t st) {
    return self ? go2<D, FP16, true>(k, v, p, dev, st) : go2<D, FP16, false>(k, v, p, dev, st);
}

}  // namespace

cudaError_t launch_small(const CUtensorMap& k, const CUtensorMap& v, const Params& p, int head_dim, bool fp16, bool self, Device dev,
                         cudaStream_t st) {
    if (head_dim == 128) return fp16 ? go3<128, true>(k, v, p, self, dev, st) : go3<128, false>(k, v, p, self, dev, st);
    return fp16 ? go3<64, true>(k, v, p, self, dev, st) : go3<64, false>(k, v, p, self, dev, st);
}

}  // namespace paged
}  // namespace plora
