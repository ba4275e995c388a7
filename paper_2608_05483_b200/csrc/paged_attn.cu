// Attention over a paged KV cache: the plan (which units a batch is cut into), the merge, and the C entry.
//
// The plan is made on the device, from lengths that only the device knows, so a step needs no copy to the
// host and can be captured in a graph.  Its first CTA writes the units; the others write what every token may see.
#include <limits.h>

#include "paged.cuh"

namespace plora {
namespace paged {

cudaError_t launch_pdl(const void* kern, dim3 grid, dim3 block, size_t smem, cudaStream_t st, void** args) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = block;
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelExC(&cfg, kern, args);
}

EncodeTiledFn encode_tiled() {
    static EncodeTiledFn fn = [] {
        void* f = nullptr;
        cudaDriverEntryPointQueryResult q;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &q) != cudaSuccess) f = nullptr;
        return reinterpret_cast<EncodeTiledFn>(f);
    }();
    return fn;
}

namespace {

constexpr int kPlanThreads = 1024;
// Splits of the tensor-core kernel (one CTA per SM).  A CTA alone is slow to start (some 4 us until its first scores), so a
// batch that gives a CTA no more than kBigOneRound keys is cut into at most one item per SM (128 of the 148: the last
// pieces are short ones); a longer one into eight per SM, which even out as they are taken from a counter.  (256 requests
// behind one prefix: 394 us with pieces of 512 keys in two rounds, 382 with one of 1024; 24 chunks behind long caches: 360
// with eight per SM, 410 with four.)
constexpr int kBigItemsOne = 128, kBigItems = kPlanSms * 8;
constexpr int kBigMinKeys = 256, kBigOneRound = 2048, kBigMaxKeys = 1 << 22;     // (tiles of keys are counted in 16 bits)
constexpr int kGroupCache = 2048;      // group starts held in shared memory
constexpr int kLargeCache = 256;       // large requests of 1024 whose units are written by a warp each (the others: by a thread)

struct Sums {        // counts that the scan carries along
    int small, big, part;
};
__device__ __forceinline__ Sums operator+(const Sums& a, const Sums& b) { return Sums{a.small + b.small, a.big + b.big, a.part + b.part}; }

__device__ __forceinline__ int clampi(int v, int lo, int hi) { return v < lo ? lo : (v > hi ? hi : v); }

// What the plan knows of a request: its tokens, its keys, and how many of them belong to its group's prefix.
struct Req {
    int tok0, n, kv, pre;
};

__device__ __forceinline__ void token_range(const Params& p, int r, int& tok0, int& n) {
    if (p.tok_start) {
        tok0 = clampi(p.tok_start[r], 0, p.n_tok);
        n = clampi(p.tok_start[r + 1], tok0, p.n_tok) - tok0;
    } else {
        tok0 = r;
        n = 1;
    }
}
__device__ __forceinline__ int kv_of(const Params& p, int r) { return clampi(p.kv_len[r], 0, p.max_kv); }

// Keys [lo, hi) visible to the token at position pos of a cache of kv tokens.
__device__ __forceinline__ TokInfo visible(const Params& p, int t, int pos, int kv) {
    TokInfo ti;
    ti.pos = pos;
    ti.lo = p.key_lo ? max(p.key_lo[t], 0) : 0;
    ti.hi = max(0, min(p.key_hi ? p.key_hi[t] : pos + 1, kv));     // (not below 0: the kernels take differences of it and keys)
    ti.pad_ = 0;
    return ti;
}

__device__ __forceinline__ Sums scan_exclusive(const Sums& v, Sums& total, Sums* warp_sums) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    Sums in = v;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const Sums a{__shfl_up_sync(0xffffffffu, in.small, d), __shfl_up_sync(0xffffffffu, in.big, d),
                     __shfl_up_sync(0xffffffffu, in.part, d)};
        if (lane >= d) in = in + a;
    }
    __syncthreads();
    if (lane == 31) warp_sums[warp] = in;
    __syncthreads();
    Sums all = warp_sums[lane];                   // (every warp scans the 32 warps' sums for itself)
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
        const Sums a{__shfl_up_sync(0xffffffffu, all.small, d), __shfl_up_sync(0xffffffffu, all.big, d),
                     __shfl_up_sync(0xffffffffu, all.part, d)};
        if (lane >= d) all = all + a;
    }
    Sums before{__shfl_sync(0xffffffffu, all.small, max(warp - 1, 0)), __shfl_sync(0xffffffffu, all.big, max(warp - 1, 0)),
                __shfl_sync(0xffffffffu, all.part, max(warp - 1, 0))};
    if (warp == 0) before = Sums{0, 0, 0};
    all = Sums{__shfl_sync(0xffffffffu, all.small, 31), __shfl_sync(0xffffffffu, all.big, 31), __shfl_sync(0xffffffffu, all.part, 31)};
    total = all;
    return Sums{before.small + in.small - v.small, before.big + in.big - v.big, before.part + in.part - v.part};
}

__device__ __forceinline__ void sum_all(long long& a, long long& b, long long (*red)[kPlanThreads / 32]) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int d = 16; d > 0; d >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, d);
        b += __shfl_xor_sync(0xffffffffu, b, d);
    }
    if (lane == 0) {
        red[0][warp] = a;
        red[1][warp] = b;
    }
    __syncthreads();
    a = red[0][lane];
    b = red[1][lane];
    for (int d = 16; d > 0; d >>= 1) {
        a += __shfl_xor_sync(0xffffffffu, a, d);
        b += __shfl_xor_sync(0xffffffffu, b, d);
    }
}

template <bool RAGGED>
__device__ __forceinline__ void write_token_info(const Params& p) {
    const int t = (blockIdx.x - 1) * kPlanThreads + threadIdx.x;
    if (t >= p.n_tok) return;
    int r = t, pos, kv;
    if (RAGGED) {
        int lo = 0, hi = p.n_req;        // the last request whose first token is not behind t
        while (hi - lo > 1) {
            const int mid = (lo + hi) >> 1;
            if (p.tok_start[mid] <= t) lo = mid;
            else hi = mid;
        }
        r = lo;
        const int end = p.tok_start[r + 1];
        kv = kv_of(p, r);
        if (t >= end || t < p.tok_start[r]) {        // a token of no request: nothing to see
            p.tok_info[t] = TokInfo{0, 0, 0, 0};
            uint4* row = reinterpret_cast<uint4*>(p.out + (size_t)t * p.n_q_heads * p.head_dim);
            for (int i = 0; i < p.n_q_heads * p.head_dim / 8; ++i) row[i] = make_uint4(0u, 0u, 0u, 0u);
            return;
        }
        pos = kv - (end - t);
    } else {
        kv = kv_of(p, r);
        pos = kv - 1;
    }
    p.tok_info[t] = visible(p, t, pos, kv);
}

// A large request, kept for the warps that write its units.
struct Large {
    Req q;
    int r, unit, part;
};

// RAGGED: token counts per request are given; GROUPED: groups are given.  (Forms of their own, because the plan's time is
// that of a few dependent loads and of fetching its code.)
template <bool RAGGED, bool GROUPED>
__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const Params p) {
    grid_wait();
    grid_launch_dependents();
    if (blockIdx.x > 0) {
        write_token_info<RAGGED>(p);
        return;
    }
    __shared__ Sums warp_sums[kPlanThreads / 32];
    __shared__ long long red[2][kPlanThreads / 32];
    __shared__ int s_group[kGroupCache + 1], s_prefix[kGroupCache];
    __shared__ int s_kv[kPlanThreads], s_tok[kPlanThreads + 1];
    __shared__ Large s_large[kLargeCache];
    __shared__ int s_merge, s_n_large;
    const int tid = threadIdx.x;
    if (tid == 0) s_merge = 0;
    // tokens of a unit: the rows of a tile of the small kernel, or two tiles of the big one
    const int TBs = max(1, kSmallRows / p.G), TBb = 2 * p.big_tile_tok;
    auto is_small = [&](int n) { return n * p.G <= kSmallRows; };       // (one token is, unless a KV head has more query heads)
    // What is looked at again and again is loaded once, all at the same time (most batches have no more requests than the
    // CTA has threads; what does not fit is read where it lies).
    const bool cached = p.n_groups <= kGroupCache, held = p.n_req <= kPlanThreads;
    if (tid < p.n_req) {
        s_kv[tid] = kv_of(p, tid);
        if (RAGGED) s_tok[tid] = clampi(p.tok_start[tid], 0, p.n_tok);
    }
    if (RAGGED && tid == 0 && held) s_tok[p.n_req] = clampi(p.tok_start[p.n_req], 0, p.n_tok);
    if (GROUPED && cached) {
        for (int g = tid; g <= p.n_groups; g += kPlanThreads) s_group[g] = clampi(p.group_start[g], 0, p.n_req);
        for (int g = tid; g < p.n_groups; g += kPlanThreads) s_prefix[g] = p.prefix_len[g];
    }
    // Ranges that do not ascend would overlap: there is no bound on the units they want, and the lists have room for what
    // ranges that share nothing can want (see caps()).  Such a batch gets no units.
    bool descends = false;
    for (int r = tid; RAGGED && r < p.n_req; r += kPlanThreads) descends |= p.tok_start[r] > p.tok_start[r + 1];
    for (int g = tid; GROUPED && g < p.n_groups; g += kPlanThreads) descends |= p.group_start[g] > p.group_start[g + 1];
    if (__syncthreads_or(descends)) {
        if (tid == 0) {
            atomicCAS(p.header, 0, PLORA_ERR_INVALID_ARG);
            p.header[kSmallUnitsWord] = p.header[kBigUnitsWord] = p.header[kMergeWord] = 0;
            p.header[kSmallNextWord] = p.header[kBigNextWord] = 0;
        }
        return;
    }
    auto kv_at = [&](int r) { return held ? s_kv[r] : kv_of(p, r); };
    auto tokens_of = [&](int r, int& tok0, int& n) {
        if (!RAGGED) {
            tok0 = r;
            n = 1;
        } else if (held) {
            tok0 = s_tok[r];
            n = max(s_tok[r + 1], tok0) - tok0;
        } else {
            token_range(p, r, tok0, n);
        }
    };
    auto gstart = [&](int g) { return cached ? s_group[g] : clampi(p.group_start[g], 0, p.n_req); };
    // tokens of the prefix that group g reads together (more than one request, one token each), 0: none
    auto read_prefix = [&](int g, int len) {
        const int s = gstart(g), e = gstart(g + 1);
        if (e - s < 2) return 0;
        int t0, t1, n;
        tokens_of(s, t0, n);
        tokens_of(e - 1, t1, n);
        return t1 + n - t0 == e - s ? clampi(len, 0, kv_at(s)) : 0;
    };
    if (GROUPED && cached) {
        for (int g = tid; g < p.n_groups; g += kPlanThreads) s_prefix[g] = read_prefix(g, s_prefix[g]);
        __syncthreads();
    }
    auto prefix_of = [&](int g) { return cached ? s_prefix[g] : read_prefix(g, p.prefix_len[g]); };
    auto request = [&](int r) {
        Req q{0, 0, 0, 0};
        if (r >= p.n_req) return q;
        tokens_of(r, q.tok0, q.n);
        q.kv = kv_at(r);
        if (GROUPED) {
            int lo = 0, hi = p.n_groups;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (gstart(mid) <= r) lo = mid;
                else hi = mid;
            }
            if (gstart(lo) <= r && r < gstart(lo + 1)) q.pre = prefix_of(lo);
        }
        return q;
    };
    // keys of block b of a request: behind the shared prefix, up to the last that one of its tokens may see (the few tokens
    // of a small unit are looked at one by one; the big kernel looks for itself)
    auto block_keys = [&](const Req& q, int b, int TB, int& k0, int& k1) {
        if (!is_small(q.n)) {
            k0 = q.pre;
            k1 = max(k0, p.key_hi ? q.kv : q.kv - q.n + min(q.n, (b + 1) * TB));
            return;
        }
        k0 = INT_MAX;
        k1 = 0;
        for (int t = q.tok0; t < q.tok0 + q.n; ++t) {
            const TokInfo ti = visible(p, t, q.kv - (q.tok0 + q.n - t), q.kv);
            if (ti.lo < ti.hi) {
                k0 = min(k0, ti.lo);
                k1 = max(k1, ti.hi);
            }
        }
        k0 = max(k0, q.pre);
        k1 = max(k0, k1);
        if (k0 == INT_MAX) k0 = k1 = 0;
    };

    // how many keys there are to read in all, over the units of each kind: the split lengths follow from it
    long long keys_s = 0, keys_b = 0;
    const Req first = request(tid);              // (kept: most batches have no more requests than the CTA has threads)
    for (int r = tid; r < p.n_req; r += kPlanThreads) {
        const Req q = r == tid ? first : request(r);
        int k0, k1;
        if (is_small(q.n)) {
            if (q.n > 0) {
                block_keys(q, 0, TBs, k0, k1);
                keys_s += k1 - k0;
            }
        } else if (p.key_hi) {           // every block may see all of the request's keys
            keys_b += (long long)((q.n + TBb - 1) / TBb) * max(0, q.kv - q.pre);
        } else if (q.kv < q.n + q.pre) {
            for (int b = 0; b * TBb < q.n; ++b) {
                block_keys(q, b, TBb, k0, k1);
                keys_b += k1 - k0;
            }
        } else {           // block b sees kv - n + min(n, (b + 1) TBb) keys
            const long long nb = (q.n + TBb - 1) / TBb;
            keys_b += nb * (q.kv - q.n - q.pre) + TBb * (nb * (nb - 1) / 2) + q.n;
        }
    }
    for (int g = tid; GROUPED && g < p.n_groups; g += kPlanThreads) {
        const int n = gstart(g + 1) - gstart(g), pre = prefix_of(g);
        if (is_small(n)) keys_s += pre;
        else keys_b += (long long)pre * ((n + TBb - 1) / TBb);
    }
    sum_all(keys_s, keys_b, red);
    const int chunk_s = small_chunk(keys_s, p.n_kv_heads);
    long long per_b = (keys_b * p.n_kv_heads + kBigItemsOne - 1) / kBigItemsOne;
    if (per_b > kBigOneRound) per_b = max((long long)kBigOneRound, (keys_b * p.n_kv_heads + kBigItems - 1) / kBigItems);
    const int chunk_b = (int)min((long long)kBigMaxKeys, max((long long)kBigMinKeys, (per_b + 127) / 128 * 128));
    auto splits_of = [&](int keys, bool small) { const int c = small ? chunk_s : chunk_b; return (keys + c - 1) / c; };
    auto put = [&](bool small, int i, const Unit& u) {
        PLORA_CHECKED(i >= 0 && i < (small ? p.cap_small : p.cap_big), p.header) (small ? p.small_units : p.big_units)[i] = checked(p, u);
    };

    Sums carry{0, 0, 0}, total;
    // the groups' prefixes: always partial results
    for (int g0 = 0; GROUPED && g0 < p.n_groups; g0 += kPlanThreads) {
        const int g = g0 + tid;
        int pre = 0, s = 0, n = 0, tok0 = 0, nn;
        if (g < p.n_groups) {
            s = gstart(g);
            n = gstart(g + 1) - s;
            pre = prefix_of(g);
            if (pre > 0) token_range(p, s, tok0, nn);
        }
        const bool small = is_small(n);
        const int TB = small ? TBs : TBb, chunk = small ? chunk_s : chunk_b;
        const int splits = splits_of(pre, small);
        const int blocks = pre > 0 ? (n + TB - 1) / TB : 0;
        const Sums want{small ? splits * blocks : 0, small ? 0 : splits * blocks, pre > 0 ? splits * n : 0};
        const Sums at = carry + scan_exclusive(want, total, warp_sums);
        if (pre > 0) {
            for (int b = 0; b < blocks; ++b) {
                const int nt = min(TB, n - b * TB);
                for (int i = 0; i < splits; ++i)
                    put(small, (small ? at.small : at.big) + b * splits + i,
                        Unit{tok0 + b * TB, nt, s, i * chunk, min(pre, (i + 1) * chunk), at.part + i * n + b * TB, {0, 0}});
            }
            for (int t = 0; t < n; ++t)
                if (row_exists(p, tok0 + t, false)) p.tok_prefix[tok0 + t] = make_int4(at.part + t, splits, n, 0);
        }
        carry = carry + total;
    }
    __syncthreads();
    // the requests' own keys
    for (int r0 = 0; r0 < p.n_req; r0 += kPlanThreads) {
        const int r = r0 + tid;
        const Req q = r0 == 0 ? first : request(r);
        const bool small = is_small(q.n);
        const int TB = small ? TBs : TBb, chunk = small ? chunk_s : chunk_b, nb = (q.n + TB - 1) / TB;
        Sums want{0, 0, 0};
        if (!small && q.kv - q.pre <= chunk && q.kv >= q.n + q.pre && !p.key_hi) {
            want.big = nb;                          // no block is split, and each has a key
            want.part = q.pre > 0 ? q.n : 0;
        } else if (!small && p.key_hi) {
            const int splits = splits_of(max(0, q.kv - q.pre), false);
            want.big = nb * splits;
            want.part = splits > 1 || q.pre > 0 ? splits * q.n : 0;
        } else {
            for (int b = 0; b < nb; ++b) {
                int k0, k1;
                block_keys(q, b, TB, k0, k1);
                const int splits = splits_of(k1 - k0, small);
                (small ? want.small : want.big) += splits;
                if (splits > 1 || q.pre > 0) want.part += splits * min(TB, q.n - b * TB);
            }
        }
        const Sums at = carry + scan_exclusive(want, total, warp_sums);
        // lists a token for the merge: `splits` partial results of its own keys from `part` on, `stride` apart, and its prefix's
        auto list = [&](int tok, int at, int part, int splits, int stride, int pre_keys) {
            const int4 pre = pre_keys > 0 ? p.tok_prefix[tok] : make_int4(0, 0, 0, 0);
            if (row_exists(p, at, false)) p.tok_merge[at] = TokMerge{tok, {part, pre.x}, {splits, pre.y}, {stride, pre.z}, 0};
        };
        // writes the units of one block, and lists its tokens if they need a merge
        auto write_block = [&](const Req& q, int r, int b, bool small, int splits, int k0, int k1, int unit, int part) {
            const int TB = small ? TBs : TBb, chunk = small ? chunk_s : chunk_b, nt = min(TB, q.n - b * TB);
            const bool direct = splits == 1 && q.pre == 0;
            for (int i = 0; i < splits; ++i)
                put(small, unit + i, Unit{q.tok0 + b * TB, nt, r, k0 + i * chunk, min(k1, k0 + (i + 1) * chunk),
                                          direct ? -1 : part + i * nt, {0, 0}});
            if (direct) return;
            const int m0 = atomicAdd(&s_merge, nt);      // (in any order: every token's result is its own)
            for (int t = 0; t < nt; ++t) list(q.tok0 + b * TB + t, m0 + t, part + t, splits, nt, q.pre);
        };
        int slot = kLargeCache;
        if (RAGGED) {
            if (tid == 0) s_n_large = 0;
            __syncthreads();
        }
        if (RAGGED && !small) slot = atomicAdd(&s_n_large, 1);
        if (slot < kLargeCache) {
            s_large[slot] = Large{q, r, at.big, at.part};
        } else if (q.n > 0) {
            // (the last block first: it sees the most keys, and the items are taken in this order)
            int unit = small ? at.small : at.big, part = at.part;
            for (int b = nb - 1; b >= 0; --b) {
                int k0, k1;
                block_keys(q, b, TB, k0, k1);
                const int splits = splits_of(k1 - k0, small);
                write_block(q, r, b, small, splits, k0, k1, unit, part);
                unit += splits;
                if (splits > 1 || q.pre > 0) part += splits * min(TB, q.n - b * TB);
            }
        }
        // large requests: a warp each, a lane per block
        if (RAGGED) __syncthreads();
        const int lane = tid & 31;
        for (int w = tid >> 5; RAGGED && w < min(s_n_large, kLargeCache); w += kPlanThreads / 32) {
            const Large big = s_large[w];
            const int blocks = (big.q.n + TBb - 1) / TBb;
            int unit = big.unit, part = big.part;
            for (int b0 = blocks - 1; b0 >= 0; b0 -= 32) {
                const int b = b0 - lane;
                int k0 = 0, k1 = 0, splits = 0, parts = 0;
                if (b >= 0) {
                    block_keys(big.q, b, TBb, k0, k1);
                    splits = splits_of(k1 - k0, false);
                    if (splits > 1 || big.q.pre > 0) parts = splits * min(TBb, big.q.n - b * TBb);
                }
                int su = splits, sp = parts;
#pragma unroll
                for (int d = 1; d < 32; d <<= 1) {
                    const int a = __shfl_up_sync(0xffffffffu, su, d), c = __shfl_up_sync(0xffffffffu, sp, d);
                    if (lane >= d) {
                        su += a;
                        sp += c;
                    }
                }
                // a block that its unit finishes is a lane's work; one with tokens to list is the warp's
                const int my_unit = unit + su - splits, my_part = part + sp - parts;
                const bool direct = splits == 1 && big.q.pre == 0;
                if (b >= 0 && direct) write_block(big.q, big.r, b, false, splits, k0, k1, my_unit, my_part);
                for (unsigned left = __ballot_sync(0xffffffffu, b >= 0 && !direct); left; left &= left - 1) {
                    const int from = __ffs(left) - 1;
                    const int bb = b0 - from, n = __shfl_sync(0xffffffffu, splits, from), u0 = __shfl_sync(0xffffffffu, my_unit, from);
                    const int p0 = __shfl_sync(0xffffffffu, my_part, from), a0 = __shfl_sync(0xffffffffu, k0, from);
                    const int a1 = __shfl_sync(0xffffffffu, k1, from), tok0 = big.q.tok0 + bb * TBb, nt = min(TBb, big.q.n - bb * TBb);
                    for (int i = lane; i < n; i += 32)
                        put(false, u0 + i, Unit{tok0, nt, big.r, a0 + i * chunk_b, min(a1, a0 + (i + 1) * chunk_b), p0 + i * nt, {0, 0}});
                    int m0 = 0;
                    if (lane == 0) m0 = atomicAdd(&s_merge, nt);
                    m0 = __shfl_sync(0xffffffffu, m0, 0);
                    for (int t = lane; t < nt; t += 32) list(tok0 + t, m0 + t, p0 + t, n, nt, big.q.pre);
                }
                unit += __shfl_sync(0xffffffffu, su, 31);
                part += __shfl_sync(0xffffffffu, sp, 31);
            }
        }
        carry = carry + total;
    }
    __syncthreads();
    if (tid == 0) {
        p.header[kSmallUnitsWord] = carry.small;
        p.header[kBigUnitsWord] = carry.big;
        p.header[kSmallNextWord] = 0;
        p.header[kBigNextWord] = 0;
        p.header[kMergeWord] = s_merge;
    }
}

// A row is a listed token's query head; D / 4 lanes share it, four dims each.  A lane looks at one partial result's maximum
// and sum, all at once (D / 4 at a time); then the outputs are added up.  Short chains of dependent loads on many rows: what
// counts is the rows under way.
template <int D, bool FP16>
__global__ void __launch_bounds__(128) merge_kernel(const Params p) {
    grid_wait();
    grid_launch_dependents();
    constexpr int L = D / 4;
    const unsigned all = 0xffffffffu;
    const int sub = threadIdx.x % L;
    const long long rows = (long long)p.header[kMergeWord] * p.n_q_heads;
    const long long step = (long long)gridDim.x * (128 / L);
    // (lanes of a warp leave together: the trip count is the warp's first row's)
    for (long long row = (long long)blockIdx.x * (128 / L) + threadIdx.x / L; row - threadIdx.x % 32 / L < rows; row += step) {
        const bool live = row < rows;
        TokMerge tm{0, {0, 0}, {0, 0}, {0, 0}, 0};
        int hq = 0;
        if (live) {
            hq = (int)(row % p.n_q_heads);
            tm = p.tok_merge[row / p.n_q_heads];
        }
        float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
        float M = -INFINITY, sum = 0.f;
        const int n = tm.n[0] + tm.n[1], n_warp = __reduce_max_sync(all, n);
        for (int i0 = 0; i0 < n_warp; i0 += L) {
            const int i = i0 + sub;
            int at = 0;
            float2 ml = make_float2(-INFINITY, 0.f);
            if (i < n) {
                at = i < tm.n[0] ? tm.base[0] + i * tm.stride[0] : tm.base[1] + (i - tm.n[0]) * tm.stride[1];
                if (row_exists(p, at, true)) ml = p.part_ml[(size_t)at * p.n_q_heads + hq];
                else at = 0;
            }
            float m = ml.x;
#pragma unroll
            for (int d = L / 2; d > 0; d >>= 1) m = fmaxf(m, __shfl_xor_sync(all, m, d));
            const float Mn = fmaxf(M, m), Me = Mn == -INFINITY ? 0.f : Mn, back = ex2(M - Me), f = ex2(ml.x - Me);
            float l = f * ml.y;
#pragma unroll
            for (int d = L / 2; d > 0; d >>= 1) l += __shfl_xor_sync(all, l, d);
            sum = sum * back + l;
            M = Mn;
            o.x *= back; o.y *= back; o.z *= back; o.w *= back;
            const int here = min(L, n_warp - i0);
#pragma unroll 4
            for (int k = 0; k < here; ++k) {
                const float fk = __shfl_sync(all, f, k, L);
                const int ak = __shfl_sync(all, at, k, L);
                if (i0 + k < n) {
                    const float4 x = *reinterpret_cast<const float4*>(p.part_o + ((size_t)ak * p.n_q_heads + hq) * D + sub * 4);
                    o.x = fmaf(fk, x.x, o.x); o.y = fmaf(fk, x.y, o.y); o.z = fmaf(fk, x.z, o.z); o.w = fmaf(fk, x.w, o.w);
                }
            }
        }
        if (live && row_exists(p, tm.tok, false)) {
            const float inv = sum > 0.f ? 1.f / sum : (sum == 0.f ? 0.f : sum);    // nothing visible: a zero row
            *reinterpret_cast<uint2*>(p.out + ((size_t)tm.tok * p.n_q_heads + hq) * D + sub * 4) =
                make_uint2(pack16<FP16>(o.x * inv, o.y * inv), pack16<FP16>(o.z * inv, o.w * inv));
        }
    }
}

size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

struct Caps {
    long long small, big, part;
};
int tile_tokens(int G) { return kBigRows / G; }
// Upper bounds of what the plan can write.  A request makes one block of each kind, a large one its tokens' more, and so does a
// group.  A split length is at least 1 / kSmallItems (1 / kBigItems) of all keys of its kind, so the units are at most one
// per block plus that many / heads, and blocks that are split make at most twice that many; or it is the longest there is
// (kSmallMaxKeys, kBigMaxKeys), and then every block is cut into at most as many pieces as the longest cache.
Caps caps(long long n_tok, long long n_req, long long max_kv, int n_kv_heads, int G) {
    const long long TBs = kSmallRows / G > 0 ? kSmallRows / G : 1, TBb = 2 * tile_tokens(G);
    const long long extra_s = (kSmallItems + n_kv_heads - 1) / n_kv_heads, extra_b = (kBigItems + n_kv_heads - 1) / n_kv_heads;
    const long long most_s = (max_kv + kSmallMaxKeys - 1) / kSmallMaxKeys, most_b = (max_kv + kBigMaxKeys - 1) / kBigMaxKeys;
    Caps c;
    c.small = 2 * n_req * most_s + extra_s + 1;
    c.big = (n_tok / TBb + 2 * n_req) * most_b + extra_b + 1;
    const long long at_longest = (most_s > 1 ? most_s : 0) + (most_b > 1 ? most_b : 0);
    const long long by_items = 2 * n_req + 4 * (extra_s * TBs + extra_b * TBb) + (n_tok + n_req) * at_longest;
    const long long by_len = n_tok * (2 * ((max_kv + kSmallMinKeys - 1) / kSmallMinKeys) + 2);
    c.part = by_items < by_len ? by_items : by_len;
    return c;
}

struct Layout {
    size_t small, big, info, merge, prefix, ml, o, total;
};
Layout layout(const Caps& c, long long n_tok, int n_q_heads, int head_dim) {
    Layout l;
    size_t at = 256;
    l.small = at; at += up256((size_t)c.small * sizeof(Unit));
    l.big = at; at += up256((size_t)c.big * sizeof(Unit));
    l.info = at; at += up256((size_t)n_tok * sizeof(TokInfo));
    l.merge = at; at += up256((size_t)n_tok * sizeof(TokMerge));
    l.prefix = at; at += up256((size_t)n_tok * sizeof(int4));
    l.ml = at; at += up256((size_t)c.part * n_q_heads * sizeof(float2));
    l.o = at; at += up256((size_t)c.part * n_q_heads * head_dim * sizeof(float));
    l.total = at;
    return l;
}

// A launch that was refused leaves its error behind in the runtime; it is reported here and must not be found by a later call.
plora_status cuda_failed() {
    (void)cudaGetLastError();
    return PLORA_ERR_CUDA;
}

bool supported(int n_q_heads, int n_kv_heads, int head_dim, int page_size) {
    if (head_dim != 64 && head_dim != 128) return false;
    if (page_size != 16 && page_size != 32 && page_size != 64 && page_size != 128) return false;
    return n_q_heads % n_kv_heads == 0 && n_q_heads / n_kv_heads <= kBigRows;
}

}  // namespace
}  // namespace paged
}  // namespace plora

using namespace plora::paged;

extern "C" PLORA_API size_t plora_attn_paged_workspace_bytes(int32_t n_tok, int32_t n_req, int32_t n_q_heads, int32_t n_kv_heads,
                                                             int32_t head_dim, int32_t page_size, int32_t max_blocks) {
    if (n_tok < 1 || n_req < 1 || n_q_heads < 1 || n_kv_heads < 1 || max_blocks < 1 || page_size < 1) return 0;
    if (!supported(n_q_heads, n_kv_heads, head_dim, page_size)) return 0;
    const Caps c = caps(n_tok, n_req, (long long)max_blocks * page_size, n_kv_heads, n_q_heads / n_kv_heads);
    return layout(c, n_tok, n_q_heads, head_dim).total;
}

extern "C" PLORA_API plora_status plora_attn_paged(const plora_paged_attn* a, void* stream) {
    if (!a || a->n_tok < 0 || a->n_req < 0 || a->n_groups < 0) return PLORA_ERR_INVALID_ARG;
    if (a->n_tok == 0) return PLORA_OK;
    if (!a->q || !a->k_cache || !a->v_cache || !a->block_table || !a->kv_len || !a->out || !a->workspace || a->n_req < 1 ||
        a->n_q_heads < 1 || a->n_kv_heads < 1 || a->n_pages < 1 || a->max_blocks < 1 || a->page_size < 1 || a->head_dim < 1)
        return PLORA_ERR_INVALID_ARG;
    if (a->type != PLORA_INPUT_BF16 && a->type != PLORA_INPUT_FP16) return PLORA_ERR_INVALID_ARG;
    if (!supported(a->n_q_heads, a->n_kv_heads, a->head_dim, a->page_size)) return PLORA_ERR_UNSUPPORTED;
    if (!a->tok_start && a->n_tok != a->n_req) return PLORA_ERR_INVALID_ARG;
    if (a->n_groups > 0 && (!a->group_start || !a->prefix_len || a->n_groups > a->n_req)) return PLORA_ERR_INVALID_ARG;
    if (!(a->softcap >= 0.f) || a->softcap > 3.0e38f || !(a->scale == a->scale)) return PLORA_ERR_INVALID_ARG;
    const long long head_row = a->head_dim, page_elems = (long long)a->n_kv_heads * a->page_size * a->head_dim;
    const long long page_stride = a->page_stride ? a->page_stride : page_elems;
    const long long q_stride = a->q_stride ? a->q_stride : (long long)a->n_q_heads * head_row;
    if (page_stride < page_elems || (page_stride & 7) || q_stride < (long long)a->n_q_heads * head_row || (q_stride & 7))
        return PLORA_ERR_INVALID_ARG;
    if (((uintptr_t)a->q & 15) || ((uintptr_t)a->k_cache & 15) || ((uintptr_t)a->v_cache & 15) || ((uintptr_t)a->out & 15) ||
        ((uintptr_t)a->workspace & 255))
        return PLORA_ERR_INVALID_ARG;
    if ((long long)a->max_blocks * a->page_size > INT32_MAX) return PLORA_ERR_UNSUPPORTED;
    Params p{};
    p.n_tok = a->n_tok; p.n_req = a->n_req; p.n_groups = a->n_groups;
    p.n_q_heads = a->n_q_heads; p.n_kv_heads = a->n_kv_heads; p.G = a->n_q_heads / a->n_kv_heads;
    p.head_dim = a->head_dim;
    p.big_tile_tok = tile_tokens(p.G);
    p.page_size = a->page_size; p.n_pages = a->n_pages; p.max_blocks = a->max_blocks;
    for (p.page_shift = 0; (1 << p.page_shift) < p.page_size; ++p.page_shift) {}
    p.max_kv = (a->max_blocks < a->n_pages ? a->max_blocks : a->n_pages) * a->page_size;
    const Caps c = caps(p.n_tok, p.n_req, p.max_kv, p.n_kv_heads, p.G);
    const Layout l = layout(c, p.n_tok, p.n_q_heads, a->head_dim);
    if (a->workspace_bytes < l.total) return PLORA_ERR_WORKSPACE;
    if (c.small * p.n_kv_heads > INT32_MAX || c.big * p.n_kv_heads > INT32_MAX || c.part > INT32_MAX) return PLORA_ERR_UNSUPPORTED;
    uint8_t* ws = static_cast<uint8_t*>(a->workspace);
    p.header = reinterpret_cast<int32_t*>(ws);
    p.small_units = reinterpret_cast<Unit*>(ws + l.small);
    p.big_units = reinterpret_cast<Unit*>(ws + l.big);
    p.tok_info = reinterpret_cast<TokInfo*>(ws + l.info);
    p.tok_merge = reinterpret_cast<TokMerge*>(ws + l.merge);
    p.tok_prefix = reinterpret_cast<int4*>(ws + l.prefix);
    p.part_ml = reinterpret_cast<float2*>(ws + l.ml);
    p.part_o = reinterpret_cast<float*>(ws + l.o);
    p.cap_small = (int32_t)c.small; p.cap_big = (int32_t)c.big; p.cap_part = (int32_t)c.part;
    p.q = static_cast<const uint16_t*>(a->q);
    p.out = static_cast<uint16_t*>(a->out);
    p.q_stride = q_stride;
    p.block_table = a->block_table; p.kv_len = a->kv_len; p.tok_start = a->tok_start;
    p.group_start = a->group_start; p.prefix_len = a->prefix_len;
    p.key_lo = a->key_lo; p.key_hi = a->key_hi; p.slopes = a->slopes;
    const float log2e = 1.4426950408889634f;
    p.scale_log2e = a->scale * log2e;
    if (a->softcap > 0.f) {
        // tanh(x) / x = c0 + c1 x^2 + ... on |x| <= 0.6, taken at x = qk * scale / cap
        const double c[5] = {0.9999999307565199, -0.33332344319327695, 0.13310648968894678, -0.05212255543054139, 0.015504650012447066};
        const double x = (double)a->scale / a->softcap;
        double power = (double)a->scale * 1.4426950408889634;
        for (int i = 0; i < 5; ++i, power *= x * x) p.cap_d[i] = (float)(c[i] * power);
        // (the square of a product must stay a number; so must the coefficients, which a cap next to nothing makes overflow)
        const double below = x != 0.0 ? 0.6 / (x < 0 ? -x : x) : 1e18;
        p.cap_poly_below = (float)(below < 1e18 ? below : 1e18);
        if (!(p.cap_d[4] - p.cap_d[4] == 0.f)) p.cap_poly_below = -1.f;
        p.cap_in = 2.f * log2e * a->scale / a->softcap;
        p.cap_log2e = a->softcap * log2e;
    }
    if (!encode_tiled()) return PLORA_ERR_UNSUPPORTED;
    const bool fp16 = a->type == PLORA_INPUT_FP16;
    // K and V as 4-D tensors [page][KV head][slot][dim]; a box is 64 dims of the slots of a page piece, 128-byte swizzled
    CUtensorMap tm[2];
    const cuuint64_t dims[4] = {(cuuint64_t)a->head_dim, (cuuint64_t)p.page_size, (cuuint64_t)p.n_kv_heads, (cuuint64_t)p.n_pages};
    const cuuint64_t strides[3] = {(cuuint64_t)a->head_dim * 2, (cuuint64_t)p.page_size * a->head_dim * 2, (cuuint64_t)page_stride * 2};
    const cuuint32_t box[4] = {64, (cuuint32_t)(p.page_size < 64 ? p.page_size : 64), 1, 1};
    const cuuint32_t es[4] = {1, 1, 1, 1};
    const void* bases[2] = {a->k_cache, a->v_cache};
    for (int i = 0; i < 2; ++i)
        if (encode_tiled()(&tm[i], fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
                           const_cast<void*>(bases[i]), dims, strides, box, es, CU_TENSOR_MAP_INTERLEAVE_NONE,
                           CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return PLORA_ERR_INVALID_ARG;
    // the queries as a 3-D tensor [token][head][dim]; a box is 64 dims of a KV head's G heads, of the tokens of a tile
    CUtensorMap tq;
    const cuuint64_t qdims[3] = {(cuuint64_t)a->head_dim, (cuuint64_t)p.n_q_heads, (cuuint64_t)p.n_tok};
    const cuuint64_t qstrides[2] = {(cuuint64_t)a->head_dim * 2, (cuuint64_t)q_stride * 2};
    const cuuint32_t qbox[3] = {64, (cuuint32_t)p.G, (cuuint32_t)p.big_tile_tok};
    if (encode_tiled()(&tq, fp16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a->q),
                       qdims, qstrides, qbox, es, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                       CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return PLORA_ERR_INVALID_ARG;
    Device dev{0, 0};
    static std::atomic<int> sms_of[64];
    if (cudaGetDevice(&dev.id) != cudaSuccess) return cuda_failed();
    if (dev.id < 64) dev.sms = sms_of[dev.id].load(std::memory_order_relaxed);
    if (dev.sms == 0) {
        if (cudaDeviceGetAttribute(&dev.sms, cudaDevAttrMultiProcessorCount, dev.id) != cudaSuccess) return cuda_failed();
        if (dev.id < 64) sms_of[dev.id].store(dev.sms, std::memory_order_relaxed);
    }
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    void* args[] = {&p};
    const bool ragged = p.tok_start != nullptr, grouped = p.n_groups > 0;
    const void* pk = ragged ? (grouped ? (const void*)plan_kernel<true, true> : (const void*)plan_kernel<true, false>)
                            : (grouped ? (const void*)plan_kernel<false, true> : (const void*)plan_kernel<false, false>);
    // Single tokens that share nothing need no plan.  (Two requests are read one by one even if they are said to share a prefix:
    // the second then finds it in L2.)
    const bool self = !ragged && p.G <= kSmallRows && p.n_req <= kSelfRequests && (!grouped || p.n_req <= 2);
    if (!self && launch_pdl(pk, dim3(1 + (p.n_tok + kPlanThreads - 1) / kPlanThreads), dim3(kPlanThreads), 0, st, args) != cudaSuccess)
        return cuda_failed();
    // a small unit holds whatever fits into its rows; single tokens that share nothing always do
    const bool big = p.G > kSmallRows || (!self && (ragged || grouped) && (long long)p.n_tok * p.G > kSmallRows);
    p.after_big = big;
    if (big && launch_big(tq, tm[0], tm[1], p, a->head_dim, fp16, dev, st) != cudaSuccess) return cuda_failed();
    if (p.G <= kSmallRows && launch_small(tm[0], tm[1], p, a->head_dim, fp16, self, dev, st) != cudaSuccess) return cuda_failed();
    const void* mk = a->head_dim == 128 ? (fp16 ? (const void*)merge_kernel<128, true> : (const void*)merge_kernel<128, false>)
                                        : (fp16 ? (const void*)merge_kernel<64, true> : (const void*)merge_kernel<64, false>);
    const int at_once = 128 / (a->head_dim / 4);
    const long long ctas = ((long long)p.n_tok * p.n_q_heads + at_once - 1) / at_once;
    const int most = dev.sms * 16;
    if (launch_pdl(mk, dim3((unsigned)(ctas < most ? ctas : most)), dim3(128), 0, st, args) != cudaSuccess) return cuda_failed();
    return PLORA_OK;
}
