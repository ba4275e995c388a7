// Attention over a paged KV cache: what the kernels of plora_attn_paged share.
//
// The batch is cut into units.  A unit is a run of consecutive query tokens (all query heads of one KV
// head: ntok * G rows) against a range of keys of one block table; a work item is a unit and a KV head.
// A request's tokens against the keys that are its own make units, and so do the tokens of a group of
// requests against the keys of their common prefix, which are then read once for the whole group.
// Where a token's keys are dealt out to more than one unit, each leaves a partial result (maximum m,
// sum l, unnormalised output o, in the base-2 domain), and the merge kernel combines them:
//     O = sum_i 2^(m_i - m) o_i / sum_i 2^(m_i - m) l_i,   m = max_i m_i.
#pragma once

#include <cuda.h>
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "plora.h"
#include "plora_internal.cuh"

namespace plora {
namespace paged {

struct Unit {       // 32 bytes
    int32_t tok0, ntok;   // query tokens
    int32_t req;          // row of the block table
    int32_t k0, k1;       // keys [k0, k1)
    int32_t part;         // first partial (counted in tokens), -1: the unit writes the output itself
    int32_t pad_[2];
};
static_assert(sizeof(Unit) == 32, "a unit is two 16-byte words");

struct TokInfo {    // 16 bytes: keys [lo, hi) are visible to the token, which stands at pos
    int32_t lo, hi, pos, pad_;
};

// A token whose result has to be put together: n[i] partial results from number base[i] on, stride[i] apart; i = 0 its
// own keys, i = 1 its group's prefix.  (None at all: a zero row.)  Tokens whose unit writes the output are not listed.
struct TokMerge {   // 32 bytes
    int32_t tok, base[2], n[2], stride[2], pad_;
};
static_assert(sizeof(TokMerge) == 32, "two 16-byte words");

// Workspace header (256 bytes, zero before the first call): word 0 the sticky status word; words 8 and
// 10 the test hook and the wait limit of plora_attn_set_debug; the rest is rewritten by every call.
constexpr int kSmallUnitsWord = 1, kBigUnitsWord = 2, kSmallNextWord = 3, kBigNextWord = 4, kMergeWord = 5;
constexpr int kHookWord = 8, kLimitWord = 10;
constexpr long long kWaitCycles = 4000000000ll;   // default limit of a wait: about two seconds of SM clock

struct Params {
    int32_t* header;
    Unit* small_units;
    Unit* big_units;
    TokInfo* tok_info;
    TokMerge* tok_merge;      // [kMergeWord's count]
    int4* tok_prefix;         // [token] {base, n, stride}: the partial results of its group's prefix
    float2* part_ml;          // [partial token][query head] {m, l}
    float* part_o;            // [partial token][query head][D]
    int32_t cap_small, cap_big, cap_part;
    int32_t after_big;        // the mma.sync kernel runs behind the tensor-core kernel of the same call
    int32_t big_tile_tok;     // query tokens in a 128-row tile of the tensor-core kernel

    const uint16_t* q;
    uint16_t* out;
    long long q_stride;       // elements between tokens
    const int32_t* block_table;
    const int32_t* kv_len;
    const int32_t* tok_start;     // nullptr: one token per request
    const int32_t* group_start;   // nullptr: no groups
    const int32_t* prefix_len;
    const int32_t* key_lo;
    const int32_t* key_hi;
    const float* slopes;
    int32_t n_tok, n_req, n_groups, n_q_heads, n_kv_heads, G, head_dim;
    int32_t page_size, page_shift, n_pages, max_blocks;
    int32_t max_kv;           // min(max_blocks, n_pages) * page_size
    float scale_log2e;        // softmax scale times log2(e): scores live in the base-2 domain
    // capped scores, cap_log2e * tanh(qk * scale / softcap): see capped()
    float cap_d[5];           // the polynomial, for |qk| <= cap_poly_below (below 0: not used)
    float cap_poly_below;
    float cap_in, cap_log2e;  // cap_in = 2 log2(e) * scale / softcap
};

// Debug build: a unit whose tokens, keys or partial results lie outside the call's is reported and becomes one without tokens.
__device__ __forceinline__ Unit checked(const Params& p, const Unit& u) {
#ifdef PLORA_DEBUG
    const bool tokens = u.tok0 >= 0 && u.ntok >= 0 && u.ntok <= p.n_tok - u.tok0, keys = u.k0 >= 0 && u.k0 <= u.k1 && u.k1 <= p.max_kv;
    if (!tokens || !keys || u.req < 0 || u.req >= p.n_req || (u.part >= 0 && u.ntok > p.cap_part - u.part)) {
        atomicCAS(p.header, 0, PLORA_ERR_DEBUG_CHECK);
        return Unit{0, 0, 0, 0, 0, -1, {0, 0}};
    }
#endif
    return u;
}
// Where rows of the output and of the partial results lie (debug build: one that does not exist is reported).
__device__ __forceinline__ bool row_exists(const Params& p, int i, bool partial) {
#ifdef PLORA_DEBUG
    PLORA_CHECKED(i >= 0 && i < (partial ? p.cap_part : p.n_tok), p.header) return true;
    return false;
#else
    return true;
#endif
}

constexpr int kSmallRows = 16;     // rows of a unit the mma.sync kernel takes
// Requests of single tokens that the mma.sync kernel deals out by itself.  Against the plan kernel (us, self-dealt / planned; 64/8
// heads): 1 request of some 1000 keys 10.8 / 14.0, 32: 38 / 44, 128: 106 / 106, 256: 193 / 185; 256 of some 100 keys 39 / 44,
// of 1000 with one KV head 40 / 53.  Arrays for more (1024) cost every call 10 us and more.
constexpr int kSelfRequests = 256;
constexpr int kBigRows = 128;      // rows of a tile of the tensor-core kernel; a unit has up to two tiles

// Keys of a split of the mma.sync kernel: its items should number about kSmallItems (eight for each of two CTAs per SM).
constexpr int kPlanSms = 148;          // the plan aims at this many SMs, whatever the device has: it sizes the workspace
constexpr int kSmallItems = kPlanSms * 2 * 8;
constexpr int kSmallMinKeys = 128, kSmallMaxKeys = 1 << 30;     // no split shorter or longer than this
__device__ __forceinline__ int small_chunk(long long keys, int n_kv_heads) {
    const long long per = (keys * n_kv_heads + kSmallItems - 1) / kSmallItems;
    return (int)min((long long)kSmallMaxKeys, max((long long)kSmallMinKeys, (per + 63) / 64 * 64));
}

// ---- PTX wrappers ---------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count));
}
__device__ __forceinline__ void mbar_init_fence() { asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory"); }
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive_expect_tx(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool mbar_try_wait(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(bar), "r"(parity)
        : "memory");
    return ok != 0;
}
// Every wait is bounded.  When one runs out, the CTA's abort flag goes up, the status word gets
// PLORA_ERR_TIMEOUT, and every role leaves its loop.
struct WaitCtl {
    volatile int* abort_flag;
    int32_t* header;
};
__device__ __forceinline__ long long wait_limit(const int32_t* header) {
    const long long v = *reinterpret_cast<const volatile long long*>(header + kLimitWord);
    return v > 0 ? v : kWaitCycles;
}
// (Kept small: it stands at some thirty places, and an unrolled loop of tries here once made the kernels' code so large that
// instruction fetch bounded them.)
__device__ __forceinline__ bool mbar_wait_slow(uint32_t bar, uint32_t parity, const WaitCtl& w) {
    const long long t0 = clock64();
#pragma unroll 1
    for (uint32_t n = 1;; ++n) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((n & 63) == 0 && (*w.abort_flag || clock64() - t0 > wait_limit(w.header))) break;
    }
    if (!*w.abort_flag) atomicCAS(w.header, 0, PLORA_ERR_TIMEOUT);
    *w.abort_flag = 1;
    return false;
}
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, const WaitCtl& w) {
    if (mbar_try_wait(bar, parity)) return true;
    return mbar_wait_slow(bar, parity, w);
}
// A last look at a barrier before a CTA leaves, whatever the abort flag says: copies in flight must land first.
__device__ __forceinline__ bool mbar_drain(uint32_t bar, uint32_t parity, long long limit) {
    const long long t0 = clock64();
#pragma unroll 1
    while (!mbar_try_wait(bar, parity))
        if (clock64() - t0 > limit) return false;
    return true;
}
__device__ __forceinline__ void bulk_g2s(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}
// Box of the 4-D cache tensor [page][KV head][slot][dim]: 64 dims of consecutive slots, 128-byte rows, swizzled.
__device__ __forceinline__ void tma_box4(uint32_t dst, const CUtensorMap* tm, int dim, int slot, int head, int page,
                                         uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
        " [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
        "l"(reinterpret_cast<uint64_t>(tm)), "r"(dim), "r"(slot), "r"(head), "r"(page), "r"(bar)
        : "memory");
}
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w) : "memory");
}
__device__ __forceinline__ uint4 lds128(uint32_t a) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
    return v;
}
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void grid_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void grid_launch_dependents() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float rcp(float x) {
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// two floats -> one word of two 16-bit values, round to nearest even (lo in the lower half)
template <bool FP16>
__device__ __forceinline__ uint32_t pack16(float lo, float hi) {
    uint32_t r;
    if (FP16) asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    else asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}
// A capped score in the base-2 domain.  Its error reaches an exponential, so it has to be small against the score, whatever the
// cap.  For |x| <= 0.6 tanh(x) is x P(x^2), P of degree 4 fitted for the least relative error (8e-8), its coefficients scaled so
// that it takes the raw product: s (d0 + s^2 (d1 + ...)).  Beyond, it is 1 - 2 / (1 + e^2x): off by 1.5e-7 of the cap, which
// is some 3e-7 of the score there (and could be any share of a small one).  (The fast tanh instruction is off by 2^-11.)
__device__ __forceinline__ float capped_far(const Params& p, float qk) {
    return fmaf(-2.f * p.cap_log2e, rcp(1.f + ex2(qk * p.cap_in)), p.cap_log2e);
}
__device__ __forceinline__ float capped(const Params& p, float qk) {
    const float u = qk * qk;
    const float near = fmaf(fmaf(fmaf(fmaf(p.cap_d[4], u, p.cap_d[3]), u, p.cap_d[2]), u, p.cap_d[1]), u, p.cap_d[0]) * qk;
    return fabsf(qk) <= p.cap_poly_below ? near : capped_far(p, qk);
}
// Score in the base-2 domain from the raw product: scale, cap, bias by distance.
template <bool CAP, bool BIAS>
__device__ __forceinline__ float score(const Params& p, float qk, float slope, int dist) {
    float s = CAP ? capped(p, qk) : qk * p.scale_log2e;
    if (BIAS) s = fmaf(-slope, fabsf((float)dist), s);
    return s;
}

// The kernel's dynamic shared memory is asked for once per device (a host call of half a microsecond otherwise).
struct Configured {
    std::atomic<uint64_t> devices{0};
    cudaError_t ensure(const void* kern, int bytes, int dev) {
        const uint64_t bit = dev < 64 ? 1ull << dev : 0;
        if (devices.load(std::memory_order_relaxed) & bit) return cudaSuccess;
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
        if (e == cudaSuccess) devices.fetch_or(bit, std::memory_order_relaxed);
        return e;
    }
};
struct Device {
    int id, sms;
};

// The driver's call that makes tensor maps (nullptr: there is none).
typedef CUresult (*EncodeTiledFn)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                                  const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                                  CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
EncodeTiledFn encode_tiled();

// ---- launches -----------------------------------------------------------------------------------------
cudaError_t launch_small(const CUtensorMap& tm_k, const CUtensorMap& tm_v, const Params& p, int head_dim, bool fp16, bool self,
                         Device dev, cudaStream_t st);
cudaError_t launch_big(const CUtensorMap& tm_q, const CUtensorMap& tm_k, const CUtensorMap& tm_v, const Params& p, int head_dim,
                       bool fp16, Device dev, cudaStream_t st);
cudaError_t launch_pdl(const void* kern, dim3 grid, dim3 block, size_t smem, cudaStream_t st, void** args);

}  // namespace paged
}  // namespace plora
