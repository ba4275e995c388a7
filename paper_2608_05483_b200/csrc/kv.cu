// Around the paged KV cache: block tables and slot maps from request lengths, rotary positions, and the write
// of rotated keys and of values to their slots.
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <limits.h>
#include <stdint.h>

#include "plora.h"

namespace plora {
namespace kv {
namespace {

// ---- block tables and slot maps ---------------------------------------------------------------------------
// Request r holds c_r tokens and gets n_r more: it needs blocks [ceil(c / P), ceil((c + n) / P)) anew, and takes
// their pages from the free list in the order of (request, block).  Both the first token and the first page of a request
// are running sums over the requests.  A few KB move; the time is that of one launch and of the scan, so there is one
// kernel and nothing is handed from CTA to CTA: every CTA scans all requests (1024 at a time) and then writes the tokens
// of its own range (a thread per token) and the pages of its own share of the chunks (a thread per page), each
// finding its request by bisection in shared memory.
constexpr int kPlanThreads = 1024;

struct PlanParams {
    const int32_t *kv_len, *new_len, *free_pages, *cursor_in;
    int32_t *block_table, *tok_start, *positions, *tok_req, *slots, *kv_len_out, *cursor_out;
    int32_t n_req, page_size, page_shift, n_free, max_blocks, max_tokens;
};

// the last i in [0, n) with a[i] <= v, given a[0] <= v (of equal entries the last: empty ones are passed over)
__device__ __forceinline__ int bisect(const int* a, int n, int v) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a[mid] <= v) lo = mid;
        else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kPlanThreads) plan_kernel(const PlanParams p) {
    __shared__ int s_tok[kPlanThreads], s_page[kPlanThreads], s_old[kPlanThreads];
    __shared__ int2 s_warp[kPlanThreads / 32];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    asm volatile("griddepcontrol.wait;" ::: "memory");
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int cursor = p.cursor_in ? *p.cursor_in : 0;
    const int t = blockIdx.x * kPlanThreads + tid;      // this thread's token
    int2 carry = make_int2(0, 0);
    for (int r0 = 0, chunk = 0; r0 < p.n_req; r0 += kPlanThreads, ++chunk) {
        const int r = r0 + tid, n_here = min(kPlanThreads, p.n_req - r0);
        int old = 0, add = 0;
        if (r < p.n_req) {
            old = max(p.kv_len[r], 0);
            add = max(p.new_len[r], 0);
        }
        const int have = (old + p.page_size - 1) >> p.page_shift, need = (old + add + p.page_size - 1) >> p.page_shift;
        int2 v = make_int2(add, need - have);
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
            const int a = __shfl_up_sync(0xffffffffu, v.x, d), b = __shfl_up_sync(0xffffffffu, v.y, d);
            if (lane >= d) {
                v.x += a;
                v.y += b;
            }
        }
        if (lane == 31) s_warp[warp] = v;
        __syncthreads();
        int2 before = carry, all = carry;
#pragma unroll 8
        for (int w = 0; w < kPlanThreads / 32; ++w) {
            const int2 x = s_warp[w];
            if (w < warp) {
                before.x += x.x;
                before.y += x.y;
            }
            all.x += x.x;
            all.y += x.y;
        }
        const int tok0 = before.x + v.x - add, page0 = before.y + v.y - (need - have);
        s_tok[tid] = tok0;
        s_page[tid] = page0;
        s_old[tid] = old;
        if (blockIdx.x == 0 && r < p.n_req) {
            p.tok_start[r] = tok0;
            p.kv_len_out[r] = old + add;
        }
        __syncthreads();
        if (t < p.max_tokens && t >= carry.x && t < all.x) {
            const int i = bisect(s_tok, n_here, t);
            const int o = s_old[i], pos = o + t - s_tok[i], b = pos >> p.page_shift;
            const int first_new = (o + p.page_size - 1) >> p.page_shift;
            int page = -1;
            if (b < p.max_blocks) {
                if (b < first_new) {
                    page = p.block_table[(size_t)(r0 + i) * p.max_blocks + b];
                } else {
                    const long long f = (long long)cursor + s_page[i] + (b - first_new);
                    if (f >= 0 && f < p.n_free) page = p.free_pages[f];
                }
            }
            p.positions[t] = pos;
            p.tok_req[t] = r0 + i;
            p.slots[t] = page < 0 ? -1 : page * p.page_size + (pos & (p.page_size - 1));
        }
        if (chunk % gridDim.x == blockIdx.x) {
            for (int g = carry.y + tid; g < all.y; g += kPlanThreads) {
                const int i = bisect(s_page, n_here, g);
                const int b = ((s_old[i] + p.page_size - 1) >> p.page_shift) + (g - s_page[i]);
                const long long f = (long long)cursor + g;
                if (b < p.max_blocks)
                    p.block_table[(size_t)(r0 + i) * p.max_blocks + b] = f >= 0 && f < p.n_free ? p.free_pages[f] : -1;
            }
        }
        __syncthreads();
        carry = all;
    }
    if (t < p.max_tokens && t >= carry.x) p.positions[t] = p.tok_req[t] = p.slots[t] = -1;
    if (blockIdx.x == 0 && tid == 0) {
        p.tok_start[p.n_req] = carry.x;
        *p.cursor_out = cursor + carry.y;
    }
}

// ---- the table of cosines and sines ----------------------------------------------------------------------------
// In 64 bits: at position 10^6 a 32-bit angle would be off by 0.03.  A set-up step, made once per model.
struct TableParams {
    plora_rope_desc d;
    float* table;
    int32_t max_pos;
};
__device__ double rope_freq(const plora_rope_desc& d, int i) {
    const double two_pi = 6.283185307179586476925;
    double base = d.base;
    if (d.scaling == PLORA_ROPE_NTK) base *= pow(d.factor, (double)d.rot_dim / (d.rot_dim - 2));
    const double f = pow(base, -2.0 * i / d.rot_dim);
    if (d.scaling == PLORA_ROPE_LINEAR) return f / d.factor;
    if (d.scaling == PLORA_ROPE_BANDS) {
        const double turns = d.orig_len * f / two_pi;      // how often the pair turns over the original length
        if (turns > d.high) return f;
        if (turns < d.low) return f / d.factor;
        const double s = (turns - d.low) / (d.high - d.low);
        return (1.0 - s) * f / d.factor + s * f;
    }
    if (d.scaling == PLORA_ROPE_RAMP) {
        const double per = d.rot_dim / (2.0 * log(d.base));     // pair that turns `turns` times: per * ln(orig_len / (2 pi turns))
        const double from = fmin(fmax(floor(per * log(d.orig_len / (two_pi * d.high))), 0.0), d.rot_dim - 1.0);
        double to = fmin(fmax(ceil(per * log(d.orig_len / (two_pi * d.low))), 0.0), d.rot_dim - 1.0);
        if (to <= from) to = from + 0.001;
        const double s = fmin(fmax((i - from) / (to - from), 0.0), 1.0);
        return f / d.factor * s + f * (1.0 - s);
    }
    return f;
}
__global__ void __launch_bounds__(256) table_kernel(const TableParams p) {
    __shared__ double s_freq[PLORA_ROPE_MAX_DIM / 2];
    const int half = p.d.rot_dim / 2;
    for (int i = threadIdx.x; i < half; i += 256) s_freq[i] = rope_freq(p.d, i);
    __syncthreads();
    const long long n = (long long)p.max_pos * half;
    for (long long j = (long long)blockIdx.x * 256 + threadIdx.x; j < n; j += (long long)gridDim.x * 256) {
        const long long pos = j / half;
        double s, c;
        sincos((double)pos * s_freq[j - pos * half], &s, &c);
        reinterpret_cast<float2*>(p.table)[j] = make_float2((float)(c * p.d.magnitude), (float)(s * p.d.magnitude));
    }
}

// ---- rotary positions and the cache write -------------------------------------------------------------------------
// A thread takes 2 V values of one head: V pairs (a, b) of the rotated part (its halves, or neighbours), or 2 V values
// of the part that passes through.  Pure streaming: every projection value is read once and leaves once; bound by HBM.
struct RopeParams {
    const void *q, *k, *v;
    long long q_stride, k_stride, v_stride;   // elements between tokens
    const int32_t *positions, *slots;
    const float* table;
    void *q_out, *k_cache, *v_cache;
    long long page_stride;
    int32_t* status;
    int32_t n_tok, n_q, n_kv, head_dim, rot_dim, max_pos, page_shift, n_pages;
    int32_t per_head, per_tok;                // chunks of a head, of a token
};

template <typename T>
__device__ __forceinline__ float to_f(T x);
template <>
__device__ __forceinline__ float to_f(float x) { return x; }
template <>
__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_f(float x, __nv_bfloat16& y) { y = __float2bfloat16_rn(x); }
__device__ __forceinline__ void from_f(float x, __half& y) { y = __float2half_rn(x); }

template <typename T, int V>
struct alignas((sizeof(T) * V) < 16 ? sizeof(T) * V : 16) Vec {
    T x[V];
};
// Two runs of V values; 32 bytes that lie together go in one access.
__device__ __forceinline__ void ld32(const void* p, uint32_t (&w)[8]) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
}
__device__ __forceinline__ void st32(void* p, const uint32_t (&w)[8]) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]),
                 "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}
template <typename T, int V, bool WIDE>
__device__ __forceinline__ void load(const T* p, int ia, int ib, float (&f)[2 * V]) {
    if (WIDE && sizeof(T) * V == 16 && ib == ia + V) {
        uint32_t w[8];
        ld32(p + ia, w);
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) f[i] = to_f(reinterpret_cast<const T*>(w)[i]);
        return;
    }
    const Vec<T, V> a = *reinterpret_cast<const Vec<T, V>*>(p + ia), b = *reinterpret_cast<const Vec<T, V>*>(p + ib);
#pragma unroll
    for (int i = 0; i < V; ++i) {
        f[i] = to_f(a.x[i]);
        f[V + i] = to_f(b.x[i]);
    }
}
template <typename T, int V, bool WIDE>
__device__ __forceinline__ void store(T* p, int ia, int ib, const float (&f)[2 * V]) {
    Vec<T, V> a, b;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        from_f(f[i], a.x[i]);
        from_f(f[V + i], b.x[i]);
    }
    if (WIDE && sizeof(T) * V == 16 && ib == ia + V) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            w[i] = reinterpret_cast<const uint32_t*>(&a)[i];
            w[4 + i] = reinterpret_cast<const uint32_t*>(&b)[i];
        }
        st32(p + ia, w);
        return;
    }
    *reinterpret_cast<Vec<T, V>*>(p + ia) = a;
    *reinterpret_cast<Vec<T, V>*>(p + ib) = b;
}

// WIDE (interleaved pairs only): bases and strides are multiples of 32 bytes, and a chunk's two runs, which lie together, go in
// one access.  Measured against two of 16 bytes: 16384 tokens of 64/8 heads, 64 of 128 dims, 122 and 126 us; 8192 of 32/32, bf16,
// 77 and 80; 4096 of 32/8, fp32 in, 30.5 and 31.8.  With halves only v and what passes through have such runs, and it was no
// faster (16384 of 32/8: 43 and 42 at 64 dims, 85 and 83 at 128).
// Eight CTAs per SM, although eight of the twelve forms of 8 values then spill 8 to 20 bytes: with six and no spills the first
// takes 136 us and the second 86; what counts is the loads under way.  (Interleaved fp32 input would be some 6 % faster.)
template <typename TI, typename TO, int V, bool INTER, bool WIDE>
__global__ void __launch_bounds__(256, 8) rope_kernel(const RopeParams p) {
    // the block's first chunk: one 64-bit division for the block, small ones for the threads
    const long long first = (long long)blockIdx.x * 256;
    const int t0 = (int)(first / p.per_tok);
    const unsigned x0 = (unsigned)(first - (long long)t0 * p.per_tok) + threadIdx.x, more = x0 / (unsigned)p.per_tok;
    const int t = t0 + (int)more, rest = (int)(x0 - more * (unsigned)p.per_tok);
    if (t >= p.n_tok) return;
    const int h = rest / p.per_head, c = rest - h * p.per_head;
    const int D = p.head_dim, half = p.rot_dim / 2, rot_chunks = half / V;
    const int pos = p.positions[t], slot = p.n_kv > 0 ? p.slots[t] : -1;
    const bool is_q = h < p.n_q, is_v = h >= p.n_q + p.n_kv;
    bool pad = pos < 0;
    if (!pad && p.rot_dim > 0 && pos >= p.max_pos) {
        if (p.status) atomicCAS(p.status, 0, PLORA_ERR_INVALID_ARG);
        pad = true;
    }
    const TI* src;
    TO* dst;
    if (is_q) {
        src = static_cast<const TI*>(p.q) + t * p.q_stride + (long long)h * D;
        dst = static_cast<TO*>(p.q_out) + ((long long)t * p.n_q + h) * D;
    } else {
        const int page = slot >> p.page_shift;
        if (slot < 0 || pad) return;
        if (page >= p.n_pages) {
            if (p.status) atomicCAS(p.status, 0, PLORA_ERR_INVALID_ARG);
            return;
        }
        const int hk = h - p.n_q - (is_v ? p.n_kv : 0), P = 1 << p.page_shift;
        src = is_v ? static_cast<const TI*>(p.v) + t * p.v_stride + (long long)hk * D
                   : static_cast<const TI*>(p.k) + t * p.k_stride + (long long)hk * D;
        dst = static_cast<TO*>(is_v ? p.v_cache : p.k_cache) + page * p.page_stride + ((long long)hk * P + (slot & (P - 1))) * D;
    }
    // where the chunk's two runs of V values lie
    const bool turns = c < rot_chunks && !is_v;
    const bool split = !INTER && c < rot_chunks;
    const int ia = split ? c * V : 2 * c * V;
    const int ib = split ? half + c * V : ia + V;
    float x[2 * V];
    if (pad) {       // a padding token: its query row is zero, its key and value go nowhere
#pragma unroll
        for (int i = 0; i < 2 * V; ++i) x[i] = 0.f;
    } else {
        load<TI, V, WIDE>(src, ia, ib, x);
        if (turns) {
            const Vec<float, 2 * V> cs = *reinterpret_cast<const Vec<float, 2 * V>*>(p.table + ((long long)pos * half + c * V) * 2);
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const int ja = INTER ? 2 * v : v, jb = INTER ? 2 * v + 1 : V + v;
                const float u = x[ja], w = x[jb], co = cs.x[2 * v], si = cs.x[2 * v + 1];
                // (written out, so that every variant of the kernel rounds alike)
                x[ja] = __fmaf_rn(u, co, -__fmul_rn(w, si));
                x[jb] = __fmaf_rn(w, co, __fmul_rn(u, si));
            }
        }
    }
    store<TO, V, WIDE>(dst, ia, ib, x);
}

// Launched so that it may start while the kernel before it drains; it waits for that kernel before it reads anything.
cudaError_t launch(const void* kern, dim3 grid, unsigned block, cudaStream_t st, void** args) {
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(block);
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    const cudaError_t e = cudaLaunchKernelExC(&cfg, kern, args);
    if (e != cudaSuccess) (void)cudaGetLastError();      // reported by the caller; a later call must not find it
    return e;
}

template <typename TI, typename TO, int V, bool WIDE>
cudaError_t rope_go(const RopeParams& p, bool inter, cudaStream_t st) {
    const long long n = (long long)p.n_tok * p.per_tok;
    // (an ordinary launch: waiting for the kernel before costs every CTA some hundred cycles, and these live for two thousand)
    const unsigned grid = (unsigned)((n + 255) / 256);
    if (inter) rope_kernel<TI, TO, V, true, WIDE><<<grid, 256, 0, st>>>(p);
    else rope_kernel<TI, TO, V, false, false><<<grid, 256, 0, st>>>(p);
    return cudaGetLastError();
}
template <typename TI, typename TO>
cudaError_t rope_go_v(const RopeParams& p, int V, bool wide, bool inter, cudaStream_t st) {
    switch (V) {
        case 8: return wide ? rope_go<TI, TO, 8, true>(p, inter, st) : rope_go<TI, TO, 8, false>(p, inter, st);
        case 4: return rope_go<TI, TO, 4, false>(p, inter, st);
        case 2: return rope_go<TI, TO, 2, false>(p, inter, st);
        default: return rope_go<TI, TO, 1, false>(p, inter, st);
    }
}

bool power_of_two(int v) { return v > 0 && (v & (v - 1)) == 0; }
int shift_of(int v) {
    int s = 0;
    while ((1 << s) < v) ++s;
    return s;
}
bool aligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

}  // namespace
}  // namespace kv
}  // namespace plora

using namespace plora::kv;

extern "C" PLORA_API plora_status plora_kv_plan(const int32_t* kv_len, const int32_t* new_len, int32_t n_req, int32_t page_size,
                                                const int32_t* free_pages, int32_t n_free, const int32_t* cursor_in,
                                                int32_t* block_table, int32_t max_blocks, int32_t max_tokens, int32_t* tok_start,
                                                int32_t* positions, int32_t* tok_req, int32_t* slots, int32_t* kv_len_out,
                                                int32_t* cursor_out, void* stream) {
    if (n_req < 0 || n_free < 0 || max_tokens < 0 || max_blocks < 1) return PLORA_ERR_INVALID_ARG;
    if (!tok_start || !cursor_out || cursor_in == cursor_out) return PLORA_ERR_INVALID_ARG;
    if (n_req > 0 && (!kv_len || !new_len || !block_table || !kv_len_out || kv_len_out == kv_len || kv_len_out == new_len))
        return PLORA_ERR_INVALID_ARG;
    if (max_tokens > 0 && (!positions || !tok_req || !slots)) return PLORA_ERR_INVALID_ARG;
    if (n_free > 0 && !free_pages) return PLORA_ERR_INVALID_ARG;
    if (!power_of_two(page_size)) return PLORA_ERR_UNSUPPORTED;
    PlanParams p{kv_len, new_len, free_pages, cursor_in, block_table, tok_start, positions, tok_req, slots, kv_len_out, cursor_out,
                 n_req, page_size, shift_of(page_size), n_free, max_blocks, max_tokens};
    const int grid = max_tokens > 0 ? (int)(((long long)max_tokens + kPlanThreads - 1) / kPlanThreads) : 1;
    void* args[] = {&p};
    return launch((const void*)plan_kernel, dim3((unsigned)grid), kPlanThreads, static_cast<cudaStream_t>(stream), args) == cudaSuccess
               ? PLORA_OK
               : PLORA_ERR_CUDA;
}

extern "C" PLORA_API plora_status plora_rope_table(const plora_rope_desc* d, int32_t max_pos, float* table, void* stream) {
    if (!d || !table || max_pos < 1 || !aligned(table, 16)) return PLORA_ERR_INVALID_ARG;
    if (d->rot_dim < 2 || (d->rot_dim & 1) || d->rot_dim > PLORA_ROPE_MAX_DIM) return PLORA_ERR_UNSUPPORTED;
    if (d->scaling < PLORA_ROPE_NONE || d->scaling > PLORA_ROPE_RAMP) return PLORA_ERR_INVALID_ARG;
    if (!(d->base > 1.0) || !(d->magnitude > 0.0)) return PLORA_ERR_INVALID_ARG;
    if (d->scaling != PLORA_ROPE_NONE && !(d->factor >= 1.0)) return PLORA_ERR_INVALID_ARG;
    if (d->scaling == PLORA_ROPE_NTK && d->rot_dim < 4) return PLORA_ERR_UNSUPPORTED;
    if ((d->scaling == PLORA_ROPE_BANDS || d->scaling == PLORA_ROPE_RAMP) &&
        (!(d->orig_len >= 1.0) || !(d->low > 0.0) || !(d->high > d->low)))
        return PLORA_ERR_INVALID_ARG;
    TableParams p{*d, table, max_pos};
    const long long n = (long long)max_pos * (d->rot_dim / 2);
    const long long grid = (n + 255) / 256;
    table_kernel<<<(unsigned)(grid < 148 * 8 ? grid : 148 * 8), 256, 0, static_cast<cudaStream_t>(stream)>>>(p);
    return cudaGetLastError() == cudaSuccess ? PLORA_OK : PLORA_ERR_CUDA;
}

extern "C" PLORA_API plora_status plora_rope_cache(const plora_rope_cache_args* a, void* stream) {
    if (!a || a->n_tok < 0 || a->n_q_heads < 0 || a->n_kv_heads < 0 || a->rot_dim < 0) return PLORA_ERR_INVALID_ARG;
    if (a->n_q_heads == 0 && a->n_kv_heads == 0) return PLORA_ERR_INVALID_ARG;
    if (a->out_type != PLORA_INPUT_BF16 && a->out_type != PLORA_INPUT_FP16) return PLORA_ERR_INVALID_ARG;
    if (a->in_type != PLORA_INPUT_FP32 && a->in_type != a->out_type) return PLORA_ERR_INVALID_ARG;
    if (a->layout != PLORA_ROPE_HALF && a->layout != PLORA_ROPE_INTERLEAVED) return PLORA_ERR_INVALID_ARG;
    if (a->head_dim < 2 || (a->head_dim & 1) || a->head_dim > PLORA_ROPE_MAX_DIM || (a->rot_dim & 1) || a->rot_dim > a->head_dim)
        return PLORA_ERR_UNSUPPORTED;
    if (a->n_tok == 0) return PLORA_OK;
    if (!a->positions || (a->n_q_heads > 0 && (!a->q || !a->q_out))) return PLORA_ERR_INVALID_ARG;
    if (a->n_kv_heads > 0 && (!a->k || !a->v || !a->slots || !a->k_cache || !a->v_cache || a->n_pages < 1)) return PLORA_ERR_INVALID_ARG;
    if (a->rot_dim > 0 && (!a->table || a->max_pos < 1 || !aligned(a->table, 16))) return PLORA_ERR_INVALID_ARG;
    if (a->n_kv_heads > 0 && !power_of_two(a->page_size)) return PLORA_ERR_UNSUPPORTED;
    RopeParams p{};
    const long long D = a->head_dim, page_elems = (long long)a->n_kv_heads * a->page_size * D;
    p.q = a->q; p.k = a->k; p.v = a->v;
    p.q_stride = a->q_stride ? a->q_stride : a->n_q_heads * D;
    p.k_stride = a->k_stride ? a->k_stride : a->n_kv_heads * D;
    p.v_stride = a->v_stride ? a->v_stride : a->n_kv_heads * D;
    p.page_stride = a->page_stride ? a->page_stride : page_elems;
    if (p.q_stride < a->n_q_heads * D || p.k_stride < a->n_kv_heads * D || p.v_stride < a->n_kv_heads * D || p.page_stride < page_elems)
        return PLORA_ERR_INVALID_ARG;
    p.positions = a->positions; p.slots = a->slots; p.table = a->table;
    p.q_out = a->q_out; p.k_cache = a->k_cache; p.v_cache = a->v_cache;
    p.status = a->status;
    p.n_tok = a->n_tok; p.n_q = a->n_q_heads; p.n_kv = a->n_kv_heads; p.head_dim = a->head_dim; p.rot_dim = a->rot_dim;
    p.max_pos = a->max_pos; p.n_pages = a->n_pages;
    p.page_shift = a->n_kv_heads > 0 ? shift_of(a->page_size) : 0;
    // the widest chunk that divides every run and whose accesses are aligned
    const size_t es = a->in_type == PLORA_INPUT_FP32 ? 4 : 2;
    int V = 8;
    for (; V > 1; V >>= 1) {
        const size_t ib = es * V < 16 ? es * V : 16, ob = 2 * V;
        if ((a->rot_dim / 2) % V || (a->head_dim - a->rot_dim) % (2 * V)) continue;
        if (p.q_stride % V || p.k_stride % V || p.v_stride % V || p.page_stride % V) continue;
        if (!aligned(a->q, ib) || !aligned(a->k, ib) || !aligned(a->v, ib)) continue;
        if (!aligned(a->q_out, ob) || !aligned(a->k_cache, ob) || !aligned(a->v_cache, ob)) continue;
        break;
    }
    if (V == 1 && (!aligned(a->q, es) || !aligned(a->k, es) || !aligned(a->v, es) || !aligned(a->q_out, 2) ||
                   !aligned(a->k_cache, 2) || !aligned(a->v_cache, 2)))
        return PLORA_ERR_INVALID_ARG;
    p.per_head = a->head_dim / (2 * V);
    p.per_tok = p.per_head * (p.n_q + 2 * p.n_kv);
    if (((long long)p.n_tok * p.per_tok + 255) / 256 > INT32_MAX) return PLORA_ERR_UNSUPPORTED;
    // 32-byte accesses where the runs lie together (16 values of a 16-bit type): every base and stride has to allow them
    const int W = 32 / (int)es;
    const bool inter = a->layout == PLORA_ROPE_INTERLEAVED;
    const bool wide = inter && V == 8 && p.q_stride % W == 0 && p.k_stride % W == 0 && p.v_stride % W == 0 && p.page_stride % 16 == 0 &&
                      a->head_dim % 16 == 0 && a->rot_dim % 16 == 0 && aligned(a->q, 32) && aligned(a->k, 32) && aligned(a->v, 32) &&
                      aligned(a->q_out, 32) && aligned(a->k_cache, 32) && aligned(a->v_cache, 32);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool f32 = a->in_type == PLORA_INPUT_FP32;
    cudaError_t e;
    if (a->out_type == PLORA_INPUT_BF16)
        e = f32 ? rope_go_v<float, __nv_bfloat16>(p, V, wide, inter, st) : rope_go_v<__nv_bfloat16, __nv_bfloat16>(p, V, wide, inter, st);
    else
        e = f32 ? rope_go_v<float, __half>(p, V, wide, inter, st) : rope_go_v<__half, __half>(p, V, wide, inter, st);
    return e == cudaSuccess ? PLORA_OK : PLORA_ERR_CUDA;
}
