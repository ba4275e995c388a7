// What stands in front of a layer's 8-bit products: the root-mean-square norm with the residual's addition, the gated
// activation of the FFN, and the set-up call that lays a weight out in 8 bits.
//
// All of them give e4m3 values q with an fp32 scale s per block, v ~ s q: s = max(max|v| / 448, 2^-126) over the block (448 is
// the largest e4m3 value; the bound keeps s, and 1 / s, a normal number for a block of zeros), q = e4m3(v / s), to nearest
// even.  Blocks are 128 columns of a row (activations) or 128 x 128 (weights).  The same pass gives v rounded to 16 bits where
// the adapters of plora_lora_delta read it.
//
// Both activation kernels are bound by HBM: they read each input once and hold it in registers.  A thread has chunks of 8
// consecutive columns; 16 lanes have a block, so its maximum is four shuffles.  Sums, the norm's factor and the products are
// fp32; each output is rounded once.
#include "w8.cuh"

namespace plora {
namespace w8 {
namespace {

constexpr float kTop = 448.f, kLeast = 1.17549435e-38f;   // largest e4m3 value; 2^-126
constexpr int kMaxNorm = 32768;     // columns of a row that a CTA of 1024 threads holds

enum Kind { kNone = -1, kBf16 = PLORA_INPUT_BF16, kFp16 = PLORA_INPUT_FP16, kFp32 = PLORA_INPUT_FP32 };
template <int K> struct TypeOf { typedef float type; };
template <> struct TypeOf<kBf16> { typedef __nv_bfloat16 type; };
template <> struct TypeOf<kFp16> { typedef __half type; };

__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
__device__ __forceinline__ void from_f(float v, float& o) { o = v; }
__device__ __forceinline__ void from_f(float v, __nv_bfloat16& o) { o = __float2bfloat16_rn(v); }
__device__ __forceinline__ void from_f(float v, __half& o) { o = __float2half_rn(v); }

template <int BYTES> struct Words { uint32_t w[BYTES / 4]; };
__device__ __forceinline__ void ld_words(const void* p, Words<16>& r) {
    const uint4 v = *static_cast<const uint4*>(p);
    r.w[0] = v.x; r.w[1] = v.y; r.w[2] = v.z; r.w[3] = v.w;
}
__device__ __forceinline__ void ld_words(const void* p, Words<32>& r) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r.w[0]), "=r"(r.w[1]), "=r"(r.w[2]), "=r"(r.w[3]), "=r"(r.w[4]), "=r"(r.w[5]), "=r"(r.w[6]), "=r"(r.w[7]) : "l"(p));
}
__device__ __forceinline__ void st_words(void* p, const Words<16>& r) { *static_cast<uint4*>(p) = make_uint4(r.w[0], r.w[1], r.w[2], r.w[3]); }
__device__ __forceinline__ void st_words(void* p, const Words<32>& r) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(r.w[0]), "r"(r.w[1]), "r"(r.w[2]), "r"(r.w[3]),
                 "r"(r.w[4]), "r"(r.w[5]), "r"(r.w[6]), "r"(r.w[7]) : "memory");
}
// Eight columns of a row.  VEC: the whole chunk lies inside the row, aligned; otherwise element by element, zeros beyond `left`.
template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T* p, int left, float (&f)[8]) {
    if (VEC) {
        Words<8 * sizeof(T)> w;
        ld_words(p, w);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = to_f(reinterpret_cast<const T*>(w.w)[i]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = i < left ? to_f(p[i]) : 0.f;
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* p, int left, const float (&f)[8]) {
    if (VEC) {
        Words<8 * sizeof(T)> w;
#pragma unroll
        for (int i = 0; i < 8; ++i) from_f(f[i], reinterpret_cast<T*>(w.w)[i]);
        st_words(p, w);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) from_f(f[i], p[i]);
    }
}
// Two e4m3 values in 16 bits, lo in the lower byte; to nearest even, finite values beyond the range to the largest.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
    return r;
}
template <bool VEC>
__device__ __forceinline__ void store_q8(uint8_t* p, int left, const float (&f)[8], float inv) {
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        w[i] = e4m3x2(f[4 * i] * inv, f[4 * i + 1] * inv) | e4m3x2(f[4 * i + 2] * inv, f[4 * i + 3] * inv) << 16;
    if (VEC) {
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = (uint8_t)(w[i >> 2] >> 8 * (i & 3));
    }
}
// The scale of a block from its largest magnitude; 1 / s is within two roundings of the true reciprocal.  (A NaN gives NaN.)
__device__ __forceinline__ float scale_of(float top, float& inv) {
    const float s = top / kTop;
    const bool least = s < kLeast;
    inv = least ? 1.f / kLeast : kTop / top;
    return least ? kLeast : s;
}
__device__ __forceinline__ float max8(const float (&f)[8]) {
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) m = f[i] != f[i] ? f[i] : m < fabsf(f[i]) ? fabsf(f[i]) : m;
    return m;
}
// max that keeps a NaN, over the 16 lanes of a block
__device__ __forceinline__ float max16(float m) {
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) {
        const float o = __shfl_xor_sync(0xffffffffu, m, d);
        m = o != o || o > m ? o : m;
    }
    return m;
}

struct NormParams {
    const void *x, *weight, *res;
    void *res_out, *y;
    uint8_t* q;
    float* scale;
    long long x_stride, res_stride, res_out_stride, y_stride, q_stride;
    int32_t n, d, blocks, weight_f32;
    float eps, offset;
};

// ROWS rows per CTA, blockDim.x / ROWS threads each (ROWS > 1: a warp), NC chunks of 8 columns per thread; at most MAXT threads.
template <int KX, int KR, int KY, int NC, int ROWS, int MAXT, bool VEC>
__global__ void __launch_bounds__(MAXT) norm_kernel(const NormParams p) {
    typedef typename TypeOf<KX>::type TX;
    typedef typename TypeOf<KR>::type TR;
    typedef typename TypeOf<KY>::type TY;
    __shared__ float part[32];
    const int T = ROWS > 1 ? 32 : blockDim.x, t = ROWS > 1 ? threadIdx.x & 31 : threadIdx.x;
    const long long row = (long long)blockIdx.x * ROWS + (ROWS > 1 ? threadIdx.x >> 5 : 0);
    paged::grid_wait();
    paged::grid_launch_dependents();
    if (ROWS > 1 && row >= p.n) return;
    float h[NC][8];
    const TX* x = static_cast<const TX*>(p.x) + row * p.x_stride;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = (i * T + t) * 8, left = p.d - c;
        if (left > 0) load8<VEC>(x + c, left, h[i]);
        else
#pragma unroll
            for (int e = 0; e < 8; ++e) h[i][e] = 0.f;
    }
    if (KR != kNone) {
        const TR* res = static_cast<const TR*>(p.res) + row * p.res_stride;
        float r[NC][8];
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = (i * T + t) * 8, left = p.d - c;
            if (left > 0) load8<VEC>(res + c, left, r[i]);
        }
        TR* out = static_cast<TR*>(p.res_out) + row * p.res_out_stride;
#pragma unroll
        for (int i = 0; i < NC; ++i) {
            const int c = (i * T + t) * 8, left = p.d - c;
            if (left > 0) {
#pragma unroll
                for (int e = 0; e < 8; ++e) h[i][e] += r[i][e];
                store8<VEC>(out + c, left, h[i]);
            }
        }
    }
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        float s = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(h[i][e], h[i][e], s);
        sum += s;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (ROWS == 1) {
        if ((t & 31) == 0) part[t >> 5] = sum;
        __syncthreads();
        sum = (t & 31) < T / 32 ? part[t & 31] : 0.f;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    }
    const float f = __frsqrt_rn(sum / (float)p.d + p.eps);
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = (i * T + t) * 8, left = p.d - c;
        if (left > 0) {
            float w[8];
            if (!p.weight) {
#pragma unroll
                for (int e = 0; e < 8; ++e) w[e] = 1.f;
            } else if (p.weight_f32) {
                load8<VEC>(static_cast<const float*>(p.weight) + c, left, w);
            } else {
                load8<VEC>(static_cast<const TY*>(p.weight) + c, left, w);
            }
#pragma unroll
            for (int e = 0; e < 8; ++e) h[i][e] *= f * (w[e] + p.offset);
            if (p.y) store8<VEC>(static_cast<TY*>(p.y) + row * p.y_stride + c, left, h[i]);
            if (!VEC)       // (what lies beyond the row takes no part in a block's maximum)
#pragma unroll
                for (int e = 0; e < 8; ++e) h[i][e] = e < left ? h[i][e] : 0.f;
        }
    }
    if (!p.q) return;
#pragma unroll
    for (int i = 0; i < NC; ++i) {
        const int c = (i * T + t) * 8, left = p.d - c;
        float inv;
        const float s = scale_of(max16(max8(h[i])), inv);
        if (left > 0) store_q8<VEC>(p.q + row * p.q_stride + c, left, h[i], inv);
        if ((t & 15) == 0 && left > 0) p.scale[row * p.blocks + c / kBlock] = s;
    }
}

struct ActParams {
    const void *gate, *up;
    void* y;
    uint8_t* q;
    float* scale;
    long long gate_stride, up_stride, y_stride, q_stride;
    int32_t n, d, blocks;
};
// sigmoid(2 z) v is v / (1 + e^-2z): silu for 2 z = v, and gelu's tanh form, v / 2 (1 + tanh z), for z = sqrt(2 / pi) (v + 0.044715 v^3)
template <int ACT>
__device__ __forceinline__ float act_of(float v) {
    if (ACT == PLORA_ACT_NONE) return v;
    const float z2 = ACT == PLORA_ACT_SILU ? v : 1.5957691216057308f * fmaf(0.044715f * v * v, v, v);
    return __fdividef(v, 1.f + expf(-z2));
}
// 16 lanes have a block of 128 columns of a row.
template <int KX, int KY, int ACT, bool GATED, bool VEC>
__global__ void __launch_bounds__(256) act_kernel(const ActParams p) {
    typedef typename TypeOf<KX>::type TX;
    typedef typename TypeOf<KY>::type TY;
    paged::grid_wait();
    paged::grid_launch_dependents();
    const unsigned g = (blockIdx.x * 256u + threadIdx.x) >> 4;
    const unsigned row = g / (unsigned)p.blocks, b = g - row * (unsigned)p.blocks;
    const int c = (int)b * kBlock + (int)(threadIdx.x & 15) * 8, left = row < (unsigned)p.n ? p.d - c : 0;
    float v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = 0.f;
    if (left > 0) {
        float u[8];
        load8<VEC>(static_cast<const TX*>(p.gate) + row * p.gate_stride + c, left, v);
        if (GATED) load8<VEC>(static_cast<const TX*>(p.up) + row * p.up_stride + c, left, u);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            v[e] = act_of<ACT>(v[e]);
            if (GATED) v[e] *= u[e];
            if (!VEC) v[e] = e < left ? v[e] : 0.f;
        }
        if (p.y) store8<VEC>(static_cast<TY*>(p.y) + row * p.y_stride + c, left, v);
    }
    if (!p.q) return;
    float inv;
    const float s = scale_of(max16(max8(v)), inv);
    if (left > 0) {
        store_q8<VEC>(p.q + row * p.q_stride + c, left, v, inv);
        if ((threadIdx.x & 15) == 0) p.scale[(size_t)row * p.blocks + b] = s;
    }
}

struct WeightParams {
    const void* w;
    uint8_t* q;
    float* scale;
    long long w_stride, q_stride;
    int32_t n, k, blocks;
};
// A CTA of 1024 threads per 128 x 128 block: a thread has two chunks of 8 columns, 64 rows apart.  (A set-up call: it does not let
// the next kernel start early, which is what allows the product to fetch weights before it has joined the stream's order.)
template <int KX, bool VEC>
__global__ void __launch_bounds__(1024) weight_kernel(const WeightParams p) {
    typedef typename TypeOf<KX>::type TX;
    __shared__ float part[32];
    const int r0 = blockIdx.y * kBlock + (threadIdx.x >> 4), c = blockIdx.x * kBlock + (threadIdx.x & 15) * 8, left = p.k - c;
    float v[2][8], m = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = r0 + 64 * i;
#pragma unroll
        for (int e = 0; e < 8; ++e) v[i][e] = 0.f;
        if (r < p.n && left > 0) load8<VEC>(static_cast<const TX*>(p.w) + r * p.w_stride + c, left, v[i]);
        const float o = max8(v[i]);
        m = o != o || o > m ? o : m;
    }
    m = max16(m);
    const float o = __shfl_xor_sync(0xffffffffu, m, 16);
    m = o != o || o > m ? o : m;
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
    __syncthreads();
    m = part[0];
#pragma unroll
    for (int i = 1; i < 32; ++i) {
        const float o = part[i];
        m = o != o || o > m ? o : m;
    }
    float inv;
    const float s = scale_of(m, inv);
    if (threadIdx.x == 0) p.scale[(size_t)blockIdx.y * p.blocks + blockIdx.x] = s;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = r0 + 64 * i;
        if (r < p.n && left > 0) store_q8<VEC>(p.q + r * p.q_stride + c, left, v[i], inv);
    }
}

// ---- host side --------------------------------------------------------------------------------------------------
cudaError_t launch(const void* kern, dim3 grid, unsigned block, cudaStream_t st, void** args) {
    const cudaError_t e = paged::launch_pdl(kern, grid, dim3(block), 0, st, args);
    if (e != cudaSuccess) (void)cudaGetLastError();      // reported by the caller; a later call must not find it
    return e;
}
bool aligned(const void* p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }
size_t size_of(int kind) { return kind == kFp32 ? 4 : 2; }
bool is16(int kind) { return kind == kBf16 || kind == kFp16; }
bool is_kind(int kind) { return is16(kind) || kind == kFp32; }
long long up16(long long v) { return (v + 15) & ~15ll; }
// Rows of a tensor: `stride` elements apart (0: packed), each of d elements.  `fits`: the stride holds a row and elements are whole.
// `wide`: chunks of 8 elements are aligned in every row.
struct Rows {
    bool fits, wide;
};
Rows rows_of(const void* p, int kind, long long& stride, long long d) {
    if (!stride) stride = d;
    const size_t es = size_of(kind);
    return {stride >= d && aligned(p, es), stride % 8 == 0 && aligned(p, 8 * es)};
}

template <int KX, int KR, int KY, bool VEC>
cudaError_t norm_go(const NormParams& p, int sms, cudaStream_t st) {
    // A warp per row up to 1024 columns.  Beyond, a CTA per row: four chunks per thread where there are rows enough to fill the
    // SMs (bytes under way), one where a row's latency is all there is.
    const int chunks = (p.d + 7) / 8;
    void* args[] = {const_cast<NormParams*>(&p)};
    if (chunks <= 128) {
        const dim3 grid((unsigned)((p.n + 7) / 8));
        if (chunks <= 32) return launch((const void*)norm_kernel<KX, KR, KY, 1, 8, 256, VEC>, grid, 256, st, args);
        return launch((const void*)norm_kernel<KX, KR, KY, 4, 8, 256, VEC>, grid, 256, st, args);
    }
    auto threads = [&](int nc) { return (unsigned)((chunks + nc * 32 - 1) / (nc * 32) * 32); };
    if (p.n <= 2 * sms && chunks <= 1024) return launch((const void*)norm_kernel<KX, KR, KY, 1, 1, 1024, VEC>, dim3(p.n), threads(1), st, args);
    if (chunks <= 1024) return launch((const void*)norm_kernel<KX, KR, KY, 4, 1, 256, VEC>, dim3(p.n), threads(4), st, args);
    return launch((const void*)norm_kernel<KX, KR, KY, 4, 1, 1024, VEC>, dim3(p.n), threads(4), st, args);
}
template <int KX, int KY>
cudaError_t norm_res(const NormParams& p, int res, bool vec, int sms, cudaStream_t st) {
    if (!p.res) return vec ? norm_go<KX, kNone, KY, true>(p, sms, st) : norm_go<KX, kNone, KY, false>(p, sms, st);
    if (res == kFp32) return vec ? norm_go<KX, kFp32, KY, true>(p, sms, st) : norm_go<KX, kFp32, KY, false>(p, sms, st);
    return vec ? norm_go<KX, KY, KY, true>(p, sms, st) : norm_go<KX, KY, KY, false>(p, sms, st);
}
template <int KX, int KY, int ACT>
cudaError_t act_go(const ActParams& p, bool vec, unsigned grid, cudaStream_t st) {
    void* args[] = {const_cast<ActParams*>(&p)};
    const void* k = p.up ? (vec ? (const void*)act_kernel<KX, KY, ACT, true, true> : (const void*)act_kernel<KX, KY, ACT, true, false>)
                         : (vec ? (const void*)act_kernel<KX, KY, ACT, false, true> : (const void*)act_kernel<KX, KY, ACT, false, false>);
    return launch(k, dim3(grid), 256, st, args);
}
template <int KX, int KY>
cudaError_t act_kind(const ActParams& p, int act, bool vec, unsigned grid, cudaStream_t st) {
    if (act == PLORA_ACT_SILU) return act_go<KX, KY, PLORA_ACT_SILU>(p, vec, grid, st);
    if (act == PLORA_ACT_GELU) return act_go<KX, KY, PLORA_ACT_GELU>(p, vec, grid, st);
    return act_go<KX, KY, PLORA_ACT_NONE>(p, vec, grid, st);
}
template <int KX>
cudaError_t weight_go(const WeightParams& p, bool vec, dim3 grid, cudaStream_t st) {
    if (vec) weight_kernel<KX, true><<<grid, 1024, 0, st>>>(p);
    else weight_kernel<KX, false><<<grid, 1024, 0, st>>>(p);
    return cudaGetLastError();
}

}  // namespace
}  // namespace w8
}  // namespace plora

using namespace plora::w8;

extern "C" PLORA_API plora_status plora_rms_norm(const plora_rms_norm_args* a, void* stream) {
    if (!a || a->n < 0 || a->d < 1) return PLORA_ERR_INVALID_ARG;
    if (!is16(a->type) || (a->in_type != kFp32 && a->in_type != a->type)) return PLORA_ERR_INVALID_ARG;
    if (a->weight && a->weight_type != kFp32 && a->weight_type != a->type) return PLORA_ERR_INVALID_ARG;
    if (a->residual && a->residual_type != kFp32 && a->residual_type != a->type) return PLORA_ERR_INVALID_ARG;
    if (!(a->eps >= 0.f) || !(a->offset - a->offset == 0.f)) return PLORA_ERR_INVALID_ARG;
    if (a->d > kMaxNorm) return PLORA_ERR_UNSUPPORTED;
    if (a->n == 0) return PLORA_OK;
    if (!a->x || (!a->residual != !a->residual_out) || (!a->q != !a->scale) || (!a->y && !a->q && !a->residual)) return PLORA_ERR_INVALID_ARG;
    NormParams p{a->x, a->weight, a->residual, a->residual_out, a->y, static_cast<uint8_t*>(a->q), a->scale, a->x_stride, a->residual_stride,
                 a->residual_out_stride, a->y_stride, a->q_stride, a->n, a->d, (a->d + kBlock - 1) / kBlock, a->weight_type == kFp32,
                 a->eps, a->offset};
    bool vec = a->d % 8 == 0;
    auto take = [&](const void* ptr, int kind, long long& stride) {
        if (!ptr) return true;
        const Rows r = rows_of(ptr, kind, stride, a->d);
        vec = vec && r.wide;
        return r.fits;
    };
    long long none = 0;
    if (!take(a->x, a->in_type, p.x_stride) || !take(a->residual, a->residual_type, p.res_stride) ||
        !take(a->residual_out, a->residual_type, p.res_out_stride) || !take(a->y, a->type, p.y_stride) ||
        !take(a->weight, a->weight_type, none))
        return PLORA_ERR_INVALID_ARG;
    if (a->q) {
        if (!p.q_stride) p.q_stride = up16(a->d);
        if (p.q_stride < a->d || p.q_stride % 16 || !aligned(a->q, 16) || !aligned(a->scale, 4)) return PLORA_ERR_INVALID_ARG;
    }
    plora::paged::Device dev;
    if (plora::w8::device(dev) != cudaSuccess) return PLORA_ERR_CUDA;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (a->type == kBf16)
        e = a->in_type == kFp32 ? norm_res<kFp32, kBf16>(p, a->residual_type, vec, dev.sms, st) : norm_res<kBf16, kBf16>(p, a->residual_type, vec, dev.sms, st);
    else
        e = a->in_type == kFp32 ? norm_res<kFp32, kFp16>(p, a->residual_type, vec, dev.sms, st) : norm_res<kFp16, kFp16>(p, a->residual_type, vec, dev.sms, st);
    return e == cudaSuccess ? PLORA_OK : PLORA_ERR_CUDA;
}

extern "C" PLORA_API plora_status plora_gated_act(const plora_gated_act_args* a, void* stream) {
    if (!a || a->n < 0 || a->d < 1) return PLORA_ERR_INVALID_ARG;
    if (!is16(a->type) || (a->in_type != kFp32 && a->in_type != a->type)) return PLORA_ERR_INVALID_ARG;
    if (a->act != PLORA_ACT_NONE && a->act != PLORA_ACT_SILU && a->act != PLORA_ACT_GELU) return PLORA_ERR_INVALID_ARG;
    if (a->n == 0) return PLORA_OK;
    if (!a->gate || (!a->q != !a->scale) || (!a->y && !a->q)) return PLORA_ERR_INVALID_ARG;
    ActParams p{a->gate, a->up, a->y, static_cast<uint8_t*>(a->q), a->scale, a->gate_stride, a->up_stride, a->y_stride, a->q_stride, a->n,
                a->d, (int)(((long long)a->d + kBlock - 1) / kBlock)};
    bool vec = a->d % 8 == 0;
    auto take = [&](const void* ptr, int kind, long long& stride) {
        if (!ptr) return true;
        const Rows r = rows_of(ptr, kind, stride, a->d);
        vec = vec && r.wide;
        return r.fits;
    };
    if (!take(a->gate, a->in_type, p.gate_stride) || !take(a->up, a->in_type, p.up_stride) || !take(a->y, a->type, p.y_stride))
        return PLORA_ERR_INVALID_ARG;
    if (a->q) {
        if (!p.q_stride) p.q_stride = up16(a->d);
        if (p.q_stride < a->d || p.q_stride % 16 || !aligned(a->q, 16) || !aligned(a->scale, 4)) return PLORA_ERR_INVALID_ARG;
    }
    const long long lanes = (long long)p.n * p.blocks * 16;     // (the kernel counts blocks of 128 in 32 bits)
    if (lanes / 16 > (1ll << 28)) return PLORA_ERR_UNSUPPORTED;
    const unsigned grid = (unsigned)((lanes + 255) / 256);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (a->type == kBf16)
        e = a->in_type == kFp32 ? act_kind<kFp32, kBf16>(p, a->act, vec, grid, st) : act_kind<kBf16, kBf16>(p, a->act, vec, grid, st);
    else
        e = a->in_type == kFp32 ? act_kind<kFp32, kFp16>(p, a->act, vec, grid, st) : act_kind<kFp16, kFp16>(p, a->act, vec, grid, st);
    return e == cudaSuccess ? PLORA_OK : PLORA_ERR_CUDA;
}

extern "C" PLORA_API plora_status plora_quant_weight(const void* w, int32_t type, int32_t n, int32_t k, int64_t w_stride, void* q,
                                                     int64_t q_stride, float* scale, void* stream) {
    if (n < 0 || k < 1 || !is_kind(type)) return PLORA_ERR_INVALID_ARG;
    if (n == 0) return PLORA_OK;
    if (!w || !q || !scale) return PLORA_ERR_INVALID_ARG;
    WeightParams p{w, static_cast<uint8_t*>(q), scale, w_stride, q_stride, n, k, (int)(((long long)k + kBlock - 1) / kBlock)};
    const Rows r = rows_of(w, type, p.w_stride, k);
    if (!p.q_stride) p.q_stride = up16(k);
    if (!r.fits || p.q_stride < k || p.q_stride % 16 || !aligned(q, 16) || !aligned(scale, 4)) return PLORA_ERR_INVALID_ARG;
    const long long rows = ((long long)n + kBlock - 1) / kBlock;
    if (rows > 65535) return PLORA_ERR_UNSUPPORTED;
    const bool vec = r.wide && k % 8 == 0;
    const dim3 grid((unsigned)p.blocks, (unsigned)rows);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = type == kFp32 ? weight_go<kFp32>(p, vec, grid, st)
                                        : type == kBf16 ? weight_go<kBf16>(p, vec, grid, st) : weight_go<kFp16>(p, vec, grid, st);
    return e == cudaSuccess ? PLORA_OK : PLORA_ERR_CUDA;
}
