// What stands in front of a layer's 8-bit products: the root-mean-square norm with the residual's addition, the gated
// activation of the FFN, and the set-up call that lays a weight out in 8 bits.
//
// All of them give e4m3 values q with an fp32 scale s per block, v ~ s q: s = max(max|v| / 448, 2^-126) over the block (448 is
// the largest e4m3 value; the bound keeps s, and 1 / s, a normal number for a block of zeros), q = e4m3(v / s), to nearest
// even.  Blocks are 128 columns of a row (activations) or 128 x 128 (weights).  The same pass gives v rounded to 16 bits where
// the adapters of plora_lora_delta read it.
//
// Norm and activation are bound by HBM: they read each input once and hold it in registers.  Measured: norm of 16384 x 8192, bf16, with a
// residual and both outputs 179 us (6.8 TB/s), of 512 x 5120, fp32 in, 5.3 us; activation of 16384 x 13824, bf16, both outputs, 226 us
// (7.0 TB/s), of 512 x 13824, fp32 in, 13.2 us (5.9 TB/s).  Sums, the norm's factor and the products are fp32; each output is rounded once.
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

// ---- eight columns of a row -----------------------------------------------------------------------------------------
typedef float2 Eight[4];
__device__ __forceinline__ uint32_t word_of(__nv_bfloat16, float2 v) { return paged::pack16<false>(v.x, v.y); }
__device__ __forceinline__ uint32_t word_of(__half, float2 v) { return paged::pack16<true>(v.x, v.y); }
__device__ __forceinline__ float2 pair_of(__nv_bfloat16, uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
__device__ __forceinline__ float2 pair_of(__half, uint32_t w) { return __half22float2(*reinterpret_cast<const __half2*>(&w)); }

__device__ __forceinline__ void unpack8(float, const uint32_t (&w)[8], Eight& f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
}
template <typename T>
__device__ __forceinline__ void unpack8(T t, const uint32_t (&w)[4], Eight& f) {
#pragma unroll
    for (int i = 0; i < 4; ++i) f[i] = pair_of(t, w[i]);
}
__device__ __forceinline__ void ld_words(const void* p, uint32_t (&w)[4]) {
    const uint4 v = *static_cast<const uint4*>(p);
    w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
}
__device__ __forceinline__ void ld_words(const void* p, uint32_t (&w)[8]) {
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
}
// A chunk on its way: 16-bit values as they lie in memory, so that they take up no more registers than that until they are worked on
// (activation of 16384 x 13824, bf16: 282 -> 225 us; norm of 16384 x 8192, bf16: 209 -> 179).
template <bool VEC, typename T> struct Raw { uint32_t w[4]; };
template <bool VEC> struct Raw<VEC, float> { Eight f; };
template <> struct Raw<false, __nv_bfloat16> { Eight f; };
template <> struct Raw<false, __half> { Eight f; };
// VEC: the whole chunk lies inside the row, aligned to its own size; otherwise element by element, zeros beyond `left`.
template <bool VEC, typename T>
__device__ __forceinline__ void load8(const T* p, int left, Eight& f) {
    if (VEC) {
        uint32_t w[2 * sizeof(T)];
        ld_words(p, w);
        unpack8(T(), w, f);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = make_float2(2 * i < left ? to_f(p[2 * i]) : 0.f, 2 * i + 1 < left ? to_f(p[2 * i + 1]) : 0.f);
    }
}
template <bool VEC, typename T>
__device__ __forceinline__ void fetch8(const T* p, int left, Raw<VEC, T>& r) {
    if constexpr (VEC && sizeof(T) == 2) ld_words(p, r.w);
    else load8<VEC>(p, left, r.f);
}
template <bool VEC, typename T>
__device__ __forceinline__ void open8(const Raw<VEC, T>& r, Eight& f) {
    if constexpr (VEC && sizeof(T) == 2) {
        unpack8(T(), r.w, f);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) f[i] = r.f[i];
    }
}
__device__ __forceinline__ void put8(float* p, const Eight& f) {
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(__float_as_uint(f[0].x)), "r"(__float_as_uint(f[0].y)),
                 "r"(__float_as_uint(f[1].x)), "r"(__float_as_uint(f[1].y)), "r"(__float_as_uint(f[2].x)), "r"(__float_as_uint(f[2].y)),
                 "r"(__float_as_uint(f[3].x)), "r"(__float_as_uint(f[3].y)) : "memory");
}
template <typename T>
__device__ __forceinline__ void put8(T* p, const Eight& f) {
    *reinterpret_cast<uint4*>(p) = make_uint4(word_of(T(), f[0]), word_of(T(), f[1]), word_of(T(), f[2]), word_of(T(), f[3]));
}
template <bool VEC, typename T>
__device__ __forceinline__ void store8(T* p, int left, const Eight& f) {
    if (VEC) {
        put8(p, f);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (2 * i < left) from_f(f[i].x, p[2 * i]);
            if (2 * i + 1 < left) from_f(f[i].y, p[2 * i + 1]);
        }
    }
}
// Two e4m3 values in 16 bits, the first in the lower byte; to nearest even, finite values beyond the range to the largest.
__device__ __forceinline__ uint32_t e4m3x2(float2 v) {
    uint16_t r;
    asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(v.y), "f"(v.x));
    return r;
}
template <bool VEC>
__device__ __forceinline__ void store_q8(uint8_t* p, int left, const Eight& f, float inv) {
    const float2 inv2 = make_float2(inv, inv);
    uint32_t w[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) w[i] = e4m3x2(__fmul2_rn(f[2 * i], inv2)) | e4m3x2(__fmul2_rn(f[2 * i + 1], inv2)) << 16;
    if (VEC) {
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < left) p[i] = (uint8_t)(w[i >> 2] >> 8 * (i & 3));
    }
}
// The scale of a block from its largest magnitude, and its reciprocal by the special-function unit: v / s is good to some 2^-22.
__device__ __forceinline__ float scale_of(float top, float& inv) {
    float s = top * (1.f / kTop);
    s = s < kLeast ? kLeast : s;             // (a NaN stays one)
    inv = paged::rcp(s);
    return s;
}
// Largest magnitude; a NaN stays one.
__device__ __forceinline__ float max_abs(float a, float b, float c) {
    float m;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}
__device__ __forceinline__ float max8(const Eight& f) {
    return max_abs(max_abs(f[0].x, f[0].y, f[1].x), max_abs(f[1].y, f[2].x, f[2].y), max_abs(f[3].x, f[3].y, 0.f));
}

// ---- a thread's part of a row ---------------------------------------------------------------------------------------
// Four lanes have a block of 128 columns, each four chunks of 8 columns that lie 32 columns apart: every access of the four is 64
// bytes (32 of the 8-bit output) in one piece, and a block's maximum is two shuffles for 32 values.  (With 16 lanes per block and a
// chunk each, instruction issue bounded these kernels: 24 instructions per value.)
constexpr int kChunks = 4;
typedef Eight Part[kChunks];
__device__ __forceinline__ int column_of(int t, int i) { return (t >> 2) * kBlock + i * 32 + (t & 3) * 8; }

// y, q and scale of the row's values v (thread t of the row).  All lanes of the warp call it.
template <int KY, bool VEC>
__device__ __forceinline__ void write_part(void* y, long long y_stride, uint8_t* q, long long q_stride, float* scale, int blocks, int d, long long row,
                                           int t, bool live, const Part& v) {
    typedef typename TypeOf<KY>::type TY;
    if (y && live) {
        TY* out = static_cast<TY*>(y) + row * y_stride;
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            const int c = column_of(t, i);
            if (c < d) store8<VEC>(out + c, d - c, v[i]);
        }
    }
    if (!q) return;
    float m = max_abs(max8(v[0]), max8(v[1]), max_abs(max8(v[2]), max8(v[3]), 0.f)), inv;
    m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, 1), 0.f);
    m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, 2), 0.f);
    const float s = scale_of(m, inv);
    if (!live) return;
    uint8_t* out = q + row * q_stride;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int c = column_of(t, i);
        if (c < d) store_q8<VEC>(out + c, d - c, v[i], inv);
    }
    if ((t & 3) == 0 && (t >> 2) < blocks) scale[row * blocks + (t >> 2)] = s;
}

// ---- norm ------------------------------------------------------------------------------------------------------------
struct NormParams {
    const void *x, *weight, *res;
    void *res_out, *y;
    uint8_t* q;
    float* scale;
    long long x_stride, res_stride, res_out_stride, y_stride, q_stride;
    int32_t n, d, blocks, weight_f32;
    int32_t lanes;               // of a row, where a warp has whole rows: a power of two
    float eps, offset;
};

// The sum of squares over the row's threads.
template <bool CTA>
__device__ __forceinline__ float row_sum(const Part& h, float* part, int t, int lanes) {
    float2 s[kChunks];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        s[i] = __fmul2_rn(h[i][0], h[i][0]);
#pragma unroll
        for (int e = 1; e < 4; ++e) s[i] = __ffma2_rn(h[i][e], h[i][e], s[i]);
    }
    const float2 two = __fadd2_rn(__fadd2_rn(s[0], s[1]), __fadd2_rn(s[2], s[3]));
    float sum = two.x + two.y;
    for (int d = lanes / 2; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    if (CTA) {
        const int warps = blockDim.x / 32;
        if ((t & 31) == 0) part[t >> 5] = sum;
        __syncthreads();
        sum = (t & 31) < warps ? part[t & 31] : 0.f;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
    }
    return sum;
}
// v = h * rsqrt(mean + eps) * (weight + offset)
__device__ __forceinline__ void scale8(Eight& h, const Eight& w, float f, float offset) {
    const float2 f2 = make_float2(f, f), o2 = make_float2(offset, offset);
#pragma unroll
    for (int e = 0; e < 4; ++e) h[e] = __fmul2_rn(h[e], __fmul2_rn(f2, __fadd2_rn(w[e], o2)));
}
template <int KY, bool VEC>
__device__ __forceinline__ void weigh(const NormParams& p, Part& h, float sum, int t) {
    typedef typename TypeOf<KY>::type TY;
    const float f = __frsqrt_rn(sum / (float)p.d + p.eps);
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int c = column_of(t, i), left = p.d - c;
        if (left > 0) {
            Eight w;
            if (!p.weight) {
#pragma unroll
                for (int e = 0; e < 4; ++e) w[e] = make_float2(1.f, 1.f);
            } else if (p.weight_f32) {
                load8<VEC>(static_cast<const float*>(p.weight) + c, left, w);
            } else {
                load8<VEC>(static_cast<const TY*>(p.weight) + c, left, w);
            }
            scale8(h[i], w, f, p.offset);
            if (!VEC)       // (what lies beyond the row takes no part in a block's maximum)
#pragma unroll
                for (int e = 0; e < 4; ++e) h[i][e] = make_float2(2 * e < left ? h[i][e].x : 0.f, 2 * e + 1 < left ? h[i][e].y : 0.f);
        }
    }
}

// CTA: a row per CTA; otherwise p.lanes lanes per row, and several rows per warp where a row has fewer than 32.
// (CTAs of MAXT threads per SM: three where x has 16 bits; fp32 chunks and short rows are faster with more registers, 16384 x 4096 fp32
// 108 us with two, 114 with three.  TIGHT: four.)
template <int KX, int KR, int KY, bool CTA, int MAXT, bool VEC, bool TIGHT = false>
__global__ void __launch_bounds__(MAXT, MAXT > 256 ? 1 : TIGHT ? 4 : CTA && KX != kFp32 ? 3 : 2) norm_kernel(const NormParams p) {
    typedef typename TypeOf<KX>::type TX;
    typedef typename TypeOf<KR>::type TR;
    __shared__ float part[32];
    const int lanes = CTA ? 32 : p.lanes, t = CTA ? threadIdx.x : threadIdx.x & (lanes - 1);
    const long long row = CTA ? blockIdx.x : ((long long)blockIdx.x * blockDim.x + threadIdx.x) / lanes;
    const bool live = row < p.n;
    paged::grid_wait();
    paged::grid_launch_dependents();
    Part h;
    Raw<VEC, TX> x8[kChunks];
    Raw<VEC, TR> r8[kChunks];
    const TX* x = static_cast<const TX*>(p.x) + row * p.x_stride;
    const TR* res = static_cast<const TR*>(p.res) + row * p.res_stride;
    TR* out = static_cast<TR*>(p.res_out) + row * p.res_out_stride;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int c = column_of(t, i), left = live ? p.d - c : 0;
        if (left > 0) {
            fetch8<VEC, TX>(x + c, left, x8[i]);
            if (KR != kNone) fetch8<VEC, TR>(res + c, left, r8[i]);
        }
    }
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int c = column_of(t, i), left = live ? p.d - c : 0;
        if (left > 0) {
            open8<VEC, TX>(x8[i], h[i]);
            if (KR != kNone) {
                Eight r;
                open8<VEC, TR>(r8[i], r);
#pragma unroll
                for (int e = 0; e < 4; ++e) h[i][e] = __fadd2_rn(h[i][e], r[e]);
                store8<VEC>(out + c, left, h[i]);
            }
        } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) h[i][e] = make_float2(0.f, 0.f);
        }
    }
    weigh<KY, VEC>(p, h, row_sum<CTA>(h, part, t, lanes), t);
    write_part<KY, VEC>(p.y, p.y_stride, p.q, p.q_stride, p.scale, p.blocks, p.d, row, t, live, h);
}

// ---- activation --------------------------------------------------------------------------------------------------------
struct ActParams {
    const void *gate, *up;
    void* y;
    uint8_t* q;
    float* scale;
    long long gate_stride, up_stride, y_stride, q_stride;
    int32_t n, d, blocks;
};
// sigmoid(2 z) v is v / (1 + e^-2z): silu for 2 z = v, and gelu's tanh form, v / 2 (1 + tanh z), for z = sqrt(2 / pi) (v + 0.044715 v^3).
// The exponential and the reciprocal are the special-function unit's: good to a few 2^-23, and to 2^-23 of the exponent.
template <int ACT>
__device__ __forceinline__ float act_of(float v) {
    if (ACT == PLORA_ACT_NONE) return v;
    const float z2 = ACT == PLORA_ACT_SILU ? v : 1.5957691216057308f * fmaf(0.044715f * v * v, v, v);
    return v * paged::rcp(1.f + paged::ex2(z2 * -1.4426950408889634f));
}
template <int KX, int KY, int ACT, bool GATED, bool VEC>
__global__ void __launch_bounds__(128, 6) act_kernel(const ActParams p) {
    typedef typename TypeOf<KX>::type TX;
    paged::grid_wait();
    paged::grid_launch_dependents();
    const unsigned g = (blockIdx.x * 128u + threadIdx.x) >> 2;
    const unsigned row = g / (unsigned)p.blocks, b = g - row * (unsigned)p.blocks;
    const int t = (int)b * 4 + (threadIdx.x & 3);
    const bool live = row < (unsigned)p.n;
    const TX *gate = static_cast<const TX*>(p.gate) + row * p.gate_stride, *up = static_cast<const TX*>(p.up) + row * p.up_stride;
    // Chunks beyond the row become zeros (which stay zeros): 16-bit ones after the loads (16384 x 13824, bf16, 245 us if before, 226 so), fp32
    // ones before (512 x 13824 15.2 us if after, 13.2 so).
    constexpr bool kLate = VEC && sizeof(TX) == 2;
    Part v;
    Raw<VEC, TX> g8[kChunks], u8[kChunks];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int c = column_of(t, i), left = live ? p.d - c : 0;
        if (left > 0) {
            fetch8<VEC, TX>(gate + c, left, g8[i]);
            if (GATED) fetch8<VEC, TX>(up + c, left, u8[i]);
        } else if (!kLate) {
            g8[i] = Raw<VEC, TX>{};
            u8[i] = Raw<VEC, TX>{};
        }
    }
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        if (kLate && (!live || column_of(t, i) >= p.d)) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[i][e] = make_float2(0.f, 0.f);
            continue;
        }
        Eight u;
        open8<VEC, TX>(g8[i], v[i]);
        if (GATED) open8<VEC, TX>(u8[i], u);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[i][e] = make_float2(act_of<ACT>(v[i][e].x), act_of<ACT>(v[i][e].y));
            if (GATED) v[i][e] = __fmul2_rn(v[i][e], u[e]);
        }
    }
    write_part<KY, VEC>(p.y, p.y_stride, p.q, p.q_stride, p.scale, p.blocks, p.d, row, t, live, v);
}

struct WeightParams {
    const void* w;
    uint8_t* q;
    float* scale;
    long long w_stride, q_stride;
    int32_t n, k, blocks;
};
// A CTA of 1024 threads per 128 x 128 block: a thread has two chunks of 8 columns, 64 rows apart.  (A set-up call: it lets
// no kernel start early.)
template <int KX, bool VEC>
__global__ void __launch_bounds__(1024) weight_kernel(const WeightParams p) {
    typedef typename TypeOf<KX>::type TX;
    __shared__ float part[32];
    const int r0 = blockIdx.y * kBlock + (threadIdx.x >> 4), c = blockIdx.x * kBlock + (threadIdx.x & 15) * 8, left = p.k - c;
    Eight v[2];
    float m = 0.f;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int r = r0 + 64 * i;
#pragma unroll
        for (int e = 0; e < 4; ++e) v[i][e] = make_float2(0.f, 0.f);
        if (r < p.n && left > 0) load8<VEC>(static_cast<const TX*>(p.w) + r * p.w_stride + c, left, v[i]);
        m = max_abs(m, max8(v[i]), 0.f);
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) m = max_abs(m, __shfl_xor_sync(0xffffffffu, m, d), 0.f);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = m;
    __syncthreads();
    m = part[0];
#pragma unroll
    for (int i = 1; i < 32; ++i) m = max_abs(m, part[i], 0.f);
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

// CTAs of `warps` warps that fit on an SM's four parts, each with registers for 512 / regs warps.
long long ctas_by_registers(int regs, int warps) { return 4 * (512 / ((regs + 7) / 8 * 8)) / warps; }
int registers_of(const void* kern) {
    cudaFuncAttributes a;
    if (cudaFuncGetAttributes(&a, kern) == cudaSuccess) return a.numRegs;
    (void)cudaGetLastError();
    return 64;
}

template <int KX, int KR, int KY, bool VEC>
cudaError_t norm_go(NormParams p, int sms, cudaStream_t st) {
    // Up to 1024 columns a row has 4 lanes per block, rounded up to a power of two; beyond, a CTA.  (Chosen by the columns alone:
    // rows sum alike in any batch.)
    void* args[] = {&p};
    if (p.blocks <= 8) {
        for (p.lanes = 4; p.lanes < 4 * p.blocks; p.lanes *= 2) {}
        const long long threads = (long long)p.n * p.lanes;
        return launch((const void*)norm_kernel<KX, KR, KY, false, 256, VEC>, dim3((unsigned)((threads + 255) / 256)), 256, st, args);
    }
    const unsigned threads = (unsigned)((p.blocks * 4 + 31) / 32 * 32);
    const void* kern = threads > 256 ? (const void*)norm_kernel<KX, KR, KY, true, 1024, VEC> : (const void*)norm_kernel<KX, KR, KY, true, 256, VEC>;
    if constexpr (VEC && (KX == kFp32) != (KR == kFp32)) {
        // fp32 rows take more than 64 registers a thread.  With 64 more of them fit at one time, which pays if all then do: 777 x 4168,
        // half with an fp32 residual, 9.2 us against 11.7; 1000 x 4096, fp32, 9.3 against 11.4.  With one round or several either way
        // it does not (512 x 4168 7.5 against 5.8, 1200 x 4168 14.9 against 14.2), nor where x and the residual are both fp32, which spills
        // 128 bytes a thread (777 x 4168 12.4 against 11.4, 1000 x 4096 14.0 against 12.3).
        static const int regs = registers_of((const void*)norm_kernel<KX, KR, KY, true, 256, VEC>);
        const int warps = (int)threads / 32;
        if (threads <= 256 && p.n > ctas_by_registers(regs, warps) * sms && p.n <= ctas_by_registers(64, warps) * sms)
            kern = (const void*)norm_kernel<KX, KR, KY, true, 256, VEC, true>;
    }
    return launch(kern, dim3(p.n), threads, st, args);
}
template <int KX, int KY>
cudaError_t norm_res(const NormParams& p, int res, bool vec, int sms, cudaStream_t st) {
    if (!p.res) return vec ? norm_go<KX, kNone, KY, true>(p, sms, st) : norm_go<KX, kNone, KY, false>(p, sms, st);
    if (res == kFp32) return vec ? norm_go<KX, kFp32, KY, true>(p, sms, st) : norm_go<KX, kFp32, KY, false>(p, sms, st);
    return vec ? norm_go<KX, KY, KY, true>(p, sms, st) : norm_go<KX, KY, KY, false>(p, sms, st);
}
template <int KX, int KY, int ACT>
cudaError_t act_go(const ActParams& p, bool vec, cudaStream_t st) {
    void* args[] = {const_cast<ActParams*>(&p)};
    const void* k = p.up ? (vec ? (const void*)act_kernel<KX, KY, ACT, true, true> : (const void*)act_kernel<KX, KY, ACT, true, false>)
                         : (vec ? (const void*)act_kernel<KX, KY, ACT, false, true> : (const void*)act_kernel<KX, KY, ACT, false, false>);
    return launch(k, dim3((unsigned)(((long long)p.n * p.blocks * 4 + 127) / 128)), 128, st, args);
}
template <int KX, int KY>
cudaError_t act_kind(const ActParams& p, int act, bool vec, cudaStream_t st) {
    if (act == PLORA_ACT_SILU) return act_go<KX, KY, PLORA_ACT_SILU>(p, vec, st);
    if (act == PLORA_ACT_GELU) return act_go<KX, KY, PLORA_ACT_GELU>(p, vec, st);
    return act_go<KX, KY, PLORA_ACT_NONE>(p, vec, st);
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
                 0, a->eps, a->offset};
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
    if (device(dev) != cudaSuccess) return PLORA_ERR_CUDA;
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
    if ((long long)p.n * p.blocks > (1ll << 29)) return PLORA_ERR_UNSUPPORTED;     // (the kernel counts its threads in 32 bits)
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t e;
    if (a->type == kBf16)
        e = a->in_type == kFp32 ? act_kind<kFp32, kBf16>(p, a->act, vec, st) : act_kind<kBf16, kBf16>(p, a->act, vec, st);
    else
        e = a->in_type == kFp32 ? act_kind<kFp32, kFp16>(p, a->act, vec, st) : act_kind<kFp16, kFp16>(p, a->act, vec, st);
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
