// Shared by the operators of pconv_dense.h (pconv_linear*.hip, pconv_norm.hip, pconv_distill.hip): storage types, 16-byte
// pieces of rows at any alignment, activations, checks of arguments.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>
#include <cstring>

#include "pconv_dense.h"
#include "pconv_internal.h"
#include "pconv_mfma_util.h"

#define PCONV_HIP(call)                                  \
    do {                                                 \
        hipError_t e_ = (call);                          \
        if (e_ != hipSuccess) {                          \
            ::pconv::set_hip_error(#call, (int)e_);      \
            return PCONV_EHIP;                           \
        }                                                \
    } while (0)

namespace pconv {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef short short4v __attribute__((ext_vector_type(4)));

// A storage type: its element, and how many of them a 16-byte piece holds.
template <int DT>
struct Store;
template <>
struct Store<PCONV_F32> {
    typedef float T;
    typedef float4v V;
    static constexpr int kPer = 4;
};
template <>
struct Store<PCONV_F16> {
    typedef _Float16 T;
    typedef half8 V;
    static constexpr int kPer = 8;
};
template <>
struct Store<PCONV_BF16> {
    typedef __bf16 T;
    typedef bf16x8 V;
    static constexpr int kPer = 8;
};

inline int elem_bytes(int dtype) { return dtype == PCONV_F32 ? 4 : 2; }

// 16 bytes from / to an address that is aligned to one element only: one wide access (the hardware takes any alignment).
__device__ __forceinline__ uint4v load16(const void* p) {
    uint4v v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
__device__ __forceinline__ void store16(void* p, uint4v v) { __builtin_memcpy(p, &v, 16); }

// The first n elements of a piece, zeros behind them; nothing behind them is read.
template <int DT>
__device__ __forceinline__ uint4v load_part(const typename Store<DT>::T* p, int n) {
    constexpr int P = Store<DT>::kPer;
    if (n >= P) return load16(p);
    typename Store<DT>::V v = {};
    if (n > 0) {                               // (one branch, and all of it under way at once)
        typename Store<DT>::T each[P];
#pragma unroll
        for (int i = 0; i < P; ++i) each[i] = p[i < n ? i : n - 1];
#pragma unroll
        for (int i = 0; i < P; ++i) v[i] = i < n ? each[i] : (typename Store<DT>::T)0.f;
    }
    return __builtin_bit_cast(uint4v, v);
}

// Eight consecutive values, as stored, and as floats; `n` of them are there.
template <int DT>
struct Eight {
    static constexpr int P = Store<DT>::kPer;
    uint4v raw[8 / P];
    __device__ __forceinline__ void load(const typename Store<DT>::T* p, int n) {
#pragma unroll
        for (int h = 0; h < 8 / P; ++h) raw[h] = load_part<DT>(p + h * P, n - h * P);
    }
    __device__ __forceinline__ void load_whole(const typename Store<DT>::T* p) {
#pragma unroll
        for (int h = 0; h < 8 / P; ++h) raw[h] = load16(p + h * P);
    }
    __device__ __forceinline__ void get(float out[8]) const {
#pragma unroll
        for (int h = 0; h < 8 / P; ++h) {
            const auto v = __builtin_bit_cast(typename Store<DT>::V, raw[h]);
#pragma unroll
            for (int i = 0; i < P; ++i) out[h * P + i] = (float)v[i];
        }
    }
};
template <int DT>
__device__ __forceinline__ void load8(const typename Store<DT>::T* p, int n, float out[8]) {
    Eight<DT> e;
    e.load(p, n);
    e.get(out);
}
// Eight consecutive values from floats, rounded once; the first n of them are stored.
template <int DT>
__device__ __forceinline__ void store8(typename Store<DT>::T* p, int n, const float in[8]) {
    typedef typename Store<DT>::T T;
    constexpr int P = Store<DT>::kPer;
#pragma unroll
    for (int h = 0; h < 8 / P; ++h) {
        typename Store<DT>::V v;
#pragma unroll
        for (int i = 0; i < P; ++i) v[i] = (T)in[h * P + i];
        if (n >= (h + 1) * P) {
            store16(p + h * P, __builtin_bit_cast(uint4v, v));
        } else {
#pragma unroll
            for (int i = 0; i < P; ++i)
                if (h * P + i < n) p[h * P + i] = v[i];
        }
    }
}

constexpr float kSqrtHalf = 0.70710678118654752f, kSqrt2OverPi = 0.79788456080286536f, kInvSqrt2Pi = 0.39894228040143268f;

// z moved into +-100: behind that an activation's curve is 0 or 1 (times z) in 32 bits, and its slope meets no inf * 0.  `tamed` leaves NaN as it
// is; `bounded`, one instruction, does not: for curves, which z itself multiplies.
__device__ __forceinline__ float tamed(float z) { return z > 100.f ? 100.f : z < -100.f ? -100.f : z; }
__device__ __forceinline__ float bounded(float z) { return __builtin_amdgcn_fmed3f(z, -100.f, 100.f); }
constexpr float kLog2E = 1.44269504088896341f, kLn2 = 0.69314718055994531f;
// An exponent in two parts, `low` being what the first one's rounding left.  WIDE (fp32): rounded as one number an exponent x costs 2^x some
// |x| units, up to a hundred in the tails; with the rest put right behind the exponential that is one.  Otherwise `low` is 0: a hundred
// units are nothing that 16 bits keep.  (fp32, 4096 x 64 -> 4096: SiLU 38 -> 40 us, GELU's tanh form 38 -> 44, GELU 48 -> 54; 2048 x 512 ->
// 2048 40.3 -> 40.7, 40.3 -> 42, 43 -> 45.)
struct Exponent {
    float x, low;
};
template <bool WIDE>
__device__ __forceinline__ float exp2_of(const Exponent& a) {
    const float e = __builtin_amdgcn_exp2f(a.x);
    if constexpr (!WIDE) return e;
    return a.x > 127.f ? e : fmaf(e, a.low * kLn2, e);             // (2^x may be infinite)
}
// t * (c + c_low)
template <bool WIDE>
__device__ __forceinline__ Exponent exponent(float t, float c, float c_low) {
    Exponent a{t * c, 0.f};
    if constexpr (WIDE) a.low = fmaf(t, c_low, fmaf(t, c, -a.x));
    return a;
}
// 1 / (1 + 2^x).  (v_exp_f32 and v_rcp_f32 are good to one unit of 32 bits each; an IEEE division is ten instructions.)
template <bool WIDE>
__device__ __forceinline__ float falling(const Exponent& a) { return __builtin_amdgcn_rcpf(1.f + exp2_of<WIDE>(a)); }

__device__ __forceinline__ float relu(float z) { return z < 0.f ? 0.f : z; }                    // (NaN stays)
__device__ __forceinline__ float relu_slope(float z) { return z > 0.f ? 1.f : z == z ? 0.f : z; }
// Phi(t), the normal distribution, and e = exp(-t^2 / 2).  WIDE: from erfc, which has no cancellation in the tail either, with the rounding
// of its argument put right by its slope.  Otherwise the tail as e times a polynomial in k = 1 / (1 + 0.27 |t|), fitted to
// exp(t^2 / 2) * Phi(-t) over 0 .. 13.2 for the least relative error, 1.2e-6.  The roundings of t^2 and of the exponent add some t^2 units
// of 2^-24: 1e-5 of the tail at t = 13, a fiftieth of fp16's half step.  (8192 x 4096 x 4096, bf16: 198 us without an activation, 248 with
// erff, 212 with the polynomial.  fp32 products wait for the matrix cores in any case.)
template <bool WIDE>
__device__ __forceinline__ float normal_share(float t, float& e) {
    if constexpr (WIDE) {
        const float h = t * t, x = -kSqrtHalf * t;
        Exponent a = exponent<true>(h, -0.5f * kLog2E, -9.62981517e-9f);
        a.low = fmaf(fmaf(t, t, -h), -0.5f * kLog2E, a.low);
        e = exp2_of<true>(a);
        const float left = fmaf(-1.21016175e-8f, t, fmaf(-kSqrtHalf, t, -x));
        return fmaf(-0.56418958f * left, e, 0.5f * erfcf(x));      // (erfc'(x) / 2 = -exp(-x^2) / sqrt(pi))
    }
    e = __builtin_amdgcn_exp2f(-0.5f * kLog2E * t * t);
    const float k = __builtin_amdgcn_rcpf(fmaf(0.27f, fabsf(t), 1.f));
    const float poly = k * fmaf(k, fmaf(k, fmaf(k, fmaf(k, fmaf(k, fmaf(k, -0.060592773f, 0.157589721f), -0.0228579642f), 0.116564072f),
                                                0.0932392658f), 0.108363624f), 0.107693477f);
    const float tail = poly * e;
    return t < 0.f ? tail : 1.f - tail;
}
template <bool WIDE>
__device__ __forceinline__ float gelu(float z) {
    float e;
    return z * normal_share<WIDE>(bounded(z), e);
}
template <bool WIDE>
__device__ __forceinline__ float gelu_slope(float z) {
    float e;
    const float t = tamed(z), share = normal_share<WIDE>(t, e);
    return fmaf(t * kInvSqrt2Pi, e, share);
}
// (1 + tanh(u)) / 2 = 1 / (1 + exp(-2u)): no cancellation where the curve nears 0.  -2u * log2(e) = t * (k + m t^2)
template <bool WIDE>
__device__ __forceinline__ float gelu_tanh_share(float t) {
    constexpr float k = -2.f * kSqrt2OverPi * kLog2E;
    if constexpr (WIDE) {
        constexpr float k0 = -2.30220819f, k0_low = -1.29484024e-8f, m = -0.102943242f, m_low = 2.01619854e-9f;
        const float h = t * t, p = m * h, p_low = fmaf(m, h, -p) + fmaf(m, fmaf(t, t, -h), m_low * h);
        const float c = k0 + p, b = c - k0, c_low = (k0 - (c - b)) + (p - b) + (p_low + k0_low);     // (the sum's rounding, either larger)
        return falling<true>(exponent<true>(t, c, c_low));
    }
    return falling<false>({t * fmaf(k * 0.044715f, t * t, k), 0.f});
}
template <bool WIDE>
__device__ __forceinline__ float gelu_tanh(float z) { return z * gelu_tanh_share<WIDE>(bounded(z)); }
template <bool WIDE>
__device__ __forceinline__ float gelu_tanh_slope(float z) {
    const float t = tamed(z), s = gelu_tanh_share<WIDE>(t);
    return fmaf(t * s * (1.f - s), fmaf(6.f * kSqrt2OverPi * 0.044715f, t * t, 2.f * kSqrt2OverPi), s);
}
template <bool WIDE>
__device__ __forceinline__ float silu_share(float t) { return falling<WIDE>(exponent<WIDE>(t, -kLog2E, -1.92596303e-8f)); }
template <bool WIDE>
__device__ __forceinline__ float silu(float z) { return z * silu_share<WIDE>(bounded(z)); }
template <bool WIDE>
__device__ __forceinline__ float silu_slope(float z) {
    const float t = tamed(z), s = silu_share<WIDE>(t);
    return s * fmaf(t, 1.f - s, 1.f);
}

// v = curve(v), or v *= slope(z), for R times eight values of a storage type
template <int DT, int R>
__device__ __forceinline__ void activate8(float v[R][8], int act) {
#define PCONV_EACH(F)                                         \
    _Pragma("unroll") for (int r = 0; r < R; ++r)             \
        _Pragma("unroll") for (int q = 0; q < 8; ++q) v[r][q] = F(v[r][q]); \
    break
    switch (act) {
        case PCONV_ACT_RELU: PCONV_EACH(relu);
        case PCONV_ACT_GELU: PCONV_EACH(gelu<DT == PCONV_F32>);
        case PCONV_ACT_GELU_TANH: PCONV_EACH(gelu_tanh<DT == PCONV_F32>);
        case PCONV_ACT_SILU: PCONV_EACH(silu<DT == PCONV_F32>);
        default: break;
    }
#undef PCONV_EACH
}
template <int DT, int R>
__device__ __forceinline__ void times_slope8(float v[R][8], const float z[R][8], int act) {
#define PCONV_EACH(F)                                         \
    _Pragma("unroll") for (int r = 0; r < R; ++r)             \
        _Pragma("unroll") for (int q = 0; q < 8; ++q) v[r][q] *= F(z[r][q]); \
    break
    switch (act) {
        case PCONV_ACT_RELU: PCONV_EACH(relu_slope);
        case PCONV_ACT_GELU: PCONV_EACH(gelu_slope<DT == PCONV_F32>);
        case PCONV_ACT_GELU_TANH: PCONV_EACH(gelu_tanh_slope<DT == PCONV_F32>);
        case PCONV_ACT_SILU: PCONV_EACH(silu_slope<DT == PCONV_F32>);
        default: break;
    }
#undef PCONV_EACH
}

// out[j] of 64 columns from `first`, by a workgroup of 256: 16 threads to four columns, each with every 16th strip
__device__ __forceinline__ void add_strips(const float* parts, int strips, int N, float* out, int first) {
    __shared__ float sums[16][64];
    const int c = threadIdx.x % 16 * 4, s = threadIdx.x / 16, j = first + c, n = N - j;
    float sum[4] = {};
    if (n > 0)
#pragma unroll 4
        for (int g = s; g < strips; g += 16) {
            const float4v v = __builtin_bit_cast(float4v, load_part<PCONV_F32>(parts + (size_t)g * N + j, n));
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] += v[e];
        }
#pragma unroll
    for (int e = 0; e < 4; ++e) sums[s][c + e] = sum[e];
    __syncthreads();
    const int d = first + threadIdx.x;
    if (threadIdx.x < 64 && d < N) {
        float all = 0.f;
#pragma unroll
        for (int q = 0; q < 16; ++q) all += sums[q][threadIdx.x];
        out[d] = all;
    }
}

constexpr long long kMostStride = 1 << 20;

inline bool is_dtype(int dtype) { return dtype == PCONV_F32 || dtype == PCONV_F16 || dtype == PCONV_BF16; }
inline bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }

// A matrix's row stride: 0 becomes `cols`
inline int check_stride(long long* ld, int cols) {
    if (*ld == 0) *ld = cols;
    if (*ld < cols) return PCONV_ESHAPE;
    if (*ld > kMostStride) return PCONV_EUNSUPPORTED;
    return PCONV_OK;
}

}  // namespace
}  // namespace pconv
