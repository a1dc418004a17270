// Distillation from a teacher's top logits (pconv_dense.h): per row of V logits the softmax of the network that is trained, the
// teacher's distribution over its k stored entries, the loss and the gradient of the logits.  Memory bounds it: the logits in
// once, the gradient out once.
//
// One workgroup per row.  The row's logits are read once, Q pieces of 16 bytes a thread, and stay in registers, first as they are
// stored, then, up to eight pieces, as their exponentials: largest, sum of the exponentials, gradient.  (A row begins at any element:
// pieces are those of memory, cut at the row's ends, so that every access is aligned.)  Longer rows are read again for the gradient,
// with the running maximum and sum of a softmax in the first pass.  The entries are one wave's work, beside the reductions of the
// others; after the row's w * T * q has been stored the entries' places are stored again with their p taken off, by the first entry of
// each index (for all that share it).
// 8192 x 32001, bf16, 64 entries: 220 us, 4.8 TB/s (a copy reaches 5.17), 239 with three tensors of logits by turns.  With the entries in
// front of the row's loads, and every exponential taken twice, it took 400.  4096 x 128000: 484 us, 4.3 TB/s (4.0 with the row read again;
// one workgroup fills a compute unit there, and the exponentials are taken twice), the gradient alone from kept statistics 424.  256 x 1000:
// 6 us, the latency of the entries' and the row's loads and four reductions.  Few rows of many logits are a compute unit's work each: one of
// 128,000 takes 20 us, the gradient alone 13.
#include "pconv_dense_util.h"

namespace pconv {
namespace {

constexpr int kMostEntries = 1024;

struct DistillArgs {
    const void* logits;
    const int32_t* indices;
    const float* values;
    const float* weight;
    float* loss;
    void* grad;
    const float* given;        // stats of an earlier call, or null
    float* stats;
    long long ldl, ldg;
    int V, k;
    float t;
    float c, c_low;            // log2(e) / T, and what is missing to it
};

// exp(d / T) for d <= 0.  WIDE: to two units of 32 bits wherever d lies, the product's rounding and c's put right behind the exponential
// (otherwise |d| / T units more: nothing that a gradient of 16 bits keeps).  d = -inf gives 0, NaN stays.
template <bool WIDE>
__device__ __forceinline__ float exp_over_t(float d, float c, float c_low) {
    const float x = d * c, e = __builtin_amdgcn_exp2f(x);
    if constexpr (!WIDE) return e;
    const float rest = fmaf(d, c_low, fmaf(d, c, -x)) * 0.693147181f;
    return fmaf(e, x < -200.f ? 0.f : rest, e);
}

template <typename F>
__device__ __forceinline__ float wave_reduce(float v, F f) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v = f(v, __shfl_xor(v, d, 64));
    return v;
}
// `room`: a float of LDS per wave, read after the barrier in here
template <int THREADS, typename F>
__device__ __forceinline__ float all_reduce(float v, float* room, F f) {
    v = wave_reduce(v, f);
    if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
    __syncthreads();
    v = room[0];
#pragma unroll
    for (int w = 1; w < THREADS / 64; ++w) v = f(v, room[w]);
    return v;
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }     // (a NaN is passed over: the sum finds it)
__device__ __forceinline__ float plus(float a, float b) { return a + b; }

// Piece `q` of the row that begins `shift` elements into a 16-byte piece of memory: elements q * P - shift .. + P - 1
template <int DT>
__device__ __forceinline__ uint4v load_piece(const typename Store<DT>::T* row, int at, int V) {
    constexpr int P = Store<DT>::kPer;
    if (at >= 0 && at + P <= V) return load16(row + at);
    typename Store<DT>::V v;
#pragma unroll
    for (int e = 0; e < P; ++e) {
        v[e] = (typename Store<DT>::T)(-__builtin_inff());
        if (at + e >= 0 && at + e < V) v[e] = row[at + e];
    }
    return __builtin_bit_cast(uint4v, v);
}
template <int DT>
__device__ __forceinline__ void store_piece(typename Store<DT>::T* row, int at, int V, const float v[Store<DT>::kPer]) {
    typedef typename Store<DT>::T T;
    constexpr int P = Store<DT>::kPer;
    typename Store<DT>::V o;
#pragma unroll
    for (int e = 0; e < P; ++e) o[e] = (T)v[e];
    if (at >= 0 && at + P <= V) {
        store16(row + at, __builtin_bit_cast(uint4v, o));
    } else {
#pragma unroll
        for (int e = 0; e < P; ++e)
            if (at + e >= 0 && at + e < V) row[at + e] = o[e];
    }
}

// Waves that a SIMD is to hold: two workgroups of 1024 threads a compute unit where 64 registers are enough
[[maybe_unused]] constexpr int waves_per_simd(int threads, int pieces) { return pieces <= 4 ? 8 : threads / 256; }

// Q = 0: the row is read again for the gradient
template <int DT, int THREADS, int Q>
__global__ __launch_bounds__(THREADS, waves_per_simd(THREADS, Q)) void distill_kernel(const DistillArgs p) {
    typedef typename Store<DT>::T T;
    typedef typename Store<DT>::V Vec;
    constexpr int P = Store<DT>::kPer;
    constexpr bool WIDE = DT == PCONV_F32;
    __shared__ float room[2][16];
    __shared__ float teacher[2];                           // largest t, sum of exp((t - largest) / T) or NaN
    extern __shared__ __align__(16) unsigned char entries[];
    const int k4 = (p.k + 3) / 4 * 4;
    int* const index = reinterpret_cast<int*>(entries);    // [k4], -1: not there
    float* const prob = reinterpret_cast<float*>(index + k4);
    float* const own = prob + k4;                          // the row's own logit at the index
    const int t = threadIdx.x, lane = t & 63;
    const long long r = blockIdx.x;
    const T* const row = static_cast<const T*>(p.logits) + r * p.ldl;
    T* const out = static_cast<T*>(p.grad) + r * p.ldg;
    const int shift = (int)(reinterpret_cast<uintptr_t>(row) % 16) / (int)sizeof(T);
    const int pieces = (int)(((long long)p.V + shift + P - 1) / P);
    const float w = p.weight ? p.weight[r] : 1.f;
    // a row that is left out (the same for the whole workgroup)
    auto leave_out = [&] {
        if (t == 0) {
            if (p.loss) p.loss[r] = 0.f;
            if (p.stats) p.stats[2 * r] = p.stats[2 * r + 1] = 0.f;
        }
        if (p.grad) {
            const float zero[P] = {};
            for (int q = t; q < pieces; q += THREADS) store_piece<DT>(out, q * P - shift, p.V, zero);
        }
    };
    if (w == 0.f) {
        leave_out();
        return;
    }
    uint4v raw[Q ? Q : 1];
    if constexpr (Q > 0) {
#pragma unroll
        for (int q = 0; q < Q; ++q) raw[q] = load_piece<DT>(row, (t + q * THREADS) * P - shift, p.V);
    }

    // the teacher's entries: the first wave's lanes, j = lane, lane + 64, ..  (t - largest before the division by T: t / T would round
    // away what the logits differ by, and overflow where they are the type's lowest value)
    if (t < 64) {
        float top = -__builtin_inff(), some = 0.f, sum = 0.f;
        for (int j = lane; j < k4; j += 64) {
            const int i = j < p.k ? p.indices[r * p.k + j] : -1;
            const bool there = i >= 0 && i < p.V;
            const float v = there ? p.values[r * p.k + j] : -__builtin_inff();
            index[j] = there ? i : -1;
            prob[j] = v;
            top = fmaxf(top, v);
            if (there && !(v == -__builtin_inff())) some = 1.f;
        }
        top = wave_reduce(top, larger);
        some = wave_reduce(some, larger);
        for (int j = lane; j < k4; j += 64)
            if (index[j] >= 0) sum += exp_over_t<true>(prob[j] - top, p.c, p.c_low);
        sum = wave_reduce(sum, plus);
        if (t == 0) {
            teacher[0] = top;
            teacher[1] = some == 0.f ? 0.f : sum;           // (a sum of 0: nothing is there; otherwise 1 or more, or NaN)
        }
    }

    // the softmax of the row: largest, then the sum of u = exp((s - largest) / T)
    const float c = p.c, c_low = p.c_low;
    // the exponentials are kept where the registers hold them beside the row (16 pieces: they are taken twice)
    constexpr bool KEEP = Q > 0 && Q <= 8;
    float u[KEEP ? Q : 1][P];
    float largest, norm = 0.f, m = -__builtin_inff();
    if (p.given) {
        largest = p.given[2 * r];
        norm = p.given[2 * r + 1];
        __syncthreads();
    } else {
        if constexpr (Q > 0) {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const Vec v = __builtin_bit_cast(Vec, raw[q]);
#pragma unroll
                for (int e = 0; e < P; ++e) m = fmaxf(m, (float)v[e]);
            }
        } else {
            for (int q = t; q < pieces; q += THREADS) {
                const Vec v = __builtin_bit_cast(Vec, load_piece<DT>(row, q * P - shift, p.V));
                float high = m;
#pragma unroll
                for (int e = 0; e < P; ++e) high = fmaxf(high, (float)v[e]);
                if (high > m) {
                    norm *= exp_over_t<WIDE>(m - high, c, c_low);
                    m = high;
                }
                // (-inf adds nothing, also where all has been -inf so far)
#pragma unroll
                for (int e = 0; e < P; ++e)
                    if (!((float)v[e] == -__builtin_inff())) norm += exp_over_t<WIDE>((float)v[e] - m, c, c_low);
            }
        }
        largest = all_reduce<THREADS>(m, room[0], larger);
    }
    const float top = teacher[0], total = teacher[1];
    if (total == 0.f) {
        leave_out();
        return;
    }
    // the row's own logits at the entries, before any of the gradient is stored: grad may be logits
    if (t < 64)
        for (int j = lane; j < p.k; j += 64) own[j] = index[j] >= 0 ? (float)row[index[j]] : 0.f;
    if constexpr (KEEP) {
        // (what lies outside the row is -inf: nothing, or NaN where the row is all -inf)
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const Vec v = __builtin_bit_cast(Vec, raw[q]);
#pragma unroll
            for (int e = 0; e < P; ++e) u[q][e] = exp_over_t<WIDE>((float)v[e] - largest, c, c_low);
        }
    }
    if (!p.given) {
        if constexpr (Q > 0) {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                [[maybe_unused]] const Vec v = __builtin_bit_cast(Vec, raw[q]);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    if constexpr (KEEP) norm += u[q][e];
                    else norm += exp_over_t<WIDE>((float)v[e] - largest, c, c_low);
                }
            }
        } else {
            if (m != largest) norm *= exp_over_t<WIDE>(m - largest, c, c_low);
            if (largest == -__builtin_inff()) norm = __builtin_nanf("");
        }
        norm = all_reduce<THREADS>(norm, room[1], plus);
        if (t == 0 && p.stats) {
            p.stats[2 * r] = largest;
            p.stats[2 * r + 1] = norm;
        }
    } else {
        __syncthreads();
    }

    // a total that is NaN makes the whole row NaN
    const float scale = w * p.t, each = scale / norm * (total / total);
    if (p.grad) {
        if constexpr (Q > 0) {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const int at = (t + q * THREADS) * P - shift;
                [[maybe_unused]] const Vec v = __builtin_bit_cast(Vec, raw[q]);
                float g[P];
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    if constexpr (KEEP) g[e] = each * u[q][e];
                    else g[e] = each * exp_over_t<WIDE>((float)v[e] - largest, c, c_low);
                }
                if (at < p.V) store_piece<DT>(out, at, p.V, g);
            }
        } else {
            for (int q = t; q < pieces; q += THREADS) {
                const int at = q * P - shift;
                const Vec v = __builtin_bit_cast(Vec, load_piece<DT>(row, at, p.V));
                float g[P];
#pragma unroll
                for (int e = 0; e < P; ++e) g[e] = each * exp_over_t<WIDE>((float)v[e] - largest, c, c_low);
                store_piece<DT>(out, at, p.V, g);
            }
        }
    }
    // the loss, and p in the place of t.  T * (log p - log q) = (t - largest t) - (s - largest s) - T * (log total - log norm): no quotient
    // by T, and no T^2, which overflow where the loss does not
    if (t < 64) {
        const float between = p.t * (logf(total) - logf(norm));
        float loss = 0.f;
        for (int j = lane; j < p.k; j += 64) {
            if (index[j] < 0) continue;
            const float d = prob[j] - top, mine = exp_over_t<true>(d, c, c_low) / total;
            if (!(mine == 0.f)) loss += mine * (d - (own[j] - largest) - between);
            prob[j] = mine;
        }
        loss = wave_reduce(loss, plus);
        if (p.loss && t == 0) p.loss[r] = scale * loss;
    }
    if (!p.grad) return;
    __syncthreads();
    for (int j = t; j < p.k; j += THREADS) {
        const int i = index[j];
        if (i < 0) continue;
        float mine = prob[j];
        int alike = 0;
        for (int o = 0; o < k4; o += 4) {
            const int4 four = *reinterpret_cast<const int4*>(index + o);
            alike += (four.x == i) + (four.y == i) + (four.z == i) + (four.w == i);
        }
        bool first = true;
        if (alike > 1)
            for (int o = 0; o < p.k; ++o)
                if (o != j && index[o] == i) {
                    if (o < j) first = false;
                    else mine += prob[o];
                }
        if (first) out[i] = (T)(each * exp_over_t<WIDE>(own[j] - largest, c, c_low) - scale * mine);
    }
}

template <int DT>
int launch_distill(DistillArgs a, int R, hipStream_t st) {
    typedef typename Store<DT>::T T;
    constexpr int P = Store<DT>::kPer;
    // (a launch holds fewer than 2^32 threads)
    constexpr int kMostAtOnce = 1 << 21;
    const int pieces = a.V / P + 2;                    // (of a row that begins anywhere)
    const size_t lds = 3 * (size_t)((a.k + 3) / 4 * 4) * 4;
    for (int rows; R > 0; R -= rows) {
        rows = std::min(R, kMostAtOnce);
#define PCONV_ROWS(THREADS, Q)                                                                                      \
    if (!done && pieces <= THREADS * Q) {                                                                           \
        hipLaunchKernelGGL((distill_kernel<DT, THREADS, Q>), dim3((unsigned)rows), dim3(THREADS), lds, st, a);      \
        done = true;                                                                                                \
    }
        bool done = false;
        PCONV_ROWS(64, 2) PCONV_ROWS(256, 2) PCONV_ROWS(256, 4) PCONV_ROWS(1024, 2) PCONV_ROWS(1024, 4) PCONV_ROWS(1024, 8) PCONV_ROWS(1024, 16)
        if (!done) hipLaunchKernelGGL((distill_kernel<DT, 1024, 0>), dim3((unsigned)rows), dim3(1024), lds, st, a);
#undef PCONV_ROWS
        PCONV_HIP(hipGetLastError());
        a.logits = static_cast<const T*>(a.logits) + rows * a.ldl;
        a.indices += (long long)rows * a.k;
        a.values += (long long)rows * a.k;
        if (a.weight) a.weight += rows;
        if (a.loss) a.loss += rows;
        if (a.grad) a.grad = static_cast<T*>(a.grad) + rows * a.ldg;
        if (a.given) a.given += 2 * (long long)rows;
        if (a.stats) a.stats += 2 * (long long)rows;
    }
    return PCONV_OK;
}

int distill(const void* logits, long long ldl, const int32_t* indices, const float* values, const float* weight, float* loss, void* grad,
            long long ldg, const float* given, float* stats, bool asked, int dtype, int R, int V, int k, float temperature, void* stream) {
    if (!is_dtype(dtype)) return PCONV_EINVAL;
    if (R < 0 || V < 1 || k < 1) return PCONV_ESHAPE;
    if (k > kMostEntries) return PCONV_EUNSUPPORTED;
    const double c = 1.4426950408889634 / (double)temperature;
    if (!(temperature > 0.f) || !(temperature < __builtin_inff()) || !(c < 0x1.ffffffp127)) return PCONV_EINVAL;    // (c: finite in fp32)
    for (int rc : {check_stride(&ldl, V), grad ? check_stride(&ldg, V) : PCONV_OK})
        if (rc) return rc;
    if (!asked) return PCONV_EINVAL;
    if (R == 0) return PCONV_OK;
    if (!logits || !indices || !values) return PCONV_EINVAL;
    if (!aligned_to(logits, elem_bytes(dtype)) || !aligned_to(grad, elem_bytes(dtype))) return PCONV_EINVAL;
    for (const void* p : {(const void*)indices, (const void*)values, (const void*)weight, (const void*)loss, (const void*)given, (const void*)stats})
        if (!aligned_to(p, 4)) return PCONV_EINVAL;
    DistillArgs a{};
    a.logits = logits; a.ldl = ldl;
    a.indices = indices; a.values = values; a.weight = weight;
    a.loss = loss;
    a.grad = grad; a.ldg = ldg;
    a.given = given; a.stats = stats;
    a.V = V; a.k = k;
    a.t = temperature;
    a.c = (float)c; a.c_low = (float)(c - (double)a.c);
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == PCONV_F32   ? launch_distill<PCONV_F32>(a, R, st)
           : dtype == PCONV_F16 ? launch_distill<PCONV_F16>(a, R, st)
                                : launch_distill<PCONV_BF16>(a, R, st);
}

}  // namespace
}  // namespace pconv

using namespace pconv;

extern "C" int pconv_distill(const void* logits, long long ldl, const int32_t* indices, const float* values, const float* weight,
                             float* loss, void* grad, long long ldg, float* stats, int dtype, int R, int V, int k, float temperature,
                             void* stream) {
    return distill(logits, ldl, indices, values, weight, loss, grad, ldg, nullptr, stats, loss || grad || stats, dtype, R, V, k, temperature, stream);
}

extern "C" int pconv_distill_grad(const void* logits, long long ldl, const int32_t* indices, const float* values, const float* weight,
                                  const float* stats, void* grad, long long ldg, int dtype, int R, int V, int k, float temperature,
                                  void* stream) {
    return distill(logits, ldl, indices, values, weight, nullptr, grad, ldg, stats, nullptr, stats && grad, dtype, R, V, k, temperature, stream);
}
