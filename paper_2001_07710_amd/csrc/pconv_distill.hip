// Distillation from a teacher's top logits (pconv_dense.h): per row of V logits the softmax of the network that is trained, the
// teacher's distribution over its k stored entries, the loss and the gradient of the logits.  Memory bounds it: the logits in
// once, the gradient out once.
//
// One workgroup per row.  The row's logits stay in registers as they are stored, Q pieces of 16 bytes a thread (a row begins at any
// element: pieces are those of memory, cut at the row's ends, so that every access is aligned): largest, sum of the
// exponentials, gradient, all from one reading.  Longer rows are read again, with the running maximum and sum of a softmax
// in the first pass.  The entries are held in LDS; after the row's w * T * q has been stored the entries' places are stored again
// with their p taken off, by the first entry of each index (for all that share it).
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
    float inv_t, t;
};

template <int THREADS, typename F>
__device__ __forceinline__ float all_reduce(float v, float* room, F f) {
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v = f(v, __shfl_xor(v, d, 64));
    if constexpr (THREADS > 64) {
        const int wave = threadIdx.x >> 6;
        __syncthreads();
        if ((threadIdx.x & 63) == 0) room[wave] = v;
        __syncthreads();
        v = room[0];
#pragma unroll
        for (int w = 1; w < THREADS / 64; ++w) v = f(v, room[w]);
    }
    return v;
}
__device__ __forceinline__ float larger(float a, float b) { return fmaxf(a, b); }     // (a NaN is passed over: the sum finds it)
__device__ __forceinline__ float plus(float a, float b) { return a + b; }

// exp(x) for x <= 0, NaN for NaN; exp(-inf) = 0
__device__ __forceinline__ float exp_of(float x) { return __expf(x); }

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

// Q = 0: the row is read again for the gradient
template <int DT, int THREADS, int Q>
__global__ __launch_bounds__(THREADS) void distill_kernel(const DistillArgs p) {
    typedef typename Store<DT>::T T;
    typedef typename Store<DT>::V Vec;
    constexpr int P = Store<DT>::kPer;
    __shared__ float room[16];
    __shared__ int index[kMostEntries];
    __shared__ float prob[kMostEntries];
    __shared__ float at_index[kMostEntries];
    const int t = threadIdx.x;
    const long long r = blockIdx.x;
    const T* const row = static_cast<const T*>(p.logits) + r * p.ldl;
    T* const out = static_cast<T*>(p.grad) + r * p.ldg;
    const int shift = (int)(reinterpret_cast<uintptr_t>(row) % 16) / (int)sizeof(T);
    const int pieces = (int)(((long long)p.V + shift + P - 1) / P);
    const float w = p.weight ? p.weight[r] : 1.f;

    // the teacher's entries
    float top = -__builtin_inff(), some = 0.f;
    for (int j = t; j < p.k; j += THREADS) {
        const int i = p.indices[r * p.k + j];
        const bool there = i >= 0 && i < p.V;
        const float v = there ? p.values[r * p.k + j] * p.inv_t : -__builtin_inff();
        index[j] = there ? i : -1;
        prob[j] = v;
        top = fmaxf(top, v);
        if (there && !(v == -__builtin_inff())) some = 1.f;
    }
    top = all_reduce<THREADS>(top, room, larger);
    some = all_reduce<THREADS>(some, room, larger);
    if (some == 0.f || w == 0.f) {                     // (the same for the whole workgroup)
        if (t == 0) {
            if (p.loss) p.loss[r] = 0.f;
            if (p.stats) p.stats[2 * r] = p.stats[2 * r + 1] = 0.f;
        }
        if (p.grad) {
            const float zero[P] = {};
            for (int q = t; q < pieces; q += THREADS) store_piece<DT>(out, q * P - shift, p.V, zero);
        }
        return;
    }
    uint4v raw[Q ? Q : 1];
    if constexpr (Q > 0) {
#pragma unroll
        for (int q = 0; q < Q; ++q) raw[q] = load_piece<DT>(row, (t + q * THREADS) * P - shift, p.V);
    }
    float sum = 0.f;
    for (int j = t; j < p.k; j += THREADS)
        if (index[j] >= 0) sum += exp_of(prob[j] - top);
    const float total = all_reduce<THREADS>(sum, room, plus);
    const float log_total = logf(total);

    // the softmax of the row
    float largest, norm;
    if (p.given) {
        largest = p.given[2 * r];
        norm = p.given[2 * r + 1];
    } else {
        float m = -__builtin_inff(), s = 0.f;
        if constexpr (Q > 0) {
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const Vec v = __builtin_bit_cast(Vec, raw[q]);
#pragma unroll
                for (int e = 0; e < P; ++e) m = fmaxf(m, (float)v[e]);
            }
            largest = all_reduce<THREADS>(m, room, larger);
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const Vec v = __builtin_bit_cast(Vec, raw[q]);
                const int at = (t + q * THREADS) * P - shift;
#pragma unroll
                for (int e = 0; e < P; ++e) s += at + e >= 0 && at + e < p.V ? exp_of(((float)v[e] - largest) * p.inv_t) : 0.f;
            }
        } else {
            for (int q = t; q < pieces; q += THREADS) {
                const Vec v = __builtin_bit_cast(Vec, load_piece<DT>(row, q * P - shift, p.V));
                float high = m;
#pragma unroll
                for (int e = 0; e < P; ++e) high = fmaxf(high, (float)v[e]);
                if (high > m) {
                    s *= exp_of((m - high) * p.inv_t);
                    m = high;
                }
                const int at = q * P - shift;
                // (all of it -inf so far: nothing to add, unless there is a NaN)
#pragma unroll
                for (int e = 0; e < P; ++e)
                    if (at + e >= 0 && at + e < p.V && !((float)v[e] == -__builtin_inff())) s += exp_of(((float)v[e] - m) * p.inv_t);
            }
            largest = all_reduce<THREADS>(m, room, larger);
            // (a thread whose logits were all -inf has a sum of 0; where every logit is, the sum is NaN)
            if (m != largest) s *= exp_of((m - largest) * p.inv_t);
            if (largest == -__builtin_inff()) s = __builtin_nanf("");
        }
        norm = all_reduce<THREADS>(s, room, plus);
        if (t == 0 && p.stats) {
            p.stats[2 * r] = largest;
            p.stats[2 * r + 1] = norm;
        }
    }
    const float log_norm = logf(norm);

    // loss, and what the entries' places will hold; an index that comes twice is looked for if the gradient is asked for
    float loss = 0.f;
    for (int j = t; j < p.k; j += THREADS) {
        const int i = index[j];
        if (i < 0) continue;
        const float log_p = prob[j] - top - log_total, mine = exp_of(log_p);
        const float z = ((float)row[i] - largest) * p.inv_t;
        if (!(mine == 0.f)) loss += mine * (log_p - (z - log_norm));
        at_index[j] = z;
        prob[j] = mine;
    }
    if (p.loss) {
        loss = all_reduce<THREADS>(loss, room, plus);
        if (t == 0) p.loss[r] = w * p.t * p.t * loss;
    }
    if (!p.grad) return;

    // a total that is NaN or +inf makes the whole row NaN
    const float scale = w * p.t, each = scale / norm * (total / total);
    __syncthreads();                                   // (every entry's logit has been read: grad may be logits)
    if constexpr (Q > 0) {
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int at = (t + q * THREADS) * P - shift;
            const Vec v = __builtin_bit_cast(Vec, raw[q]);
            float g[P];
#pragma unroll
            for (int e = 0; e < P; ++e) g[e] = each * exp_of(((float)v[e] - largest) * p.inv_t);
            if (at < p.V) store_piece<DT>(out, at, p.V, g);
        }
    } else {
        for (int q = t; q < pieces; q += THREADS) {
            const int at = q * P - shift;
            const Vec v = __builtin_bit_cast(Vec, load_piece<DT>(row, at, p.V));
            float g[P];
#pragma unroll
            for (int e = 0; e < P; ++e) g[e] = each * exp_of(((float)v[e] - largest) * p.inv_t);
            store_piece<DT>(out, at, p.V, g);
        }
    }
    __syncthreads();
    for (int j = t; j < p.k; j += THREADS) {
        const int i = index[j];
        if (i < 0) continue;
        float mine = prob[j];
        bool first = true;
        for (int o = 0; o < p.k; ++o)
            if (o != j && index[o] == i) {
                if (o < j) first = false;
                else mine += prob[o];
            }
        if (first) out[i] = (T)(each * exp_of(at_index[j]) - scale * mine);
    }
}

template <int DT>
int launch_distill(const DistillArgs& a, int R, hipStream_t st) {
    constexpr int P = Store<DT>::kPer;
    const int pieces = a.V / P + 2;                    // (of a row that begins anywhere)
#define PCONV_ROWS(THREADS, Q)                                                                                   \
    if (!done && pieces <= THREADS * Q) {                                                                        \
        hipLaunchKernelGGL((distill_kernel<DT, THREADS, Q>), dim3((unsigned)R), dim3(THREADS), 0, st, a);        \
        done = true;                                                                                             \
    }
    bool done = false;
    PCONV_ROWS(64, 2) PCONV_ROWS(256, 2) PCONV_ROWS(256, 4) PCONV_ROWS(1024, 2) PCONV_ROWS(1024, 4) PCONV_ROWS(1024, 8)
    if (!done) hipLaunchKernelGGL((distill_kernel<DT, 1024, 0>), dim3((unsigned)R), dim3(1024), 0, st, a);
#undef PCONV_ROWS
    PCONV_HIP(hipGetLastError());
    return PCONV_OK;
}

int distill(const void* logits, long long ldl, const int32_t* indices, const float* values, const float* weight, float* loss, void* grad,
            long long ldg, const float* given, float* stats, bool asked, int dtype, int R, int V, int k, float temperature, void* stream) {
    if (!is_dtype(dtype)) return PCONV_EINVAL;
    if (R < 0 || V < 1 || k < 1) return PCONV_ESHAPE;
    if (k > kMostEntries) return PCONV_EUNSUPPORTED;
    if (!(temperature > 0.f) || !(temperature < __builtin_inff()) || !(1.f / temperature < __builtin_inff())) return PCONV_EINVAL;
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
    a.t = temperature; a.inv_t = 1.f / temperature;
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
