// Layer norm over the rows of a matrix, forward and backward (pconv_dense.h).  Memory bounds both: x in and y out, and dy and x
// in and dx out.
//
// A row is held in registers by TPR threads, Q pieces of 16 bytes each, so that it is read once: mean, then the squares around
// it (or, backward, the two sums of g and g * h), each a reduction over those threads by shuffles, across waves through LDS.
// Workgroups walk over the rows, so that a thread's gamma and beta stay in registers too; in the backward pass so do its columns'
// sums of dy * h and dy, which meet at the end: the threads with the same columns in LDS, the workgroups in the workspace.
// Longer rows (than 1024 threads hold) are read twice or three times, from the caches.
#include "pconv_dense_util.h"

namespace pconv {
namespace {

// Sum over groups of L consecutive lanes (a power of two), in every lane.
template <int L>
__device__ __forceinline__ float lanes_sum(float v) {
#pragma unroll
    for (int d = 1; d < L; d *= 2) v += __shfl_xor(v, d, 64);
    return v;
}

// Sums of two values over the TPR threads that hold a row.  `room`: 2 * waves floats of LDS for each of two turns, used in turn,
// so that one barrier a sum is enough.
template <int TPR>
struct RowSum {
    float (*room)[2][16];
    int turn = 0;
    __device__ __forceinline__ void operator()(float& a, float& b) {
        a = lanes_sum<(TPR < 64 ? TPR : 64)>(a);
        b = lanes_sum<(TPR < 64 ? TPR : 64)>(b);
        if constexpr (TPR > 64) {
            constexpr int W = TPR / 64;
            const int wave = threadIdx.x >> 6, first = wave / W * W;
            if ((threadIdx.x & 63) == 0) {
                room[turn][0][wave] = a;
                room[turn][1][wave] = b;
            }
            __syncthreads();
            a = b = 0.f;
#pragma unroll
            for (int w = 0; w < W; ++w) {
                a += room[turn][0][first + w];
                b += room[turn][1][first + w];
            }
            turn ^= 1;
        }
    }
};

struct NormArgs {
    const void* x;
    const void* dy;
    void* out;                  // y, or dx (or null)
    const float* gamma;
    const float* beta;
    float* mean;
    float* rstd;
    float* dgamma;              // backward: [workgroup][D] parts, or null
    float* dbeta;
    long long ldx, lddy, ldo;
    int rows, D;
    float eps;
};

template <int DT, int TPR, int Q, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_kernel(const NormArgs p) {
    typedef typename Store<DT>::T T;
    typedef typename Store<DT>::V V;
    constexpr int P = Store<DT>::kPer, GROUPS = THREADS / TPR;
    __shared__ float room[2][2][16];
    RowSum<TPR> row_sum{room};
    const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    float gamma[Q][P], beta[Q][P];
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int e = 0; e < P; ++e) {
            const int d = (t + q * TPR) * P + e;
            gamma[q][e] = d < p.D && p.gamma ? p.gamma[d] : 1.f;
            beta[q][e] = d < p.D && p.beta ? p.beta[d] : 0.f;
        }
    const float inv = 1.f / (float)p.D;
    const long long step = (long long)gridDim.x * GROUPS;
    const long long turns = (p.rows + step - 1) / step;         // (the same for every thread: row_sum has barriers)
    for (long long k = 0; k < turns; ++k) {
        const long long r = k * step + (long long)blockIdx.x * GROUPS + group;
        const bool there = r < p.rows;
        const T* const x = static_cast<const T*>(p.x) + (there ? r : 0) * p.ldx;
        uint4v raw[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) raw[q] = load_part<DT>(x + (t + q * TPR) * P, there ? p.D - (t + q * TPR) * P : 0);
        float sum = 0.f, none = 0.f;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const V v = __builtin_bit_cast(V, raw[q]);
#pragma unroll
            for (int e = 0; e < P; ++e) sum += (float)v[e];
        }
        row_sum(sum, none);
        const float mean = sum * inv;
        float squares = 0.f;
        none = 0.f;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const V v = __builtin_bit_cast(V, raw[q]);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const float d = (float)v[e] - mean;
                squares += (t + q * TPR) * P + e < p.D ? d * d : 0.f;
            }
        }
        row_sum(squares, none);
        const float rstd = 1.f / sqrtf(squares * inv + p.eps);
        if (!there) continue;
        if (t == 0) {
            if (p.mean) p.mean[r] = mean;
            if (p.rstd) p.rstd[r] = rstd;
        }
        T* const y = static_cast<T*>(p.out) + r * p.ldo;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const V v = __builtin_bit_cast(V, raw[q]);
            const int d = (t + q * TPR) * P, n = p.D - d;
            V o;
#pragma unroll
            for (int e = 0; e < P; ++e) o[e] = (T)(((float)v[e] - mean) * rstd * gamma[q][e] + beta[q][e]);
            if (n >= P) store16(y + d, __builtin_bit_cast(uint4v, o));
            else
#pragma unroll
                for (int e = 0; e < P; ++e)
                    if (e < n) y[d + e] = o[e];
        }
    }
}

template <int DT, int TPR, int Q, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(const NormArgs p) {
    typedef typename Store<DT>::T T;
    typedef typename Store<DT>::V V;
    constexpr int P = Store<DT>::kPer, GROUPS = THREADS / TPR;
    __shared__ float room[2][2][16];
    __shared__ __align__(16) float columns[GROUPS > 1 ? THREADS * P : 1];
    RowSum<TPR> row_sum{room};
    const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    float gamma[Q][P], dg[Q][P], db[Q][P];
#pragma unroll
    for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int e = 0; e < P; ++e) {
            const int d = (t + q * TPR) * P + e;
            gamma[q][e] = d < p.D ? p.gamma ? p.gamma[d] : 1.f : 0.f;
            dg[q][e] = db[q][e] = 0.f;
        }
    const float inv = 1.f / (float)p.D;
    const long long step = (long long)gridDim.x * GROUPS;
    const long long turns = (p.rows + step - 1) / step;
    for (long long k = 0; k < turns; ++k) {
        const long long r = k * step + (long long)blockIdx.x * GROUPS + group;
        const bool there = r < p.rows;
        const T* const x = static_cast<const T*>(p.x) + (there ? r : 0) * p.ldx;
        const T* const dy = static_cast<const T*>(p.dy) + (there ? r : 0) * p.lddy;
        uint4v rx[Q], rd[Q];
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const int d = (t + q * TPR) * P, n = there ? p.D - d : 0;
            rx[q] = load_part<DT>(x + d, n);
            rd[q] = load_part<DT>(dy + d, n);
        }
        const float mean = there ? p.mean[r] : 0.f, rstd = there ? p.rstd[r] : 0.f;
        float s1 = 0.f, s2 = 0.f;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const V vx = __builtin_bit_cast(V, rx[q]), vd = __builtin_bit_cast(V, rd[q]);
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const float h = ((float)vx[e] - mean) * rstd, d = (float)vd[e], g = d * gamma[q][e];
                // (columns behind the row: dy and gamma are zeros there, h is finite wherever the row's statistics are)
                s1 += g;
                s2 += (t + q * TPR) * P + e < p.D ? g * h : 0.f;
                db[q][e] += d;
                dg[q][e] += d * h;
            }
        }
        row_sum(s1, s2);
        if (!there || !p.out) continue;
        s1 *= inv;
        s2 *= inv;
        T* const dx = static_cast<T*>(p.out) + r * p.ldo;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            const V vx = __builtin_bit_cast(V, rx[q]), vd = __builtin_bit_cast(V, rd[q]);
            const int d = (t + q * TPR) * P, n = p.D - d;
            V o;
#pragma unroll
            for (int e = 0; e < P; ++e) {
                const float h = ((float)vx[e] - mean) * rstd;
                o[e] = (T)(rstd * ((float)vd[e] * gamma[q][e] - s1 - h * s2));
            }
            if (n >= P) store16(dx + d, __builtin_bit_cast(uint4v, o));
            else
#pragma unroll
                for (int e = 0; e < P; ++e)
                    if (e < n) dx[d + e] = o[e];
        }
    }
    // the groups' sums of a column, in their order
    for (int which = 0; which < 2; ++which) {
        float* const out = which ? p.dbeta : p.dgamma;
        if (!out) continue;
#pragma unroll
        for (int q = 0; q < Q; ++q) {
            float sum[P];
#pragma unroll
            for (int e = 0; e < P; ++e) sum[e] = which ? db[q][e] : dg[q][e];
            if constexpr (GROUPS > 1) {
                __syncthreads();
#pragma unroll
                for (int e = 0; e < P; ++e) columns[threadIdx.x * P + e] = sum[e];
                __syncthreads();
                if (group == 0)
                    for (int g = 1; g < GROUPS; ++g)
#pragma unroll
                        for (int e = 0; e < P; ++e) sum[e] += columns[(g * TPR + t) * P + e];
            }
            if (group == 0)
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    const int d = (t + q * TPR) * P + e;
                    if (d < p.D) out[(size_t)blockIdx.x * p.D + d] = sum[e];
                }
        }
    }
}

// Rows that no workgroup holds: one workgroup a row, in several readings.
constexpr int kLong = 1024;
template <int DT>
__global__ __launch_bounds__(kLong) void norm_long_kernel(const NormArgs p) {
    typedef typename Store<DT>::T T;
    __shared__ float room[2][2][16];
    RowSum<kLong> row_sum{room};
    for (long long r = blockIdx.x; r < p.rows; r += gridDim.x) {
        const T* const x = static_cast<const T*>(p.x) + r * p.ldx;
        T* const y = static_cast<T*>(p.out) + r * p.ldo;
        float sum = 0.f, none = 0.f, v[8];
        for (int d = threadIdx.x * 8; d < p.D; d += kLong * 8) {
            load8<DT>(x + d, p.D - d, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum += v[e];
        }
        row_sum(sum, none);
        const float mean = sum / (float)p.D;
        float squares = 0.f;
        none = 0.f;
        for (int d = threadIdx.x * 8; d < p.D; d += kLong * 8) {
            load8<DT>(x + d, p.D - d, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) squares += d + e < p.D ? (v[e] - mean) * (v[e] - mean) : 0.f;
        }
        row_sum(squares, none);
        const float rstd = 1.f / sqrtf(squares / (float)p.D + p.eps);
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[r] = mean;
            if (p.rstd) p.rstd[r] = rstd;
        }
        for (int d = threadIdx.x * 8; d < p.D; d += kLong * 8) {
            const int n = p.D - d;
            load8<DT>(x + d, n, v);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                v[e] = (v[e] - mean) * rstd * (p.gamma && e < n ? p.gamma[d + e] : 1.f) + (p.beta && e < n ? p.beta[d + e] : 0.f);
            store8<DT>(y + d, n, v);
        }
    }
}

template <int DT>
__global__ __launch_bounds__(kLong) void norm_grad_long_kernel(const NormArgs p) {
    typedef typename Store<DT>::T T;
    __shared__ float room[2][2][16];
    RowSum<kLong> row_sum{room};
    for (long long r = blockIdx.x; r < p.rows; r += gridDim.x) {
        const T* const x = static_cast<const T*>(p.x) + r * p.ldx;
        const T* const dy = static_cast<const T*>(p.dy) + r * p.lddy;
        T* const dx = static_cast<T*>(p.out) + r * p.ldo;
        const float mean = p.mean[r], rstd = p.rstd[r];
        float s1 = 0.f, s2 = 0.f, vx[8], vd[8];
        for (int d = threadIdx.x * 8; d < p.D; d += kLong * 8) {
            const int n = p.D - d;
            load8<DT>(x + d, n, vx);
            load8<DT>(dy + d, n, vd);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e < n) {
                    const float g = vd[e] * (p.gamma ? p.gamma[d + e] : 1.f);
                    s1 += g;
                    s2 += g * ((vx[e] - mean) * rstd);
                }
        }
        row_sum(s1, s2);
        s1 /= (float)p.D;
        s2 /= (float)p.D;
        for (int d = threadIdx.x * 8; d < p.D; d += kLong * 8) {
            const int n = p.D - d;
            load8<DT>(x + d, n, vx);
            load8<DT>(dy + d, n, vd);
#pragma unroll
            for (int e = 0; e < 8; ++e)
                vd[e] = rstd * (vd[e] * (p.gamma && e < n ? p.gamma[d + e] : 1.f) - s1 - (vx[e] - mean) * rstd * s2);
            store8<DT>(dx + d, n, vd);
        }
    }
}

// Column sums of dy * h and dy over a strip of rows: a wave's lanes hold eight columns each, its workgroup's four waves take turns.
constexpr int kSumCols = 512;
template <int DT>
__global__ __launch_bounds__(256) void norm_columns_kernel(const NormArgs p, int per) {
    typedef typename Store<DT>::T T;
    __shared__ __align__(16) float part[3][2][kSumCols];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int j = blockIdx.x * kSumCols + lane * 8, n = p.D - j;
    const long long r0 = (long long)blockIdx.y * per, r1 = min((long long)p.rows, r0 + per);
    float dg[8] = {}, db[8] = {}, vx[8], vd[8];
    if (n > 0)
        for (long long r = r0 + wave; r < r1; r += 4) {
            load8<DT>(static_cast<const T*>(p.x) + r * p.ldx + j, n, vx);
            load8<DT>(static_cast<const T*>(p.dy) + r * p.lddy + j, n, vd);
            const float mean = p.mean[r], rstd = p.rstd[r];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                dg[q] += vd[q] * ((vx[q] - mean) * rstd);
                db[q] += vd[q];
            }
        }
    if (wave) {
        store8<PCONV_F32>(&part[wave - 1][0][lane * 8], 8, dg);
        store8<PCONV_F32>(&part[wave - 1][1][lane * 8], 8, db);
    }
    __syncthreads();
    if (wave == 0 && n > 0) {
        for (int s = 0; s < 3; ++s)
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                dg[q] += part[s][0][lane * 8 + q];
                db[q] += part[s][1][lane * 8 + q];
            }
        if (p.dgamma) store8<PCONV_F32>(p.dgamma + (size_t)blockIdx.y * p.D + j, n, dg);
        if (p.dbeta) store8<PCONV_F32>(p.dbeta + (size_t)blockIdx.y * p.D + j, n, db);
    }
}

// out[d] = sum of the parts [part][d]: 32 columns a workgroup, eight threads to a column, each a run of the parts
__global__ __launch_bounds__(256) void norm_add_kernel(const float* dgamma_parts, const float* dbeta_parts, int parts, int D, float* dgamma,
                                                       float* dbeta) {
    __shared__ float sums[8][32];
    const float* const from = blockIdx.y ? dbeta_parts : dgamma_parts;
    float* const to = blockIdx.y ? dbeta : dgamma;
    if (!to) return;
    const int c = threadIdx.x & 31, s = threadIdx.x >> 5, d = blockIdx.x * 32 + c, per = (parts + 7) / 8;
    float sum = 0.f;
    if (d < D)
        for (int g = s * per; g < min(parts, (s + 1) * per); ++g) sum += from[(size_t)g * D + d];
    sums[s][c] = sum;
    __syncthreads();
    if (s == 0 && d < D) {
        for (int q = 1; q < 8; ++q) sum += sums[q][c];
        to[d] = sum;
    }
}

__global__ __launch_bounds__(256) void norm_zero_kernel(float* a, float* b, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) {
        if (a) a[i] = 0.f;
        if (b) b[i] = 0.f;
    }
}

// How a row of `pieces` 16-byte pieces is spread: threads of a row, pieces of a thread, threads of a workgroup; tpr = 0: too long
struct Spread { int tpr, q, threads; };
Spread spread(int pieces) {
    if (pieces <= 8) return {8, 1, 256};
    if (pieces <= 16) return {16, 1, 256};
    if (pieces <= 32) return {32, 1, 256};
    if (pieces <= 64) return {64, 1, 256};
    if (pieces <= 128) return {64, 2, 256};
    if (pieces <= 256) return {256, 1, 256};
    if (pieces <= 512) return {256, 2, 256};
    if (pieces <= 1024) return {512, 2, 512};
    if (pieces <= 2048) return {1024, 2, 1024};
    if (pieces <= 4096) return {1024, 4, 1024};
    return {0, 0, kLong};
}

int workgroups(const Spread& s, int rows) {
    const int groups = s.tpr ? s.threads / s.tpr : 1;
    const long long wanted = ((long long)rows + groups - 1) / groups;
    return (int)std::min<long long>(wanted, 256ll * (2048 / s.threads));
}
int grad_workgroups(const Spread& s, int rows) {
    const int groups = s.tpr ? s.threads / s.tpr : 1;
    const long long wanted = ((long long)rows + groups - 1) / groups;
    return (int)std::min<long long>(wanted, 256ll * std::max(1, 1024 / s.threads));
}
int strips(int rows, int D) { return std::max(1, std::min({64, (int)((rows + 63ll) / 64), 512 / ((D + kSumCols - 1) / kSumCols) + 1})); }

#define PCONV_SPREADS(X) X(8, 1, 256) X(16, 1, 256) X(32, 1, 256) X(64, 1, 256) X(64, 2, 256) X(256, 1, 256) X(256, 2, 256) X(512, 2, 512) X(1024, 2, 1024) X(1024, 4, 1024)

template <int DT>
int launch_norm(const NormArgs& a, hipStream_t st) {
    const Spread s = spread((a.D + Store<DT>::kPer - 1) / Store<DT>::kPer);
    const dim3 grid((unsigned)workgroups(s, a.rows));
#define X(TPR, Q, THREADS) \
    if (s.tpr == TPR && s.q == Q) hipLaunchKernelGGL((norm_kernel<DT, TPR, Q, THREADS>), grid, dim3(THREADS), 0, st, a);
    PCONV_SPREADS(X)
#undef X
    if (!s.tpr) hipLaunchKernelGGL(norm_long_kernel<DT>, grid, dim3(kLong), 0, st, a);
    PCONV_HIP(hipGetLastError());
    return PCONV_OK;
}

int grad_parts(int dtype, int rows, int D) {
    const int per = 16 / elem_bytes(dtype);
    const Spread s = spread((D + per - 1) / per);
    return s.tpr ? grad_workgroups(s, rows) : strips(rows, D);
}

template <int DT>
int launch_norm_grad(NormArgs a, float* dgamma, float* dbeta, float* parts, hipStream_t st) {
    const Spread s = spread((a.D + Store<DT>::kPer - 1) / Store<DT>::kPer);
    const int n = grad_parts(DT, a.rows, a.D);
    // (a single part is the result)
    a.dgamma = dgamma ? n > 1 ? parts : dgamma : nullptr;
    a.dbeta = dbeta ? n > 1 ? parts + (size_t)n * a.D : dbeta : nullptr;
    const dim3 grid((unsigned)grad_workgroups(s, a.rows));
#define X(TPR, Q, THREADS) \
    if (s.tpr == TPR && s.q == Q) hipLaunchKernelGGL((norm_grad_kernel<DT, TPR, Q, THREADS>), grid, dim3(THREADS), 0, st, a);
    PCONV_SPREADS(X)
#undef X
    if (!s.tpr) {
        // (the columns first: dx may be written over x or dy)
        if (dgamma || dbeta) {
            hipLaunchKernelGGL(norm_columns_kernel<DT>, dim3((a.D + kSumCols - 1) / kSumCols, n), dim3(256), 0, st, a, (int)((a.rows + (long long)n - 1) / n));
            PCONV_HIP(hipGetLastError());
        }
        if (a.out) hipLaunchKernelGGL(norm_grad_long_kernel<DT>, grid, dim3(kLong), 0, st, a);
    }
    PCONV_HIP(hipGetLastError());
    if (n > 1 && (dgamma || dbeta)) {
        hipLaunchKernelGGL(norm_add_kernel, dim3((a.D + 31) / 32, 2), dim3(256), 0, st, a.dgamma, a.dbeta, n, a.D, dgamma, dbeta);
        PCONV_HIP(hipGetLastError());
    }
    return PCONV_OK;
}

int check_sizes(int dtype, int rows, int D) {
    if (!is_dtype(dtype)) return PCONV_EINVAL;
    if (rows < 0 || D < 1) return PCONV_ESHAPE;
    return PCONV_OK;
}

}  // namespace
}  // namespace pconv

using namespace pconv;

extern "C" int pconv_layer_norm(const void* x, long long ldx, const float* gamma, const float* beta, float eps, void* y, long long ldy,
                                float* mean, float* rstd, int dtype, int rows, int D, void* stream) {
    if (int rc = check_sizes(dtype, rows, D)) return rc;
    if (!(eps >= 0.f)) return PCONV_EINVAL;
    for (int rc : {check_stride(&ldx, D), check_stride(&ldy, D)})
        if (rc) return rc;
    if (rows == 0) return PCONV_OK;
    if (!x || !y || !aligned_to(x, elem_bytes(dtype)) || !aligned_to(y, elem_bytes(dtype))) return PCONV_EINVAL;
    for (const void* p : {(const void*)gamma, (const void*)beta, (const void*)mean, (const void*)rstd})
        if (!aligned_to(p, 4)) return PCONV_EINVAL;
    NormArgs a{};
    a.x = x; a.ldx = ldx;
    a.out = y; a.ldo = ldy;
    a.gamma = gamma; a.beta = beta;
    a.mean = mean; a.rstd = rstd;
    a.rows = rows; a.D = D; a.eps = eps;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == PCONV_F32 ? launch_norm<PCONV_F32>(a, st) : dtype == PCONV_F16 ? launch_norm<PCONV_F16>(a, st) : launch_norm<PCONV_BF16>(a, st);
}

extern "C" int pconv_layer_norm_grad_workspace(int dtype, int rows, int D, size_t* bytes) {
    if (!bytes) return PCONV_EINVAL;
    *bytes = 0;
    if (int rc = check_sizes(dtype, rows, D)) return rc;
    const int n = rows > 0 ? grad_parts(dtype, rows, D) : 0;
    if (n > 1) *bytes = 2 * (size_t)n * D * sizeof(float);
    return PCONV_OK;
}

extern "C" int pconv_layer_norm_grad(const void* dy, long long lddy, const void* x, long long ldx, const float* gamma, const float* mean,
                                     const float* rstd, void* dx, long long lddx, float* dgamma, float* dbeta, int dtype, int rows, int D,
                                     void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = check_sizes(dtype, rows, D)) return rc;
    for (int rc : {check_stride(&lddy, D), check_stride(&ldx, D), dx ? check_stride(&lddx, D) : PCONV_OK})
        if (rc) return rc;
    for (const void* p : {(const void*)gamma, (const void*)mean, (const void*)rstd, (const void*)dgamma, (const void*)dbeta})
        if (!aligned_to(p, 4)) return PCONV_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (rows == 0) {
        if (dgamma || dbeta) {
            hipLaunchKernelGGL(norm_zero_kernel, dim3((D + 255) / 256), dim3(256), 0, st, dgamma, dbeta, D);
            PCONV_HIP(hipGetLastError());
        }
        return PCONV_OK;
    }
    if (!dx && !dgamma && !dbeta) return PCONV_OK;
    if (!dy || !x || !mean || !rstd) return PCONV_EINVAL;
    for (const void* p : {dy, x, (const void*)dx})
        if (!aligned_to(p, elem_bytes(dtype))) return PCONV_EINVAL;
    const int n = grad_parts(dtype, rows, D);
    if ((dgamma || dbeta) && n > 1 && (!workspace || workspace_bytes < 2 * (size_t)n * D * sizeof(float) || !aligned_to(workspace, 16)))
        return PCONV_EINVAL;
    NormArgs a{};
    a.x = x; a.ldx = ldx;
    a.dy = dy; a.lddy = lddy;
    a.out = dx; a.ldo = lddx;
    a.gamma = gamma;
    a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd);
    a.rows = rows; a.D = D;
    float* const parts = static_cast<float*>(workspace);
    return dtype == PCONV_F32   ? launch_norm_grad<PCONV_F32>(a, dgamma, dbeta, parts, st)
           : dtype == PCONV_F16 ? launch_norm_grad<PCONV_F16>(a, dgamma, dbeta, parts, st)
                                : launch_norm_grad<PCONV_BF16>(a, dgamma, dbeta, parts, st);
}
