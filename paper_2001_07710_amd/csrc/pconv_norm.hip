// Layer norm over the rows of a matrix, forward and backward (pconv_dense.h).  Memory bounds both: x in and y out, and dy and x
// in and dx out.
//
// A row is held in registers by TPR threads, Q pieces of 16 bytes each, so that it is read once: sum, then the sums of the deviations
// from the mean and of their squares (or, backward, the two sums of g and g * h), each a reduction over those threads by shuffles, across
// waves through LDS.  The sum's and the quotient's roundings leave the first mean off by units of the row's level, which may be more than
// its spread; the deviations' own mean, `rest`, is what is missing to it (deviations of values near the mean are exact).
// Workgroups walk over the rows, several short ones at a time, the next ones under way while these are worked on, so that a
// thread's gamma and beta stay in registers too; in the backward pass so do its columns' sums of dy * h and dy, which meet at the
// end: the threads with the same columns in LDS, the workgroups in the workspace, one part for a compute unit, added in a second launch.
// Longer rows (than 1024 threads hold) are read twice or three times, from the caches, one workgroup to a row: 2000 x 25088, fp16, 64 us
// forward, 112 backward in three launches (once through memory: 39 and 58); 64 rows 8 and 15.
// 16384 x 4096, bf16: forward 48 us (5.5 TB/s, part of it from the cache behind L2), backward 77 us with the column sums (5.2 TB/s; a
// copy reaches 5.17).  200704 x 64, fp16: forward 15 us (3.4 TB/s), backward 20 (3.9): there a wave's row is one load of its
// lanes, and the shuffles of eight rows at a time are a third of its instructions.  (Forward without `rest`: 47 and 14.2.)
#include <type_traits>

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

// The sums of two values, at the price of one more exchange than those of one: even lanes take the first further, odd ones the second.
template <int L>
__device__ __forceinline__ void lanes_sums(float& a, float& b) {
    const bool odd = threadIdx.x & 1;
    float v = (odd ? b : a) + __shfl_xor(odd ? a : b, 1, 64);
#pragma unroll
    for (int d = 2; d < L; d *= 2) v += __shfl_xor(v, d, 64);
    const float other = __shfl_xor(v, 1, 64);
    a = odd ? other : v;
    b = odd ? v : other;
}

// Sums of N values over the TPR threads that hold a row (of THREADS that meet at the barrier).  The waves' sums lie in one half of
// `room` or the other by turns, so that one barrier is enough.  PAIRS: two by two (not where registers are short: the backward pass of
// 16384 x 4096 takes 90 us with it, 77 without).
template <int TPR, int N, bool PAIRS = false>
struct RowSum {
    float (*room)[N][16];
    int turn = 0;
    __device__ __forceinline__ void operator()(float (&v)[N]) {
        constexpr int L = TPR < 64 ? TPR : 64;
#pragma unroll
        for (int n = 0; n < N; n += PAIRS ? 2 : 1)
            if constexpr (PAIRS) lanes_sums<L>(v[n], v[n + 1]);
            else v[n] = lanes_sum<L>(v[n]);
        if constexpr (TPR > 64) {
            constexpr int W = TPR / 64;
            const int wave = threadIdx.x >> 6, first = wave / W * W;
            if ((threadIdx.x & 63) == 0)
#pragma unroll
                for (int n = 0; n < N; ++n) room[turn][n][wave] = v[n];
            __syncthreads();
#pragma unroll
            for (int n = 0; n < N; ++n) {
                v[n] = 0.f;
#pragma unroll
                for (int w = 0; w < W; ++w) v[n] += room[turn][n][first + w];
            }
            turn ^= 1;
        }
    }
};

// A thread's columns of gamma or beta, in wide pieces; `none` where there is no such vector, `outside` behind its end.
template <int P>
__device__ __forceinline__ void load_columns(const float* v, int d, int D, float none, float outside, float (&out)[P]) {
#pragma unroll
    for (int e = 0; e < P; ++e) out[e] = d + e < D ? none : outside;
    if (!v) return;
    if (d + P <= D) {
#pragma unroll
        for (int h = 0; h < P; h += 4) {
            const float4v w = __builtin_bit_cast(float4v, load16(v + d + h));
#pragma unroll
            for (int e = 0; e < 4; ++e) out[h + e] = w[e];
        }
    } else {
#pragma unroll
        for (int e = 0; e < P; ++e)
            if (d + e < D) out[e] = v[d + e];
    }
}

// v / D, rounded once, from v * (1 / D) and what that leaves (which is NaN where v is infinite)
struct Mean {
    float D, inv;
    __device__ __forceinline__ float operator()(float v) const {
        const float q = v * inv, left = fmaf(-q, D, v);
        return left == left ? fmaf(left, inv, q) : q;
    }
};
// 1 / sqrt(variance + eps) from the mean of the squares around a value that the mean is `rest` away from (NaN stays)
__device__ __forceinline__ float rstd_of(float squares, float rest, float eps) {
    const float variance = squares - rest * rest;
    return 1.f / sqrtf((variance < 0.f ? 0.f : variance) + eps);
}

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

// One reading of a thread's pieces of U rows, asked for one turn ahead of their use.
template <int DT, int TPR, int Q, int U>
struct Rows {
    uint4v raw[U][Q];
    __device__ __forceinline__ void load(const void* m, long long ld, long long r, long long between, int rows, int D, int t) {
        constexpr int P = Store<DT>::kPer;
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool there = r + u * between < rows;
            const auto* const at = static_cast<const typename Store<DT>::T*>(m) + (there ? r + u * between : 0) * ld;
#pragma unroll
            for (int q = 0; q < Q; ++q) raw[u][q] = load_part<DT>(at + (t + q * TPR) * P, there ? D - (t + q * TPR) * P : 0);
        }
    }
};

template <int DT, int TPR, int Q, int U, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_kernel(const NormArgs p) {
    typedef typename Store<DT>::T T;
    typedef typename Store<DT>::V V;
    constexpr int P = Store<DT>::kPer, GROUPS = THREADS / TPR;
    __shared__ float room[2][U][16], pair_room[2][2 * U][16];
    RowSum<TPR, U> row_sum{room};
    RowSum<TPR, 2 * U, true> row_sums{pair_room};
    const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const long long step = (long long)gridDim.x * GROUPS, first = (long long)blockIdx.x * GROUPS + group;
    const long long turns = (p.rows + step * U - 1) / (step * U);    // (the same for every thread: row_sum has barriers)
    Rows<DT, TPR, Q, U> rows;
    rows.load(p.x, p.ldx, first, step, p.rows, p.D, t);
    float gamma[Q][P], beta[Q][P];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        load_columns(p.gamma, (t + q * TPR) * P, p.D, 1.f, 1.f, gamma[q]);
        load_columns(p.beta, (t + q * TPR) * P, p.D, 0.f, 0.f, beta[q]);
    }
    const Mean mean_of{(float)p.D, 1.f / (float)p.D};
    for (long long k = 0; k < turns; ++k) {
        const long long r0 = k * step * U + first;
        // (the next rows are under way while these are worked on)
        const Rows<DT, TPR, Q, U> now = rows;
        if (k + 1 < turns) rows.load(p.x, p.ldx, r0 + step * U, step, p.rows, p.D, t);
        float mean[U], s[2 * U], away[U][Q][P];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            mean[u] = 0.f;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const V v = __builtin_bit_cast(V, now.raw[u][q]);
#pragma unroll
                for (int e = 0; e < P; ++e) mean[u] += (float)v[e];
            }
        }
        row_sum(mean);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            mean[u] *= mean_of.inv;
            s[2 * u] = s[2 * u + 1] = 0.f;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const V v = __builtin_bit_cast(V, now.raw[u][q]);
                const int n = p.D - (t + q * TPR) * P;
                // (what is behind the row is held as zeros, which deviate by nothing from a mean of 0)
                const float m = n > 0 ? mean[u] : 0.f;
#pragma unroll
                for (int e = 0; e < P; ++e) away[u][q][e] = (float)v[e] - m;
                if (n > 0 && n < P) {
#pragma unroll
                    for (int e = 1; e < P; ++e) away[u][q][e] = e < n ? away[u][q][e] : 0.f;
                }
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    s[2 * u] += away[u][q][e];
                    s[2 * u + 1] = fmaf(away[u][q][e], away[u][q][e], s[2 * u + 1]);
                }
            }
        }
        row_sums(s);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long r = r0 + u * step;
            if (r >= p.rows) break;
            const float rest = mean_of(s[2 * u]), rstd = rstd_of(mean_of(s[2 * u + 1]), rest, p.eps);
            if (t == 0) {
                if (p.mean) p.mean[r] = mean[u] + rest;
                if (p.rstd) p.rstd[r] = rstd;
            }
            T* const y = static_cast<T*>(p.out) + r * p.ldo;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const int d = (t + q * TPR) * P, n = p.D - d;
                V o;
#pragma unroll
                for (int e = 0; e < P; ++e) o[e] = (T)fmaf((away[u][q][e] - rest) * rstd, gamma[q][e], beta[q][e]);
                if (n >= P) store16(y + d, __builtin_bit_cast(uint4v, o));
                else
#pragma unroll
                    for (int e = 0; e < P; ++e)
                        if (e < n) y[d + e] = o[e];
            }
        }
    }
}

template <int DT, int TPR, int Q, int U, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_grad_kernel(const NormArgs p) {
    typedef typename Store<DT>::T T;
    typedef typename Store<DT>::V V;
    constexpr int P = Store<DT>::kPer, GROUPS = THREADS / TPR;
    __shared__ float room[2][2 * U][16];
    __shared__ __align__(16) float columns[GROUPS > 1 ? THREADS * P : 1];
    RowSum<TPR, 2 * U> row_sum{room};
    const int t = threadIdx.x % TPR, group = threadIdx.x / TPR;
    const long long step = (long long)gridDim.x * GROUPS, first = (long long)blockIdx.x * GROUPS + group;
    const long long turns = (p.rows + step * U - 1) / (step * U);
    Rows<DT, TPR, Q, U> xs, dys;
    float mean_next[U], rstd_next[U];
    auto load = [&](long long r) {
        xs.load(p.x, p.ldx, r, step, p.rows, p.D, t);
        dys.load(p.dy, p.lddy, r, step, p.rows, p.D, t);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool there = r + u * step < p.rows;
            mean_next[u] = there ? p.mean[r + u * step] : 0.f;
            rstd_next[u] = there ? p.rstd[r + u * step] : 0.f;
        }
    };
    load(first);
    float gamma[Q][P], dg[Q][P], db[Q][P];
#pragma unroll
    for (int q = 0; q < Q; ++q) {
        load_columns(p.gamma, (t + q * TPR) * P, p.D, 1.f, 0.f, gamma[q]);
#pragma unroll
        for (int e = 0; e < P; ++e) dg[q][e] = db[q][e] = 0.f;
    }
    const float inv = 1.f / (float)p.D;
    for (long long k = 0; k < turns; ++k) {
        const long long r0 = k * step * U + first;
        constexpr bool AHEAD = THREADS < 1024;
        if (!AHEAD && k) load(r0);
        const Rows<DT, TPR, Q, U> x = xs, dy = dys;
        float mean[U], rstd[U], s[2 * U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            mean[u] = mean_next[u];
            rstd[u] = rstd_next[u];
        }
        if (AHEAD && k + 1 < turns) load(r0 + step * U);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const V vx = __builtin_bit_cast(V, x.raw[u][q]), vd = __builtin_bit_cast(V, dy.raw[u][q]);
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    const float h = ((float)vx[e] - mean[u]) * rstd[u], d = (float)vd[e], g = d * gamma[q][e];
                    // (columns behind the row: dy and gamma are zeros there)
                    s1 += g;
                    s2 += (t + q * TPR) * P + e < p.D ? g * h : 0.f;
                    db[q][e] += d;
                    dg[q][e] += d * h;
                }
            }
            s[2 * u] = s1;
            s[2 * u + 1] = s2;
        }
        if (!p.out) continue;
        row_sum(s);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const long long r = r0 + u * step;
            if (r >= p.rows) break;
            const float s1 = s[2 * u] * inv, s2 = s[2 * u + 1] * inv;
            T* const dx = static_cast<T*>(p.out) + r * p.ldo;
#pragma unroll
            for (int q = 0; q < Q; ++q) {
                const V vx = __builtin_bit_cast(V, x.raw[u][q]), vd = __builtin_bit_cast(V, dy.raw[u][q]);
                const int d = (t + q * TPR) * P, n = p.D - d;
                V o;
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    const float h = ((float)vx[e] - mean[u]) * rstd[u];
                    o[e] = (T)(rstd[u] * ((float)vd[e] * gamma[q][e] - s1 - h * s2));
                }
                if (n >= P) store16(dx + d, __builtin_bit_cast(uint4v, o));
                else
#pragma unroll
                    for (int e = 0; e < P; ++e)
                        if (e < n) dx[d + e] = o[e];
            }
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
                // (a column of TPR * P at this q is one thread's: its groups' sums are TPR * P apart)
                for (int c = threadIdx.x; c < TPR * P; c += THREADS) {
                    float all = 0.f;
                    for (int g = 0; g < GROUPS; ++g) all += columns[g * TPR * P + c];
                    const int d = q * TPR * P + c;
                    if (d < p.D) out[(size_t)blockIdx.x * p.D + d] = all;
                }
            } else {
#pragma unroll
                for (int e = 0; e < P; ++e) {
                    const int d = (t + q * TPR) * P + e;
                    if (d < p.D) out[(size_t)blockIdx.x * p.D + d] = sum[e];
                }
            }
        }
    }
}

// Rows that no workgroup holds: one workgroup a row, in several readings, the first from memory.
constexpr int kLong = 1024;
// body(d, whole) for a thread's eights of a row's columns, from d on; whole: all eight are there
template <typename F>
__device__ __forceinline__ void along_row(int D, F body) {
    int d = threadIdx.x * 8;
#pragma unroll 4
    for (; d + 8 <= D; d += kLong * 8) body(d, std::true_type{});
    if (d < D) body(d, std::false_type{});
}
template <int DT, bool WHOLE>
__device__ __forceinline__ void load_eight(const typename Store<DT>::T* p, int n, float (&v)[8]) {
    Eight<DT> e;
    if constexpr (WHOLE) e.load_whole(p);
    else e.load(p, n);
    e.get(v);
}

template <int DT>
__global__ __launch_bounds__(kLong) void norm_long_kernel(const NormArgs p) {
    typedef typename Store<DT>::T T;
    __shared__ float room[2][1][16], pair_room[2][2][16];
    RowSum<kLong, 1> row_sum{room};
    RowSum<kLong, 2, true> row_sums{pair_room};
    for (long long r = blockIdx.x; r < p.rows; r += gridDim.x) {
        const T* const x = static_cast<const T*>(p.x) + r * p.ldx;
        T* const y = static_cast<T*>(p.out) + r * p.ldo;
        float sum[1] = {}, s[2] = {};
        along_row(p.D, [&](int d, auto whole) {
            float v[8];
            load_eight<DT, whole>(x + d, p.D - d, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) sum[0] += v[e];
        });
        row_sum(sum);
        const float mean = sum[0] / (float)p.D;
        along_row(p.D, [&](int d, auto whole) {
            float v[8];
            load_eight<DT, whole>(x + d, p.D - d, v);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float away = whole || d + e < p.D ? v[e] - mean : 0.f;
                s[0] += away;
                s[1] = fmaf(away, away, s[1]);
            }
        });
        row_sums(s);
        const float rest = s[0] / (float)p.D, rstd = rstd_of(s[1] / (float)p.D, rest, p.eps);
        if (threadIdx.x == 0) {
            if (p.mean) p.mean[r] = mean + rest;
            if (p.rstd) p.rstd[r] = rstd;
        }
        along_row(p.D, [&](int d, auto whole) {
            float v[8], gamma[8], beta[8];
            load_eight<DT, whole>(x + d, p.D - d, v);
            load_columns(p.gamma, d, p.D, 1.f, 1.f, gamma);
            load_columns(p.beta, d, p.D, 0.f, 0.f, beta);
#pragma unroll
            for (int e = 0; e < 8; ++e) v[e] = fmaf((v[e] - mean - rest) * rstd, gamma[e], beta[e]);
            store8<DT>(y + d, whole ? 8 : p.D - d, v);
        });
    }
}

template <int DT>
__global__ __launch_bounds__(kLong) void norm_grad_long_kernel(const NormArgs p) {
    typedef typename Store<DT>::T T;
    __shared__ float room[2][2][16];
    RowSum<kLong, 2> row_sum{room};
    for (long long r = blockIdx.x; r < p.rows; r += gridDim.x) {
        const T* const x = static_cast<const T*>(p.x) + r * p.ldx;
        const T* const dy = static_cast<const T*>(p.dy) + r * p.lddy;
        T* const dx = static_cast<T*>(p.out) + r * p.ldo;
        const float mean = p.mean[r], rstd = p.rstd[r];
        float s[2] = {};
        along_row(p.D, [&](int d, auto whole) {
            float vx[8], vd[8], gamma[8];
            load_eight<DT, whole>(x + d, p.D - d, vx);
            load_eight<DT, whole>(dy + d, p.D - d, vd);
            load_columns(p.gamma, d, p.D, 1.f, 0.f, gamma);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float g = vd[e] * gamma[e];
                s[0] += g;
                s[1] += whole || d + e < p.D ? g * ((vx[e] - mean) * rstd) : 0.f;
            }
        });
        row_sum(s);
        const float s1 = s[0] / (float)p.D, s2 = s[1] / (float)p.D;
        along_row(p.D, [&](int d, auto whole) {
            float vx[8], vd[8], gamma[8];
            load_eight<DT, whole>(x + d, p.D - d, vx);
            load_eight<DT, whole>(dy + d, p.D - d, vd);
            load_columns(p.gamma, d, p.D, 1.f, 0.f, gamma);
#pragma unroll
            for (int e = 0; e < 8; ++e) vd[e] = rstd * (vd[e] * gamma[e] - s1 - (vx[e] - mean) * rstd * s2);
            store8<DT>(dx + d, whole ? 8 : p.D - d, vd);
        });
    }
}

// Column sums of dy * h and dy over a strip of rows: a wave's lanes hold eight columns each, its workgroup's four waves take turns.  (Four
// rows ahead in 16 bits take all 256 registers, one wave a SIMD: 2000 x 25088, fp16, 37 us, what memory takes.)
constexpr int kSumCols = 512;
template <int DT>
__global__ __launch_bounds__(256) void norm_columns_kernel(const NormArgs p, int per) {
    typedef typename Store<DT>::T T;
    __shared__ __align__(16) float part[3][2][kSumCols];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int j = blockIdx.x * kSumCols + lane * 8, n = p.D - j;
    const long long r0 = (long long)blockIdx.y * per, r1 = min((long long)p.rows, r0 + per);
    float dg[8] = {}, db[8] = {}, vx[8], vd[8];
    auto rows = [&](auto whole) {
#pragma unroll 4
        for (long long r = r0 + wave; r < r1; r += 4) {
            Eight<DT> ex, ed;
            if constexpr (whole) {
                ex.load_whole(static_cast<const T*>(p.x) + r * p.ldx + j);
                ed.load_whole(static_cast<const T*>(p.dy) + r * p.lddy + j);
            } else {
                ex.load(static_cast<const T*>(p.x) + r * p.ldx + j, n);
                ed.load(static_cast<const T*>(p.dy) + r * p.lddy + j, n);
            }
            ex.get(vx);
            ed.get(vd);
            const float mean = p.mean[r], rstd = p.rstd[r];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                dg[q] += vd[q] * ((vx[q] - mean) * rstd);
                db[q] += vd[q];
            }
        }
    };
    if (n >= 8) rows(std::true_type{});
    else if (n > 0) rows(std::false_type{});
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

// out[d] = sum of the parts [part][d]: 64 columns a workgroup, four a thread (one where D is no multiple of four), and 16 (4)
// threads to a column, each with every 16th (4th) part, eight of them asked for at a time
template <int C>
__global__ __launch_bounds__(256) void norm_add_kernel(const float* dgamma_parts, const float* dbeta_parts, int parts, int D, float* dgamma,
                                                       float* dbeta) {
    constexpr int W = 64 / C, S = 256 / W;
    typedef float Vc __attribute__((ext_vector_type(C)));
    __shared__ float sums[S][64];
    const float* const from = blockIdx.y ? dbeta_parts : dgamma_parts;
    float* const to = blockIdx.y ? dbeta : dgamma;
    if (!to) return;
    const int c = threadIdx.x % W * C, s = threadIdx.x / W, d = blockIdx.x * 64 + c;
    float sum[C] = {};
    if (d < D)
#pragma unroll 8
        for (int g = s; g < parts; g += S) {
            const Vc v = *reinterpret_cast<const Vc*>(from + (size_t)g * D + d);
#pragma unroll
            for (int e = 0; e < C; ++e)
                if constexpr (C > 1) sum[e] += v[e];
                else sum[e] += v[0];
        }
#pragma unroll
    for (int e = 0; e < C; ++e) sums[s][c + e] = sum[e];
    __syncthreads();
    if (threadIdx.x < 64 && blockIdx.x * 64 + threadIdx.x < D) {
        float all = 0.f;
#pragma unroll
        for (int q = 0; q < S; ++q) all += sums[q][threadIdx.x];
        to[blockIdx.x * 64 + threadIdx.x] = all;
    }
}

__global__ __launch_bounds__(256) void norm_zero_kernel(float* a, float* b, int n) {
    const int i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) {
        if (a) a[i] = 0.f;
        if (b) b[i] = 0.f;
    }
}

// How a row of `pieces` 16-byte pieces is spread: threads of a row, pieces of a thread, rows at a time; tpr = 0: too long
struct Spread { int tpr, q, u; };
Spread spread(int pieces) {
    if (pieces <= 8) return {8, 1, 4};
    if (pieces <= 16) return {16, 1, 4};
    if (pieces <= 32) return {32, 1, 4};
    if (pieces <= 64) return {64, 1, 4};
    if (pieces <= 128) return {64, 2, 2};
    if (pieces <= 256) return {256, 1, 2};
    if (pieces <= 512) return {256, 2, 1};
    if (pieces <= 1024) return {512, 2, 1};
    if (pieces <= 2048) return {1024, 2, 1};
    return {0, 0, 1};
}
#define PCONV_SPREADS(X) X(8, 1, 4) X(16, 1, 4) X(32, 1, 4) X(64, 1, 4) X(64, 2, 2) X(256, 1, 2) X(256, 2, 1) X(512, 2, 1) X(1024, 2, 1)
// (the backward pass needs three times the registers; 1024 threads with two pieces of 16 bits have 128 each, and 68 bytes a lane do not fit:
// 4096 x 16384, bf16, 97 us, where memory takes 78)
Spread grad_spread(int pieces) {
    if (pieces <= 8) return {8, 1, 2};
    if (pieces <= 16) return {16, 1, 2};
    if (pieces <= 32) return {32, 1, 2};
    if (pieces <= 64) return {64, 1, 2};
    if (pieces <= 128) return {64, 2, 1};
    if (pieces <= 256) return {256, 1, 1};
    if (pieces <= 512) return {256, 2, 1};
    if (pieces <= 1024) return {512, 2, 1};
    if (pieces <= 2048) return {1024, 2, 1};
    return {0, 0, 1};
}
#define PCONV_GRAD_SPREADS(X) X(8, 1, 2) X(16, 1, 2) X(32, 1, 2) X(64, 1, 2) X(64, 2, 1) X(256, 1, 1) X(256, 2, 1) X(512, 2, 1) X(1024, 2, 1)

// 1024 threads for a compute unit: more workgroups read gamma and beta more often than they hide (16384 x 4096, bf16, of 256 threads:
// one for a compute unit 87 us, two 57, four 45, eight 46)
constexpr int forward_threads(int tpr) { return tpr > 256 ? tpr : 256; }
int workgroups(const Spread& s, int rows) {
    const int threads = s.tpr ? forward_threads(s.tpr) : kLong, groups = s.tpr ? threads / s.tpr : 1;
    const long long wanted = ((long long)rows + groups - 1) / groups;
    return (int)std::min<long long>(wanted, 256ll * (1024 / threads));
}
// (backward: one workgroup for a compute unit, so that there are few parts to add)
constexpr int backward_threads(int tpr) { return tpr > 512 ? tpr : 512; }
int grad_workgroups(const Spread& s, int rows) {
    const int groups = s.tpr ? backward_threads(s.tpr) / s.tpr : 1;
    return (int)std::min<long long>(((long long)rows + groups - 1) / groups, 256);
}
int strips(int rows, int D) { return std::max(1, std::min({64, (int)((rows + 15ll) / 16), 512 / ((D + kSumCols - 1) / kSumCols) + 1})); }

template <int DT>
int launch_norm(const NormArgs& a, hipStream_t st) {
    const Spread s = spread((a.D + Store<DT>::kPer - 1) / Store<DT>::kPer);
    const dim3 grid((unsigned)workgroups(s, a.rows));
#define X(TPR, Q, U)              \
    if (s.tpr == TPR && s.q == Q) \
        hipLaunchKernelGGL((norm_kernel<DT, TPR, Q, U, forward_threads(TPR)>), grid, dim3(forward_threads(TPR)), 0, st, a);
    PCONV_SPREADS(X)
#undef X
    if (!s.tpr) hipLaunchKernelGGL(norm_long_kernel<DT>, grid, dim3(kLong), 0, st, a);
    PCONV_HIP(hipGetLastError());
    return PCONV_OK;
}

int grad_parts(int dtype, int rows, int D) {
    const int per = 16 / elem_bytes(dtype);
    const Spread s = grad_spread((D + per - 1) / per);
    return s.tpr ? grad_workgroups(s, rows) : strips(rows, D);
}

template <int DT>
int launch_norm_grad(NormArgs a, float* dgamma, float* dbeta, float* parts, hipStream_t st) {
    const Spread s = grad_spread((a.D + Store<DT>::kPer - 1) / Store<DT>::kPer);
    const int n = grad_parts(DT, a.rows, a.D);
    // (a single part is the result)
    a.dgamma = dgamma ? n > 1 ? parts : dgamma : nullptr;
    a.dbeta = dbeta ? n > 1 ? parts + (size_t)n * a.D : dbeta : nullptr;
    const dim3 grid((unsigned)grad_workgroups(s, a.rows));
#define X(TPR, Q, U)              \
    if (s.tpr == TPR && s.q == Q) \
        hipLaunchKernelGGL((norm_grad_kernel<DT, TPR, Q, U, backward_threads(TPR)>), grid, dim3(backward_threads(TPR)), 0, st, a);
    PCONV_GRAD_SPREADS(X)
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
        const dim3 blocks((a.D + 63) / 64, 2);
        if (a.D % 4 == 0) hipLaunchKernelGGL(norm_add_kernel<4>, blocks, dim3(256), 0, st, a.dgamma, a.dbeta, n, a.D, dgamma, dbeta);
        else hipLaunchKernelGGL(norm_add_kernel<1>, blocks, dim3(256), 0, st, a.dgamma, a.dbeta, n, a.D, dgamma, dbeta);
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
