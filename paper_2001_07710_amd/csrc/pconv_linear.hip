// Entry points of the matrix products of pconv_dense.h: checks, the choice of tile and of how many workgroups share a tile, the
// column sums of the bias gradient, the gradient in front of an activation.  The products themselves: pconv_linear_kernels.h.
#include "pconv_dense_util.h"
#include "pconv_linear.h"

namespace pconv {
namespace {

constexpr int kMostRows = 1 << 30;          // (the kernels count rows, and stages of a product over rows, in 32 bits)

struct Plan {
    int tile = 0;                           // kTiles: the kernel for few rows
    int splits = 1, c_per = 0;
    size_t part_bytes = 0;
};

// What a workgroup of a tile takes, in microseconds, fitted to 45 products of 64 to 10,000 rows and columns, in every split (half of the
// choices are the best measured one, none is 30 % off): `fixed` for its launch, first stages and results, per stage `alone`, bound by
// the latency of a stage, or `shared` where more workgroups of a compute unit than that would fill are under way.
struct TileCost {
    int resident;
    double fixed, alone, shared;
};
constexpr TileCost kCost16[kTiles] = {{1, 8.0, 1.1, 1.25}, {2, 2.5, 0.67, 0.55}, {4, 1.5, 0.29, 0.2}};
constexpr TileCost kCost32 = {4, 1.5, 0.65, 0.48};
constexpr int kMostSplits = 128;

// Tile and split of a product of I x J results over C: the cheapest by these prices.  A split costs a second launch and its parts, written
// and read again at about 4.5 TB/s.
// The prices are those of rows that are aligned to 16 bytes.  Others go through registers, 0.6 us a stage on the smallest tile, and the middle
// tile stands in for the largest, with the same split: the workspace does not depend on strides.
Plan plan_product(int dtype, int I, int J, int C, bool forward) {
    Plan p;
    const int stage = kStageBytes / elem_bytes(dtype);
    const int stages = (C + stage - 1) / stage;
    long long splits = 1;
    if (forward && I <= kFewRows) {
        // (a workgroup of eight waves for 16 rows of w.  One alone draws little of what memory gives, so that all compute units are to have one:
        // 25088 -> 1024, fp16, one row, 64 workgroups 30.1 us, 256 15.1; -> 2000, 125 31.2, 250 23.5.  What is saved has to pay for a second
        // launch and the parts, some 56 stages: 4096 -> 1000, 63 workgroups 7.1 us, 252 7.7; -> 256, 16 rows, 64 8.5, 128 7.6)
        p.tile = kTiles;
        const long long tiles = (J + 15ll) / 16, most = std::max(1ll, std::min({kComputeUnits / tiles, stages / 8ll, 16ll}));
        splits = stages - stages / most >= 56 ? most : 1;
    } else {
        double best = 0;
        for (int t = dtype == PCONV_F32 ? 2 : 0; t < kTiles; ++t) {
            const TileCost& c = dtype == PCONV_F32 ? kCost32 : kCost16[t];
            const long long e = kTileEdges[t], tiles = ((I + e - 1) / e) * ((J + e - 1) / e);
            long long tried = 0;
            for (long long s = 1; s <= std::min(kMostSplits, stages); s = s < 4 ? s + 1 : s + s / 2) {
                const int per = (int)((stages + s - 1) / s);
                const long long real = (stages + per - 1) / per, work = tiles * real;
                if (real == tried) continue;
                tried = real;
                if (s > 1 && work > 2 * c.resident * kComputeUnits) break;
                const long long full = work / (c.resident * kComputeUnits), rest = work % (c.resident * kComputeUnits);
                auto round = [&](long long w) { return c.fixed + per * std::max(c.alone, c.shared * (double)((w + kComputeUnits - 1) / kComputeUnits)); };
                double us = full * round(c.resident * kComputeUnits) + (rest ? round(rest) : 0.0);
                if (real > 1) us += 2.5 + 2.0 * real * I * J * 4 / 4.5e6;
                if (best == 0 || us < best) {
                    best = us;
                    p.tile = t;
                    splits = real;
                }
            }
        }
    }
    const int per = (int)((stages + splits - 1) / splits);
    p.splits = (stages + per - 1) / per;
    p.c_per = per * stage;
    if (p.splits > 1) p.part_bytes = (size_t)p.splits * (size_t)I * (size_t)J * sizeof(float);
    return p;
}

int launch(int dtype, const Product& p, bool few, void* stream) {
    switch (dtype) {
        case PCONV_F32: return few ? launch_few_rows_f32(p, stream) : launch_product_f32(p, stream);
        case PCONV_F16: return few ? launch_few_rows_f16(p, stream) : launch_product_f16(p, stream);
        default: return few ? launch_few_rows_bf16(p, stream) : launch_product_bf16(p, stream);
    }
}

int run(int dtype, Product& p, const Plan& plan, void* workspace, void* stream) {
    p.tile = plan.tile;
    p.splits = plan.splits;
    p.c_per = plan.c_per;
    p.parts = static_cast<float*>(workspace);
    return launch(dtype, p, plan.tile == kTiles, stream);
}

int check_sizes(int dtype, int M, int N, int K) {
    if (!is_dtype(dtype)) return PCONV_EINVAL;
    if (M < 0 || N < 1 || K < 1) return PCONV_ESHAPE;
    if (M > kMostRows || N > kMostStride || K > kMostStride) return PCONV_EUNSUPPORTED;
    return PCONV_OK;
}
bool bad_element_alignment(int dtype, const void* p) { return !aligned_to(p, elem_bytes(dtype)); }
bool bad_act(int act) { return act < PCONV_ACT_NONE || act > PCONV_ACT_SILU; }
bool bad_workspace(const void* ws, size_t have, size_t need) { return need && (!ws || have < need || !aligned_to(ws, 16)); }

// ---- column sums of dz (the bias gradient): a workgroup sums a strip of rows for 512 columns, in the order of the rows.  8192 x 4096, bf16: 13
// us, what memory takes for dz.  (Few columns leave most lanes idle, and there are 64 strips at most: 200,000 x 64, bf16, 177 us.)
constexpr int kSumCols = 512, kMostStrips = 64;
int sum_strips(int M, int N) {
    const int wide = (N + kSumCols - 1) / kSumCols;
    return std::max(1, std::min({kMostStrips, (int)((M + 63ll) / 64), (2 * kComputeUnits + wide - 1) / wide}));
}

template <int DT>
__global__ __launch_bounds__(256) void column_sums_kernel(const typename Store<DT>::T* m, long long ld, int M, int N, int per, float* out) {
    __shared__ __align__(16) float part[3][kSumCols];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int j = blockIdx.x * kSumCols + lane * 8, n = N - j;
    const long long r0 = (long long)blockIdx.y * per, r1 = min((long long)M, r0 + per);
    float sum[8] = {}, v[8];
    if (n > 0)
#pragma unroll 4
        for (long long r = r0 + wave; r < r1; r += 4) {
            load8<DT>(m + r * ld + j, n, v);
#pragma unroll
            for (int q = 0; q < 8; ++q) sum[q] += v[q];
        }
    if (wave) store8<PCONV_F32>(&part[wave - 1][lane * 8], 8, sum);
    __syncthreads();
    if (wave == 0 && n > 0) {
        for (int s = 0; s < 3; ++s)
#pragma unroll
            for (int q = 0; q < 8; ++q) sum[q] += part[s][lane * 8 + q];
        store8<PCONV_F32>(out + (size_t)blockIdx.y * N + j, n, sum);
    }
}
__global__ __launch_bounds__(256) void add_strips_kernel(Strips s) { add_strips(s.parts, s.strips, s.N, s.out, blockIdx.x * 64); }
constexpr unsigned kMostThreads = 1u << 28;     // of the launches of one thread for each piece (HIP takes fewer than 2^32)
__global__ __launch_bounds__(256) void fill_zero_kernel(float* out, unsigned n) {
    const unsigned i = blockIdx.x * 256 + threadIdx.x;
    if (i < n) out[i] = 0.f;
}
int fill_zero(float* out, unsigned long long n, hipStream_t st) {
    for (unsigned now; n > 0; n -= now, out += now) {
        now = (unsigned)std::min<unsigned long long>(n, kMostThreads);
        hipLaunchKernelGGL(fill_zero_kernel, dim3((now + 255) / 256), dim3(256), 0, st, out, now);
        PCONV_HIP(hipGetLastError());
    }
    return PCONV_OK;
}

// Column sums of m, but for the adding of strips where there are several
template <int DT>
int column_sums(const void* m, long long ld, int M, int N, float* parts, float* out, Strips* left, hipStream_t st) {
    const int strips = sum_strips(M, N), per = (M + strips - 1) / strips;
    hipLaunchKernelGGL(column_sums_kernel<DT>, dim3((N + kSumCols - 1) / kSumCols, strips), dim3(256), 0, st,
                       static_cast<const typename Store<DT>::T*>(m), ld, M, N, per, strips > 1 ? parts : out);
    PCONV_HIP(hipGetLastError());
    if (strips > 1) *left = Strips{parts, strips, N, out};
    return PCONV_OK;
}
size_t strip_bytes(int M, int N) {
    const int strips = sum_strips(M, N);
    return strips > 1 ? ((size_t)strips * N * sizeof(float) + 15) / 16 * 16 : 0;
}

// dz = dy * act'(z), eight values a thread: memory bounds it.  8192 x 4096, bf16: 37 us with ReLU, 39 with GELU (5.2 to 5.4 TB/s, part of it
// from the cache behind L2); 64 x 4096: 4.5 us, a launch.
template <int DT>
__global__ __launch_bounds__(256) void activation_grad_kernel(const typename Store<DT>::T* dy, long long lddy, const typename Store<DT>::T* z,
                                                              long long ldz, typename Store<DT>::T* dz, long long lddz, int M, int N, int act) {
    const unsigned per_row = (unsigned)(N + 7) / 8, at = blockIdx.x * 256 + threadIdx.x;
    const long long i = at / per_row;
    if (i >= M) return;
    const int j = (int)(at % per_row) * 8, n = N - j;
    float v[1][8], a[1][8];
    load8<DT>(dy + i * lddy + j, n, v[0]);
    load8<DT>(z + i * ldz + j, n, a[0]);
    times_slope8<DT, 1>(v, a, act);
    store8<DT>(dz + i * lddz + j, n, v[0]);
}

template <int DT>
int activation_grad(const void* dy, long long lddy, const void* z, long long ldz, void* dz, long long lddz, int M, int N, int act, hipStream_t st) {
    typedef typename Store<DT>::T T;
    const T *gradient = static_cast<const T*>(dy), *argument = static_cast<const T*>(z);
    T* out = static_cast<T*>(dz);
    const int per_row = (N + 7) / 8, most = (int)(kMostThreads / per_row);
    for (int rows; M > 0; M -= rows) {
        rows = std::min(M, most);
        hipLaunchKernelGGL(activation_grad_kernel<DT>, dim3((unsigned)(((long long)rows * per_row + 255) / 256)), dim3(256), 0, st, gradient, lddy,
                           argument, ldz, out, lddz, rows, N, act);
        PCONV_HIP(hipGetLastError());
        gradient += rows * lddy;
        argument += rows * ldz;
        out += rows * lddz;
    }
    return PCONV_OK;
}

}  // namespace
}  // namespace pconv

using namespace pconv;

extern "C" int pconv_linear_workspace(int dtype, int M, int N, int K, size_t* bytes) {
    if (!bytes) return PCONV_EINVAL;
    *bytes = 0;
    if (int rc = check_sizes(dtype, M, N, K)) return rc;
    if (M > 0) *bytes = plan_product(dtype, M, N, K, true).part_bytes;
    return PCONV_OK;
}

extern "C" int pconv_linear(const void* x, long long ldx, const void* w, long long ldw, const float* bias, const void* residual,
                            long long ldr, void* z, void* y, long long ldy, int dtype, int M, int N, int K, int act, unsigned flags,
                            void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = check_sizes(dtype, M, N, K)) return rc;
    if (bad_act(act) || (flags & ~(unsigned)PCONV_FLAG_RESIDUAL_FIRST)) return PCONV_EINVAL;
    for (int rc : {check_stride(&ldx, K), check_stride(&ldw, K), residual ? check_stride(&ldr, N) : PCONV_OK, check_stride(&ldy, N)})
        if (rc) return rc;
    if (M == 0) return PCONV_OK;
    if (!x || !w || !y) return PCONV_EINVAL;
    for (const void* p : {x, w, residual, (const void*)z, (const void*)y})
        if (bad_element_alignment(dtype, p)) return PCONV_EINVAL;
    if (!aligned_to(bias, 4)) return PCONV_EINVAL;
    const Plan plan = plan_product(dtype, M, N, K, true);
    if (bad_workspace(workspace, workspace_bytes, plan.part_bytes)) return PCONV_EINVAL;
    Product p{};
    p.a = x; p.lda = ldx; p.b = w; p.ldb = ldw;
    p.I = M; p.J = N; p.C = K;
    p.f.kind = kForward;
    p.f.act = act;
    p.f.first = (flags & PCONV_FLAG_RESIDUAL_FIRST) != 0;
    p.f.bias = bias;
    p.f.add = residual; p.f.ld_add = ldr;
    p.f.z = z;
    p.f.out = y; p.f.ld_out = ldy;
    return run(dtype, p, plan, workspace, stream);
}

extern "C" int pconv_linear_grad_input_workspace(int dtype, int M, int N, int K, size_t* bytes) {
    if (!bytes) return PCONV_EINVAL;
    *bytes = 0;
    if (int rc = check_sizes(dtype, M, N, K)) return rc;
    if (M > 0) *bytes = plan_product(dtype, M, K, N, false).part_bytes;
    return PCONV_OK;
}

extern "C" int pconv_linear_grad_input(const void* dz, long long lddz, const void* w, long long ldw, const void* z, long long ldz,
                                       int act, const void* add, long long lda, void* dx, long long lddx, int dtype, int M, int N,
                                       int K, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = check_sizes(dtype, M, N, K)) return rc;
    if (bad_act(act) || (act != PCONV_ACT_NONE && !z && M > 0)) return PCONV_EINVAL;
    for (int rc : {check_stride(&lddz, N), check_stride(&ldw, K), z ? check_stride(&ldz, K) : PCONV_OK,
                   add ? check_stride(&lda, K) : PCONV_OK, check_stride(&lddx, K)})
        if (rc) return rc;
    if (M == 0) return PCONV_OK;
    if (!dz || !w || !dx) return PCONV_EINVAL;
    for (const void* p : {dz, w, z, add, (const void*)dx})
        if (bad_element_alignment(dtype, p)) return PCONV_EINVAL;
    const Plan plan = plan_product(dtype, M, K, N, false);
    if (bad_workspace(workspace, workspace_bytes, plan.part_bytes)) return PCONV_EINVAL;
    Product p{};
    p.a = dz; p.lda = lddz; p.b = w; p.ldb = ldw;
    p.I = M; p.J = K; p.C = N;
    p.b_rows = true;
    p.f.kind = kGradInput;
    p.f.act = act;
    p.f.zin = act == PCONV_ACT_NONE ? nullptr : z; p.f.ld_zin = ldz;
    p.f.add = add; p.f.ld_add = lda;
    p.f.out = dx; p.f.ld_out = lddx;
    return run(dtype, p, plan, workspace, stream);
}

extern "C" int pconv_linear_grad_weight_workspace(int dtype, int M, int N, int K, size_t* bytes) {
    if (!bytes) return PCONV_EINVAL;
    *bytes = 0;
    if (int rc = check_sizes(dtype, M, N, K)) return rc;
    // (the strips of the bias gradient's sums first, the product's parts behind them)
    if (M > 0) *bytes = strip_bytes(M, N) + plan_product(dtype, N, K, M, false).part_bytes;
    return PCONV_OK;
}

extern "C" int pconv_linear_grad_weight(const void* dz, long long lddz, const void* x, long long ldx, float* dw, float* db, int dtype,
                                        int M, int N, int K, void* workspace, size_t workspace_bytes, void* stream) {
    if (int rc = check_sizes(dtype, M, N, K)) return rc;
    for (int rc : {check_stride(&lddz, N), check_stride(&ldx, K)})
        if (rc) return rc;
    if (!dw || !aligned_to(dw, 4) || !aligned_to(db, 4)) return PCONV_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (M == 0) {
        if (int rc = fill_zero(dw, (unsigned long long)N * K, st)) return rc;
        return db ? fill_zero(db, N, st) : PCONV_OK;
    }
    if (!dz || !x) return PCONV_EINVAL;
    for (const void* p : {dz, x})
        if (bad_element_alignment(dtype, p)) return PCONV_EINVAL;
    const Plan plan = plan_product(dtype, N, K, M, false);
    const size_t strips = strip_bytes(M, N);
    if (bad_workspace(workspace, workspace_bytes, strips + plan.part_bytes)) return PCONV_EINVAL;
    Product p{};
    if (db) {
        float* const parts = static_cast<float*>(workspace);
        int rc = dtype == PCONV_F32   ? column_sums<PCONV_F32>(dz, lddz, M, N, parts, db, &p.strips, st)
                 : dtype == PCONV_F16 ? column_sums<PCONV_F16>(dz, lddz, M, N, parts, db, &p.strips, st)
                                      : column_sums<PCONV_BF16>(dz, lddz, M, N, parts, db, &p.strips, st);
        if (rc) return rc;
        if (p.strips.parts && plan.splits == 1) {
            hipLaunchKernelGGL(add_strips_kernel, dim3((N + 63) / 64), dim3(256), 0, st, p.strips);
            PCONV_HIP(hipGetLastError());
        }
    }
    p.a = dz; p.lda = lddz; p.b = x; p.ldb = ldx;
    p.I = N; p.J = K; p.C = M;
    p.a_rows = p.b_rows = true;
    p.f.kind = kFloat;
    p.f.out = dw; p.f.ld_out = K;
    return run(dtype, p, plan, workspace ? static_cast<char*>(workspace) + strips : nullptr, stream);
}

extern "C" int pconv_activation_grad(const void* dy, long long lddy, const void* z, long long ldz, void* dz, long long lddz, int dtype,
                                     int M, int N, int act, void* stream) {
    if (int rc = check_sizes(dtype, M, N, 1)) return rc;
    if (bad_act(act)) return PCONV_EINVAL;
    for (int rc : {check_stride(&lddy, N), check_stride(&ldz, N), check_stride(&lddz, N)})
        if (rc) return rc;
    if (M == 0) return PCONV_OK;
    if (!dy || !z || !dz) return PCONV_EINVAL;
    for (const void* p : {dy, z, (const void*)dz})
        if (bad_element_alignment(dtype, p)) return PCONV_EINVAL;
    hipStream_t st = static_cast<hipStream_t>(stream);
    return dtype == PCONV_F32   ? activation_grad<PCONV_F32>(dy, lddy, z, ldz, dz, lddz, M, N, act, st)
           : dtype == PCONV_F16 ? activation_grad<PCONV_F16>(dy, lddy, z, ldz, dz, lddz, M, N, act, st)
                                : activation_grad<PCONV_BF16>(dy, lddy, z, ldz, dz, lddz, M, N, act, st);
}
