// Matrix products with an epilogue on the matrix cores, for one storage type (PCONV_LINEAR_DT) per translation unit.
//
// R[i][j] = sum over c of A(i, c) * B(j, c), each operand stored with c along its rows ("c-minor": x and w of the forward
// pass, dz of the input gradient) or across them ("rows": w of the input gradient, both operands of the weight gradient).
//
// A workgroup owns a tile of TI x TJ results and walks over c in stages of 128 bytes of a row (64 elements, 32 for fp32), two
// stages in LDS: while one is multiplied the next is under way.
//   c-minor operand: [row][8 pieces of 16 bytes]; piece p of a row lies at place p ^ swizzle(row), so that the 32 rows an
//       operand read touches at one piece spread over the banks;
//   rows operand:    [c][pieces of 16 bytes]; piece p lies at p ^ swizzle(c) likewise, and is read with
//       ds_read_b64_tr_b16: four c of 16 rows a group of 16 lanes, handed over transposed (fp32: single words).
// Where rows are aligned to 16 bytes the pieces go from memory to LDS without registers (buffer_load ... lds: a wave's 64
// pieces land side by side, so the swizzle is applied to what each lane asks for); otherwise through registers.
// Pieces outside the matrix are outside the buffer descriptor and read as zeros.
//
// The matrix instructions get B as their rows and A as their columns: a lane of the result then holds four consecutive j of one i.
// They leave through a window of LDS that belongs to the wave, 32 i at a time, so that eight lanes store one 128-byte line.
#include "pconv_dense_util.h"
#include "pconv_linear.h"

namespace pconv {
namespace {

typedef __attribute__((address_space(3))) void* lds_ptr;
typedef __attribute__((address_space(3))) short4v* lds_short4;

constexpr int DT = PCONV_LINEAR_DT;
typedef Store<DT>::T T;
constexpr int ES = (int)sizeof(T);
constexpr int PER = 16 / ES;                 // elements of a piece
constexpr int BK = kStageBytes / ES;         // elements of c in a stage
constexpr int KS = 4;                        // steps of a stage: two pieces of c each

// acc += rows x columns over two pieces of c: lanes 0-31 hold the first, lanes 32-63 the second, of row / column lane % 32
__device__ __forceinline__ float16v mma(uint4v a, uint4v b, float16v acc) {
    if constexpr (DT == PCONV_F16)
        return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), acc, 0, 0, 0);
    else if constexpr (DT == PCONV_BF16)
        return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    else {
        const float4v x = __builtin_bit_cast(float4v, a), y = __builtin_bit_cast(float4v, b);
#pragma unroll
        for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_mfma_f32_32x32x2f32(x[q], y[q], acc, 0, 0, 0);
        return acc;
    }
}

struct Args {
    const unsigned char* a;
    const unsigned char* b;
    long long lda, ldb;                       // bytes
    unsigned long long a_span, b_span;        // bytes from the first element to behind the last
    int I, J, C, c_per, tiles_i, tiles_j;
    Finish f;
    float* parts;
};

// What the epilogue of eight results reads besides them: asked for ahead of their use.
struct Beside {
    Eight<DT> add, zin;
    __device__ __forceinline__ void load(const Finish& f, long long i, int j, int n) {
        if (f.kind == kFloat || n <= 0) return;
        if (f.add) add.load(static_cast<const T*>(f.add) + i * f.ld_add + j, n);
        if (f.kind == kGradInput && f.zin) zin.load(static_cast<const T*>(f.zin) + i * f.ld_zin + j, n);
    }
};

// Results v[0..7] at (i, j..j+7), n of them inside the matrix
__device__ __forceinline__ void finish8(const Finish& f, float v[8], const float bias[8], const Beside& beside, long long i, int j, int n) {
    if (f.kind == kFloat) {
        store8<PCONV_F32>(static_cast<float*>(f.out) + i * f.ld_out + j, n, v);
        return;
    }
    float add[8] = {};
    if (f.add) beside.add.get(add);
    if (f.kind == kForward) {
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] += bias[q];
        if (f.add && f.first)
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] += add[q];
        if (f.z) store8<DT>(static_cast<T*>(f.z) + i * f.ld_out + j, n, v);
        activate8(v, f.act);
        if (f.add && !f.first)
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] += add[q];
    } else {
        if (f.zin) {
            float z[8];
            beside.zin.get(z);
            times_slope8(v, z, f.act);
        }
        if (f.add)
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] += add[q];
    }
    store8<DT>(static_cast<T*>(f.out) + i * f.ld_out + j, n, v);
}
__device__ __forceinline__ void bias8(const Finish& f, int j, int n, float bias[8]) {
#pragma unroll
    for (int q = 0; q < 8; ++q) bias[q] = f.kind == kForward && f.bias && q < n ? f.bias[j + q] : 0.f;
}

// Workgroup b of G onto the work in order: consecutive workgroups go to different XCDs, an XCD's workgroups take consecutive work.
__device__ __forceinline__ unsigned by_xcd(unsigned b, unsigned G) {
    const unsigned x = b % 8, q = G / 8, r = G % 8;
    return x * q + (x < r ? x : r) + b / 8;
}

// How one operand of W rows (i or j) is staged and read.  ROWS: stored with c across its rows.
template <bool ROWS, int W, int THREADS>
struct Operand {
    static constexpr bool kRows = ROWS;
    static constexpr int kBytes = W * kStageBytes;
    static constexpr int kLineBytes = ROWS ? W * ES : kStageBytes;       // of one line in LDS
    static constexpr int kLinePieces = kLineBytes / 16;
    static constexpr int kPieces = kBytes / 16 / THREADS;                // per thread
    static constexpr int kLinesPer = THREADS / kLinePieces;              // lines that the workgroup's threads cover at once
    static_assert(THREADS % kLinePieces == 0 && kBytes % (16 * THREADS) == 0, "a thread's pieces lie under each other");
    static __device__ __forceinline__ int swizzle(int line) {
        if constexpr (!ROWS) return (line >> 1) & 7;
        // four lines of 64 bytes are read at once: they go to different quarters of 256 bytes
        else return kLinePieces >= 16 ? (line & 3) * 4 : ((line >> 1) & 1) * 4;
    }
    static constexpr int kPeriod = ROWS ? 4 : 16;
    static_assert(kLinesPer % kPeriod == 0 || kPieces == 1 || kLinesPer < kPeriod, "");

    // line and piece of the matrix that thread t's piece q holds
    static __device__ __forceinline__ void where(int t, int q, int* line, int* piece) {
        *line = t / kLinePieces + q * kLinesPer;
        *piece = (t % kLinePieces) ^ swizzle(*line);
    }
    // operand registers of 32-row block `blk` at step s
    static __device__ __forceinline__ uint4v read(const unsigned char* lds, int blk, int s, int lane) {
        const int r = lane & 31, h = lane >> 5;
        if constexpr (!ROWS) {
            const int row = blk * 32 + r;
            return *reinterpret_cast<const uint4v*>(lds + row * kStageBytes + (((2 * s + h) ^ swizzle(row)) * 16));
        } else if constexpr (ES == 2) {
            uint4v v;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int u = lane & 15, c = 16 * s + 8 * h + 4 * q + (u >> 2);
                const int at = (blk * 32 + 16 * ((lane >> 4) & 1) + 4 * (u & 3)) * 2;
                const unsigned char* p = lds + c * kLineBytes + (((at >> 4) ^ swizzle(c)) << 4) + (at & 15);
                const short4v w = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4)p);
                const uint2v d = __builtin_bit_cast(uint2v, w);
                if (q) { v.z = d.x; v.w = d.y; } else { v.x = d.x; v.y = d.y; }
            }
            return v;
        } else {
            float4v v;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = 8 * s + 4 * h + q, at = (blk * 32 + r) * 4;
                v[q] = *reinterpret_cast<const float*>(lds + c * kLineBytes + (((at >> 4) ^ swizzle(c)) << 4) + (at & 15));
            }
            return __builtin_bit_cast(uint4v, v);
        }
    }
};

template <bool AR, bool BR, int WI, int WJ, int AF, int BF, bool DIRECT>
__global__ __launch_bounds__(WI * WJ * 64) void product_kernel(const Args p) {
    constexpr int THREADS = WI * WJ * 64, TI = 32 * AF * WI, TJ = 32 * BF * WJ;
    typedef Operand<AR, TI, THREADS> OA;
    typedef Operand<BR, TJ, THREADS> OB;
    constexpr int STAGE = OA::kBytes + OB::kBytes;
    extern __shared__ __align__(16) unsigned char lds[];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wi = wave % WI, wj = wave / WI;

    // tile: groups of eight tile rows, column by column inside a group
    const unsigned tiles = (unsigned)p.tiles_i * p.tiles_j;
    const unsigned id = by_xcd(blockIdx.x, gridDim.x), split = id / tiles, tile = id % tiles;
    const unsigned per_group = 8u * p.tiles_j, group = tile / per_group, in = tile % per_group;
    const unsigned high = min(8u, (unsigned)p.tiles_i - group * 8);
    const int i0 = (int)(group * 8 + in % high) * TI, j0 = (int)(in / high) * TJ;
    const int c0 = (int)split * p.c_per, c1 = min(p.C, c0 + p.c_per);
    const int stages = (c1 - c0 + BK - 1) / BK;

    // where the operands' next stage begins, and the bytes from there to the matrix's end
    const unsigned long long a_at = AR ? (unsigned long long)c0 * p.lda + (unsigned long long)i0 * ES
                                       : (unsigned long long)i0 * p.lda + (unsigned long long)c0 * ES;
    const unsigned long long b_at = BR ? (unsigned long long)c0 * p.ldb + (unsigned long long)j0 * ES
                                       : (unsigned long long)j0 * p.ldb + (unsigned long long)c0 * ES;
    const unsigned char *pa = p.a + a_at, *pb = p.b + b_at;
    unsigned long long a_left = p.a_span - a_at, b_left = p.b_span - b_at;
    const unsigned long long a_step = AR ? (unsigned long long)p.lda * BK : kStageBytes;
    const unsigned long long b_step = BR ? (unsigned long long)p.ldb * BK : kStageBytes;
    int c_left = c1 - c0;

    float16v acc[AF][BF];
#pragma unroll
    for (int a = 0; a < AF; ++a)
#pragma unroll
        for (int b = 0; b < BF; ++b)
#pragma unroll
            for (int r = 0; r < 16; ++r) acc[a][b][r] = 0.f;

    uint4v ra[DIRECT ? 1 : OA::kPieces], rb[DIRECT ? 1 : OB::kPieces];
    // one operand's stage: into LDS (DIRECT), or into registers
    auto ask = [&](auto tag, const unsigned char* at, unsigned long long left, long long ld, int rows, unsigned char* to, uint4v* regs) {
        typedef decltype(tag) O;
        constexpr bool R = O::kRows;
        if constexpr (DIRECT) {
            const auto rsrc = make_rsrc(at, (uint32_t)min(left, 0x7FFFFFFFull));
            int line, piece;
            O::where(t, 0, &line, &piece);
            unsigned off = (unsigned)(line * ld) + piece * 16;
            if (!R && piece * PER >= c_left) off = kInvalid;
#pragma unroll
            for (int q = 0; q < O::kPieces; ++q)
                __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (lds_ptr)(to + (q * THREADS + wave * 64) * 16), 16,
                                                         (int)(off + (unsigned)(q * O::kLinesPer * ld)), 0, 0, 0);
        } else {
#pragma unroll
            for (int q = 0; q < O::kPieces; ++q) {
                int line, piece;
                O::where(t, q, &line, &piece);
                const int lines = R ? c_left : rows, along = (R ? rows : c_left) - piece * PER;
                regs[q] = uint4v{0, 0, 0, 0};
                if (line < lines && along > 0)
                    regs[q] = load_part<DT>(reinterpret_cast<const T*>(at + line * ld) + piece * PER, along);
            }
        }
    };
    auto ask_stage = [&](int buf) {
        unsigned char* const to = lds + buf * STAGE;
        ask(OA{}, pa, a_left, p.lda, p.I - i0, to, ra);
        ask(OB{}, pb, b_left, p.ldb, p.J - j0, to + OA::kBytes, rb);
        pa += a_step;
        pb += b_step;
        a_left -= a_step;
        b_left -= b_step;
        c_left -= BK;
    };
    auto put_stage = [&](int buf) {
        if constexpr (!DIRECT) {
            unsigned char* const to = lds + buf * STAGE;
#pragma unroll
            for (int q = 0; q < OA::kPieces; ++q) *reinterpret_cast<uint4v*>(to + (q * THREADS + t) * 16) = ra[q];
#pragma unroll
            for (int q = 0; q < OB::kPieces; ++q) *reinterpret_cast<uint4v*>(to + OA::kBytes + (q * THREADS + t) * 16) = rb[q];
        }
    };

    ask_stage(0);
    put_stage(0);
    for (int s = 0; s < stages; ++s) {
        const int buf = s & 1;
        __builtin_amdgcn_s_waitcnt(0x0F70);    // vmcnt(0): this wave's pieces of stage s are in LDS
        __syncthreads();                       // so are the other waves', and none reads the other half any more
        if (s + 1 < stages) ask_stage(buf ^ 1);
        const unsigned char *la = lds + buf * STAGE, *lb = la + OA::kBytes;
#pragma unroll
        for (int k = 0; k < KS; ++k) {
            uint4v fa[AF], fb[BF];
#pragma unroll
            for (int b = 0; b < BF; ++b) fb[b] = OB::read(lb, wj * BF + b, k, lane);
#pragma unroll
            for (int a = 0; a < AF; ++a) fa[a] = OA::read(la, wi * AF + a, k, lane);
#pragma unroll
            for (int a = 0; a < AF; ++a)
#pragma unroll
                for (int b = 0; b < BF; ++b) acc[a][b] = mma(fb[b], fa[a], acc[a][b]);
        }
        if (s + 1 < stages) put_stage(buf ^ 1);
    }
    __syncthreads();

    // results: a window of 32 i x 32 BF j floats for each wave, a pitch that spreads the rows over the banks
    constexpr int PITCH = (32 * BF + 4) * 4, ROW_LANES = 4 * BF, ROWS_AT_ONCE = 64 / ROW_LANES;
    static_assert(WI * WJ * 32 * PITCH <= 2 * STAGE, "the windows fit the stages");
    unsigned char* const win = lds + wave * 32 * PITCH;
    Finish f = p.f;
    if (p.parts) {
        f.kind = kFloat;
        f.out = p.parts + (unsigned long long)split * p.I * p.J;
        f.ld_out = p.J;
    }
    const int j = j0 + wj * 32 * BF + (lane % ROW_LANES) * 8, n = p.J - j;
    float bias[8];
    bias8(f, j, n, bias);
    auto put_block = [&](const float16v (&block)[BF]) {
#pragma unroll
        for (int b = 0; b < BF; ++b)
#pragma unroll
            for (int g = 0; g < 4; ++g)
                *reinterpret_cast<float4v*>(win + (lane & 31) * PITCH + (b * 32 + g * 8 + (lane >> 5) * 4) * 4) =
                    float4v{block[b][4 * g], block[b][4 * g + 1], block[b][4 * g + 2], block[b][4 * g + 3]};
    };
    constexpr int TIMES = 32 / ROWS_AT_ONCE;
#pragma unroll 1
    for (int a = 0; a < AF; ++a) {
        const int i = i0 + (wi * AF + a) * 32 + lane / ROW_LANES;
        Beside beside[TIMES];
#pragma unroll
        for (int r = 0; r < TIMES; ++r)
            if (i + r * ROWS_AT_ONCE < p.I) beside[r].load(f, i + r * ROWS_AT_ONCE, j, n);
#pragma unroll
        for (int b = 0; b < AF; ++b)
            if (a == b) put_block(acc[b]);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int r = 0; r < TIMES; ++r) {
            const unsigned char* const at = win + (lane / ROW_LANES + r * ROWS_AT_ONCE) * PITCH + (lane % ROW_LANES) * 32;
            const float4v lo = *reinterpret_cast<const float4v*>(at), hi = *reinterpret_cast<const float4v*>(at + 16);
            float v[8] = {lo.x, lo.y, lo.z, lo.w, hi.x, hi.y, hi.z, hi.w};
            if (i + r * ROWS_AT_ONCE < p.I && n > 0) finish8(f, v, bias, beside[r], i + r * ROWS_AT_ONCE, j, n);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
}

// The parts of a product that several workgroups share, added in their order, and its epilogue: eight results a thread.
__global__ __launch_bounds__(256) void add_parts_kernel(const float* parts, int splits, int I, int J, Finish f) {
    const int per_row = (J + 7) / 8;
    const unsigned long long at = (unsigned long long)blockIdx.x * 256 + threadIdx.x;
    const unsigned long long i = at / per_row;
    if (i >= (unsigned long long)I) return;
    const int j = (int)(at % per_row) * 8, n = J - j;
    float v[8] = {}, w[8], bias[8];
    for (int s = 0; s < splits; ++s) {
        load8<PCONV_F32>(parts + ((unsigned long long)s * I + i) * J + j, n, w);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[q] += w[q];
    }
    bias8(f, j, n, bias);
    Beside beside;
    beside.load(f, (long long)i, j, n);
    finish8(f, v, bias, beside, (long long)i, j, n);
}

// Few rows of x (up to 16) with weights that are read once, straight into registers: memory bounds it, no operand is shared.  A
// workgroup owns 16 rows of w; its waves take turns along k (a wave's 64 lanes: 16 rows x 4 pieces), and their sums meet in LDS
// in the order of the waves.  v_mfma_f32_16x16x32: rows of the result are rows of w, its columns rows of x.
constexpr int kFewWaves = 8;
__device__ __forceinline__ float4v mma16(uint4v a, uint4v b, float4v acc) {
    if constexpr (DT == PCONV_F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), acc, 0, 0, 0);
    else if constexpr (DT == PCONV_BF16)
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), acc, 0, 0, 0);
    else {
        const float4v x = __builtin_bit_cast(float4v, a), y = __builtin_bit_cast(float4v, b);
#pragma unroll
        for (int q = 0; q < 4; ++q) acc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[q], y[q], acc, 0, 0, 0);
        return acc;
    }
}

__global__ __launch_bounds__(kFewWaves * 64) void few_rows_kernel(const Args p) {
    __shared__ __align__(16) float sums[kFewWaves][16][20];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const unsigned tiles = (unsigned)p.tiles_j, split = blockIdx.x / tiles, tile = blockIdx.x % tiles;
    const int j0 = (int)tile * 16, c0 = (int)split * p.c_per, c1 = min(p.C, c0 + p.c_per);
    const int r = lane & 15, piece = lane >> 4;
    const bool has_w = j0 + r < p.J, has_x = r < p.I;
    const T* pw = reinterpret_cast<const T*>(p.b + (has_w ? j0 + r : 0) * p.ldb);
    const T* px = reinterpret_cast<const T*>(p.a + (has_x ? r : 0) * p.lda);
    constexpr int STEP = 4 * PER, U = 4;                    // elements of k of one step of a wave; steps in flight
    float4v acc = {0.f, 0.f, 0.f, 0.f};
    int c = c0 + wave * STEP * U;
    for (; c + STEP * U <= c1; c += kFewWaves * STEP * U) {
        uint4v w[U], x[U];
#pragma unroll
        for (int u = 0; u < U; ++u) w[u] = load16(pw + c + u * STEP + piece * PER);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            x[u] = uint4v{0, 0, 0, 0};
            if (has_x) x[u] = load16(px + c + u * STEP + piece * PER);
        }
#pragma unroll
        for (int u = 0; u < U; ++u) acc = mma16(w[u], x[u], acc);
    }
    if (c < c1) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = c + u * STEP + piece * PER;
            const uint4v w = load_part<DT>(pw + at, c1 - at);
            uint4v x = {0, 0, 0, 0};
            if (has_x) x = load_part<DT>(px + at, c1 - at);
            acc = mma16(w, x, acc);
        }
    }
    *reinterpret_cast<float4v*>(&sums[wave][r][4 * piece]) = acc;            // [row of x][row of w]
    __syncthreads();
    if (t < 32) {
        const int i = t >> 1, j = j0 + (t & 1) * 8, n = p.J - j;
        if (i < p.I && n > 0) {
            float v[8] = {}, bias[8];
            for (int s = 0; s < kFewWaves; ++s)
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] += sums[s][i][(t & 1) * 8 + q];
            Finish f = p.f;
            if (p.parts) {
                f.kind = kFloat;
                f.out = p.parts + (unsigned long long)split * p.I * p.J;
                f.ld_out = p.J;
            }
            bias8(f, j, n, bias);
            Beside beside;
            beside.load(f, i, j, n);
            finish8(f, v, bias, beside, i, j, n);
        }
    }
}

Args make_args(const Product& p, int tile_i, int tile_j) {
    Args a;
    a.a = static_cast<const unsigned char*>(p.a);
    a.b = static_cast<const unsigned char*>(p.b);
    a.lda = p.lda * ES;
    a.ldb = p.ldb * ES;
    a.I = p.I;
    a.J = p.J;
    a.C = p.C;
    a.c_per = p.c_per;
    const long long ra = p.a_rows ? p.C : p.I, la = p.a_rows ? p.I : p.C, rb = p.b_rows ? p.C : p.J, lb = p.b_rows ? p.J : p.C;
    // (up to the end of the last element's 16 bytes, which lie in its page: a piece that begins inside is read whole)
    a.a_span = ((unsigned long long)((ra - 1) * a.lda + la * ES) + 15) / 16 * 16;
    a.b_span = ((unsigned long long)((rb - 1) * a.ldb + lb * ES) + 15) / 16 * 16;
    a.tiles_i = (int)(((long long)p.I + tile_i - 1) / tile_i);
    a.tiles_j = (int)(((long long)p.J + tile_j - 1) / tile_j);
    a.f = p.f;
    a.parts = p.splits > 1 ? p.parts : nullptr;
    return a;
}

int add_parts(const Product& p, hipStream_t st) {
    if (p.splits <= 1) return PCONV_OK;
    const unsigned long long threads = (unsigned long long)p.I * ((p.J + 7) / 8);
    hipLaunchKernelGGL(add_parts_kernel, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, st, p.parts, p.splits, p.I, p.J, p.f);
    PCONV_HIP(hipGetLastError());
    return PCONV_OK;
}

template <bool AR, bool BR, int WI, int WJ, int AF, int BF>
int launch_tile(const Product& p, bool direct, hipStream_t st) {
    constexpr int TI = 32 * AF * WI, TJ = 32 * BF * WJ;
    const Args a = make_args(p, TI, TJ);
    const size_t lds = 2 * (size_t)(TI + TJ) * kStageBytes;
    const unsigned long long grid = (unsigned long long)a.tiles_i * a.tiles_j * p.splits;
    if (grid > 0x7FFFFFFFull) return PCONV_EUNSUPPORTED;
#define PCONV_PRODUCT(DIRECT)                                                                                           \
    {                                                                                                                   \
        auto kern = product_kernel<AR, BR, WI, WJ, AF, BF, DIRECT>;                                                     \
        static LdsAllowance allowed;                                                                                    \
        if (lds > 64 * 1024) PCONV_HIP(allowed.ask((const void*)kern));                                                 \
        hipLaunchKernelGGL(kern, dim3((unsigned)grid), dim3(WI * WJ * 64), lds, st, a);                                 \
    }
    if (direct) PCONV_PRODUCT(true) else PCONV_PRODUCT(false)
#undef PCONV_PRODUCT
    PCONV_HIP(hipGetLastError());
    return add_parts(p, st);
}

template <bool AR, bool BR>
int launch_form(const Product& p, hipStream_t st) {
    // straight to LDS: pieces of 16 bytes are aligned, and (c-minor) none of them is cut by the end of c
    auto fits = [&](const void* m, long long ld, bool rows) {
        return aligned_to(m, 16) && ld * ES % 16 == 0 && (rows || (long long)p.C * ES % 16 == 0);
    };
    const bool direct = fits(p.a, p.lda, AR) && fits(p.b, p.ldb, BR);
    switch (p.tile) {
        case 0: return launch_tile<AR, BR, 2, 4, 4, 2>(p, direct, st);
        case 1: return launch_tile<AR, BR, 2, 2, 2, 2>(p, direct, st);
        default: return launch_tile<AR, BR, 2, 2, 1, 1>(p, direct, st);
    }
}

int launch_product(const Product& p, void* stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    if (!p.a_rows && !p.b_rows) return launch_form<false, false>(p, st);
    if (!p.a_rows) return launch_form<false, true>(p, st);
    return launch_form<true, true>(p, st);
}

int launch_few_rows(const Product& p, void* stream) {
    hipStream_t st = static_cast<hipStream_t>(stream);
    const Args a = make_args(p, kFewRows, 16);
    const unsigned long long grid = (unsigned long long)a.tiles_j * p.splits;
    if (grid > 0x7FFFFFFFull) return PCONV_EUNSUPPORTED;
    hipLaunchKernelGGL(few_rows_kernel, dim3((unsigned)grid), dim3(kFewWaves * 64), 0, st, a);
    PCONV_HIP(hipGetLastError());
    return add_parts(p, st);
}

}  // namespace
}  // namespace pconv
