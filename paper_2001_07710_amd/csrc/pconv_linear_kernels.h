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
#include <type_traits>
#include <utility>

#include "pconv_dense_util.h"
#include "pconv_linear.h"

namespace pconv {
namespace {

typedef __attribute__((address_space(3))) void* lds_ptr;
typedef __attribute__((address_space(3))) unsigned char* lds_bytes;
typedef __attribute__((address_space(3))) short4v* lds_short4;
typedef const __attribute__((address_space(3))) uint4v* lds_uint4;
typedef const __attribute__((address_space(3))) float* lds_float;

constexpr int DT = PCONV_LINEAR_DT;
typedef Store<DT>::T T;
constexpr int ES = (int)sizeof(T);
constexpr int PER = 16 / ES;                 // elements of a piece
constexpr int BK = kStageBytes / ES;         // elements of c in a stage
constexpr int KS = kStageBytes / 64;         // steps of a stage: four pieces of c each

// acc += rows x columns over four pieces of c: lanes 16 g .. 16 g + 15 hold piece g of row / column lane % 16.  (16 x 16 x 32 and not
// 32 x 32 x 16: the same rate by the clock, but half the traffic of accumulators, and the chip's power is what bounds large products:
// 2195 against 2010 TFLOP/s on random operands in registers, bf16.)
__device__ __forceinline__ float4v mma(uint4v a, uint4v b, float4v acc) {
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

// f(0), f(1), .. f(N - 1) with constants (the unroller gives up on bodies of this size)
template <typename F, int... I>
__device__ __forceinline__ void each_of(std::integer_sequence<int, I...>, F f) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F f) {
    each_of(std::make_integer_sequence<int, N>{}, f);
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
        else if constexpr (ES == 4) return ((line >> 2) & 3) * 4;              // lines 4 g + q: to different 64 bytes of 256
        // lines 8 g + 4 q + 0..3, 32 bytes of each: to different 32 bytes of 256 for two g (lines of 128 bytes lie so by halves)
        else return kLinePieces >= 16 ? ((line & 3) | ((line >> 1) & 4)) * 2 : (((line >> 1) & 1) | ((line >> 2) & 2)) * 2;
    }
    static constexpr int kReads = ROWS ? ES == 2 ? 2 : 4 : 1;             // LDS reads of one operand
    static constexpr int kPeriod = 16;                                    // of the swizzle, in lines
    static constexpr int kVariants = kLinesPer % kPeriod == 0 ? 1 : kPeriod / kLinesPer;     // of a thread's piece, by q
    static_assert(kLinesPer % kPeriod == 0 || kPeriod % kLinesPer == 0, "");

    // line and piece of the matrix that thread t's piece q holds
    static __device__ __forceinline__ void where(int t, int q, int* line, int* piece) {
        *line = t / kLinePieces + q * kLinesPer;
        *piece = (t % kLinePieces) ^ swizzle(*line);
    }
    // operand registers of 16-row block `blk` at step s
    static __device__ __forceinline__ uint4v read(lds_bytes lds, int blk, int s, int lane) {
        const int r = lane & 15, g = lane >> 4;
        if constexpr (!ROWS) {
            const int row = blk * 16 + r;
            return *(lds_uint4)(lds + row * kStageBytes + (((4 * s + g) ^ swizzle(row)) * 16));
        } else if constexpr (ES == 2) {
            uint4v v;
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                const int c = 32 * s + 8 * g + 4 * q + (r >> 2), at = (blk * 16 + 4 * (r & 3)) * 2;
                const lds_bytes p = lds + c * kLineBytes + (((at >> 4) ^ swizzle(c)) << 4) + (at & 15);
                const uint2v d = __builtin_bit_cast(uint2v, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_short4)p));
                if (q) { v.z = d.x; v.w = d.y; } else { v.x = d.x; v.y = d.y; }
            }
            return v;
        } else {
            float4v v;
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int c = 16 * s + 4 * g + q, at = (blk * 16 + r) * 4;
                v[q] = *(lds_float)(lds + c * kLineBytes + (((at >> 4) ^ swizzle(c)) << 4) + (at & 15));
            }
            return __builtin_bit_cast(uint4v, v);
        }
    }
};

template <bool AR, bool BR, int WI, int WJ, int AF, int BF, bool DIRECT>
__global__ __launch_bounds__(WI * WJ * 64) void product_kernel(const Args p) {
    constexpr int THREADS = WI * WJ * 64, TI = 16 * AF * WI, TJ = 16 * BF * WJ;
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

    float4v acc[AF][BF];
#pragma unroll
    for (int a = 0; a < AF; ++a)
#pragma unroll
        for (int b = 0; b < BF; ++b) acc[a][b] = float4v{0.f, 0.f, 0.f, 0.f};

    // DIRECT: the stage that is being asked for, a piece at a time
    constexpr int PIECES = OA::kPieces + OB::kPieces;
    __amdgpu_buffer_rsrc_t rsrc_a, rsrc_b;
    unsigned off_a[OA::kVariants], off_b[OB::kVariants];
    int to_stage = 0;
    auto begin_stage = [&](int buf) {
        auto offsets = [&](auto tag, long long ld, unsigned* off) {
            typedef decltype(tag) O;
#pragma unroll
            for (int v = 0; v < O::kVariants; ++v) {
                int line, piece;
                O::where(t, v, &line, &piece);
                off[v] = !O::kRows && piece * PER >= c_left ? kInvalid : (unsigned)(line * ld) + piece * 16;
            }
        };
        // (behind the last stage nothing is there: zeros, which nobody reads)
        rsrc_a = make_rsrc(pa, c_left > 0 ? (uint32_t)min(a_left, 0x7FFFFFFFull) : 0);
        rsrc_b = make_rsrc(pb, c_left > 0 ? (uint32_t)min(b_left, 0x7FFFFFFFull) : 0);
        offsets(OA{}, p.lda, off_a);
        offsets(OB{}, p.ldb, off_b);
        to_stage = buf * STAGE + wave * 1024;
        pa += a_step;
        pb += b_step;
        a_left -= a_step;
        b_left -= b_step;
        c_left -= BK;
    };
    auto ask_piece = [&](lds_bytes into, int q) {
        if (q < OA::kPieces) {
            const int v = q % OA::kVariants;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_a, (lds_ptr)(into + to_stage + q * THREADS * 16), 16,
                                                     (int)(off_a[v] + (unsigned)((q - v) * OA::kLinesPer * p.lda)), 0, 0, 0);
        } else {
            const int o = q - OA::kPieces, v = o % OB::kVariants;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_b, (lds_ptr)(into + to_stage + OA::kBytes + o * THREADS * 16), 16,
                                                     (int)(off_b[v] + (unsigned)((o - v) * OB::kLinesPer * p.ldb)), 0, 0, 0);
        }
    };
    // through registers: a stage's pieces
    uint4v ra[DIRECT ? 1 : OA::kPieces], rb[DIRECT ? 1 : OB::kPieces];
    auto fetch = [&](auto tag, const unsigned char* at, long long ld, int rows, uint4v* regs) {
        typedef decltype(tag) O;
#pragma unroll
        for (int q = 0; q < O::kPieces; ++q) {
            int line, piece;
            O::where(t, q, &line, &piece);
            const int lines = O::kRows ? c_left : rows, along = (O::kRows ? rows : c_left) - piece * PER;
            regs[q] = uint4v{0, 0, 0, 0};
            if (line < lines && along > 0) regs[q] = load_part<DT>(reinterpret_cast<const T*>(at + line * ld) + piece * PER, along);
        }
    };
    auto fetch_stage = [&] {
        fetch(OA{}, pa, p.lda, p.I - i0, ra);
        fetch(OB{}, pb, p.ldb, p.J - j0, rb);
        pa += a_step;
        pb += b_step;
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

    typedef uint4v FragA[AF];
    typedef uint4v FragB[BF];
    auto read_one = [&](lds_bytes from, int buf, int k, int q, FragA& fa, FragB& fb) {
        const lds_bytes la = from + buf * STAGE, lb = la + OA::kBytes;
        if (q < BF) fb[q] = OB::read(lb, wj * BF + q, k, lane);
        else fa[q - BF] = OA::read(la, wi * AF + q - BF, k, lane);
    };
    if constexpr (DIRECT) {
        // A step's operands are read while the step before is multiplied, across stages too: the barrier that publishes stage
        // s + 1 stands in front of stage s's last step, whose operands are in registers by then, so that stage s + 2 can be asked
        // for into the same half: a piece at a time between the MFMAs of that step (asked for together they stand in the way of
        // every wave's next instructions until the memory pipeline has taken them).
        static_assert(KS == 2, "");
        constexpr int MFMAS = AF * BF, READS = AF + BF;
        // (two pointers to the stages, said not to alias, or the compiler waits for every piece that is under way in front of each
        // ds_read_b64_tr_b16: what keeps them apart are the waits and barriers below)
        auto main_loop = [&](const lds_bytes __restrict into, const lds_bytes __restrict from) {
            FragA fa[2];
            FragB fb[2];
            auto step = [&](auto kk, int buf) {
                constexpr int k = kk;
                each<MFMAS>([&](auto mm) {
                    constexpr int m = mm;
                    // (behind the last stage: what is there, and not used)
                    each<READS>([&](auto q) {
                        if constexpr (q * MFMAS / READS == m) read_one(from, k == 0 ? buf : buf ^ 1, k ^ 1, q, fa[k ^ 1], fb[k ^ 1]);
                    });
                    if constexpr (k == 1)
                        each<PIECES>([&](auto q) {
                            if constexpr (q * MFMAS / PIECES == m) ask_piece(into, q);
                        });
                    acc[m / BF][m % BF] = mma(fb[k][m % BF], fa[k][m / BF], acc[m / BF][m % BF]);
                    __builtin_amdgcn_sched_barrier(0);
                });
            };
            each<2>([&](auto s) {
                begin_stage(s);
                each<PIECES>([&](auto q) { ask_piece(into, q); });
            });
            __builtin_amdgcn_s_waitcnt(0x0F70 | (PIECES & 15) | (PIECES >> 4) << 14);      // vmcnt: all but the pieces of stage 1
            __syncthreads();
            each<READS>([&](auto q) { read_one(from, 0, 0, q, fa[0], fb[0]); });
            for (int s = 0; s < stages; ++s) {
                step(std::integral_constant<int, 0>{}, s & 1);
                __builtin_amdgcn_s_waitcnt(0x0F70);        // vmcnt(0): this wave's pieces of stage s + 1 are in LDS
                __syncthreads();                           // so are the other waves', and all have read stage s
                begin_stage(s & 1);
                __builtin_amdgcn_sched_barrier(0);
                step(std::integral_constant<int, 1>{}, s & 1);
            }
        };
        lds_bytes into = (lds_bytes)lds, from = into;
        asm("" : "+s"(into), "+s"(from));              // (or it knows that they are the same)
        main_loop(into, from);
        __builtin_amdgcn_s_waitcnt(0x0F70);
    } else {
        fetch_stage();
        put_stage(0);
        for (int s = 0; s < stages; ++s) {
            const int buf = s & 1;
            __syncthreads();                   // stage s is in LDS for every wave, and no wave reads the other half any more
            if (s + 1 < stages) fetch_stage();
#pragma unroll
            for (int k = 0; k < KS; ++k) {
                FragA fa;
                FragB fb;
#pragma unroll
                for (int q = 0; q < AF + BF; ++q) read_one((lds_bytes)lds, buf, k, q, fa, fb);
#pragma unroll
                for (int m = 0; m < AF * BF; ++m) acc[m / BF][m % BF] = mma(fb[m % BF], fa[m / BF], acc[m / BF][m % BF]);
            }
            if (s + 1 < stages) put_stage(buf ^ 1);
        }
    }
    __syncthreads();

    // results: a window of 16 i x 16 BF j floats for each wave, a pitch that spreads the rows over the banks
    constexpr int PITCH = (16 * BF + 4) * 4, ROW_LANES = 2 * BF, ROWS_AT_ONCE = 64 / ROW_LANES;
    static_assert(WI * WJ * 16 * PITCH <= 2 * STAGE && 16 % ROWS_AT_ONCE == 0, "the windows fit the stages");
    unsigned char* const win = lds + wave * 16 * PITCH;
    Finish f = p.f;
    if (p.parts) {
        f.kind = kFloat;
        f.out = p.parts + (unsigned long long)split * p.I * p.J;
        f.ld_out = p.J;
    }
    const int j = j0 + wj * 16 * BF + (lane % ROW_LANES) * 8, n = p.J - j;
    float bias[8];
    bias8(f, j, n, bias);
    auto put_block = [&](const float4v (&block)[BF]) {
#pragma unroll
        for (int b = 0; b < BF; ++b)
            *reinterpret_cast<float4v*>(win + (lane & 15) * PITCH + (b * 16 + (lane >> 4) * 4) * 4) = block[b];
    };
    constexpr int TIMES = 16 / ROWS_AT_ONCE;
#pragma unroll 1
    for (int a = 0; a < AF; ++a) {
        const int i = i0 + (wi * AF + a) * 16 + lane / ROW_LANES;
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
        for (int u = 0; u < U; ++u) acc = mma(w[u], x[u], acc);
    }
    if (c < c1) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const int at = c + u * STEP + piece * PER;
            const uint4v w = load_part<DT>(pw + at, c1 - at);
            uint4v x = {0, 0, 0, 0};
            if (has_x) x = load_part<DT>(px + at, c1 - at);
            acc = mma(w, x, acc);
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
    constexpr int TI = 16 * AF * WI, TJ = 16 * BF * WJ;
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
        case 0: return launch_tile<AR, BR, 2, 2, 8, 8>(p, direct, st);
        case 1: return launch_tile<AR, BR, 2, 2, 4, 4>(p, direct, st);
        default: return launch_tile<AR, BR, 2, 2, 2, 2>(p, direct, st);
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
