// Matrix products with an epilogue on the matrix cores, for one storage type (PCONV_LINEAR_DT) per translation unit.
//
// R[i][j] = sum over c of A(i, c) * B(j, c), each operand stored with c along its rows ("c-minor": x and w of the forward
// pass, dz of the input gradient) or across them ("rows": w of the input gradient, both operands of the weight gradient).
//
// A workgroup of four waves owns a tile of TI x TJ results (256, 128 or 64 each way; a wave half of it each way) and walks over c in
// stages of 128 bytes of a row (64 elements, 32 for fp32), three stages of A and two of B in LDS:
//   c-minor operand: [row][8 pieces of 16 bytes]; piece p of a row lies at place p ^ swizzle(row), so that the 16 rows an
//       operand read touches at one piece spread over the banks;
//   rows operand:    [c][pieces of 16 bytes]; piece p lies at p ^ swizzle(c) likewise, and is read with
//       ds_read_b64_tr_b16: four c of 16 rows a group of 16 lanes, handed over transposed (fp32: single words).
// (No bank conflict is counted for any of the three forms.)
// Where rows are aligned to 16 bytes the pieces go from memory to LDS without registers (buffer_load ... lds: a wave's 64
// pieces land side by side, so the swizzle is applied to what each lane asks for); otherwise through registers.
// Pieces outside the matrix are outside the buffer descriptor and read as zeros.
//
// The matrix instructions get B as their rows and A as their columns: a lane of the result then holds four consecutive j of one i.
// They leave through a window of LDS that belongs to the wave, 16 i at a time, so that 16 lanes store 256 bytes of a row (of the
// largest tile; through no window they would be pieces of 8 bytes).
//
// What bounds it.  Large products: the chip's power.  With fewer stalls a stage (2,570 clocks of which 2,048 are MFMAs on the largest tile)
// the clock falls and the time stays: 1.4 to 2 GHz under these loops.  8192 x 4096 -> 16384, bf16, medians of calls in a row: 787 us,
// 1.40 PFLOP/s, with z kept and GELU 838; the library's plain product there 709.  Gradients of 8192 x 4096 -> 4096: input 208 us
// (1.32 PFLOP/s), with GELU's slope 226, weights 203.  (The means of a kernel trace are 5 to 12 % longer.)  Per tile of 256 x 256 the results
// take 13,000 clocks, during which nothing is multiplied: a wave has its SIMD's registers to itself.
// Small products: a launch, the latency of two stages, and the results' way out (512^3: 5.4 us).
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

// A barrier that waits for the wave's accesses to LDS but not for those to memory, as __syncthreads() would
__device__ __forceinline__ void meet() {
    asm volatile("" : : : "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);        // lgkmcnt(0)
    __builtin_amdgcn_s_barrier();
    asm volatile("" : : : "memory");
}

struct Args {
    const unsigned char* a;
    const unsigned char* b;
    long long lda, ldb;                       // bytes
    unsigned long long a_span, b_span;        // bytes from the first element to behind the last
    int I, J, C, c_per, tiles_i, tiles_j;
    unsigned work;                            // tiles x splits
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
    template <bool ADD, bool ZIN>
    __device__ __forceinline__ void load_whole(const Finish& f, long long i, int j) {
        if constexpr (ADD) add.load_whole(static_cast<const T*>(f.add) + i * f.ld_add + j);
        if constexpr (ZIN) zin.load_whole(static_cast<const T*>(f.zin) + i * f.ld_zin + j);
    }
};

// Results v[r][0..7] at (i + r * between, j..j+7), n of them inside the matrix.  ADD, ZIN: there may be such an operand
template <bool ADD, bool ZIN, int R>
__device__ __forceinline__ void finish_rows(const Finish& f, float v[R][8], const float bias[8], const Beside beside[R], long long i,
                                            int between, int j, int n) {
    if (f.kind == kFloat) {
#pragma unroll
        for (int r = 0; r < R; ++r) store8<PCONV_F32>(static_cast<float*>(f.out) + (i + r * between) * f.ld_out + j, n, v[r]);
        return;
    }
    auto plus = [&] {
#pragma unroll
        for (int r = 0; r < R; ++r) {
            float add[8];
            beside[r].add.get(add);
#pragma unroll
            for (int q = 0; q < 8; ++q) v[r][q] += add[q];
        }
    };
    if (f.kind == kForward) {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int q = 0; q < 8; ++q) v[r][q] += bias[q];
        if (ADD && f.add && f.first) plus();
        if (f.z)
#pragma unroll
            for (int r = 0; r < R; ++r) store8<DT>(static_cast<T*>(f.z) + (i + r * between) * f.ld_out + j, n, v[r]);
        activate8<DT, R>(v, f.act);
        if (ADD && f.add && !f.first) plus();
    } else {
        if (ZIN && f.zin) {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                float z[1][8];
                beside[r].zin.get(z[0]);
                times_slope8<DT, 1>(v + r, z, f.act);
            }
        }
        if (ADD && f.add) plus();
    }
#pragma unroll
    for (int r = 0; r < R; ++r) store8<DT>(static_cast<T*>(f.out) + (i + r * between) * f.ld_out + j, n, v[r]);
}
__device__ __forceinline__ void finish8(const Finish& f, float v[1][8], const float bias[8], long long i, int j, int n) {
    Beside beside[1];
    beside[0].load(f, i, j, n);
    finish_rows<true, true, 1>(f, v, bias, beside, i, 0, j, n);
}
__device__ __forceinline__ void bias8(const Finish& f, int j, int n, float bias[8]) {
#pragma unroll
    for (int q = 0; q < 8; ++q) bias[q] = f.kind == kForward && f.bias && q < n ? f.bias[j + q] : 0.f;
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
__global__ __launch_bounds__(WI * WJ * 64, AF * BF == 64 ? 1 : 2) void product_kernel(const Args p) {
    constexpr int THREADS = WI * WJ * 64, TI = 16 * AF * WI, TJ = 16 * BF * WJ;
    typedef Operand<AR, TI, THREADS> OA;
    typedef Operand<BR, TJ, THREADS> OB;
    // LDS: three stages of A, two of B; a wave's window for the results lies in the stage of A that is not in use then
    constexpr int B_AT = 3 * OA::kBytes;
    extern __shared__ __align__(16) unsigned char lds[];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int wi = wave % WI, wj = wave / WI;

    // The workgroups of an XCD (every eighth) take turns along a range of the work of their own.  A piece of work: a split of c and a
    // tile, tiles in groups of eight tile rows, column by column inside a group, so that those under way at a time share operands.
    const unsigned tiles = (unsigned)p.tiles_i * p.tiles_j, xcd = blockIdx.x % 8, turn = gridDim.x / 8;
    const unsigned first = (unsigned)((unsigned long long)p.work * xcd / 8) + blockIdx.x / 8;
    const unsigned end = (unsigned)((unsigned long long)p.work * (xcd + 1) / 8);
    if (first >= end) return;
    // Where a piece of work's operands begin, the bytes from there to the matrices' ends, and how much of c is left; none: zeros
    struct Work {
        int i0, j0, split, stages;
        const unsigned char *pa, *pb;
        unsigned long long a_left, b_left;
        int c_left;
    };
    const unsigned long long a_step = AR ? (unsigned long long)p.lda * BK : kStageBytes;
    const unsigned long long b_step = BR ? (unsigned long long)p.ldb * BK : kStageBytes;
    auto work_at = [&](unsigned id) {
        Work w{};
        if (id >= end) return w;
        const unsigned split = id / tiles, tile = id % tiles;
        const unsigned per_group = 8u * p.tiles_j, group = tile / per_group, in = tile % per_group;
        const unsigned high = min(8u, (unsigned)p.tiles_i - group * 8);
        const int c0 = (int)split * p.c_per;
        w.i0 = (int)(group * 8 + in % high) * TI;
        w.j0 = (int)(in / high) * TJ;
        w.split = (int)split;
        w.c_left = min(p.C, c0 + p.c_per) - c0;
        w.stages = max(2, (w.c_left + BK - 1) / BK);           // (two at least, the second of zeros where there is one: see main_loop)
        const unsigned long long a_at = AR ? (unsigned long long)c0 * p.lda + (unsigned long long)w.i0 * ES
                                           : (unsigned long long)w.i0 * p.lda + (unsigned long long)c0 * ES;
        const unsigned long long b_at = BR ? (unsigned long long)c0 * p.ldb + (unsigned long long)w.j0 * ES
                                           : (unsigned long long)w.j0 * p.ldb + (unsigned long long)c0 * ES;
        w.pa = p.a + a_at;
        w.pb = p.b + b_at;
        w.a_left = p.a_span - a_at;
        w.b_left = p.b_span - b_at;
        return w;
    };
    Work now = work_at(first);
    // the operands' next stage
    const unsigned char *pa = now.pa, *pb = now.pb;
    unsigned long long a_left = now.a_left, b_left = now.b_left;
    int c_left = now.c_left;
    float4v acc[AF][BF];

    // DIRECT: the stage that is being asked for, a piece at a time
    __amdgpu_buffer_rsrc_t rsrc_a, rsrc_b;
    unsigned off_a[OA::kVariants], off_b[OB::kVariants];
    auto begin_stage = [&] {
        auto offsets = [&](auto tag, long long ld, unsigned* off) {
            typedef decltype(tag) O;
#pragma unroll
            for (int v = 0; v < O::kVariants; ++v) {
                int line, piece;
                O::where(t, v, &line, &piece);
                off[v] = !O::kRows && piece * PER >= c_left ? kInvalid : (unsigned)(line * ld) + piece * 16;
            }
        };
        // (where nothing is left: zeros)
        rsrc_a = make_rsrc(pa, c_left > 0 ? (uint32_t)min(a_left, 0x7FFFFFFFull) : 0);
        rsrc_b = make_rsrc(pb, c_left > 0 ? (uint32_t)min(b_left, 0x7FFFFFFFull) : 0);
        offsets(OA{}, p.lda, off_a);
        offsets(OB{}, p.ldb, off_b);
        pa += a_step;
        pb += b_step;
        a_left -= a_step;
        b_left -= b_step;
        c_left -= BK;
    };
    // piece q of an operand's stage, into the LDS at `to`
    auto ask_a = [&](lds_bytes to, int q) {
        const int v = q % OA::kVariants;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_a, (lds_ptr)(to + wave * 1024 + q * THREADS * 16), 16,
                                                 (int)(off_a[v] + (unsigned)((q - v) * OA::kLinesPer * p.lda)), 0, 0, 0);
    };
    auto ask_b = [&](lds_bytes to, int q) {
        const int v = q % OB::kVariants;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc_b, (lds_ptr)(to + wave * 1024 + q * THREADS * 16), 16,
                                                 (int)(off_b[v] + (unsigned)((q - v) * OB::kLinesPer * p.ldb)), 0, 0, 0);
    };
    // through registers: a stage's pieces
    constexpr int AHEAD = DIRECT ? 1 : OA::kPieces + OB::kPieces <= 4 ? 4 : 2;
    uint4v ra[AHEAD][DIRECT ? 1 : OA::kPieces], rb[AHEAD][DIRECT ? 1 : OB::kPieces];
    auto fetch = [&](auto tag, const unsigned char* at, unsigned long long left, long long ld, int rows, uint4v* regs) {
        typedef decltype(tag) O;
#pragma unroll
        for (int q = 0; q < O::kPieces; ++q) {
            int line, piece;
            O::where(t, q, &line, &piece);
            const int lines = O::kRows ? c_left : rows;
            int along = (O::kRows ? rows : c_left) - piece * PER;
            regs[q] = uint4v{0, 0, 0, 0};
            // (what stands behind the end of a line of i or j gives results that nobody stores: read whole, up to the matrix's end)
            if (O::kRows && along > 0 && (unsigned long long)(line * ld) + piece * 16 + 16 <= left) along = PER;
            if (line < lines && along > 0) regs[q] = load_part<DT>(reinterpret_cast<const T*>(at + line * ld) + piece * PER, along);
        }
    };
    auto fetch_stage = [&](int slot) {
        fetch(OA{}, pa, a_left, p.lda, p.I - now.i0, ra[slot]);
        fetch(OB{}, pb, b_left, p.ldb, p.J - now.j0, rb[slot]);
        a_left -= a_step;
        b_left -= b_step;
        pa += a_step;
        pb += b_step;
        c_left -= BK;
    };
    auto put_stage = [&](int slot, int buf) {
        if constexpr (!DIRECT) {
#pragma unroll
            for (int q = 0; q < OA::kPieces; ++q) *reinterpret_cast<uint4v*>(lds + buf * OA::kBytes + (q * THREADS + t) * 16) = ra[slot][q];
#pragma unroll
            for (int q = 0; q < OB::kPieces; ++q) *reinterpret_cast<uint4v*>(lds + B_AT + buf * OB::kBytes + (q * THREADS + t) * 16) = rb[slot][q];
        }
    };

    typedef uint4v FragA[AF];
    typedef uint4v FragB[BF];
    auto read_one = [&](lds_bytes la, lds_bytes lb, int k, int q, FragA& fa, FragB& fb) {
        if (q < BF) fb[q] = OB::read(lb, wj * BF + q, k, lane);
        else fa[q - BF] = OA::read(la, wi * AF + q - BF, k, lane);
    };
    auto clear = [&] {
#pragma unroll
        for (int a = 0; a < AF; ++a)
#pragma unroll
            for (int b = 0; b < BF; ++b) acc[a][b] = float4v{0.f, 0.f, 0.f, 0.f};
    };
    // Results leave through a window of 16 i x 16 BF j floats for each wave; of a row's 16-byte pieces, piece q lies at q ^ row, which
    // spreads the rows over the banks.
    constexpr int PITCH = 16 * BF * 4, ROW_LANES = 2 * BF, ROWS_AT_ONCE = 64 / ROW_LANES, TIMES = 16 / ROWS_AT_ONCE;
    static_assert(16 % ROWS_AT_ONCE == 0 && WI * WJ * 16 * PITCH <= OA::kBytes, "the windows fit a stage of A");
    constexpr int SPREAD = 4 * BF < 16 ? 4 * BF - 1 : 15;
    auto put_block = [&](unsigned char* win, const float4v (&block)[BF]) {
        const int row = lane & 15;
#pragma unroll
        for (int b = 0; b < BF; ++b) {
            float4v v;
            asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v.x) : "a"(block[b].x));
            asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v.y) : "a"(block[b].y));
            asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v.z) : "a"(block[b].z));
            asm volatile("v_accvgpr_read_b32 %0, %1" : "=v"(v.w) : "a"(block[b].w));
            *reinterpret_cast<float4v*>(win + row * PITCH + ((b * 4 + (lane >> 4)) ^ (row & SPREAD)) * 16) = v;
        }
    };
    auto finish = [&](int at) {
        unsigned char* const win = lds + at + wave * 16 * PITCH;
        // (the reads of accumulators in put_block are the assembler's: no wait is put in front of them; the last MFMA, of 8 passes at
        // most, is done 11 wait states behind it)
        asm volatile("s_nop 15\n\ts_nop 15");
        Finish f = p.f;
        if (p.parts) {
            f.kind = kFloat;
            f.out = p.parts + (unsigned long long)now.split * p.I * p.J;
            f.ld_out = p.J;
        }
        const int j = now.j0 + wj * 16 * BF + (lane % ROW_LANES) * 8, n = p.J - j, i_first = now.i0 + wi * AF * 16 + lane / ROW_LANES;
        float bias[8];
        bias8(f, j, n, bias);
        auto put = [&](int a) {
#pragma unroll
            for (int b = 0; b < AF; ++b)
                if (a == b) put_block(win, acc[b]);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };
        auto get = [&](int r, float (&v)[8]) {
            const int row = lane / ROW_LANES + r * ROWS_AT_ONCE, q = (lane % ROW_LANES) * 2;
            const float4v lo = *reinterpret_cast<const float4v*>(win + row * PITCH + (q ^ (row & SPREAD)) * 16);
            const float4v hi = *reinterpret_cast<const float4v*>(win + row * PITCH + ((q + 1) ^ (row & SPREAD)) * 16);
            v[0] = lo.x; v[1] = lo.y; v[2] = lo.z; v[3] = lo.w;
            v[4] = hi.x; v[5] = hi.y; v[6] = hi.z; v[7] = hi.w;
        };
        auto done = [&] {
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
        };
        if (now.i0 + TI <= p.I && now.j0 + TJ <= p.J) {
            // A whole tile, with what it reads besides known to the compiler: loads in a branch, or none, would be waited for in front of
            // every window, and with them the stores of the window before.
            [[maybe_unused]] auto whole = [&](auto kind, auto add, auto zin) {
                f.kind = kind;
                if constexpr (!add) f.add = nullptr;
                if constexpr (!zin) f.zin = nullptr;
                Beside next[TIMES];
                auto load = [&](int a) {
                    if constexpr (add || zin)
#pragma unroll
                        for (int r = 0; r < TIMES; ++r) next[r].template load_whole<add, zin>(f, i_first + a * 16 + r * ROWS_AT_ONCE, j);
                };
                auto window = [&](int a) {
                    Beside beside[TIMES];
#pragma unroll
                    for (int r = 0; r < TIMES; ++r) beside[r] = next[r];
                    put(a);
                    load(a + 1 < AF ? a + 1 : a);
                    float v[TIMES][8];
#pragma unroll
                    for (int r = 0; r < TIMES; ++r) get(r, v[r]);
                    finish_rows<add, zin, TIMES>(f, v, bias, beside, i_first + a * 16, ROWS_AT_ONCE, j, 8);
                    done();
                };
                load(0);
                // (the first one by itself: in front of the loop the same stores stand behind the loads as at its end, and a window's
                // wait for its loads is none for the stores of the window before)
                constexpr int PEELED = add || zin ? 1 : 0;
                if constexpr (PEELED) window(0);
#pragma unroll 1
                for (int a = PEELED; a < AF; ++a) window(a);
            };
            [[maybe_unused]] constexpr std::true_type yes{};
            [[maybe_unused]] constexpr std::false_type no{};
            if (f.kind == kFloat) {
                // (floats leave as they are, 16 bytes a lane side by side)
                float* const out = static_cast<float*>(f.out) + now.j0 + wj * 16 * BF + (lane % ROW_LANES) * 4;
#pragma unroll 1
                for (int a = 0; a < AF; ++a) {
                    put(a);
                    float4v v[TIMES][2];
#pragma unroll
                    for (int r = 0; r < TIMES; ++r)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const int row = lane / ROW_LANES + r * ROWS_AT_ONCE, q = lane % ROW_LANES + h * ROW_LANES;
                            v[r][h] = *reinterpret_cast<const float4v*>(win + row * PITCH + (q ^ (row & SPREAD)) * 16);
                        }
#pragma unroll
                    for (int r = 0; r < TIMES; ++r)
#pragma unroll
                        for (int h = 0; h < 2; ++h)
                            store16(out + (long long)(i_first + a * 16 + r * ROWS_AT_ONCE) * f.ld_out + h * ROW_LANES * 4,
                                    __builtin_bit_cast(uint4v, v[r][h]));
                    done();
                }
            } else if constexpr (!BR) {
                if (f.add) whole(std::integral_constant<int, kForward>{}, yes, no);
                else whole(std::integral_constant<int, kForward>{}, no, no);
            } else if constexpr (!AR) {
                if (f.add && f.zin) whole(std::integral_constant<int, kGradInput>{}, yes, yes);
                else if (f.add) whole(std::integral_constant<int, kGradInput>{}, yes, no);
                else if (f.zin) whole(std::integral_constant<int, kGradInput>{}, no, yes);
                else whole(std::integral_constant<int, kGradInput>{}, no, no);
            }
            return;
        }
#pragma unroll 1
        for (int a = 0; a < AF; ++a) {
            put(a);
#pragma unroll 1
            for (int r = 0; r < TIMES; ++r) {
                const int i = i_first + a * 16 + r * ROWS_AT_ONCE;
                float v[1][8];
                get(r, v[0]);
                if (i < p.I && n > 0) finish8(f, v, bias, i, j, n);
            }
            done();
        }
    };

    if constexpr (DIRECT) {
        // One sequence of stages over all of the workgroup's work.  A step's operands are read while the step before is multiplied,
        // across stages too: the barrier that publishes stage s + 1 stands in front of stage s's last step, whose operands are in
        // registers by then.  Stage s + 2 is asked for in the course of stage s, a piece at a time between MFMAs (together they stand in
        // the way of every wave's next instructions until the memory pipeline has taken them, and workgroups that run in step ask
        // for more than L2 gives at a time): A in the first step, into a third stage of its own, B in the last one, into stage s's, which
        // all waves have read then.  At the end of a piece of work the next one's first two stages are in LDS.
        static_assert(KS == 2, "");
        constexpr int MFMAS = AF * BF, READS = AF + BF;
        // (two pointers to the stages, said not to alias, or the compiler waits for every piece that is under way in front of each
        // ds_read_b64_tr_b16: what keeps them apart are the waits and barriers below)
        auto main_loop = [&](const lds_bytes __restrict into, const lds_bytes __restrict from) {
            FragA fa[2];
            FragB fb[2];
            // where the stages of A lie, s, s + 1, s + 2, and of B, s, s + 1
            int a0 = 0, a1 = OA::kBytes, a2 = 2 * OA::kBytes, b0 = B_AT, b1 = B_AT + OB::kBytes;
            auto step = [&](auto kk) {
                constexpr int k = kk, ASKS = k ? OB::kPieces : OA::kPieces;
                each<MFMAS>([&](auto mm) {
                    constexpr int m = mm;
                    // (behind the last stage: what is there, and not used)
                    each<READS>([&](auto q) {
                        if constexpr (q * MFMAS / READS == m) read_one(from + (k ? a1 : a0), from + (k ? b1 : b0), k ^ 1, q, fa[k ^ 1], fb[k ^ 1]);
                    });
                    each<ASKS>([&](auto q) {
                        if constexpr ((2 * q + 1) * MFMAS / (2 * ASKS) == m) {
                            if constexpr (k == 0) ask_a(into + a2, q);
                            else ask_b(into + b0, q);
                        }
                    });
                    acc[m / BF][m % BF] = mma(fb[k][m % BF], fa[k][m / BF], acc[m / BF][m % BF]);
                    asm volatile("" : "+a"(acc[m / BF][m % BF]));          // (it stays where it is)
                    __builtin_amdgcn_sched_barrier(0);
                });
            };
            each<2>([&](auto s) {
                begin_stage();
                each<OA::kPieces>([&](auto q) { ask_a(into + s * OA::kBytes, q); });
                each<OB::kPieces>([&](auto q) { ask_b(into + B_AT + s * OB::kBytes, q); });
            });
            constexpr int PIECES = OA::kPieces + OB::kPieces;
            __builtin_amdgcn_s_waitcnt(0x0F70 | (PIECES & 15) | (PIECES >> 4) << 14);      // vmcnt: all but the pieces of stage 1
            meet();
            int known = -1;                                    // the stage behind which this wave's pieces are known to be in LDS
            for (unsigned id = first; id < end; id += turn) {
                const Work then = work_at(id + turn);
                clear();
                // (not kept from the last stage before: the registers are needed in between)
                each<READS>([&](auto q) { read_one(from + a0, from + b0, 0, q, fa[0], fb[0]); });
                // (no branch in this loop: with one the accumulators are copied from block to block)
                for (int s = 0, more = 1; more; ++s) {
                    const bool over = s == now.stages - 2;     // the work's last stage has been asked for: the next one's first two
                    pa = over ? then.pa : pa;
                    pb = over ? then.pb : pb;
                    a_left = over ? then.a_left : a_left;
                    b_left = over ? then.b_left : b_left;
                    c_left = over ? then.c_left : c_left;
                    begin_stage();
                    __builtin_amdgcn_sched_barrier(0);
                    step(std::integral_constant<int, 0>{});
                    // this wave's pieces of stage s + 1 are in LDS: all but those of A that were asked for just now
                    asm volatile("s_cmp_eq_u32 %0, %1\n\ts_cbranch_scc1 .Lthere%=\n\ts_waitcnt vmcnt(%2)\n.Lthere%=:" : : "s"(s), "s"(known), "i"(OA::kPieces) : "scc", "memory");
                    meet();                                    // so are the other waves', and all have read stage s
                    __builtin_amdgcn_sched_barrier(0);
                    step(std::integral_constant<int, 1>{});
                    const int a = a0, b = b0;
                    a0 = a1;
                    a1 = a2;
                    a2 = a;
                    b0 = b1;
                    b1 = b;
                    more = now.stages - 1 - s;
                    asm("" : "+s"(more));                      // (or it peels the last stage off)
                }
                // (vmcnt(0), here: the wait in stage 0 would be one for the results' stores too)
                __builtin_amdgcn_s_waitcnt(0x0F70);
                known = 0;
                finish(a2);
                meet();                                        // the windows are free again
                now = then;
            }
        };
        lds_bytes into = (lds_bytes)lds, from = into;
        asm("" : "+s"(into), "+s"(from));              // (or it knows that they are the same)
        main_loop(into, from);
    } else {
        for (unsigned id = first; id < end; id += turn) {
            now = work_at(id);
            pa = now.pa;
            pb = now.pb;
            a_left = now.a_left;
            b_left = now.b_left;
            c_left = now.c_left;
            clear();
            // (AHEAD stages are under way: a stage is short for a load from memory)
            each<AHEAD>([&](auto d) { fetch_stage(d); });
            put_stage(0, 0);
            for (int s0 = 0; s0 < now.stages; s0 += AHEAD)
                each<AHEAD>([&](auto d) {
                    const int s = s0 + d, buf = s & 1;
                    if (s >= now.stages) return;
                    __syncthreads();               // stage s is in LDS for every wave, and no wave reads the other half any more
                    fetch_stage(d);
                    each<KS>([&](auto k) {
                        FragA fa;
                        FragB fb;
                        each<AF + BF>([&](auto q) {
                            read_one((lds_bytes)(lds + buf * OA::kBytes), (lds_bytes)(lds + B_AT + buf * OB::kBytes), k, q, fa, fb);
                        });
                        each<AF * BF>([&](auto m) {
                            acc[m / BF][m % BF] = mma(fb[m % BF], fa[m / BF], acc[m / BF][m % BF]);
                            asm volatile("" : "+a"(acc[m / BF][m % BF]));
                        });
                    });
                    put_stage((d + 1) % AHEAD, buf ^ 1);
                });
            finish(2 * OA::kBytes);
            __syncthreads();
        }
    }
}

// The parts of a product that several workgroups share, added in their order, and its epilogue: eight results a thread.
// (The workgroups behind those add strips of column sums.)
__global__ __launch_bounds__(256) void add_parts_kernel(const float* parts, int splits, int I, int J, Finish f, unsigned blocks, Strips strips) {
    if (blockIdx.x >= blocks) {
        add_strips(strips.parts, strips.strips, strips.N, strips.out, (int)(blockIdx.x - blocks) * 64);
        return;
    }
    const int per_row = (J + 7) / 8;
    const unsigned long long at = (unsigned long long)blockIdx.x * 256 + threadIdx.x;
    const unsigned long long i = at / per_row;
    if (i >= (unsigned long long)I) return;
    const int j = (int)(at % per_row) * 8, n = J - j;
    float v[1][8] = {}, w[8], bias[8];
#pragma unroll 8
    for (int s = 0; s < splits; ++s) {
        load8<PCONV_F32>(parts + ((unsigned long long)s * I + i) * J + j, n, w);
#pragma unroll
        for (int q = 0; q < 8; ++q) v[0][q] += w[q];
    }
    bias8(f, j, n, bias);
    finish8(f, v, bias, (long long)i, j, n);
}

// Few rows of x (up to 16) with weights that are read once, straight into registers: memory bounds it, no operand is shared.  A
// workgroup owns 16 rows of w; its waves take turns along k (a wave's 64 lanes: 16 rows x 4 pieces), and their sums meet in LDS
// in the order of the waves.  Rows of the matrix instructions' results are rows of w, their columns rows of x: for one row fifteen
// sixteenths of them are idle, and still far ahead of memory.  25088 -> 4096, fp16, one row: 38.5 us, 5.3 TB/s, what a copy reaches.
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
            float v[1][8] = {}, bias[8];
            for (int s = 0; s < kFewWaves; ++s)
#pragma unroll
                for (int q = 0; q < 8; ++q) v[0][q] += sums[s][i][(t & 1) * 8 + q];
            Finish f = p.f;
            if (p.parts) {
                f.kind = kFloat;
                f.out = p.parts + (unsigned long long)split * p.I * p.J;
                f.ld_out = p.J;
            }
            bias8(f, j, n, bias);
            finish8(f, v, bias, i, j, n);
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
    // (of a matrix that begins at a multiple of 16 bytes, up to the end of the last element's 16, which lie in its page: a piece that
    // begins inside is read whole)
    auto span = [](const void* m, long long rows, long long ld, long long cols) {
        const unsigned long long n = (unsigned long long)((rows - 1) * ld + cols * ES);
        return aligned_to(m, 16) ? (n + 15) / 16 * 16 : n;
    };
    a.a_span = span(p.a, ra, a.lda, la);
    a.b_span = span(p.b, rb, a.ldb, lb);
    a.tiles_i = (int)(((long long)p.I + tile_i - 1) / tile_i);
    a.tiles_j = (int)(((long long)p.J + tile_j - 1) / tile_j);
    a.f = p.f;
    a.parts = p.splits > 1 ? p.parts : nullptr;
    return a;
}

int add_parts(const Product& p, hipStream_t st) {
    if (p.splits <= 1) return PCONV_OK;
    const unsigned long long threads = (unsigned long long)p.I * ((p.J + 7) / 8);
    const unsigned blocks = (unsigned)((threads + 255) / 256), more = p.strips.parts ? (unsigned)(p.strips.N + 63) / 64 : 0;
    hipLaunchKernelGGL(add_parts_kernel, dim3(blocks + more), dim3(256), 0, st, p.parts, p.splits, p.I, p.J, p.f, blocks, p.strips);
    PCONV_HIP(hipGetLastError());
    return PCONV_OK;
}

template <bool AR, bool BR, bool DIRECT, int WI, int WJ, int AF, int BF>
int launch_tile(const Product& p, hipStream_t st) {
    constexpr int TI = 16 * AF * WI, TJ = 16 * BF * WJ;
    Args a = make_args(p, TI, TJ);
    constexpr size_t lds = (3 * TI + 2 * TJ) * (size_t)kStageBytes;
    const unsigned long long work = (unsigned long long)a.tiles_i * a.tiles_j * p.splits;
    if (work > 0x7FFFFFFFull) return PCONV_EUNSUPPORTED;
    a.work = (unsigned)work;
    // as many workgroups as are resident, the same number on each XCD
    const unsigned grid = (unsigned)std::min<unsigned long long>((work + 7) / 8 * 8, kComputeUnits * (160 * 1024 / lds));
    auto kern = product_kernel<AR, BR, WI, WJ, AF, BF, DIRECT>;
    static LdsAllowance allowed;
    if (lds > 64 * 1024) PCONV_HIP(allowed.ask((const void*)kern));
    hipLaunchKernelGGL(kern, dim3(grid), dim3(WI * WJ * 64), lds, st, a);
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
    // (fp32: the matrix cores' rate is so low that the smallest tile feeds them, 2048^3: 131 us against 134 and 532 of the larger ones)
    if constexpr (ES == 4)
        return direct ? launch_tile<AR, BR, true, 2, 2, 2, 2>(p, st) : launch_tile<AR, BR, false, 2, 2, 2, 2>(p, st);
    else {
        // (through registers the largest tile has none left to look ahead)
        if (!direct) return p.tile < 2 ? launch_tile<AR, BR, false, 2, 2, 4, 4>(p, st) : launch_tile<AR, BR, false, 2, 2, 2, 2>(p, st);
        switch (p.tile) {
            case 0: return launch_tile<AR, BR, true, 2, 2, 8, 8>(p, st);
            case 1: return launch_tile<AR, BR, true, 2, 2, 4, 4>(p, st);
            default: return launch_tile<AR, BR, true, 2, 2, 2, 2>(p, st);
        }
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
