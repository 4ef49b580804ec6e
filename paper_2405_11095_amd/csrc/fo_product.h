// Products of two matrices whose rows run along the summed axis, out[q][p] = sum_k Q[q][k] P[p][k], on the matrix cores.
//
// One engine serves 8-bit codes (exact 32-bit integer sums) and 16-bit floats (fp32 sums): both matrix instructions, 16x16x64 in
// i8 and 16x16x32 in f16, take 16 bytes of a row from every lane and issue in the same time, so that a tile's bytes travel the
// same way.
//
// A workgroup forms a tile of outputs, each of its waves a part of it in registers.  The summed axis is taken
// 128 bytes of every row at a time (a "stage"), loaded straight into LDS, DEPTH stages there at once.  A stage is two half steps of
// 64 bytes.  While a half step's matrix instructions run on one set of registers, the next half step's fragments are read into
// the other; the one barrier of a stage stands in front of its second half step, whose fragments are in registers by then:
// behind it the stage's buffer is free for the loads of the stage DEPTH further on, and the next stage has arrived.
//
// EXACT: operands in two parts of fp16 each.  The matrix cores round a sum after every eight products; with every run of stages it goes
// into a second one and starts again at zero (kRun).
//
// P may come turned, its summed axis running down the columns (16-bit floats only): a stage of it is 64 rows of a tile's columns,
// and its fragments are read through the LDS's transposing load, which hands lane c of 16 column c of 4 rows by 16 columns.
#pragma once
#include "fo_device.h"

namespace fo {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));

constexpr uint32_t kStageBytes = 128;  // of a row, a stage
constexpr uint32_t kMatrices = 64;     // matrices of one call

struct OpI8 {
    typedef i32x4 Acc;
    static __device__ __forceinline__ Acc mfma(i32x4 p, i32x4 q, Acc c) { return __builtin_amdgcn_mfma_i32_16x16x64_i8(p, q, c, 0, 0, 0); }
};
struct OpF16 {
    typedef f32x4 Acc;
    static __device__ __forceinline__ Acc mfma(i32x4 p, i32x4 q, Acc c)
    {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, p), __builtin_bit_cast(f16x8, q), c, 0, 0, 0);
    }
};

struct ProductArgs {
    const char *q, *p;        // rows of ld bytes (a multiple of 128), 16-byte aligned; P turned: 64 stages rows, rows_p a multiple of 64
    uint64_t ld_q, ld_p;
    uint64_t next_q, next_p;  // bytes from one matrix of the call to the next
    uint32_t rows_q, rows_p;
    uint32_t stages;          // of a row
    uint32_t segments;        // 1, or 3: the pairs of parts one after the other
    uint64_t part_q, part_p;  // bytes from the first part to the second
    uint32_t tiles_q, tiles_p;
    uint32_t symmetric;       // Q = P: tiles on and above the diagonal only
    uint32_t count;           // matrices
};

// EXACT: a run is one stage as long as there are kShortSum of them, which leaves a rounding of the whole sum every 64 products (orthogonalised
// updates of 257 x 1025: off by 1.4e-6 with one every 256 and without the product of the second parts, 9e-7 so).  In longer sums those
// roundings would take over: a sum of n squares, all of one sign, is off by some sqrt(n / 64) half steps, and by n / 64 of them
// where the squares are alike.  There a run is kRun stages, and what adding it to the second sum loses is taken into the next run
// (in bf16: in fp32 it does not fit the registers of TileMid).  Off, in runs of one stage and so: 131072 x 32, 5.4e-6 and
// 1.7e-6; 4 x 524288 of +-1, 8e-4 and 4e-6; in the same time (32 x 131072 4.8 ms, 4096 x 11008 12.0, 6000 x 6000 15.8 and 15.4).
constexpr uint32_t kShortSum = 64, kRun = 8;

// The tile of a workgroup.  Workgroups go round the eight XCDs, each with an L2 of its own: each gets a contiguous run of the
// tiles instead, and a run goes down bands of eight tiles, whose operands the L2 holds.
struct TileAt {
    uint32_t matrix, q, p;
};
__device__ __forceinline__ TileAt tile_at(const ProductArgs &a, uint32_t id, uint32_t total)
{
    const uint32_t per = total / 8u, rest = total % 8u, x = id % 8u;
    uint32_t t = x * per + (x < rest ? x : rest) + id / 8u;
    const uint32_t each = a.symmetric ? a.tiles_q * (a.tiles_q + 1u) / 2u : a.tiles_q * a.tiles_p;
    TileAt r;
    r.matrix = t / each;
    t -= r.matrix * each;
    if (a.symmetric) { // row by row of the upper triangle
        uint32_t q = 0, left = a.tiles_q;
        while (t >= left) { t -= left; --left; ++q; }
        r.q = q;
        r.p = q + t;
        return r;
    }
    const uint32_t band = t / (8u * a.tiles_p);
    const uint32_t high = a.tiles_q - band * 8u < 8u ? a.tiles_q - band * 8u : 8u;
    t -= band * 8u * a.tiles_p;
    r.q = band * 8u + t % high;
    r.p = t / high;
    return r;
}

// A tile's shape: WQ x WP waves, each NQ x NP fragments of 16 x 16 outputs; DEPTH stages of both operands in LDS, in PARTS parts.
// Operands in two parts: with PARTS = 2 a stage holds all four and their four products are taken at once; with PARTS = 1 the
// summed axis runs through three pairs of parts one after the other, second with second left out (2^-24 of the sum, and a third more).
template <int WQ_, int WP_, int NQ_, int NP_, int DEPTH_, int PARTS_ = 1>
struct TileShape {
    static constexpr int WQ = WQ_, WP = WP_, NQ = NQ_, NP = NP_, DEPTH = DEPTH_, PARTS = PARTS_;
    static constexpr uint32_t Q = WQ * NQ * 16, P = WP * NP * 16, threads = WQ * WP * 64;
    static constexpr uint32_t part = (Q + P) * kStageBytes, buffer = PARTS * part, lds = DEPTH * buffer;
};

// Which row of an operand stands at place m (0 .. 15) of fragment n is free.  Rows of Q go to fragments so that the NQ fragments
// of a wave hold, at place m, NQ neighbouring rows, m NQ ..; rows of P so that the four places 4 g .. 4 g + 3 of all NP fragments,
// which are the outputs of lane group g, hold 4 NP neighbouring rows.  A lane's outputs then are a block of NQ by 4 NP, and are
// stored along either side in whole vectors.  (Scalar stores of the transposed half: 11008 x 4096 in fp16, update product 392 us,
// 355 so.)
// In LDS a fragment's rows follow one another; row `at` of the stage there is this row of the tile:
template <int N>
__device__ __forceinline__ uint32_t row_q(uint32_t at) { return at / (16u * N) * (16u * N) + at % 16u * N + at / 16u % N; }
template <int N>
__device__ __forceinline__ uint32_t row_p(uint32_t at) { return at / (16u * N) * (16u * N) + at % 16u / 4u * (4u * N) + at / 16u % N * 4u + at % 4u; }
// 16-byte piece c of the stage's row r lies at piece c ^ (r & 7): the 16 rows of a fragment meet no bank twice.
__device__ __forceinline__ uint32_t swizzle(uint32_t r, uint32_t c) { return r * kStageBytes + ((c ^ (r & 7u)) << 4); }

// Turned, columns stay in their order, 16 neighbours a fragment, and lane group g's outputs are columns 4 g .. 4 g + 3 of every 16;
// lane groups trade them in the end, for blocks of neighbours as above.  A transposing load takes 32 lanes at once: 32 bytes of eight rows, k & 3 and bit 3 of k.  The rows move them to 32-byte pieces of
// their own.  (Columns in blocks of 4 NP as above would read half of every 16 bytes: 11008 x 4096, update product 399 us, 329 so.)
template <typename Shape>
__device__ __forceinline__ uint32_t swizzle_turned(uint32_t k)
{
    static_assert(Shape::P >= 128 || Shape::P == 64, "rows of 256 bytes and more, or two rows in 256 bytes");
    return Shape::P >= 128 ? (k & 3u) | (k >> 1 & 4u) : (k >> 1 & 1u) | (k >> 2 & 2u);
}

// 16 bytes a lane from a base that is the same in every lane, plus a lane's offset, to LDS address `lds` + 16 x lane.  In assembly,
// since in front of a read from LDS the compiler waits for all such loads of its own making wherever it cannot tell their
// addresses apart (transposing reads; a second object in LDS), which takes the prefetch away: 11008 x 4096, update product
// 381 us, 323 so.  It has no output to be overwritten; loads_done() waits for it.  The wait states are those between M0 and the load
// (1) and between a base from the vector unit and the load (5).
__device__ __forceinline__ void load_to_lds(const char *base, uint32_t off, uint32_t lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(off), "s"(base) : "memory", "m0");
}
// All but the last `behind` loads of this wave to LDS have arrived: in front of each barrier that publishes a stage.
template <int behind>
__device__ __forceinline__ void loads_done()
{
    static_assert(behind >= 0 && behind < 64, "six bits");
    __builtin_amdgcn_s_waitcnt(0x0F70 | (behind & 15) | (behind >> 4) << 14); // vmcnt
}

// Element r of a in the upper one of every two groups of N lanes trades places with element r of b in the lower one.
template <int N>
__device__ __forceinline__ void trade(f32x4 &a, f32x4 &b, int r)
{
    const float x = a[r], y = b[r];
    const auto t = N == 32 ? __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(y), false, false)
                           : __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(y), false, false);
    a[r] = __uint_as_float(t[0]);
    b[r] = __uint_as_float(t[1]);
}

// Epi: void operator()(const TileAt &, uint32_t q, uint32_t p, const Acc (&)[NQ][NP]): the lane's outputs, of which element r of
// [i][j] is (q + i, p + 4 j + r); rows past the matrices' ends are among them
// RUNS: EXACT in runs of more than one stage
template <typename Op, typename Shape, bool TURNED, bool EXACT, bool RUNS, typename Epi>
__global__ __launch_bounds__(Shape::threads, 2) void k_product(const ProductArgs a, const Epi epi)
{
    constexpr int NQ = Shape::NQ, NP = Shape::NP, PARTS = Shape::PARTS;
    constexpr int waves = Shape::WQ * Shape::WP, LQ = Shape::Q / 8 / waves, LP = Shape::P / 8 / waves; // loads of 8 rows, a wave
    constexpr uint32_t kOperand = Shape::Q * kStageBytes, kBuffer = Shape::buffer;
    typedef typename Op::Acc Acc;
    __shared__ __align__(16) char lds[Shape::lds];

    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const TileAt at = tile_at(a, blockIdx.x, gridDim.x);
    const uint32_t q0 = at.q * Shape::Q, p0 = at.p * Shape::P;
    const char *const base_q = a.q + at.matrix * a.next_q + (uint64_t)q0 * a.ld_q;
    const char *const base_p = a.p + at.matrix * a.next_p + (TURNED ? (uint64_t)p0 * 2u : (uint64_t)p0 * a.ld_p);

    // where this lane's pieces come from: rows past the end are the last row again, their outputs are not stored
    uint32_t off_q[LQ], off_p[LP];
#pragma unroll
    for (int i = 0; i < LQ; ++i) {
        const uint32_t at = 8u * (waves * i + wave) + (lane >> 3), r = row_q<NQ>(at);
        off_q[i] = (uint32_t)((q0 + r < a.rows_q ? r : a.rows_q - 1u - q0) * a.ld_q) + (((lane ^ at) & 7u) << 4);
    }
#pragma unroll
    for (int i = 0; i < LP; ++i) {
        if constexpr (TURNED) {
            constexpr uint32_t pieces = Shape::P / 8; // of 16 bytes
            const uint32_t n = 64u * (waves * i + wave) + lane, r = n / pieces, c = (n % pieces) ^ (swizzle_turned<Shape>(r) << 1);
            off_p[i] = (uint32_t)(r * a.ld_p) + (p0 + c * 8u < a.rows_p ? c : 0u) * 16u;
        } else {
            const uint32_t at = 8u * (waves * i + wave) + (lane >> 3), r = row_p<NP>(at);
            off_p[i] = (uint32_t)((p0 + r < a.rows_p ? r : a.rows_p - 1u - p0) * a.ld_p) + (((lane ^ at) & 7u) << 4);
        }
    }
    const uint32_t total = a.stages * a.segments;
    uint32_t seg = 3u - a.segments, k = 0; // the stage to load next; segments 0 and 1 are those of the second parts
    const uint32_t lds_at = (uint32_t)reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) char *)lds);
    const char *bq, *bp; // the stage that is being loaded
    auto load_begin = [&]() {
        // two parts: the small products first, whose sums round by little
        bq = base_q + (seg == 0u ? a.part_q : 0u) + (uint64_t)k * kStageBytes;
        bp = base_p + (seg == 1u ? a.part_p : 0u) + (TURNED ? (uint64_t)k * 64u * a.ld_p : (uint64_t)k * kStageBytes);
        const bool last = ++k == a.stages;
        k = last ? 0u : k;
        seg += last;
    };
    auto load = [&](uint32_t buffer, int i) { // the i-th of PARTS (LQ + LP) loads
        const int n = i / (LQ + LP);
        i -= n * (LQ + LP);
        const uint32_t to = lds_at + buffer + n * Shape::part + wave * 1024u;
        if (i < LQ) load_to_lds(bq + (n ? a.part_q : 0u), off_q[i < LQ ? i : 0], to + i * waves * 1024u);
        else load_to_lds(bp + (n ? a.part_p : 0u), off_p[i < LQ ? 0 : i - LQ], to + kOperand + (i - LQ) * waves * 1024u);
    };

    // fragments: piece (lane >> 4) + 4 half of the row at place lane & 15
    const uint32_t wq = wave % Shape::WQ * (NQ * 16u), wp = wave / Shape::WQ * (NP * 16u);
    uint32_t at_q[2], at_p[2]; // of fragment 0
#pragma unroll
    for (int h = 0; h < 2; ++h) {
        at_q[h] = swizzle(wq + (lane & 15u), (lane >> 4) + 4u * h);
        // turned: row 32 h + 8 (lane >> 4) + (lane >> 2 & 3), and the one four further on; four columns from 4 (lane & 3) on
        at_p[h] = kOperand + (TURNED ? (32u * h + 8u * (lane >> 4) + (lane >> 2 & 3u)) * (Shape::P * 2u) + (lane & 3u) * 8u
                                     : swizzle(wp + (lane & 15u), (lane >> 4) + 4u * h));
    }
    i32x4 fq[2][PARTS][NQ], fp[2][PARTS][NP];
    Acc acc[NQ][NP] = {}, low[PARTS == 2 ? NQ : 1][NP] = {}, sum[EXACT ? NQ : 1][NP] = {}; // low: the products with second parts
    bf16x4 lost[RUNS ? NQ : 1][NP] = {};
    uint32_t column[NP]; // turned: where the 16 columns of a fragment lie in a row
#pragma unroll
    for (int i = 0; i < NP; ++i) column[i] = ((wp / 16u + i) ^ swizzle_turned<Shape>(8u * (lane >> 4) + (lane >> 2 & 3u))) << 5;
    constexpr int kReads = PARTS * (NQ + NP), least = (kReads + NQ - 1) / NQ, kReadsOfGroup = least < 2 * PARTS ? 2 * PARTS : least;
    auto read = [&](int h, uint32_t buffer, int i) { // the i-th of a half step's fragments
        const int n = i / (NQ + NP);
        i -= n * (NQ + NP);
        buffer += n * Shape::part;
        if (i >= NP) {
            fq[h][n][i - NP] = *(const i32x4 *)(lds + buffer + at_q[h] + (i - NP) * 16 * kStageBytes);
        } else if constexpr (TURNED) {
            const uint32_t at = buffer + at_p[h] + column[i];
            typedef short s16x4 __attribute__((ext_vector_type(4)));
            const auto first = (__attribute__((address_space(3))) s16x4 *)(lds + at), next = (__attribute__((address_space(3))) s16x4 *)(lds + at + 4u * Shape::P * 2u);
            const s16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(first), v1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16(next);
            fp[h][n][i] = __builtin_bit_cast(i32x4, __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7));
        } else {
            fp[h][n][i] = *(const i32x4 *)(lds + buffer + at_p[h] + i * 16 * kStageBytes);
        }
    };
    // one half step: NQ groups of matrix instructions on fragments `h`; in front of each group two or so (of a part) of the reads of the
    // next half step's fragments (so that the last ones have time to arrive) and its share of the loads
    constexpr int each = PARTS * (LQ + LP), most = (each + NQ - 1) / NQ;
    auto half = [&](auto h, uint32_t from, auto loads, uint32_t to) {
        constexpr int H = decltype(h)::value;
        static_for<NQ>([&](auto g) {
            constexpr int i = decltype(g)::value;
            if constexpr (decltype(loads)::value)
                static_for<most>([&](auto l) {
                    if constexpr (i * most + decltype(l)::value < each) load(to, i * most + decltype(l)::value);
                });
            static_for<kReadsOfGroup>([&](auto l) {
                constexpr int n = kReadsOfGroup * i + decltype(l)::value;
                if constexpr (n < kReads) read(1 - H, from, n);
            });
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                if constexpr (EXACT && !RUNS && H == 0) { // sums start anew with every stage
                    sum[i][j] += acc[i][j];
                    acc[i][j] = Op::mfma(fp[H][0][j], fq[H][0][i], Acc{});
                } else {
                    acc[i][j] = Op::mfma(fp[H][0][j], fq[H][0][i], acc[i][j]);
                }
                if constexpr (PARTS == 2) {
                    low[i][j] = Op::mfma(fp[H][1][j], fq[H][1][i], low[i][j]);
                    low[i][j] = Op::mfma(fp[H][1][j], fq[H][0][i], low[i][j]);
                    low[i][j] = Op::mfma(fp[H][0][j], fq[H][1][i], low[i][j]);
                }
            }
        });
        static_for<NQ>([&](auto g) { // that order for the compiler's scheduler
            constexpr int i = decltype(g)::value;
            constexpr int reads = [] {
                int r = 0;
                for (int n = kReadsOfGroup * i; n < kReadsOfGroup * (i + 1) && n < kReads; ++n) r += TURNED && n % (NQ + NP) < NP ? 2 : 1;
                return r;
            }();
            if constexpr (reads > 0) __builtin_amdgcn_sched_group_barrier(0x100, reads, 0);
            __builtin_amdgcn_sched_group_barrier(0x008, NP * (PARTS == 2 ? 4 : 1), 0);
        });
    };
    constexpr std::integral_constant<int, 0> first{};
    constexpr std::integral_constant<int, 1> second{};

    constexpr int D = Shape::DEPTH;
    static_for<D>([&](auto d) {
        if ((uint32_t)decltype(d)::value < total) {
            load_begin();
            static_for<each>([&](auto i) { load(decltype(d)::value * kBuffer, decltype(i)::value); });
        }
    });
    if (total >= (uint32_t)D) loads_done<(D - 1) * each>();
    else loads_done<0>();
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kReads; ++i) read(0, 0, i);
    uint32_t buffer = 0, left = (a.segments - 1u) * a.stages + kRun; // (what second parts add is small, and goes with the first run)
    auto run = [&]() {
        if constexpr (RUNS) {
            if (left-- != 0u) return;
            left = kRun - 1u;
#pragma unroll
            for (int i = 0; i < NQ; ++i)
#pragma unroll
                for (int j = 0; j < NP; ++j) {
                    const Acc add = acc[i][j] - __builtin_convertvector(lost[i][j], Acc), to = sum[i][j] + add;
                    lost[i][j] = __builtin_convertvector((to - sum[i][j]) - add, bf16x4);
                    sum[i][j] = to;
                    acc[i][j] = Acc{};
                }
        }
    };
    auto follow = [&](uint32_t b) { return b + kBuffer == D * kBuffer ? 0u : b + kBuffer; };
    for (uint32_t s = D; s < total; ++s) {
        run();
        half(first, buffer, std::false_type{}, 0);
        loads_done<(D - 2) * each>();
        __syncthreads();
        load_begin();
        half(second, follow(buffer), std::true_type{}, buffer);
        buffer = follow(buffer);
    }
    for (uint32_t s = total < (uint32_t)D ? total : D; s; --s) { // nothing left to load; what the very last half step reads is not used
        run();
        half(first, buffer, std::false_type{}, 0);
        loads_done<0>();
        __syncthreads();
        half(second, follow(buffer), std::false_type{}, 0);
        buffer = follow(buffer);
    }
    if constexpr (EXACT)
#pragma unroll
        for (int i = 0; i < NQ; ++i)
#pragma unroll
            for (int j = 0; j < NP; ++j) {
                if constexpr (RUNS) acc[i][j] -= __builtin_convertvector(lost[i][j], Acc);
                if constexpr (PARTS == 2) acc[i][j] += low[i][j];
                acc[i][j] += sum[i][j];
            }
    if constexpr (TURNED) { // piece g' of fragment j is lane group g''s: fragments to lane groups, pieces to registers
#pragma unroll
        for (int i = 0; i < NQ; ++i)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
                if constexpr (NP == 4) {
                    trade<32>(acc[i][0], acc[i][2], r);
                    trade<32>(acc[i][1], acc[i][3], r);
                    trade<16>(acc[i][0], acc[i][1], r);
                    trade<16>(acc[i][2], acc[i][3], r);
                } else {
                    trade<32>(acc[i][0], acc[i][1], r);
                    trade<16>(acc[i][0], acc[i][1], r);
                }
            }
    }
    epi(at, q0 + wq + (lane & 15u) * NQ, p0 + wp + (lane >> 4) * (4u * NP), acc);
}

// ---- which tile ----------------------------------------------------------------------------------------------------------------
// A compute unit holds one workgroup of TileBig or TileLarge, two of TileMid or TileDeep, five of TileSmall.  What bounds a stage is
// the way from the L2 to LDS, at 2.4 GHz some 19 bytes a cycle and compute unit with one workgroup (Large, 4096 x 4096 x 11008) and 24 to 33 with
// five (4096 x 4096 x 4096): large tiles move the fewest bytes for an output, small ones use more of the 256 units.
// us, each kernel by itself in a trace, fp16 (i8 where said); full products are those down the columns:
//   tiles of 256 / 192 / 128 sides                    Big   Large   Mid  Small  Deep
//   688 /    - / 2752  4096 x 11008 x 4096            303           354   521   548
//   256 /    - / 1024  4096 x 4096 x 4096             118           148   210   236
//   136 / 253 / 528    the same, upper half            98     88    109   147   160
//   136 / 253 / 528    4096 x 4096 x 11008, upper half 224   188    271   438   458
//   192 /    - / 768   12 of 1024 x 1024 x 1024        31            33    40    46
//   144 / 231 / 544    4000 x 2057 x 16384, i8        181    135    190   226   217
//   120 / 252 / 432    12 of 1024, upper halves        28     27     21    25    27
//    80 / 168 / 288    8 of 1024 x 1024 x 4096, upper halves  80  65  58   70    62
//    66 / 120 / 253    2800 x 2800 x 8192, upper half 147    113     87   104   153
//    45 /  78 / 171    2300 x 2300 x 8192, upper half 141    106     79    73    98
//    64 /    - / 256   2048 x 2048 x 2048              44            26    29    31
//    36 /  66 / 136    2048, upper half                42     34     23    20    23
//    32 /  66 / 128    512 x 4096 x 4096, i8           49     35     25    18    18
//    10 /  21 /  36    1024 x 1024 x 6336, upper half 109     80     65    46    26
//    56 /  75 / 112    77 x 14336 x 4096, i8           42     31     26    20    16
// So: Mid from 200 of them on, as long as a round takes them all; where Mid would need a second round, Large if every one of those
// has a unit to itself, and Big otherwise.  Fewer: Small, and Deep (four stages instead of two, two workgroups a unit) as long as
// one round takes them all.  (Large has three rows to a lane, for twelve waves, three a SIMD; turned operands have no use for it.)
typedef TileShape<2, 4, 8, 4, 2> TileBig;
typedef TileShape<4, 3, 3, 4, 2> TileLarge;
typedef TileShape<2, 2, 4, 4, 2> TileMid;
typedef TileShape<2, 2, 2, 2, 2> TileSmall;
typedef TileShape<2, 2, 2, 2, 4> TileDeep;
typedef TileShape<2, 2, 2, 2, 2, 2> TilePairs; // small tiles of operands in two parts: a third of the stages
typedef TileShape<2, 2, 2, 2, 4, 2> TilePairsDeep;

inline uint64_t product_tiles(const ProductArgs &a, uint32_t side)
{
    const uint64_t q = (a.rows_q + side - 1u) / side, p = (a.rows_p + side - 1u) / side;
    return a.count * (a.symmetric ? q * (q + 1u) / 2u : q * p);
}

template <typename Op, bool TURNED, bool EXACT, typename Shape, bool RUNS = false, typename Epi>
void launch_product_as(ProductArgs a, const Epi &epi, hipStream_t st)
{
    a.segments = EXACT && Shape::PARTS == 1 ? 3u : 1u; // EXACT: operands in two parts
    static_assert(Shape::Q == Shape::P, "the upper triangle of a symmetric product is one of square tiles");
    a.tiles_q = (a.rows_q + Shape::Q - 1u) / Shape::Q;
    a.tiles_p = (a.rows_p + Shape::P - 1u) / Shape::P;
    const dim3 grid((unsigned)product_tiles(a, Shape::Q)), block(Shape::threads);
    if constexpr (RUNS)
        if (a.stages > kShortSum) {
            hipLaunchKernelGGL((k_product<Op, Shape, TURNED, EXACT, true, Epi>), grid, block, 0, st, a, epi);
            return;
        }
    hipLaunchKernelGGL((k_product<Op, Shape, TURNED, EXACT, false, Epi>), grid, block, 0, st, a, epi);
}
template <typename Op, bool TURNED = false, bool EXACT = false, typename Epi>
void launch_product(const ProductArgs &a, const Epi &epi, hipStream_t st)
{
    if constexpr (EXACT) {
        // (No Big: a second set of sums does not fit the registers.)  A unit holds two tiles of Mid or Pairs, or one of PairsDeep, which is
        // ahead as long as every tile has a unit to itself.  Mid is behind where its tiles hardly make a round, and ahead from two
        // rounds on.  us, each kernel by itself in a trace:
        //   tiles of 128 / 64                                Mid  Pairs  PairsDeep
        //    36 /  136    1000 x 1000 x 2050, upper half      64     23     22
        //    78 /  300    1500 x 1500 x 1500, upper half      50     25     32
        //   136 /  528    2000 x 2000 x 2000, upper half      64     54     62
        //   136 /  528    1000 x 2050 x 1000                  38     29     38
        //   253 /  990    2800 x 2800 x 2800, upper half     100     96    118
        //   256 / 1024    2048 x 2048 x 2048                  74     71     93
        //   320 / 1280    20 of 512 x 512 x 512               32     27     38
        //   432 / 1632    12 of 1024, upper halves            59     62     81
        //   484 / 1936    2800 x 2800 x 2800                 151    187    249
        //   528 / 2080    4096 x 4096 x 11008, upper half    872    934    943
        //  2752 / 11008   4096 x 11008 x 4096               1124   1424   1767
        // A sum longer than kShortSum over few outputs is one of Gram's: in the other products it is no longer than either side.
        constexpr bool longer = Epi::sums_longer_than_sides;
        constexpr uint32_t least = ((kShortSum + 1u) * 64u + 127u) / 128u; // tiles of 128 along a side as long as such a sum
        static_assert(least * (least + 1u) / 2u >= 256u, "which are Mid's");
        if (product_tiles(a, 128u) >= 256u) launch_product_as<Op, TURNED, EXACT, TileMid, true>(a, epi, st);
        else if (product_tiles(a, 64u) > 256u) launch_product_as<Op, TURNED, EXACT, TilePairs, longer>(a, epi, st);
        else launch_product_as<Op, TURNED, EXACT, TilePairsDeep, longer>(a, epi, st);
    } else {
        if constexpr (!TURNED)
            if (product_tiles(a, 128u) > 512u && product_tiles(a, 192u) <= 256u) return launch_product_as<Op, TURNED, EXACT, TileLarge>(a, epi, st);
        if (product_tiles(a, 128u) > 512u) launch_product_as<Op, TURNED, EXACT, TileBig>(a, epi, st);
        else if (product_tiles(a, 128u) >= 200u) launch_product_as<Op, TURNED, EXACT, TileMid>(a, epi, st);
        else if (product_tiles(a, 64u) > 512u) launch_product_as<Op, TURNED, EXACT, TileSmall>(a, epi, st);
        else launch_product_as<Op, TURNED, EXACT, TileDeep>(a, epi, st);
    }
}

} // namespace fo
