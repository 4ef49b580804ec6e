// Rows of a matrix as 8-bit codes with one amplitude a row (fo_rows_encode), on gfx950.
//
// A row (or, transposed, a column) x of `len` values, zero-padded to `stride` coordinates, becomes y = H_b D_eps x, block by block
// of b = 2^k coordinates (k = 0: y = x), then q = rint(127 y / max|y| [+ u / 2]) with u the dither.  Both operands of a product use
// the same eps, so the transforms cancel in it: (H D x) . (H D w) = b (x . w).  The stages of a transform go from the lowest
// coordinate bit to the highest in both kernels, so that a matrix and its transpose give the same codes to the bit.
#pragma once
#include "fo_device.h"

namespace fo {

constexpr uint32_t kDomainRowDither = 3u; // coordinate i = row * stride + k: 16 bits, half i & 1 of word (i >> 1) & 3 of call i >> 3
constexpr uint32_t kRowSegment = 1024;    // coordinates a wave holds, 16 a lane: lane l has 8 l .. 8 l + 7 of either half

struct RowsArgs {
    const void *x;
    uint64_t ld;        // elements from one row of x in memory to the next
    uint64_t rows;      // coded rows
    uint32_t len, stride, block;
    uint32_t dither;
    uint32_t k0, k1, round_lo, eps_party, party;
    float unflatten;    // 1 / sqrt(b)
    int8_t *codes;
    float *scales;
};

template <typename T>
__device__ __forceinline__ float widen(T v)
{
    if constexpr (std::is_same_v<T, uint16_t>) return __uint_as_float((uint32_t)v << 16); // bf16
    else return (float)v;
}

// Walsh-Hadamard stage on lane bit K of 16 values.  On bits 0 to 3 the upper lane gets its own value minus its partner's instead of
// the other way round, one multiply-add with +-1 that reads the partner's register in place: everything that the value meets later
// has the same sign then, so that one sign per lane, lane_sign(), is put right in the factor at the end.
#define FO_FMAC_DPP(n, from, perm) "v_fmac_f32_dpp %" #n ", %" #from ", %[s] " perm " row_mask:0xf bank_mask:0xf\n\t"
#define FO_FMAC_DPP_8(v, perm)                                                                                                           \
    asm volatile("s_nop 1\n\t" FO_FMAC_DPP(0, 0, perm) FO_FMAC_DPP(1, 1, perm) FO_FMAC_DPP(2, 2, perm) FO_FMAC_DPP(3, 3, perm)                \
                     FO_FMAC_DPP(4, 4, perm) FO_FMAC_DPP(5, 5, perm) FO_FMAC_DPP(6, 6, perm) FO_FMAC_DPP(7, 7, perm) "s_nop 1"               \
                 : "+v"((v)[0]), "+v"((v)[1]), "+v"((v)[2]), "+v"((v)[3]), "+v"((v)[4]), "+v"((v)[5]), "+v"((v)[6]), "+v"((v)[7])           \
                 : [s] "v"(sign))
#define FO_FMAC_DPP_FROM_8(v, t, perm)                                                                                                   \
    asm volatile("s_nop 1\n\t" FO_FMAC_DPP(0, 8, perm) FO_FMAC_DPP(1, 9, perm) FO_FMAC_DPP(2, 10, perm) FO_FMAC_DPP(3, 11, perm)              \
                     FO_FMAC_DPP(4, 12, perm) FO_FMAC_DPP(5, 13, perm) FO_FMAC_DPP(6, 14, perm) FO_FMAC_DPP(7, 15, perm) "s_nop 1"           \
                 : "+v"((v)[0]), "+v"((v)[1]), "+v"((v)[2]), "+v"((v)[3]), "+v"((v)[4]), "+v"((v)[5]), "+v"((v)[6]), "+v"((v)[7])           \
                 : "v"((t)[0]), "v"((t)[1]), "v"((t)[2]), "v"((t)[3]), "v"((t)[4]), "v"((t)[5]), "v"((t)[6]), "v"((t)[7]), [s] "v"(sign))
// (The wait states are those between a vector instruction and one that reads its result in another lane.)
template <int K>
__device__ __forceinline__ void bfly_lane(float (&v)[16], uint32_t lane)
{
    const float sign = lane >> K & 1u ? -1.f : 1.f;
    if constexpr (K == 0) {
        FO_FMAC_DPP_8(v, "quad_perm:[1,0,3,2]");
        FO_FMAC_DPP_8(v + 8, "quad_perm:[1,0,3,2]");
    } else if constexpr (K == 1) {
        FO_FMAC_DPP_8(v, "quad_perm:[2,3,0,1]");
        FO_FMAC_DPP_8(v + 8, "quad_perm:[2,3,0,1]");
    } else if constexpr (K == 2) { // row_half_mirror and then quad_perm 3,2,1,0: lane ^ 7 ^ 3
        float t[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) t[k] = __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(v[k]), 0x141, 0xf, 0xf, true));
        FO_FMAC_DPP_FROM_8(v, t, "quad_perm:[3,2,1,0]");
        FO_FMAC_DPP_FROM_8(v + 8, t + 8, "quad_perm:[3,2,1,0]");
    } else if constexpr (K == 3) {
        FO_FMAC_DPP_8(v, "row_ror:8");
        FO_FMAC_DPP_8(v + 8, "row_ror:8");
    } else if constexpr (K == 4) { // as bfly_lane5, with rows of 16 lanes
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v[k]), __float_as_uint(v[k + 8]), false, false);
            const float x = __uint_as_float(r[0]), y = __uint_as_float(r[1]);
            r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x + y), __float_as_uint(x - y), false, false);
            v[k] = __uint_as_float(r[0]);
            v[k + 8] = __uint_as_float(r[1]);
        }
    } else {
        bfly_lane5(v);
    }
}
#undef FO_FMAC_DPP_FROM_8
#undef FO_FMAC_DPP_8
#undef FO_FMAC_DPP
__device__ __forceinline__ uint32_t lane_sign(uint32_t lane, uint32_t block) // the sign bit: parity of the lane bits below 4 that had a stage
{
    return block ? (uint32_t)__builtin_popcount(lane & (block > 6u ? 15u : 7u)) << 31 : 0u;
}

// Largest magnitude as the bits of a float: an infinity or a NaN is larger than every number
constexpr uint32_t kInfinity = 0x7F800000u, kNotFinite = 0xFFFFFFFFu;
__device__ __forceinline__ uint32_t magnitude(float v) { return __float_as_uint(v) & 0x7FFFFFFFu; }
__device__ __forceinline__ uint32_t wave_max(uint32_t m) // in registers, the steps of wave_sum
{
    auto larger = [](uint32_t a, uint32_t b) { return a > b ? a : b; };
    m = larger(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0xB1, 0xf, 0xf, true));
    m = larger(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x4E, 0xf, 0xf, true));
    m = larger(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x141, 0xf, 0xf, true));
    m = larger(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, 0x140, 0xf, 0xf, true));
    auto r = __builtin_amdgcn_permlane16_swap(m, m, false, false);
    m = larger(r[0], r[1]);
    r = __builtin_amdgcn_permlane32_swap(m, m, false, false);
    return larger(r[0], r[1]);
}

// The factor that takes a row's largest magnitude to 127, and the amplitude its codes stand for.  A magnitude under 2^-64 is taken
// up by 2^64 first (exactly), so that the factor stays finite.  Not finite: factor 0 and amplitude NaN.
struct RowFactor {
    float up, inv;
    bool finite;
};
__device__ __forceinline__ RowFactor row_factor(uint32_t max_bits)
{
    RowFactor f;
    const float m = __uint_as_float(max_bits);
    f.finite = max_bits < kInfinity;
    f.up = m < 0x1p-64f ? 0x1p64f : 1.f;
    f.inv = f.finite && m > 0.f ? __fmul_rn(127.f, 1.f / (m * f.up)) : 0.f;
    return f;
}
__device__ __forceinline__ float row_scale(uint32_t max_bits, float unflatten)
{
    return max_bits < kInfinity ? __uint_as_float(max_bits) * (1.f / 127.f) * unflatten : __builtin_nanf("");
}

// A code in the low byte: adding 1.5 2^23 rounds to the nearest integer, ties to even.  Without dither |127 y / max| is at most
// 127 (1 + 2^-22), which rounds to 127.
// The product is rounded before anything is added to it, in every kernel: a matrix and its transpose give the same codes.
__device__ __forceinline__ uint32_t row_code(float y, float inv)
{
#pragma clang fp contract(off)
    const float v = y * inv;
    return __float_as_uint(v + 12582912.f);
}
__device__ __forceinline__ uint32_t row_code(float y, float inv, float half_dither)
{
#pragma clang fp contract(off)
    const float v = y * inv;
    return __float_as_uint(__builtin_amdgcn_fmed3f(v + half_dither, -127.f, 127.f) + 12582912.f);
}
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d)
{
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(d, c, 0x0C0C0400u), __builtin_amdgcn_perm(b, a, 0x0C0C0400u), 0x05040100u);
}
// u / 2 of 16 random bits: an odd multiple of 2^-17 in (-1/2, 1/2).  Sixteen bits bring E[q] within 2^-17 of what is rounded, which itself is off
// from 127 y / max by three roundings of 2^-24 of up to 127 (2^-15.4 at most, found over all 2^16 dithers of 4000 values).
__device__ __forceinline__ float half_dither_of(uint32_t r16) { return (float)(int32_t)(2u * r16 + 1u - 65536u) * 0x1p-17f; }

// Blocks of up to 2^10 finite values add up to as much as 2^138.  A row whose transform leaves fp32's range is transformed once more, 2^-16
// of it (exact for whatever its codes can tell), by a workgroup of N threads, 1024 coordinates at a time in LDS, with the
// same additions in the same order; x[k step] is its coordinate k.  Rare, and apart from the kernels' loops, where it would take 3 to 12 %
// of their time.  Called by the whole workgroup, for a row without infinities and NaN.
template <typename T, uint32_t N>
__device__ __forceinline__ void encode_lowered(const RowsArgs &a, const T *x, uint64_t step, uint64_t row, float *y, uint32_t *most)
{
    const uint32_t t = threadIdx.x;
    const RngKey eps{ a.k0, a.k1, kDomainEps, a.round_lo, a.eps_party }, dither{ a.k0, a.k1, kDomainRowDither, a.round_lo, a.party };
    uint32_t m = 0;
    RowFactor f;
    for (int pass = 0; pass < 2; ++pass) { // the largest magnitude, the codes
        for (uint32_t k0 = 0; k0 < a.stride; k0 += 1024u) {
            __syncthreads(); // y has been read
            for (uint32_t i = t; i < 1024u; i += N) {
                const uint32_t k = k0 + i;
                uint32_t w[4];
                philox(k / 128u, eps, w);
                const uint32_t w0 = w[0], w1 = w[1], w2 = w[2], w3 = w[3], low = k & 32u ? w1 : w0, high = k & 32u ? w3 : w2, n = k & 64u ? high : low;
                y[i] = k < a.len ? flip_by_bit31(widen(x[k * step]) * 0x1p-16f, n << (31u - k % 32u)) : 0.f;
            }
            for (uint32_t b = 0; b < a.block; ++b) {
                __syncthreads();
                for (uint32_t p = t; p < 512u; p += N) {
                    const uint32_t i = p >> b << (b + 1u) | (p & ((1u << b) - 1u)), j = i | 1u << b;
                    const float u = y[i], v = y[j];
                    y[i] = u + v;
                    y[j] = u - v;
                }
            }
            __syncthreads();
            for (uint32_t i = 4u * t; i < 1024u && k0 + i < a.stride; i += 4u * N) {
                if (pass == 0) {
                    for (uint32_t c = 0; c < 4u; ++c) m = m > magnitude(y[i + c]) ? m : magnitude(y[i + c]);
                    continue;
                }
                const uint64_t at = row * a.stride + k0 + i;
                auto store = [&](uint32_t q0, uint32_t q1, uint32_t q2, uint32_t q3) {
                    *reinterpret_cast<uint32_t *>(a.codes + at) = pack4(q0, q1, q2, q3);
                };
                if (a.dither) {
                    uint32_t w[4];
                    philox((uint32_t)(at >> 3), dither, w);
                    const uint32_t w0 = w[0], w1 = w[1], w2 = w[2], w3 = w[3], low = at & 4u ? w2 : w0, high = at & 4u ? w3 : w1;
                    store(row_code(y[i], f.inv, half_dither_of(low & 0xFFFFu)), row_code(y[i + 1u], f.inv, half_dither_of(low >> 16)),
                          row_code(y[i + 2u], f.inv, half_dither_of(high & 0xFFFFu)), row_code(y[i + 3u], f.inv, half_dither_of(high >> 16)));
                } else {
                    store(row_code(y[i], f.inv), row_code(y[i + 1u], f.inv), row_code(y[i + 2u], f.inv), row_code(y[i + 3u], f.inv));
                }
            }
        }
        if (pass) return;
        m = wave_max(m);
        if ((t & 63u) == 0u) most[t >> 6] = m;
        __syncthreads();
        for (uint32_t w = 0; w < N / 64u; ++w) m = m > most[w] ? m : most[w];
        f = row_factor(m);
        if (t == 0) a.scales[row] = row_scale(m, a.unflatten) * 0x1p16f;
    }
}

// A lane's 16 values of a segment, x[k] .. x[k + 7] and x[k + 512] .. x[k + 519], zero from `len` on, two (of 16 bits) or one in a
// register.  (Where the whole segment lies in front of it both loads are on their way before either is waited for.)
template <typename T>
struct Segment {
    static constexpr int N = 4 * sizeof(T);
    uint32_t w[N];
    __device__ __forceinline__ void load(const T *x, uint32_t k, uint32_t segment_end, uint32_t len)
    {
        if (segment_end <= len) { // (elements may lie at any multiple of their size)
            __builtin_memcpy(w, x + k, 2 * N);
            __builtin_memcpy(w + N / 2, x + k + 512u, 2 * N);
        } else {
            T t[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const uint32_t at = k + (i & 7) + 512u * (i / 8);
                t[i] = at < len ? x[at] : T(0);
            }
            __builtin_memcpy(w, t, sizeof(w));
        }
    }
    // flips: for the i-th two values the first one's at bit 15, the second one's at bit 31
    __device__ __forceinline__ void flip(int i, uint32_t mask)
    {
        if constexpr (sizeof(T) == 2) {
            w[i] ^= mask;
        } else {
            w[2 * i] ^= mask << 16;
            w[2 * i + 1] = __builtin_amdgcn_bitop3_b32(w[2 * i + 1], mask, 0x80000000u, 0x78);
        }
    }
    __device__ __forceinline__ void values(float (&v)[16]) const
    {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            if constexpr (std::is_same_v<T, uint16_t>) v[i] = __uint_as_float(i % 2 ? w[i / 2] & 0xFFFF0000u : w[i / 2] << 16);
            else if constexpr (sizeof(T) == 2) v[i] = (float)__builtin_bit_cast(_Float16, (uint16_t)(w[i / 2] >> (16 * (i % 2))));
            else v[i] = __uint_as_float(w[i]);
        }
    }
};

// One workgroup of W waves a row at a time; a wave holds 1024 coordinates.  FEW: the row fits the workgroup, which reads it once, the
// next row's values on their way meanwhile, and keeps every coordinate's sign flip in place; other rows are read twice.
// 8192 rows of 4096 bf16 in blocks of 256, 100 MB: 25 us, 4.0 TB/s, vector instructions at 70 % of their rate (a butterfly across lanes as
// a move and an addition, and sign flips spread anew for each row: 28.6 us).
template <typename T, int W, bool FEW>
__global__ __launch_bounds__(W * 64) void k_rows_encode(const RowsArgs a)
{
    constexpr uint32_t kFlips = FEW ? W * kRowSegment / 2 : (1u << 17) / 32; // FEW: one for two coordinates; else bits
    __shared__ __align__(16) uint32_t flips[kFlips < 1024u ? 1024u : kFlips];
    __shared__ uint32_t most[16];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    if (a.block) {
        __shared__ __align__(16) uint32_t words[FEW ? W * kRowSegment / 32 : 4];
        const RngKey key{ a.k0, a.k1, kDomainEps, a.round_lo, a.eps_party };
        for (uint32_t c = threadIdx.x; c < (FEW ? W * kRowSegment : a.stride) / 128u; c += W * 64) { // (past the row: signs of zeros)
            uint32_t w[4];
            philox(c, key, w);
            *reinterpret_cast<uint4 *>((FEW ? words : flips) + 4u * c) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        __syncthreads();
        if constexpr (FEW) { // every thread spreads half a word
            const uint32_t n = words[threadIdx.x / 2u] >> (threadIdx.x % 2u * 16u);
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                uint32_t m[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) m[k] = (n >> (2 * (i + k)) & 1u) << 15 | (n >> (2 * (i + k) + 1)) << 31;
                *reinterpret_cast<uint4 *>(flips + threadIdx.x * 8u + i) = make_uint4(m[0], m[1], m[2], m[3]);
            }
            __syncthreads();
        }
    }
    const RngKey key{ a.k0, a.k1, kDomainRowDither, a.round_lo, a.party };
    const uint32_t segments = (a.stride + kRowSegment - 1u) / kRowSegment;
    const uint32_t sign = lane_sign(lane, a.block);
    Segment<T> in;
    float v[16];
    auto flattened = [&](uint32_t seg) { // y (up to the lane's sign) from what was loaded
        const uint32_t k = seg * kRowSegment + lane * 8u;
        if (a.block) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t at = k + 512u * h;
                if constexpr (FEW) {
                    const uint4 m = *reinterpret_cast<const uint4 *>(flips + at / 2u);
                    in.flip(4 * h, m.x);
                    in.flip(4 * h + 1, m.y);
                    in.flip(4 * h + 2, m.z);
                    in.flip(4 * h + 3, m.w);
                } else {
                    const uint32_t n = (at < a.stride ? flips[at >> 5] : 0u) >> (at & 31u);
#pragma unroll
                    for (int i = 0; i < 4; ++i) in.flip(4 * h + i, (n >> (2 * i) & 1u) << 15 | (n >> (2 * i + 1)) << 31);
                }
            }
        }
        in.values(v);
        if (!a.block) return;
        bfly<float, 0>(v);
        bfly<float, 1>(v);
        bfly<float, 2>(v);
        bfly_lane<0>(v, lane);
        bfly_lane<1>(v, lane);
        bfly_lane<2>(v, lane);
        if (a.block > 6) bfly_lane<3>(v, lane);
        if (a.block > 7) bfly_lane<4>(v, lane);
        if (a.block > 8) bfly_lane<5>(v, lane);
        if (a.block > 9) bfly<float, 3>(v);
    };
    auto load = [&](uint64_t row, uint32_t seg) {
        in.load(static_cast<const T *>(a.x) + row * a.ld, seg * kRowSegment + lane * 8u, (seg + 1u) * kRowSegment, a.len);
    };

    uint32_t largest = 0; // over the rows
    if (FEW) load(blockIdx.x, wave);
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        uint32_t m = 0;
        for (uint32_t seg = wave; seg < (FEW ? wave + 1u : segments); seg += W) {
            if (!FEW) load(row, seg);
            flattened(seg);
#pragma unroll
            for (int i = 0; i < 16; ++i) m = m > magnitude(v[i]) ? m : magnitude(v[i]);
        }
        if (FEW && row + gridDim.x < a.rows) load(row + gridDim.x, wave);
        m = wave_max(m);
        if constexpr (W > 1) {
            __syncthreads(); // the last row's maxima have been read
            if (lane == 0) most[wave] = m;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < W; ++w) m = m > most[w] ? m : most[w];
        }
        largest = largest > m ? largest : m;
        const RowFactor f = row_factor(m);
        if (threadIdx.x == 0) a.scales[row] = row_scale(m, a.unflatten);
        const float inv = __uint_as_float(__float_as_uint(f.inv) ^ sign);
        for (uint32_t seg = wave; seg < (FEW ? wave + 1u : segments); seg += W) {
            if (!FEW) {
                load(row, seg);
                flattened(seg);
            }
            if (f.up != 1.f)
#pragma unroll
                for (int i = 0; i < 16; ++i) v[i] *= f.up;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t k = seg * kRowSegment + 512u * h + lane * 8u;
                const uint64_t i = row * a.stride + k;
                uint32_t q[8];
                if (a.dither) {
                    uint32_t w[4];
                    philox((uint32_t)(i >> 3), key, w);
#pragma unroll
                    for (int c = 0; c < 8; ++c) q[c] = row_code(v[8 * h + c], inv, half_dither_of((w[c >> 1] >> (16 * (c & 1))) & 0xFFFFu));
                } else {
#pragma unroll
                    for (int c = 0; c < 8; ++c) q[c] = row_code(v[8 * h + c], inv);
                }
                const uint2 out = make_uint2(pack4(q[0], q[1], q[2], q[3]), pack4(q[4], q[5], q[6], q[7]));
                if (k < a.stride) *reinterpret_cast<uint2 *>(a.codes + i) = f.finite ? out : make_uint2(0u, 0u);
            }
        }
    }
    if (!a.block || __builtin_amdgcn_readfirstlane((int)largest) < (int)kInfinity) return;
    __syncthreads(); // the amplitudes are there, the flips have been read
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        if (magnitude(a.scales[row]) <= kInfinity) continue;
        const T *const x = static_cast<const T *>(a.x) + row * a.ld;
        uint32_t m = 0; // of the row itself: an infinity or a NaN of its own?
        for (uint32_t k = threadIdx.x; k < a.len; k += W * 64) m = m > magnitude(widen(x[k])) ? m : magnitude(widen(x[k]));
        m = wave_max(m);
        __syncthreads(); // the last maxima have been read
        if (lane == 0) most[wave] = m;
        __syncthreads();
        for (int w = 0; w < W; ++w) m = m > most[w] ? m : most[w];
        if (m < kInfinity) encode_lowered<T, W * 64>(a, x, 1u, row, reinterpret_cast<float *>(flips), most);
    }
}

// Columns of x as coded rows.  A workgroup takes C columns by 2^LOGK coordinates (C 2^(LOGK - 6) threads, 64 values each): a thread
// first has 64 consecutive coordinates of its column (stages 0 to 5 in registers, every load 64 or 32 neighbouring columns), then,
// through LDS, all coordinates that agree in the low six bits for 64 / 2^(LOGK - 6) values of those.  The amplitude needs a whole
// column: a first pass takes the maxima (an integer maximum in memory, the same in any order), a second one reads x again, from
// the last-level cache where it fits, and quantises.  4096 columns of 8192 bf16, dithered: 21 and 39 us, the second half draws
// (vector instructions at three quarters of their rate); with each load waited for before the next 118 us together.
enum ColumnsPass { COLUMNS_MAX, COLUMNS_CODES };
template <typename T, int LOGK, ColumnsPass PASS>
__global__ __launch_bounds__((LOGK == 8 ? 64 : 32) << (LOGK - 6)) void k_columns_encode(const RowsArgs a)
{
    constexpr uint32_t C = LOGK == 8 ? 64 : 32, HI = 1u << (LOGK - 6), LOW = 64 / HI, K = 1u << LOGK;
    __shared__ float y[K * C / 2];
    __shared__ uint32_t eps[K / 32];
    const uint32_t c = threadIdx.x % C, g = threadIdx.x / C;
    // workgroups that follow one another take neighbouring columns, whose lines lie side by side in memory
    const uint32_t across_rows = (uint32_t)((a.rows + C - 1u) / C);
    const uint32_t kt = blockIdx.x / across_rows * K;
    const uint64_t row = (uint64_t)(blockIdx.x % across_rows) * C + c;
    const bool in = row < a.rows;
    if (a.block) {
        if (threadIdx.x < K / 128u) {
            const RngKey key{ a.k0, a.k1, kDomainEps, a.round_lo, a.eps_party };
            uint32_t w[4];
            philox(kt / 128u + threadIdx.x, key, w);
            *reinterpret_cast<uint4 *>(eps + 4u * threadIdx.x) = make_uint4(w[0], w[1], w[2], w[3]);
        }
        __syncthreads();
    }
    float v[64];
    {
        // all on their way before the first is waited for: past the end, the last row again and zero in its place
        const T *const x = static_cast<const T *>(a.x) + (in ? row : 0u);
        T w[64];
#pragma unroll
        for (int r = 0; r < 64; ++r) {
            const uint32_t k = kt + g * 64u + r;
            w[r] = x[(uint64_t)(k < a.len ? k : a.len - 1u) * a.ld];
        }
#pragma unroll
        for (int r = 0; r < 64; ++r) v[r] = in && kt + g * 64u + r < a.len ? widen(w[r]) : 0.f;
    }
    uint32_t at = g * 64u; // coordinate of v[0] in the tile
    if (a.block) {
#pragma unroll
        for (int r = 0; r < 64; ++r) v[r] = flip_by_bit31(v[r], eps[2u * g + r / 32] << (31 - r % 32));
        bfly<float, 0, 64>(v);
        bfly<float, 1, 64>(v);
        bfly<float, 2, 64>(v);
        bfly<float, 3, 64>(v);
        bfly<float, 4, 64>(v);
        bfly<float, 5, 64>(v);
    }
    const bool across = a.block > 6;
    if (across) {
        // in two halves, those of every LOW neighbours: half the LDS, twice the workgroups of a compute unit
        constexpr uint32_t HALF = LOW / 2;
#pragma unroll
        for (uint32_t part = 0; part < 2; ++part) {
            if (part) __syncthreads();
#pragma unroll
            for (uint32_t r = 0; r < 64; ++r)
                if (r % LOW / HALF == part) y[(g * 32u + r / LOW * HALF + r % HALF) * C + c] = v[r];
            __syncthreads();
#pragma unroll
            for (uint32_t h = 0; h < HI; ++h)
#pragma unroll
                for (uint32_t l = 0; l < HALF; ++l) v[h * LOW + part * HALF + l] = y[(h * 32u + g * HALF + l) * C + c];
        }
        static_for<LOGK - 6>([&](auto i) {
            if (a.block > 6u + decltype(i)::value) bfly<float, (LOGK == 8 ? 4 : 2) + decltype(i)::value, 64>(v);
        });
        at = g * LOW;
    }
    if constexpr (PASS == COLUMNS_MAX) {
        uint32_t m = 0;
#pragma unroll
        for (int r = 0; r < 64; ++r) m = m > magnitude(v[r]) ? m : magnitude(v[r]);
        if (m >= kInfinity) { // an infinity or a NaN of the column's own, or sums that left the range?
            const T *const x = static_cast<const T *>(a.x) + row;
            m = kInfinity;
#pragma unroll 8
            for (uint32_t k = kt + g * 64u; k < kt + g * 64u + 64u; ++k)
                if (magnitude(widen(x[(uint64_t)(k < a.len ? k : a.len - 1u) * a.ld])) >= kInfinity) m = kNotFinite;
        }
        if (in) atomicMax(reinterpret_cast<uint32_t *>(a.scales) + row, m);
    } else {
        if (!in) return;
        const RowFactor f = row_factor(__float_as_uint(a.scales[row]));
        if (f.up != 1.f)
#pragma unroll
            for (int r = 0; r < 64; ++r) v[r] *= f.up;
        const RngKey key{ a.k0, a.k1, kDomainRowDither, a.round_lo, a.party };
        // runs of neighbours: behind the exchange LOW of them, in front of it all 64; stored 16 (or 4) at a time
        constexpr uint32_t RUN = LOW < 16 ? LOW : 16;
#pragma unroll
        for (uint32_t r0 = 0; r0 < 64; r0 += RUN) {
            const uint32_t k = kt + (across ? at + r0 / LOW * 64u + r0 % LOW : at + r0);
            const uint64_t i0 = row * a.stride + k;
            uint32_t q[RUN / 4];
#pragma unroll
            for (uint32_t r = r0; r < r0 + RUN; r += 4) {
                const uint64_t i = i0 + (r - r0);
                uint32_t c[4];
                if (a.dither) {
                    uint32_t w[4];
                    philox((uint32_t)(i >> 3), key, w); // (the same call for two fours of a run: the compiler makes it once)
                    const uint32_t w0 = i & 4u ? w[2] : w[0], w1 = i & 4u ? w[3] : w[1];
                    c[0] = row_code(v[r], f.inv, half_dither_of(w0 & 0xFFFFu));
                    c[1] = row_code(v[r + 1], f.inv, half_dither_of(w0 >> 16));
                    c[2] = row_code(v[r + 2], f.inv, half_dither_of(w1 & 0xFFFFu));
                    c[3] = row_code(v[r + 3], f.inv, half_dither_of(w1 >> 16));
                } else {
#pragma unroll
                    for (int n = 0; n < 4; ++n) c[n] = row_code(v[r + n], f.inv);
                }
                q[(r - r0) / 4] = f.finite ? pack4(c[0], c[1], c[2], c[3]) : 0u;
            }
            if (k >= a.stride) continue;
            if constexpr (RUN == 16) *reinterpret_cast<uint4 *>(a.codes + i0) = make_uint4(q[0], q[1], q[2], q[3]);
            else *reinterpret_cast<uint32_t *>(a.codes + i0) = q[0];
        }
    }
}

__global__ __launch_bounds__(256) void k_columns_begin(float *scales, uint64_t rows)
{
    const uint64_t j = blockIdx.x * (uint64_t)256 + threadIdx.x;
    if (j < rows) scales[j] = 0.f;
}
// Maxima become amplitudes; columns whose transform left the range (kInfinity; kNotFinite is one with an infinity or a NaN) are coded here
constexpr uint32_t kColumnsEnd = 256; // columns of a workgroup, and its threads
template <typename T>
__global__ __launch_bounds__(kColumnsEnd) void k_columns_end(const RowsArgs a)
{
    __shared__ float y[1024];
    __shared__ uint32_t most[kColumnsEnd / 64], list[kColumnsEnd], listed;
    if (threadIdx.x == 0) listed = 0;
    __syncthreads();
    const uint64_t j = (uint64_t)blockIdx.x * kColumnsEnd + threadIdx.x;
    if (j < a.rows) {
        const uint32_t m = __float_as_uint(a.scales[j]);
        a.scales[j] = row_scale(m, a.unflatten);
        if (m == kInfinity) list[atomicAdd(&listed, 1u)] = threadIdx.x; // (each by itself, in any order)
    }
    __syncthreads();
    for (uint32_t i = 0; i < listed; ++i) {
        const uint64_t row = (uint64_t)blockIdx.x * kColumnsEnd + list[i];
        encode_lowered<T, kColumnsEnd>(a, static_cast<const T *>(a.x) + row, a.ld, row, y, most);
    }
}

} // namespace fo
