// 8-bit rows and their products (fo_rows_encode, fo_rows_product): argument checks, kernel choice, launches.
#include "fo_host.h"
#include "fo_product.h"
#include "fo_rows.h"

using namespace fo;
using namespace fo_host;

namespace {

struct RowsOut {
    const float *scales_q, *scales_p;
    void *out;
    uint64_t ld;
    uint32_t rows_q, rows_p;
};
template <typename T>
struct RowsEpilogue : RowsOut {
    template <int NQ, int NP>
    __device__ __forceinline__ void operator()(const TileAt &, uint32_t q, uint32_t p, const i32x4 (&acc)[NQ][NP]) const
    {
        constexpr int W = 16 / sizeof(T);
        constexpr int N = 4 * NP;
        typedef T V __attribute__((ext_vector_type(W)));
        if (p >= rows_p) return;
        float sp[N];
#pragma unroll
        for (int k = 0; k < N; ++k) sp[k] = scales_p[p + k < rows_p ? p + k : p];
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if (q + i >= rows_q) return;
            const float s = scales_q[q + i];
            T *const to = static_cast<T *>(out) + (q + i) * ld + p;
            T o[N];
#pragma unroll
            for (int k = 0; k < N; ++k) o[k] = (T)((float)acc[i][k / 4][k % 4] * s * sp[k]);
            if (N % W == 0 && p + N <= rows_p) {
#pragma unroll
                for (int k = 0; k + W <= N; k += W) {
                    V v;
#pragma unroll
                    for (int w = 0; w < W; ++w) v[w] = o[k + w];
                    __builtin_memcpy(to + k, &v, sizeof(v)); // (at any element)
                }
            } else {
#pragma unroll
                for (int k = 0; k < N; ++k)
                    if (p + k < rows_p) to[k] = o[k];
            }
        }
    }
};

// Few rows of Q (16 NQ at most): the bytes of P bound it, so every workgroup takes 16 rows of P, whose stages its eight waves share
// out among themselves and whose pieces go from memory into the registers they are needed in.  One token on weights of 4096 x 4096,
// 16.8 MB: 5.1 us, of which 3.3 at the rate of a large copy (tiles of 64 through LDS take 15 us for up to 512 tokens).
constexpr int kTogether = 4; // stages a wave loads at once: all of a row of 4096
template <int NQ, typename T>
__global__ __launch_bounds__(512) void k_product_few(const ProductArgs a, const RowsEpilogue<T> epi)
{
    __shared__ i32x4 part[8][NQ][64];
    const uint32_t lane = threadIdx.x & 63u, wave = threadIdx.x >> 6;
    const uint32_t p0 = blockIdx.x * 16u, r = lane & 15u;
    const char *const p = a.p + (uint64_t)(p0 + r < a.rows_p ? p0 + r : a.rows_p - 1u) * a.ld_p + (lane >> 4) * 16u;
    const char *q[NQ];
#pragma unroll
    for (int n = 0; n < NQ; ++n) q[n] = a.q + (uint64_t)(16u * n + r < a.rows_q ? 16u * n + r : a.rows_q - 1u) * a.ld_q + (lane >> 4) * 16u;
    i32x4 acc[NQ] = {};
    for (uint32_t s = wave; s < a.stages; s += 8u * kTogether) {
        i32x4 fp[kTogether][2], fq[kTogether][NQ][2];
#pragma unroll
        for (int u = 0; u < kTogether; ++u) { // behind the end: the last stage once more, times zero
            const uint32_t t = s + 8u * u;
            const uint64_t k = (uint64_t)(t < a.stages ? t : a.stages - 1u) * kStageBytes;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                fp[u][h] = *(const i32x4 *)(p + k + 64u * h);
#pragma unroll
                for (int n = 0; n < NQ; ++n) fq[u][n][h] = *(const i32x4 *)(q[n] + k + 64u * h);
            }
        }
#pragma unroll
        for (int u = 0; u < kTogether; ++u)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                if (s + 8u * u >= a.stages) fp[u][h] = i32x4{};
#pragma unroll
                for (int n = 0; n < NQ; ++n) acc[n] = OpI8::mfma(fp[u][h], fq[u][n][h], acc[n]);
            }
    }
#pragma unroll
    for (int n = 0; n < NQ; ++n) part[wave][n][lane] = acc[n];
    __syncthreads();
    if (wave < NQ) {
        i32x4 sum = part[0][wave][lane];
#pragma unroll
        for (int w = 1; w < 8; ++w) sum += part[w][wave][lane];
        const uint32_t row = 16u * wave + r, col = p0 + 4u * (lane >> 4);
        const i32x4 block[1][1] = { { sum } };
        epi(TileAt{}, row, col, block);
    }
}

bool launched(const char *what) { return hip_ok(hipGetLastError(), what); }

template <typename T>
int launch_rows_product(const ProductArgs &a, const RowsOut &o, hipStream_t st)
{
    RowsEpilogue<T> epi;
    static_cast<RowsOut &>(epi) = o;
    if (a.rows_q <= 32u) {
        const dim3 grid((a.rows_p + 15u) / 16u), block(512);
        if (a.rows_q <= 16u) hipLaunchKernelGGL((k_product_few<1, T>), grid, block, 0, st, a, epi);
        else hipLaunchKernelGGL((k_product_few<2, T>), grid, block, 0, st, a, epi);
        return launched("k_product_few") ? FO_OK : FO_EHIP;
    }
    launch_product<OpI8>(a, epi, st);
    return launched("k_product") ? FO_OK : FO_EHIP;
}

template <typename T>
int launch_rows_encode(const RowsArgs &a, bool transposed, hipStream_t st)
{
    if (transposed) {
        const unsigned n = (unsigned)((a.rows + 255u) / 256u);
        hipLaunchKernelGGL(k_columns_begin, dim3(n), dim3(256), 0, st, a.scales, a.rows);
        const bool far = a.block > 8;
        const uint64_t tiles = far ? (a.rows + 31u) / 32u * ((a.stride + 1023u) / 1024u) : (a.rows + 63u) / 64u * ((a.stride + 255u) / 256u);
        const dim3 grid((unsigned)tiles);
        if (far) {
            hipLaunchKernelGGL((k_columns_encode<T, 10, COLUMNS_MAX>), grid, dim3(512), 0, st, a);
            hipLaunchKernelGGL((k_columns_encode<T, 10, COLUMNS_CODES>), grid, dim3(512), 0, st, a);
        } else {
            hipLaunchKernelGGL((k_columns_encode<T, 8, COLUMNS_MAX>), grid, dim3(256), 0, st, a);
            hipLaunchKernelGGL((k_columns_encode<T, 8, COLUMNS_CODES>), grid, dim3(256), 0, st, a);
        }
        hipLaunchKernelGGL((k_columns_end<T>), dim3((unsigned)((a.rows + kColumnsEnd - 1u) / kColumnsEnd)), dim3(kColumnsEnd), 0, st, a);
        return launched("k_columns_encode") ? FO_OK : FO_EHIP;
    }
    const uint32_t segments = (a.stride + kRowSegment - 1u) / kRowSegment;
    // eight waves a SIMD at most, so that the sign flips are drawn for several rows
    auto grid = [&](uint32_t waves) { return dim3((unsigned)(a.rows < 8192u / waves ? a.rows : 8192u / waves)); };
    if (segments <= 1u) hipLaunchKernelGGL((k_rows_encode<T, 1, true>), grid(1), dim3(64), 0, st, a);
    else if (segments <= 4u) hipLaunchKernelGGL((k_rows_encode<T, 4, true>), grid(4), dim3(256), 0, st, a);
    else if (segments <= 8u) hipLaunchKernelGGL((k_rows_encode<T, 8, true>), grid(8), dim3(512), 0, st, a);
    else if (segments <= 16u) hipLaunchKernelGGL((k_rows_encode<T, 16, true>), grid(16), dim3(1024), 0, st, a);
    else hipLaunchKernelGGL((k_rows_encode<T, 16, false>), grid(16), dim3(1024), 0, st, a);
    return launched("k_rows_encode") ? FO_OK : FO_EHIP;
}

// A launch has at most 2^32 threads: 32 for every row of P in k_product_few, one for 64 codes or outputs in the others
constexpr uint64_t kMostRows = (uint64_t)1 << 26, kMost = (uint64_t)1 << 37;
uint32_t element_bytes(uint32_t type) { return type == FO_F32 ? 4u : 2u; }

} // namespace

extern "C" size_t fo_rows_stride(uint64_t len, uint32_t block_log2)
{
    if (len < 1 || len > FO_MAX_ROW || (block_log2 != 0 && (block_log2 < 6 || block_log2 > 10))) return 0;
    const uint64_t unit = block_log2 > 7 ? (uint64_t)1 << block_log2 : 128u;
    return (size_t)((len + unit - 1u) / unit * unit);
}

extern "C" int fo_rows_encode(const fo_rows_params *q, const void *x, uint64_t round, uint32_t party, int8_t *codes, float *scales,
                              void *hip_stream)
{
    if (!q || !x || !codes || !scales) return FO_EINVAL;
    const uint64_t stride = fo_rows_stride(q->len, q->block_log2);
    if (!stride || q->rows < 1 || q->rows > kMostRows || q->type > FO_F16 || q->transposed > 1u) return FO_EINVAL;
    if (q->dither != FO_DITHER_UNIFORM && q->dither != FO_DITHER_NONE) return FO_EINVAL;
    if (q->ld < (q->transposed ? q->rows : q->len) || q->ld > ((uint64_t)1 << 40)) return FO_EINVAL;
    if (q->rows * stride > kMost) return FO_EINVAL;
    if (q->dither == FO_DITHER_UNIFORM && q->rows * stride > ((uint64_t)1 << 35)) return FO_EINVAL; // the generator's 32-bit counter
    if (!aligned(x, element_bytes(q->type)) || !aligned(codes, 16) || !aligned(scales, 4)) return FO_EALIGN;
    RowsArgs a;
    std::memset(&a, 0, sizeof(a));
    a.x = x;
    a.ld = q->ld;
    a.rows = q->rows;
    a.len = (uint32_t)q->len;
    a.stride = (uint32_t)stride;
    a.block = q->block_log2;
    a.dither = q->dither == FO_DITHER_UNIFORM;
    a.k0 = (uint32_t)q->seed;
    a.k1 = (uint32_t)(q->seed >> 32) ^ (uint32_t)(round >> 32);
    a.round_lo = (uint32_t)round;
    a.eps_party = kPartyAllWorkers;
    a.party = party;
    a.unflatten = (float)std::exp2(-0.5 * (double)q->block_log2);
    a.codes = codes;
    a.scales = scales;
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (q->type == FO_F32) return launch_rows_encode<float>(a, q->transposed, st);
    if (q->type == FO_BF16) return launch_rows_encode<uint16_t>(a, q->transposed, st);
    return launch_rows_encode<_Float16>(a, q->transposed, st);
}

extern "C" int fo_rows_product(const int8_t *a, const float *scales_a, uint64_t rows_a, const int8_t *b, const float *scales_b,
                               uint64_t rows_b, uint64_t stride, void *out, uint32_t type, uint64_t ld_out, void *hip_stream)
{
    if (!a || !scales_a || !b || !scales_b || !out) return FO_EINVAL;
    if (rows_a < 1 || rows_a > kMostRows || rows_b < 1 || rows_b > kMostRows || type > FO_F16) return FO_EINVAL;
    if (stride < kStageBytes || stride > FO_MAX_ROW || stride % kStageBytes || ld_out < rows_b || ld_out > ((uint64_t)1 << 40)) return FO_EINVAL;
    if (rows_a * rows_b > kMost) return FO_EINVAL;
    const uint32_t size = element_bytes(type);
    if (!aligned(a, 16) || !aligned(b, 16) || !aligned(scales_a, 4) || !aligned(scales_b, 4) || !aligned(out, size)) return FO_EALIGN;
    ProductArgs p;
    std::memset(&p, 0, sizeof(p));
    p.q = reinterpret_cast<const char *>(a);
    p.p = reinterpret_cast<const char *>(b);
    p.ld_q = p.ld_p = stride;
    p.rows_q = (uint32_t)rows_a;
    p.rows_p = (uint32_t)rows_b;
    p.stages = (uint32_t)(stride / kStageBytes);
    p.count = 1;
    const RowsOut o{ scales_a, scales_b, out, ld_out, (uint32_t)rows_a, (uint32_t)rows_b };
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (type == FO_F32) return launch_rows_product<float>(p, o, st);
    if (type == FO_BF16) return launch_rows_product<__bf16>(p, o, st);
    return launch_rows_product<_Float16>(p, o, st);
}
