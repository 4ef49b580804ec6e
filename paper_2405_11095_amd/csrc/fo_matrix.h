// Kernels around the products of fo_orthogonalize and fo_matrix_step: momentum and norm, the first iterate, and what happens to
// the outputs of the three products of a Newton-Schulz step.
//
// Iterates live in scratch in fp16 scaled by 2^12, in one part (HALF) or two (SINGLE: the second holds what the first's rounding
// lost), with sides padded to multiples of 64 by zeros, which every step keeps.  X has the shorter side m as its rows (so it is the
// transpose of a matrix that is taller than wide); A = X X^T sums along its rows, X <- B X with B = a I + b A + c A^2 down its
// columns.  (Adding a X in fp32 instead, behind the product, is no more exact, and has to read X once more.)  Entries stay below the spectral norm, about 1.2, far from fp16's 16 x 2^12, and 2^12 keeps the small ones
// normal: those of X = G / ||G||_F are about 2^-12 for 4096 x 4096.  One part's roundings, 2^-12 of an entry each, come to 1e-3 of the result for
// large well conditioned updates (4096 x 4096), less than rounding it to bf16 costs (1.66e-3), which is what one part is meant for.
#pragma once
#include "fo_product.h"

namespace fo {

constexpr float kUp = 4096.f, kDown = 1.f / 4096.f;

struct MatrixTab {
    void *p[kMatrices];
};

template <typename T>
__device__ __forceinline__ float to_float(T v) { return (float)v; }

struct Parts {
    _Float16 hi, lo;
};
__device__ __forceinline__ Parts split(float v) // v already scaled
{
    Parts r;
    r.hi = (_Float16)v;
    r.lo = (_Float16)(v - (float)r.hi);
    return r;
}

// N neighbouring elements at any element, of which n (1 at least) are there, and their values, zero from the n-th on.  Apart, so
// that loads can be on their way together.
template <typename T, int N>
struct Some {
    T w[N];
    __device__ __forceinline__ void load(const T *p, uint64_t n)
    {
        if (n >= (uint64_t)N) {
            __builtin_memcpy(w, p, sizeof(w));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i) w[i] = p[(uint64_t)i < n ? i : 0];
        }
    }
    __device__ __forceinline__ void store(T *p, uint64_t n) const
    {
        if (n >= (uint64_t)N) {
            __builtin_memcpy(p, w, sizeof(w));
        } else {
#pragma unroll
            for (int i = 0; i < N; ++i)
                if ((uint64_t)i < n) p[i] = w[i];
        }
    }
    __device__ __forceinline__ float value(int i, uint64_t n) const { return (uint64_t)i < n ? to_float(w[i]) : 0.f; }
};
// Whole rows pass through in units of two vectors of 16 bytes a thread, each neighbour to its neighbour's (32 bytes in one thread
// instead: momentum of 8 of 1024 x 4096 in 159 us, so 95, 4.2 TB/s); element of vector h of this thread
constexpr uint32_t kUnit = 512; // vectors
template <typename T>
constexpr uint32_t kVector = 16 / sizeof(T);
template <typename T>
__device__ __forceinline__ uint64_t element_of(uint64_t unit, int h) { return (unit * kUnit + 256u * h + threadIdx.x) * kVector<T>; }

struct NormArgs {
    MatrixTab g;
    uint64_t rows, cols, ld; // a contiguous matrix comes as one row
    double *partials;        // [count][gridDim.x]
};

__device__ __forceinline__ void block_partial(double s, double *to)
{
    __shared__ double part[4];
    s = wave_sum(s, 6);
    if ((threadIdx.x & 63u) == 0u) part[threadIdx.x >> 6] = s;
    __syncthreads();
    if (threadIdx.x == 0) *to = part[0] + part[1] + part[2] + part[3];
}

// Sums of squares, in fp64: squares of fp32 neither overflow nor vanish there
template <typename T>
__global__ __launch_bounds__(256) void k_matrix_norm(const NormArgs a)
{
    const T *const g = static_cast<const T *>(a.g.p[blockIdx.y]);
    constexpr uint32_t V = kVector<T>, U = kUnit * V;
    const uint64_t per = (a.cols + U - 1u) / U, units = a.rows * per;
    double s = 0.0;
    for (uint64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const uint64_t r = u / per;
        Some<T, V> w[2];
        uint64_t n[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint64_t c = element_of<T>(u - r * per, h);
            n[h] = c < a.cols ? a.cols - c : 0u;
            if (n[h]) w[h].load(g + r * a.ld + c, n[h]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
            for (uint32_t i = 0; i < V; ++i) s = fma((double)w[h].value(i, n[h]), (double)w[h].value(i, n[h]), s);
    }
    block_partial(s, a.partials + (uint64_t)blockIdx.y * gridDim.x + blockIdx.x);
}

struct MomentumArgs {
    MatrixTab g, m;
    uint64_t n; // elements of a matrix
    float mu;
    uint32_t nesterov;
    double *partials;
};
__device__ __forceinline__ float momentum_update(float g, float m, const float mu, const bool nesterov) { return nesterov ? fmaf(mu, m, g) : m; }

// m <- mu m + g, and the sum of squares of what is orthogonalised
__global__ __launch_bounds__(256) void k_matrix_momentum(const MomentumArgs a)
{
    const float *const g = static_cast<const float *>(a.g.p[blockIdx.y]);
    float *const m = static_cast<float *>(a.m.p[blockIdx.y]);
    double s = 0.0;
    constexpr uint32_t V = kVector<float>, U = kUnit * V;
    for (uint64_t u = blockIdx.x; u < (a.n + U - 1u) / U; u += gridDim.x) {
        Some<float, V> gv[2], mv[2];
        uint64_t n[2];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint64_t i = element_of<float>(u, h);
            n[h] = i < a.n ? a.n - i : 0u;
            if (!n[h]) continue;
            gv[h].load(g + i, n[h]);
            mv[h].load(m + i, n[h]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (uint32_t k = 0; k < V; ++k) {
                const float gk = gv[h].value(k, n[h]);
                mv[h].w[k] = fmaf(a.mu, mv[h].value(k, n[h]), gk);
                const double x = (double)momentum_update(gk, mv[h].w[k], a.mu, a.nesterov);
                s = fma(x, x, s);
            }
            if (n[h]) mv[h].store(m + element_of<float>(u, h), n[h]);
        }
    }
    block_partial(s, a.partials + (uint64_t)blockIdx.y * gridDim.x + blockIdx.x);
}

// What takes a matrix with this sum of squares to X_0, scaled: m 2^e, as much of it in m as fits (a subnormal v stays exact: |v m| is
// 2^12 at most, and no smaller than |v|'s share of that while e = 0).  Zero stays zero, an infinity or a NaN spoils every entry.
// (A product in fp64 for every element instead: the conversions take most of the kernel, 22 us for 12 of 1024 x 1024, now 11.)
struct FirstFactor {
    float m;
    int e;
    __device__ __forceinline__ explicit FirstFactor(double sum)
    {
        const double f = sum > 0.0 ? (sum < __builtin_inf() ? (double)kUp / sqrt(sum) : __builtin_nan("")) : sum == 0.0 ? 0.0 : __builtin_nan("");
        e = f == f ? __builtin_amdgcn_frexp_exp(f) : 0;
        const int in_m = e > 120 ? 120 : e < -120 ? -120 : e;
        e -= in_m;
        m = __builtin_amdgcn_ldexpf((float)__builtin_amdgcn_frexp_mant(f), in_m);
    }
    __device__ __forceinline__ float operator()(float v) const { return __builtin_amdgcn_ldexpf(v * m, e); }
};

struct BeginArgs {
    MatrixTab g, m;     // m: fo_matrix_step's new momentum
    uint64_t rows, cols, ld;
    float mu;
    uint32_t nesterov, momentum; // momentum: the matrix is formed from g and m
    const double *partials;
    uint32_t nparts;
    uint32_t parts;     // 1 or 2
    uint32_t rows64, cols64; // padded sides
    _Float16 *x;        // [rows64][cols64] of the first matrix; TALL: [cols64][rows64]
    uint64_t part, next; // elements from part to part, matrix to matrix
};

// X_0 = G / ||G||_F, or its transpose, a square of 64 by 64 a workgroup
template <typename T, bool TALL>
__global__ __launch_bounds__(256) void k_matrix_begin(const BeginArgs a)
{
    __shared__ float tile[64][65];
    __shared__ double part[4];
    const uint32_t t = threadIdx.x, lane = t & 63u, wave = t >> 6;
    const uint32_t across = a.cols64 / 64u;
    const uint32_t r0 = blockIdx.x / across * 64u, c0 = blockIdx.x % across * 64u;
    const uint32_t tr = t >> 3, tc = (t & 7u) * 8u; // a thread's eights: rows tr and tr + 32
    const T *const g = static_cast<const T *>(a.g.p[blockIdx.y]);
    const float *const m = static_cast<const float *>(a.m.p[blockIdx.y]);
    float v[2][8] = {};
    {
        Some<T, 8> gv[2] = {};
        Some<float, 8> mv[2] = {};
        auto elements = [&](auto whole) { // (all loads on their way before the first is waited for)
            constexpr bool W = decltype(whole)::value;
            uint64_t n[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint64_t r = r0 + tr + 32u * h, c = c0 + tc, k = r * a.ld + c;
                n[h] = W ? 8u : r < a.rows && c < a.cols ? a.cols - c : 0u;
                if (!n[h]) continue;
                if (!a.momentum || a.nesterov) gv[h].load(g + k, n[h]);
                if (a.momentum) mv[h].load(m + k, n[h]);
            }
#pragma unroll
            for (int h = 0; h < 2; ++h)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    v[h][i] = a.momentum ? momentum_update(gv[h].value(i, n[h]), mv[h].value(i, n[h]), a.mu, a.nesterov) : gv[h].value(i, n[h]);
        };
        if (r0 + 64u <= a.rows && c0 + 64u <= a.cols) elements(std::true_type{});
        else elements(std::false_type{});
    }
    {
        double s = 0.0;
        for (uint32_t i = t; i < a.nparts; i += 256u) s += a.partials[(uint64_t)blockIdx.y * a.nparts + i];
        s = wave_sum(s, 6);
        if (lane == 0) part[wave] = s;
    }
    __syncthreads();
    const FirstFactor factor(part[0] + part[1] + part[2] + part[3]);
    _Float16 *const x = a.x + blockIdx.y * a.next;
    auto store = [&](_Float16 *to, const float (&w)[8]) {
        f16x8 hi, lo;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const Parts p = split(w[i]);
            hi[i] = p.hi;
            lo[i] = p.lo;
        }
        *reinterpret_cast<f16x8 *>(to) = hi;
        if (a.parts == 2u) *reinterpret_cast<f16x8 *>(to + a.part) = lo;
    };
#pragma unroll
    for (int h = 0; h < 2; ++h) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[h][i] = factor(v[h][i]);
            if constexpr (TALL) tile[tr + 32u * h][tc + i] = v[h][i];
        }
        if constexpr (!TALL) store(x + (uint64_t)(r0 + tr + 32u * h) * a.cols64 + c0 + tc, v[h]);
    }
    if constexpr (TALL) {
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            float w[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) w[i] = tile[tc + i][tr + 32u * h];
            store(x + (uint64_t)(c0 + tr + 32u * h) * a.rows64 + r0 + tc, w);
        }
    }
}

// ---- what happens to the outputs of the products -------------------------------------------------------------------------------

// A matrix of iterates: `parts` parts of fp16, rows of ld elements.  Sides are multiples of 64, so that a lane's block lies inside
// or outside as a whole, but for three rows (TileLarge).
template <int N>
__device__ __forceinline__ void read_half(const _Float16 *p, float (&v)[N]) // N neighbours
{
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        const f32x4 x = __builtin_convertvector(*reinterpret_cast<const f16x4 *>(p + i), f32x4);
#pragma unroll
        for (int k = 0; k < 4; ++k) v[i + k] += x[k];
    }
}
struct Iterate {
    _Float16 *x;
    uint64_t ld, part, next;
    template <bool TWO, int N>
    __device__ __forceinline__ void read(uint32_t matrix, uint32_t r, uint32_t c, float (&v)[N]) const
    {
        const _Float16 *const p = x + matrix * next + r * ld + c;
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = 0.f;
        read_half(p, v);
        if constexpr (TWO) read_half(p + part, v);
    }
    template <bool TWO, int N>
    __device__ __forceinline__ void write(uint32_t matrix, uint32_t r, uint32_t c, const float (&v)[N]) const
    {
        typedef _Float16 V __attribute__((ext_vector_type(N < 8 ? N : 8)));
        constexpr int W = N < 8 ? N : 8;
        _Float16 *const p = x + matrix * next + r * ld + c;
#pragma unroll
        for (int i = 0; i < N; i += W) {
            V hi, lo;
#pragma unroll
            for (int k = 0; k < W; ++k) {
                const Parts s = split(v[i + k]);
                hi[k] = s.hi;
                lo[k] = s.lo;
            }
            *reinterpret_cast<V *>(p + i) = hi;
            if constexpr (TWO) *reinterpret_cast<V *>(p + i + part) = lo;
        }
    }
    // columns c .. c + NQ - 1 of rows r .. r + 4 NP - 1, from v[column][row]; n of the columns are there
    template <bool TWO, int NQ, int NR>
    __device__ __forceinline__ void write_turned(uint32_t matrix, uint32_t r, uint32_t c, const float (&v)[NQ][NR], uint32_t n) const
    {
#pragma unroll
        for (int k = 0; k < NR; ++k) {
            float w[NQ];
#pragma unroll
            for (int i = 0; i < NQ; ++i) w[i] = v[i][k];
            if constexpr (64 % NQ == 0) {
                write<TWO>(matrix, r + k, c, w);
            } else {
                static_assert(!TWO, "one part");
                _Float16 *const p = x + matrix * next + (r + k) * ld + c;
                if (n >= (uint32_t)NQ) {
                    _Float16 h[NQ];
#pragma unroll
                    for (int i = 0; i < NQ; ++i) h[i] = (_Float16)w[i];
                    __builtin_memcpy(p, h, sizeof(h));
                } else {
#pragma unroll
                    for (int i = 0; i < NQ; ++i)
                        if ((uint32_t)i < n) p[i] = (_Float16)w[i];
                }
            }
        }
    }
};

// A = X X^T
template <bool TWO>
struct GramEpilogue {
    static constexpr bool sums_longer_than_sides = true;
    Iterate a;
    uint32_t side;
    template <int NQ, int NP>
    __device__ __forceinline__ void operator()(const TileAt &at, uint32_t q, uint32_t p, const f32x4 (&acc)[NQ][NP]) const
    {
        if (q >= side || p >= side) return;
        float v[NQ][4 * NP];
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if (64 % NQ != 0 && q + i >= side) continue;
#pragma unroll
            for (int k = 0; k < 4 * NP; ++k) v[i][k] = acc[i][k / 4][k % 4] * kDown;
            a.write<TWO>(at.matrix, q + i, p, v[i]);
        }
        if (at.q != at.p) a.write_turned<TWO>(at.matrix, p, q, v, side - q);
    }
};
// An entry of B = a I + b A + c A^2, the terms that cancel first, one rounding each (in fp64 hardly closer, 1.3 us a product slower)
__device__ __forceinline__ float polynomial(float a, float square, float ka, float kb, float kc, bool diagonal)
{
    return fmaf(kc, square, fmaf(kb, a, diagonal ? ka : 0.f));
}
// B = a I + b A + c A^2
template <bool TWO>
struct PolyEpilogue {
    static constexpr bool sums_longer_than_sides = false;
    Iterate a, b;
    uint32_t side;
    float ka, kb, kc; // ka times 2^12, kc times 2^-12
    template <int NQ, int NP>
    __device__ __forceinline__ void operator()(const TileAt &at, uint32_t q, uint32_t p, const f32x4 (&acc)[NQ][NP]) const
    {
        if (q >= side || p >= side) return;
        float v[NQ][4 * NP];
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            if (64 % NQ != 0 && q + i >= side) continue;
            a.read<TWO>(at.matrix, q + i, p, v[i]);
#pragma unroll
            for (int k = 0; k < 4 * NP; ++k) v[i][k] = polynomial(v[i][k], acc[i][k / 4][k % 4], ka, kb, kc, q + i == p + k);
            b.write<TWO>(at.matrix, q + i, p, v[i]);
        }
        if (at.q != at.p) b.write_turned<TWO>(at.matrix, p, q, v, side - q);
    }
};
// X <- B X
template <bool TWO>
struct UpdateEpilogue {
    static constexpr bool sums_longer_than_sides = false;
    Iterate to;
    uint32_t rows, cols;
    template <int NQ, int NP>
    __device__ __forceinline__ void operator()(const TileAt &at, uint32_t q, uint32_t p, const f32x4 (&acc)[NQ][NP]) const
    {
        if (q >= rows || p >= cols) return;
#pragma unroll
        for (int i = 0; i < NQ; ++i) {
            float v[4 * NP];
#pragma unroll
            for (int k = 0; k < 4 * NP; ++k) v[k] = kDown * acc[i][k / 4][k % 4];
            to.write<TWO>(at.matrix, q + i, p, v);
        }
    }
};
// The last step's, into the caller's matrices, rows x cols, or turned where these are taller than wide: out = O, or x <- keep x - by O
template <typename T, bool STEP, bool TALL>
struct LastEpilogue {
    static constexpr bool sums_longer_than_sides = false;
    MatrixTab out;
    uint64_t ld;
    uint32_t rows, cols; // of X without padding
    float keep, by;
    template <int N>
    __device__ __forceinline__ void store(T *to, const float (&v)[N], uint32_t n) const // n of the N neighbours
    {
        constexpr int W = N * sizeof(T) < 16 ? N : 16 / sizeof(T);
        typedef T V __attribute__((ext_vector_type(W)));
        if (n >= (uint32_t)N) { // (vectors at any element)
#pragma unroll
            for (int k = 0; k < N; k += W) {
                V o;
                if constexpr (STEP) __builtin_memcpy(&o, to + k, sizeof(o));
#pragma unroll
                for (int w = 0; w < W; ++w) o[w] = (T)(STEP ? keep * to_float(o[w]) - by * v[k + w] : v[k + w]);
                __builtin_memcpy(to + k, &o, sizeof(o));
            }
        } else {
#pragma unroll
            for (int k = 0; k < N; ++k)
                if ((uint32_t)k < n) to[k] = (T)(STEP ? keep * to_float(to[k]) - by * v[k] : v[k]);
        }
    }
    template <int NQ, int NP>
    __device__ __forceinline__ void operator()(const TileAt &at, uint32_t q, uint32_t p, const f32x4 (&acc)[NQ][NP]) const
    {
        if (q >= rows || p >= cols) return;
        T *const to = static_cast<T *>(out.p[at.matrix]);
        if constexpr (!TALL) {
#pragma unroll
            for (int i = 0; i < NQ; ++i) {
                float v[4 * NP];
#pragma unroll
                for (int k = 0; k < 4 * NP; ++k) v[k] = acc[i][k / 4][k % 4] * (kDown * kDown);
                if (q + i < rows) store(to + (uint64_t)(q + i) * ld + p, v, cols - p);
            }
        } else {
#pragma unroll
            for (int k = 0; k < 4 * NP; ++k) {
                float v[NQ];
#pragma unroll
                for (int i = 0; i < NQ; ++i) v[i] = acc[i][k / 4][k % 4] * (kDown * kDown);
                if (p + k < cols) store(to + (uint64_t)(p + k) * ld + q, v, rows - q);
            }
        }
    }
};

// ---- matrices of at most 128 x 128 --------------------------------------------------------------------------------------------
// One workgroup does everything: momentum, norm and all steps, X and A (or B) in LDS, sides padded to multiples of 32.  Outputs go
// round the eight waves in blocks of 32 x 32, those of A and B on and above the diagonal only.  (Launch by launch 128 x 96 in two
// parts takes 17 launches, 72 us, nearly all of it latency.)
//
// Rows of 128 in LDS, 256 bytes, 16-byte piece c of row r at piece c ^ spread(r): the 16 rows of a fragment and the eight rows
// (r & 3, r & 8) of a transposing load, 32 bytes each, meet no bank twice.
struct SmallArgs {
    MatrixTab g, m, out; // m: fo_matrix_step's momentum
    uint64_t ld_g, ld_out;
    uint32_t rows, cols; // as the caller has them
    uint32_t steps;
    float ka, kb, kc;    // as in PolyEpilogue
    float mu, keep, by;
    uint32_t nesterov;
};

template <typename T, bool STEP, bool TWO>
__global__ __launch_bounds__(512) void k_matrix_small(const SmallArgs a)
{
    typedef std::conditional_t<STEP, float, T> G;
    constexpr uint32_t SIDE = 128, kPart = SIDE * SIDE * 2u, kMatrix = kPart * (TWO ? 2u : 1u); // bytes
    __shared__ __align__(16) char lds[2 * kMatrix];
    __shared__ double part[8];
    const uint32_t t = threadIdx.x, lane = t & 63u, wave = t >> 6;
    const bool tall = a.rows > a.cols;
    const uint32_t side_m = tall ? a.cols : a.rows, side_n = tall ? a.rows : a.cols;
    const uint32_t blocks_m = (side_m + 31u) / 32u, blocks_n = (side_n + 31u) / 32u;
    constexpr uint32_t X = 0, A = kMatrix;
    auto spread = [](uint32_t r) { return (r & 3u) << 1 | (r & 8u) | (r >> 2 & 1u); };
    auto at = [&](uint32_t r, uint32_t c) { return r * 256u + (((c >> 3) ^ spread(r)) << 4) + (c & 7u) * 2u; }; // bytes, of element (r, c)

    // momentum and norm: a thread's columns lane and lane + 64 of every eighth row
    float v[16][2];
    double s = 0.0;
    {
        const G *const g = static_cast<const G *>(a.g.p[blockIdx.x]);
        float *const m = static_cast<float *>(a.m.p[blockIdx.x]);
        // (all on their way before the first is waited for; outside the matrix, its first element and zero in its place)
        G gv[16][2];
        float mv[16][2] = {};
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t r = wave + 8u * i, c = lane + 64u * h;
                const uint64_t k = r < a.rows && c < a.cols ? r * a.ld_g + c : 0u;
                gv[i][h] = g[k];
                if constexpr (STEP) mv[i][h] = m[k];
            }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < 16; ++i)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t r = wave + 8u * i, c = lane + 64u * h;
                const bool in = r < a.rows && c < a.cols;
                float x = to_float(gv[i][h]);
                if constexpr (STEP) {
                    const float mi = fmaf(a.mu, mv[i][h], x);
                    if (in) m[r * a.ld_g + c] = mi;
                    x = momentum_update(x, mi, a.mu, a.nesterov);
                }
                v[i][h] = x = in ? x : 0.f;
                s = fma((double)x, (double)x, s);
            }
        s = wave_sum(s, 6);
        if (lane == 0) part[wave] = s;
    }
    __syncthreads();
    const double sum = ((part[0] + part[1]) + (part[2] + part[3])) + ((part[4] + part[5]) + (part[6] + part[7]));
    const FirstFactor factor(sum);
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t r = wave + 8u * i, c = lane + 64u * h;
            const Parts p = split(factor(v[i][h]));
            const uint32_t to = X + (tall ? at(c, r) : at(r, c));
            *reinterpret_cast<_Float16 *>(lds + to) = p.hi;
            if constexpr (TWO) *reinterpret_cast<_Float16 *>(lds + to + kPart) = p.lo;
        }
    __syncthreads();

    // Block (bq, bp) = rows of Q with rows (turned: columns) of P over 32 `steps` coordinates.  Fragments of the next 32 are read
    // while those at hand are multiplied.
    const uint32_t l = lane & 15u, grp = lane >> 4;
    constexpr int parts = TWO ? 2 : 1;
    struct Fragments {
        i32x4 q[parts][2], p[parts][2];
    };
    const uint32_t by_rows = l * 256u + ((grp ^ spread(l)) << 4);                       // row l, coordinates 8 grp ..
    const uint32_t k8 = 8u * grp + (lane >> 2 & 3u);                                    // turned: rows k8 and k8 + 4, columns 4 (lane & 3) ..
    const uint32_t by_columns = k8 * 256u + (((lane & 3u) >> 1 ^ spread(k8 & 15u)) << 4) + (lane & 1u) * 8u;
    auto read = [&](Fragments &f, uint32_t Q, uint32_t bq, uint32_t P, uint32_t bp, auto turned, uint32_t k) {
#pragma unroll
        for (int n = 0; n < parts; ++n)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                f.q[n][i] = *reinterpret_cast<const i32x4 *>(lds + Q + n * kPart + bq * 8192u + (by_rows ^ k * 64u) + i * 4096u);
                if constexpr (decltype(turned)::value) {
                    typedef short s16x4 __attribute__((ext_vector_type(4)));
                    const uint32_t x = P + n * kPart + k * 8192u + (by_columns ^ (bp * 64u + i * 32u));
                    const s16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(lds + x));
                    const s16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4 *)(lds + ((x ^ 16u) + 1024u)));
                    f.p[n][i] = __builtin_bit_cast(i32x4, __builtin_shufflevector(x0, x1, 0, 1, 2, 3, 4, 5, 6, 7));
                } else {
                    f.p[n][i] = *reinterpret_cast<const i32x4 *>(lds + P + n * kPart + bp * 8192u + (by_rows ^ k * 64u) + i * 4096u);
                }
            }
    };
    auto multiply = [&](f32x4 (&acc)[2][2], f32x4 (&low)[2][2], const Fragments &f) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                acc[i][j] = OpF16::mfma(f.p[0][j], f.q[0][i], acc[i][j]);
                if constexpr (TWO) { // the products with second parts
                    low[i][j] = OpF16::mfma(f.p[1][j], f.q[1][i], low[i][j]);
                    low[i][j] = OpF16::mfma(f.p[1][j], f.q[0][i], low[i][j]);
                    low[i][j] = OpF16::mfma(f.p[0][j], f.q[1][i], low[i][j]);
                }
            }
    };
    auto product = [&](f32x4 (&sum)[2][2], uint32_t Q, uint32_t bq, uint32_t P, uint32_t bp, auto turned, uint32_t steps) {
        f32x4 acc[2][2] = {}, low[2][2] = {};
        auto add = [&](f32x4 (&from)[2][2], bool first) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    sum[i][j] = first ? from[i][j] : sum[i][j] + from[i][j];
                    from[i][j] = f32x4{};
                }
        };
        Fragments f0, f1;
        read(f0, Q, bq, P, bp, turned, 0);
        for (uint32_t k = 0; k < steps; k += 2u) { // (behind the last 32 coordinates: the last ones again, not used)
            read(f1, Q, bq, P, bp, turned, k + 1u < steps ? k + 1u : k);
            multiply(acc, low, f0);
            read(f0, Q, bq, P, bp, turned, k + 2u < steps ? k + 2u : k);
            if (k + 1u < steps) multiply(acc, low, f1);
            if constexpr (TWO) add(acc, k == 0u); // as EXACT in k_product: sums start anew every 64 coordinates
        }
        if constexpr (TWO) add(low, false);
        else add(acc, true);
    };
    // outputs (32 bq + 16 i + l, 32 bp + 16 j + 4 grp ..) to rows of LDS, and to their mirror images'
    auto put = [&](uint32_t M, uint32_t bq, uint32_t bp, const f32x4 (&acc)[2][2], bool mirrored) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const uint32_t q = 32u * bq + 16u * i + l, p = 32u * bp + 16u * j + 4u * grp;
                const f16x4 hi = __builtin_convertvector(acc[i][j], f16x4);
                const f16x4 lo = __builtin_convertvector(acc[i][j] - __builtin_convertvector(hi, f32x4), f16x4);
                *reinterpret_cast<f16x4 *>(lds + M + at(q, p)) = hi;
                if constexpr (TWO) *reinterpret_cast<f16x4 *>(lds + M + kPart + at(q, p)) = lo;
                if (mirrored)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        *reinterpret_cast<_Float16 *>(lds + M + at(p + k, q)) = hi[k];
                        if constexpr (TWO) *reinterpret_cast<_Float16 *>(lds + M + kPart + at(p + k, q)) = lo[k];
                    }
            }
    };
    constexpr std::false_type rows_of{};
    constexpr std::true_type columns_of{};
    // a wave's blocks: the upper triangle has at most 10, X at most 16
    const uint32_t triangle = blocks_m * (blocks_m + 1u) / 2u;
    auto upper = [&](uint32_t n, uint32_t &bq, uint32_t &bp) {
        bq = 0;
        while (n >= blocks_m - bq) n -= blocks_m - bq++;
        bp = bq + n;
    };
    f32x4 acc[2][2][2];
    for (uint32_t step = 0; step < a.steps; ++step) {
        for (uint32_t n = wave; n < triangle; n += 8u) { // A = X X^T
            uint32_t bq, bp;
            upper(n, bq, bp);
            product(acc[0], X, bq, X, bp, rows_of, blocks_n);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[0][i][j] *= kDown;
            put(A, bq, bp, acc[0], bq != bp);
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) { // B = a I + b A + c A^2
            const uint32_t n = wave + 8u * h;
            if (n >= triangle) continue;
            uint32_t bq, bp;
            upper(n, bq, bp);
            product(acc[h], A, bq, A, bp, rows_of, blocks_m);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    const uint32_t q = 32u * bq + 16u * i + l, p = 32u * bp + 16u * j + 4u * grp;
                    f32x4 x = __builtin_convertvector(*reinterpret_cast<const f16x4 *>(lds + A + at(q, p)), f32x4);
                    if constexpr (TWO) x += __builtin_convertvector(*reinterpret_cast<const f16x4 *>(lds + A + kPart + at(q, p)), f32x4);
#pragma unroll
                    for (int k = 0; k < 4; ++k) acc[h][i][j][k] = polynomial(x[k], acc[h][i][j][k], a.ka, a.kb, a.kc, q == p + k);
                }
        }
        __syncthreads(); // everybody has read A
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t n = wave + 8u * h;
            if (n >= triangle) continue;
            uint32_t bq, bp;
            upper(n, bq, bp);
            put(A, bq, bp, acc[h], bq != bp);
        }
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) { // X <- B X
            const uint32_t n = wave + 8u * h;
            if (n < blocks_m * blocks_n) product(acc[h], A, n / blocks_n, X, n % blocks_n, columns_of, blocks_m);
        }
        __syncthreads(); // everybody has read X
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const uint32_t n = wave + 8u * h, bq = n / blocks_n, bp = n % blocks_n;
            if (n >= blocks_m * blocks_n) continue;
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[h][i][j] *= kDown;
            if (step + 1u < a.steps) {
                put(X, bq, bp, acc[h], false);
                continue;
            }
            T *const out = static_cast<T *>(a.out.p[blockIdx.x]);
#pragma unroll
            for (int i = 0; i < 2; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j)
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        const uint32_t q = 32u * bq + 16u * i + l, p = 32u * bp + 16u * j + 4u * grp + k;
                        if (q >= side_m || p >= side_n) continue;
                        T *const to = out + (tall ? p * a.ld_out + q : q * a.ld_out + p);
                        const float o = acc[h][i][j][k] * kDown;
                        *to = (T)(STEP ? a.keep * to_float(*to) - a.by * o : o);
                    }
        }
        __syncthreads();
    }
}

} // namespace fo
