// Orthogonalised updates (fo_orthogonalize, fo_matrix_step): plan, argument checks, launches.
#include "fo_host.h"
#include "fo_matrix.h"

#include <algorithm>

using namespace fo;
using namespace fo_host;

struct fo_matrix_plan {
    fo_matrix_params p;
    int device;
    bool tall;             // rows > cols: X is G^T
    bool small;            // k_matrix_small: no scratch
    uint64_t m, n;         // shorter and longer side
    uint32_t m64, n64;     // padded
    uint32_t parts;        // of an iterate
    uint32_t nparts;       // partial sums of squares a matrix
    char *scratch;
    size_t scratch_bytes;
    // [count][parts][...] each
    _Float16 *x[2];        // X, m64 x n64, read by one product while the next iterate is written
    _Float16 *a, *b;       // m64 x m64
    double *partials;      // [count][nparts]
};

namespace {

bool launched(const char *what) { return hip_ok(hipGetLastError(), what); }

template <bool TWO, bool TURNED = false, typename Epi>
int launch_half(const ProductArgs &a, const Epi &epi, hipStream_t st)
{
    launch_product<OpF16, TURNED, TWO>(a, epi, st);
    return launched("k_product") ? FO_OK : FO_EHIP;
}

struct Last { // where the last step's result goes
    MatrixTab out;
    uint64_t ld;
    float keep, by;
};

template <typename T, bool STEP, bool TALL, bool TWO>
int launch_steps(const fo_matrix_plan *pl, const Last &last, hipStream_t st)
{
    const uint64_t mn = (uint64_t)pl->m64 * pl->n64, mm = (uint64_t)pl->m64 * pl->m64;
    const uint32_t parts = pl->parts;
    const Iterate a{ pl->a, pl->m64, mm, mm * parts }, b{ pl->b, pl->m64, mm, mm * parts };
    auto product = [&](const Iterate &q, const Iterate &p, uint32_t rows_p, bool symmetric) { // m64 rows of q
        ProductArgs r;
        std::memset(&r, 0, sizeof(r));
        r.q = reinterpret_cast<const char *>(q.x);
        r.p = reinterpret_cast<const char *>(p.x);
        r.ld_q = 2u * q.ld;
        r.ld_p = 2u * p.ld;
        r.next_q = 2u * q.next;
        r.next_p = 2u * p.next;
        r.part_q = 2u * q.part;
        r.part_p = 2u * p.part;
        r.rows_q = pl->m64;
        r.rows_p = rows_p;
        r.stages = (uint32_t)(r.ld_q / kStageBytes);
        r.symmetric = symmetric;
        r.count = pl->p.count;
        return r;
    };
    for (uint32_t s = 0; s < pl->p.steps; ++s) {
        const Iterate x{ pl->x[s & 1u], pl->n64, mn, mn * parts }, to{ pl->x[1u - (s & 1u)], pl->n64, mn, mn * parts };
        FO_TRY(launch_half<TWO>(product(x, x, pl->m64, true), GramEpilogue<TWO>{ a, pl->m64 }, st));
        FO_TRY(launch_half<TWO>(product(a, a, pl->m64, true), PolyEpilogue<TWO>{ a, b, pl->m64, pl->p.a * kUp, pl->p.b, pl->p.c * kDown }, st));
        if (s + 1u < pl->p.steps) {
            FO_TRY((launch_half<TWO, true>(product(b, x, pl->n64, false), UpdateEpilogue<TWO>{ to, pl->m64, pl->n64 }, st)));
        } else {
            const LastEpilogue<T, STEP, TALL> epi{ last.out, last.ld, (uint32_t)pl->m, (uint32_t)pl->n, last.keep, last.by };
            FO_TRY((launch_half<TWO, true>(product(b, x, pl->n64, false), epi, st)));
        }
    }
    return FO_OK;
}

template <typename T, bool STEP>
int launch_steps(const fo_matrix_plan *pl, const Last &last, hipStream_t st)
{
    if (pl->tall) return pl->parts == 2u ? launch_steps<T, STEP, true, true>(pl, last, st) : launch_steps<T, STEP, true, false>(pl, last, st);
    return pl->parts == 2u ? launch_steps<T, STEP, false, true>(pl, last, st) : launch_steps<T, STEP, false, false>(pl, last, st);
}
template <bool STEP>
int launch_steps(const fo_matrix_plan *pl, const Last &last, hipStream_t st)
{
    if (pl->p.type == FO_F32) return launch_steps<float, STEP>(pl, last, st);
    if (pl->p.type == FO_BF16) return launch_steps<__bf16, STEP>(pl, last, st);
    return launch_steps<_Float16, STEP>(pl, last, st);
}

template <typename T>
int launch_begin(const fo_matrix_plan *pl, BeginArgs b, hipStream_t st)
{
    b.rows = pl->p.rows;
    b.cols = pl->p.cols;
    b.partials = pl->partials;
    b.nparts = pl->nparts;
    b.parts = pl->parts;
    b.rows64 = pl->tall ? pl->n64 : pl->m64;
    b.cols64 = pl->tall ? pl->m64 : pl->n64;
    b.x = pl->x[0];
    b.part = (uint64_t)pl->m64 * pl->n64;
    b.next = b.part * pl->parts;
    const dim3 grid((b.rows64 / 64u) * (b.cols64 / 64u), pl->p.count);
    if (pl->tall) hipLaunchKernelGGL((k_matrix_begin<T, true>), grid, dim3(256), 0, st, b);
    else hipLaunchKernelGGL((k_matrix_begin<T, false>), grid, dim3(256), 0, st, b);
    return launched("k_matrix_begin") ? FO_OK : FO_EHIP;
}

template <typename T>
int launch_orthogonalize(const fo_matrix_plan *pl, const MatrixTab &g, uint64_t ld_g, hipStream_t st)
{
    const bool one = ld_g == pl->p.cols;
    const NormArgs n{ g, one ? 1u : pl->p.rows, one ? pl->p.rows * pl->p.cols : pl->p.cols, ld_g, pl->partials };
    hipLaunchKernelGGL((k_matrix_norm<T>), dim3(pl->nparts, pl->p.count), dim3(256), 0, st, n);
    if (!launched("k_matrix_norm")) return FO_EHIP;
    BeginArgs b;
    std::memset(&b, 0, sizeof(b));
    b.g = g;
    b.ld = ld_g;
    return launch_begin<T>(pl, b, st);
}

template <typename T, bool STEP>
int launch_small(const fo_matrix_plan *pl, const SmallArgs &a, hipStream_t st)
{
    if (pl->parts == 2u) hipLaunchKernelGGL((k_matrix_small<T, STEP, true>), dim3(pl->p.count), dim3(512), 0, st, a);
    else hipLaunchKernelGGL((k_matrix_small<T, STEP, false>), dim3(pl->p.count), dim3(512), 0, st, a);
    return launched("k_matrix_small") ? FO_OK : FO_EHIP;
}
template <bool STEP>
int launch_small(const fo_matrix_plan *pl, SmallArgs &a, hipStream_t st)
{
    a.rows = (uint32_t)pl->p.rows;
    a.cols = (uint32_t)pl->p.cols;
    a.steps = pl->p.steps;
    a.ka = pl->p.a * kUp;
    a.kb = pl->p.b;
    a.kc = pl->p.c * kDown;
    if (pl->p.type == FO_F32) return launch_small<float, STEP>(pl, a, st);
    if (pl->p.type == FO_BF16) return launch_small<__bf16, STEP>(pl, a, st);
    return launch_small<_Float16, STEP>(pl, a, st);
}

uint32_t element_bytes(uint32_t type) { return type == FO_F32 ? 4u : 2u; }

// The pointers of a host array, checked
template <typename P>
int take(const fo_matrix_plan *pl, const P *from, uint32_t size, MatrixTab &to)
{
    std::memset(&to, 0, sizeof(to));
    for (uint32_t i = 0; i < pl->p.count; ++i) {
        if (!from[i]) return FO_EINVAL;
        if (!aligned(from[i], size)) return FO_EALIGN;
        to.p[i] = const_cast<void *>(static_cast<const void *>(from[i]));
    }
    return FO_OK;
}

// Whether stretches of memory lie apart from one another
struct Range {
    uintptr_t at, bytes;
};
bool apart(Range *r, uint32_t n)
{
    std::sort(r, r + n, [](const Range &a, const Range &b) { return a.at < b.at; });
    for (uint32_t i = 1; i < n; ++i)
        if (r[i].at - r[i - 1].at < r[i - 1].bytes) return false;
    return true;
}

// Whether two matrices have memory in common: `rows` rows of `bytes` each, which follow one another after step_a or step_b bytes.
// (Matrices may lie side by side in a larger one, so that their stretches of memory alone do not tell.)
bool meet(uintptr_t a, uint64_t step_a, uintptr_t b, uint64_t step_b, uint64_t rows, uint64_t bytes)
{
    const uint64_t last_a = (rows - 1u) * step_a, last_b = (rows - 1u) * step_b;
    if (a + last_a + bytes <= b || b + last_b + bytes <= a) return false;
    const int64_t from = (int64_t)(a - b), end = (int64_t)(last_b + bytes), step = (int64_t)step_b, row = (int64_t)bytes;
    if (step_a == step_b) { // the rows of a lie in the rows of b all in the same way
        const int64_t in = ((from % step) + step) % step, down = (from - in) / step, most = (int64_t)rows - 1;
        return (in < row && down >= -most && down <= most) || (in + row > step && down + 1 >= -most && down + 1 <= most);
    }
    for (uint64_t i = 0; i < rows; ++i) {
        const int64_t x = from + (int64_t)(i * step_a);
        if (x <= -row) continue;
        if (x >= end) return false;
        const int64_t in = ((x % step) + step) % step;
        if (in < row || in + row > step) return true;
    }
    return false;
}

int on_device(const fo_matrix_plan *pl)
{
    int dev = -1;
    if (!hip_ok(hipGetDevice(&dev), "hipGetDevice")) return FO_EHIP;
    return dev == pl->device ? FO_OK : FO_EINVAL;
}

} // namespace

extern "C" int fo_matrix_plan_create(const fo_matrix_params *params, fo_matrix_plan **out)
{
    if (!params || !out) return FO_EINVAL;
    *out = nullptr;
    const fo_matrix_params &q = *params;
    const uint64_t m = q.rows < q.cols ? q.rows : q.cols, n = q.rows < q.cols ? q.cols : q.rows;
    if (m < 1 || m > FO_MAX_MATRIX_SHORT || n > FO_MAX_MATRIX_LONG) return FO_EINVAL;
    if (q.count < 1 || q.count > FO_MAX_MATRICES || q.type > FO_F16 || q.products > FO_PRODUCTS_SINGLE) return FO_EINVAL;
    if (q.steps < 1 || q.steps > FO_MAX_STEPS || !std::isfinite(q.a) || !std::isfinite(q.b) || !std::isfinite(q.c)) return FO_EINVAL;
    fo_matrix_plan *pl = new (std::nothrow) fo_matrix_plan();
    if (!pl) return FO_ENOMEM;
    pl->p = q;
    pl->tall = q.rows > q.cols;
    pl->small = n <= 128;
    pl->m = m;
    pl->n = n;
    pl->m64 = (uint32_t)((m + 63u) & ~(uint64_t)63u);
    pl->n64 = (uint32_t)((n + 63u) & ~(uint64_t)63u);
    pl->parts = q.products == FO_PRODUCTS_SINGLE ? 2u : 1u;
    const uint64_t work = (m * n + 2047u) / 2048u; // a unit of two vectors of fp32 a thread (16-bit ones need half the workgroups)
    pl->nparts = (uint32_t)(work < 1024u ? work : 1024u);
    if (!hip_ok(hipGetDevice(&pl->device), "hipGetDevice")) {
        delete pl;
        return FO_EHIP;
    }
    if (pl->small) {
        *out = pl;
        return FO_OK;
    }
    const size_t each = (size_t)q.count * pl->parts * sizeof(_Float16);
    const size_t sz_x = each * pl->m64 * pl->n64, sz_a = each * pl->m64 * pl->m64; // multiples of 4096 bytes
    pl->scratch_bytes = 2 * sz_x + 2 * sz_a + (size_t)q.count * pl->nparts * sizeof(double);
    void *mem = nullptr;
    const hipError_t e = hipMalloc(&mem, pl->scratch_bytes);
    if (e != hipSuccess) {
        hip_ok(e, "hipMalloc(matrix plan scratch)");
        delete pl;
        return e == hipErrorOutOfMemory ? FO_ENOMEM : FO_EHIP;
    }
    char *c = pl->scratch = static_cast<char *>(mem);
    pl->x[0] = reinterpret_cast<_Float16 *>(c); c += sz_x;
    pl->x[1] = reinterpret_cast<_Float16 *>(c); c += sz_x;
    pl->a = reinterpret_cast<_Float16 *>(c); c += sz_a;
    pl->b = reinterpret_cast<_Float16 *>(c); c += sz_a;
    pl->partials = reinterpret_cast<double *>(c);
    *out = pl;
    return FO_OK;
}

extern "C" void fo_matrix_plan_destroy(fo_matrix_plan *plan)
{
    if (!plan) return;
    if (plan->scratch) (void)hipFree(plan->scratch);
    delete plan;
}

extern "C" size_t fo_matrix_scratch_bytes(const fo_matrix_plan *p) { return p ? p->scratch_bytes : 0; }

extern "C" int fo_orthogonalize(fo_matrix_plan *pl, const void *const *g, uint64_t ld_g, void *const *out, uint64_t ld_out,
                                void *hip_stream)
{
    if (!pl || !g || !out) return FO_EINVAL;
    if (ld_g < pl->p.cols || ld_out < pl->p.cols || ld_g > ((uint64_t)1 << 40) || ld_out > ((uint64_t)1 << 40)) return FO_EINVAL;
    const uint32_t size = element_bytes(pl->p.type);
    MatrixTab from;
    Last last;
    FO_TRY(take(pl, g, size, from));
    FO_TRY(take(pl, out, size, last.out));
    const uint64_t rows = pl->p.rows, bytes = pl->p.cols * size, step_g = ld_g * size, step_out = ld_out * size;
    for (uint32_t i = 0; i < pl->p.count; ++i)
        for (uint32_t j = 0; j < pl->p.count; ++j) {
            const uintptr_t o = reinterpret_cast<uintptr_t>(out[i]), o2 = reinterpret_cast<uintptr_t>(out[j]), x = reinterpret_cast<uintptr_t>(g[j]);
            if (j < i && meet(o, step_out, o2, step_out, rows, bytes)) return FO_EINVAL;
            if (!(i == j && o == x && ld_g == ld_out) && meet(o, step_out, x, step_g, rows, bytes)) return FO_EINVAL;
        }
    FO_TRY(on_device(pl));
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    if (pl->small) {
        SmallArgs a;
        std::memset(&a, 0, sizeof(a));
        a.g = from;
        a.out = last.out;
        a.ld_g = ld_g;
        a.ld_out = ld_out;
        return launch_small<false>(pl, a, st);
    }
    last.ld = ld_out;
    last.keep = last.by = 0.f;
    if (pl->p.type == FO_F32) FO_TRY(launch_orthogonalize<float>(pl, from, ld_g, st));
    else if (pl->p.type == FO_BF16) FO_TRY(launch_orthogonalize<__bf16>(pl, from, ld_g, st));
    else FO_TRY(launch_orthogonalize<_Float16>(pl, from, ld_g, st));
    return launch_steps<false>(pl, last, st);
}

extern "C" int fo_matrix_step(fo_matrix_plan *pl, const float *const *g, float *const *momentum, void *const *x,
                              const fo_matrix_update *u, void *hip_stream)
{
    if (!pl || !g || !momentum || !x || !u) return FO_EINVAL;
    if (!(u->mu >= 0.f && u->mu < 1.f) || u->nesterov > 1u) return FO_EINVAL;
    if (!std::isfinite(u->delta) || !std::isfinite(u->scale) || !std::isfinite(u->decay)) return FO_EINVAL;
    BeginArgs b;
    std::memset(&b, 0, sizeof(b));
    Last last;
    FO_TRY(take(pl, g, 4, b.g));
    FO_TRY(take(pl, momentum, 4, b.m));
    FO_TRY(take(pl, x, element_bytes(pl->p.type), last.out));
    const uintptr_t elements = (uintptr_t)(pl->p.rows * pl->p.cols);
    Range ranges[3 * FO_MAX_MATRICES];
    for (uint32_t i = 0; i < pl->p.count; ++i) {
        ranges[3 * i] = { reinterpret_cast<uintptr_t>(g[i]), elements * 4u };
        ranges[3 * i + 1] = { reinterpret_cast<uintptr_t>(momentum[i]), elements * 4u };
        ranges[3 * i + 2] = { reinterpret_cast<uintptr_t>(x[i]), elements * element_bytes(pl->p.type) };
    }
    if (!apart(ranges, 3u * pl->p.count)) return FO_EINVAL;
    FO_TRY(on_device(pl));
    hipStream_t st = static_cast<hipStream_t>(hip_stream);
    last.ld = pl->p.cols;
    last.keep = (float)(1.0 - (double)u->delta * (double)u->decay);
    last.by = (float)((double)u->delta * (double)u->scale);
    if (pl->small) {
        SmallArgs a;
        std::memset(&a, 0, sizeof(a));
        a.g = b.g;
        a.m = b.m;
        a.out = last.out;
        a.ld_g = a.ld_out = pl->p.cols;
        a.mu = u->mu;
        a.nesterov = u->nesterov;
        a.keep = last.keep;
        a.by = last.by;
        return launch_small<true>(pl, a, st);
    }
    const MomentumArgs m{ b.g, b.m, pl->p.rows * pl->p.cols, u->mu, u->nesterov, pl->partials };
    hipLaunchKernelGGL(k_matrix_momentum, dim3(pl->nparts, pl->p.count), dim3(256), 0, st, m);
    if (!launched("k_matrix_momentum")) return FO_EHIP;
    b.ld = pl->p.cols;
    b.mu = u->mu;
    b.nesterov = u->nesterov;
    b.momentum = 1;
    FO_TRY(launch_begin<float>(pl, b, st));
    return launch_steps<true>(pl, last, st);
}
