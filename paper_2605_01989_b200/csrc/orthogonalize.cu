// dblp_orthogonalize: Newton-Schulz products on the shorter side of each matrix.
//
// f16 carries 11 bits where bf16 carries 8, and the entries' range is known: |X| is at most about 1.2 in every singular value, so
// X scaled by 2^10 and A by 2^8 sit in the middle of f16's range.  What would still go wrong is the rounding of X itself: the
// polynomial multiplies a small singular value by up to a per step (3.4^5 = 485 in five), noise as well as signal.  X is
// therefore two f16 words (22 bits); for bf16 results the products read the first, and only the term a X, the one that amplifies what
// lies outside the strong directions, reads both.  (In 64-bit simulation of a matrix of rank 8: 4e-2 of the result's norm with one
// word, 5e-4 with two; one bf16 word 3e-1.)  For fp32 and f16 results, and in the last steps
// of small matrices, products read both words of X, A and B.
#include <math.h>

#include "product.cuh"

namespace dblp {

constexpr int kUpdThreads = 256;
constexpr uint32_t kMaxSquares = 256;            // partial sums of squares a matrix
constexpr double kScaleX = 1024.0;
constexpr float kScaleA = 256.0f;
// Bf16 results come of products of one word where single roundings average out over many rows and columns: from kAverages on the shorter
// side 1.1 to 1.5 times as far from 64 bits as the result's rounding alone (1.7 where all singular values are alike).  Smaller matrices multiply both words in their last
// three steps, whose roundings reach the result (up to 1.6 times with one word, alike 2.8, with both 1.0 to 1.1: 129 x 200 78 and 99 us, 384 x
// 640 92 and 134 us), and in all steps below kFew, where single roundings show (sides of two: up to 1.6e-2 of the norm, with both 1.7e-3; 16 x 16 45 and
// 60 us).
constexpr uint32_t kAverages = 512, kFew = 64, kLastSteps = 3;

struct UpdIn {
    Source x;
    int64_t each;
    uint32_t rows, cols, parts;
    FastDiv by_row;                              // groups of eight in a row; rows * groups < 2^32
    double* squares;                             // [batch][parts]
    float eps;
    Words out;
};

__device__ __forceinline__ double block_sum(double t, double* part)
{
#pragma unroll
    for (int m = 16; m; m >>= 1) t += __shfl_xor_sync(0xFFFFFFFFu, t, m);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = t;
    __syncthreads();
    t = 0.0;
#pragma unroll
    for (int i = 0; i < kUpdThreads / 32; ++i) t += part[i];
    return t;
}

// Groups of eight columns, row by row, dealt to the blocks of a matrix in contiguous shares.
__global__ void __launch_bounds__(kUpdThreads) k_squares(const __grid_constant__ UpdIn a)
{
    __shared__ double part[kUpdThreads / 32];
    after_start();
    const uint32_t per_row = (a.cols + 7) / 8, b = blockIdx.y;
    const uint64_t groups = (uint64_t)a.rows * per_row, share = (groups + a.parts - 1) / a.parts;
    const uint64_t g0 = blockIdx.x * share, g1 = min(groups, g0 + share);
    Source x = a.x;
    x.p = (const char*)x.p + b * a.each * (x.dtype == DBLP_F32 ? 4 : 2);
    double t = 0.0;
    for (uint64_t g = g0 + threadIdx.x; g < g1; g += 4 * kUpdThreads) {             // four groups on their way
        float v[4][8];
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u) {
            const uint64_t h = min(g + u * kUpdThreads, groups - 1);
            const uint32_t r = a.by_row.div((uint32_t)h), c = ((uint32_t)h - r * per_row) * 8;
            load8(x, r, c, min(8u, a.cols - c), v[u]);
        }
#pragma unroll
        for (uint32_t u = 0; u < 4; ++u)
            if (g + u * kUpdThreads < g1)
#pragma unroll
                for (int i = 0; i < 8; ++i) t = fma((double)v[u][i], (double)v[u][i], t);
    }
    t = block_sum(t, part);
    if (threadIdx.x == 0) a.squares[(size_t)b * a.parts + blockIdx.x] = t;
}

// X = x / (norm + eps) in two words.
__global__ void __launch_bounds__(kUpdThreads) k_normalize(const __grid_constant__ UpdIn a)
{
    __shared__ double part[kUpdThreads / 32];
    wait_before();
    after_start();
    const uint32_t per_row = (a.cols + 15) / 16, b = blockIdx.y;
    const uint64_t groups = (uint64_t)a.rows * per_row;
    const double norm = sqrt(block_sum(threadIdx.x < a.parts ? a.squares[(size_t)b * a.parts + threadIdx.x] : 0.0, part)) + (double)a.eps;
    const double f = norm == 0.0 ? 0.0 : kScaleX / norm;
    const bool plain = f > 1e-30 && f < 1e30;        // an fp32 factor and fp32 products (2^-24) are enough for 22 bits
    Source x = a.x;
    x.p = (const char*)x.p + b * a.each * (x.dtype == DBLP_F32 ? 4 : 2);
    for (uint64_t g = (uint64_t)blockIdx.x * kUpdThreads + threadIdx.x; g < groups; g += (uint64_t)gridDim.x * kUpdThreads) {
        const uint32_t r = (uint32_t)(g / per_row), c = (uint32_t)(g - (uint64_t)r * per_row) * 16, left = min(16u, a.cols - c);
        float v[16];
        load8(x, r, c, min(8u, left), v);
        load8(x, r, c + 8, left > 8 ? left - 8 : 0, v + 8);
        if (plain) {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] *= (float)f;
        } else {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] = (float)((double)v[i] * f);
        }
        a.out.store(b, r, c, v, ToMemory());
    }
}

struct UpdPlan {
    uint32_t low;                                // the shorter side
    bool tall;
    bool one, both;                              // products of one word, of both, occur
    uint32_t xs, as;                             // row strides of X and of A, B
    size_t x_bytes, a_bytes, squares_bytes;      // one word of X, of A; sums
    uint32_t parts;
};

static UpdPlan plan_update(const dblp_orthogonalize_t* u)
{
    UpdPlan p{};
    p.tall = u->rows > u->cols;
    p.low = p.tall ? u->cols : u->rows;
    p.one = u->out_dtype == DBLP_BF16 && p.low >= kFew;
    p.both = !p.one || p.low < kAverages;
    p.xs = (u->cols + 15) & ~15u;
    p.as = (p.low + 15) & ~15u;
    auto padded = [](size_t b) { return (b + 255) & ~(size_t)255; };
    p.x_bytes = padded((size_t)u->batch * u->rows * p.xs * 2);
    p.a_bytes = padded((size_t)u->batch * p.low * p.as * 2);
    const uint64_t groups = (uint64_t)u->rows * ((u->cols + 7) / 8), want = (groups + 4 * kUpdThreads - 1) / (4 * kUpdThreads);
    p.parts = (uint32_t)(want < kMaxSquares ? want : kMaxSquares);
    p.squares_bytes = padded((size_t)u->batch * p.parts * 8);
    return p;
}

static Product gram_product(const dblp_orthogonalize_t* u, const UpdPlan& p, const Words& x, bool both)
{
    Product g{};
    g.a = Operand{x.hi, both ? x.lo : nullptr, x.stride, x.each, p.tall};
    g.b = g.a;
    g.M = g.N = p.low;
    g.K = p.tall ? u->rows : u->cols;
    g.batch = u->batch;
    g.dtype = DBLP_F16;
    g.terms = both ? 3 : 1;
    g.symmetric = true;
    return g;
}
static Product square_product(const dblp_orthogonalize_t* u, const UpdPlan& p, const Words& a, bool both)
{
    Product g = gram_product(u, p, a, both);
    g.a = g.b = Operand{a.hi, both ? a.lo : nullptr, a.stride, a.each, false};
    g.K = p.low;
    return g;
}
// B X, or X B where X is tall
static Product step_product(const dblp_orthogonalize_t* u, const UpdPlan& p, const Words& b, const Words& x, bool both)
{
    Product g = square_product(u, p, b, both);
    const Operand ox{x.hi, both ? x.lo : nullptr, x.stride, x.each, !p.tall};
    if (p.tall) g.a = ox;
    else g.b = ox;
    g.M = u->rows;
    g.N = u->cols;
    g.symmetric = false;
    return g;
}

struct UpdSpace {
    Words x, y, a, b;
    double* squares;
    void* products;
    size_t bytes;
};
static UpdSpace space_of(const dblp_orthogonalize_t* u, const UpdPlan& p, void* ws)
{
    UpdSpace s{};
    char* at = (char*)ws;
    auto take = [&](size_t bytes) { char* q = at; at += bytes; return q; };
    const int64_t xe = (int64_t)u->rows * p.xs, ae = (int64_t)p.low * p.as;
    auto words = [&](size_t bytes, bool two, int64_t each, uint32_t stride) {
        Words w{};
        w.hi = (__half*)take(bytes);
        w.lo = two ? (__half*)take(bytes) : nullptr;
        w.each = each;
        w.stride = stride;
        return w;
    };
    s.x = words(p.x_bytes, true, xe, p.xs);
    s.y = words(p.x_bytes, true, xe, p.xs);
    s.a = words(p.a_bytes, p.both, ae, p.as);
    s.b = words(p.a_bytes, p.both, ae, p.as);
    s.squares = (double*)take(p.squares_bytes);
    s.products = at;
    size_t most = 0;
    for (bool both : {false, true})
        if (both ? p.both : p.one)
            for (const Product& g : {gram_product(u, p, s.x, both), square_product(u, p, s.a, both), step_product(u, p, s.b, s.x, both)}) most = max(most, product_space(g));
    s.bytes = (size_t)(at - (char*)ws) + most;
    return s;
}

static bool whole(const void* p, int64_t row_stride, int64_t batch_stride, const dblp_orthogonalize_t* u, int dtype, uint32_t bytes)
{
    const uint64_t es = element_bytes(dtype), rows = u->rows > 1 ? row_stride * es : 0, batches = u->batch > 1 ? batch_stride * es : 0;
    return ((uintptr_t)p | rows | batches) % bytes == 0;
}

// Products of both words take their sums in short runs; F32 and F16 results know no other.
template <bool ONE_WORD, typename E> static int product(const Product& p, const E& e, void* ws, cudaStream_t s)
{
    if constexpr (ONE_WORD)
        if (p.terms == 1) return run_product<false>(p, e, ws, true, s);
    return run_product<true>(p, e, ws, true, s);
}

static int check_update(const char* who, const dblp_orthogonalize_t* u)
{
    DBLP_REQUIRE(u, DBLP_EINVAL, "%s: null argument", who);
    DBLP_REQUIRE(known_dtype(u->x_dtype) && known_dtype(u->out_dtype), DBLP_EINVAL, "%s: unknown dtype %d or %d", who, u->x_dtype, u->out_dtype);
    DBLP_REQUIRE(u->rows <= 32768 && u->cols <= 32768 && u->batch < 65536, DBLP_ECAPACITY, "%s: rows and columns up to 32768, batch below 65536", who);
    return DBLP_OK;
}

// no two elements of an output in one place
static bool clear_output(const dblp_orthogonalize_t* u)
{
    const int64_t row = u->out_row_stride, each = u->out_batch_stride, cols = u->cols, rows = u->rows, batch = u->batch;
    const bool rows_clear = rows <= 1 || row >= cols;
    const int64_t reach = rows <= 1 ? cols : (rows - 1) * row + cols;
    if (batch <= 1) return rows_clear;
    if (rows_clear && each >= reach) return true;                                   // one matrix after the other
    return each >= cols && (rows <= 1 || row >= (batch - 1) * each + cols);         // side by side
}

}  // namespace dblp

using namespace dblp;

#define DBLP_TRY(call)                      \
    do {                                    \
        const int rc_ = (call);             \
        if (rc_ != DBLP_OK) return rc_;     \
    } while (0)

extern "C" int dblp_orthogonalize_workspace_bytes(const dblp_orthogonalize_t* u, size_t* bytes)
{
    DBLP_TRY(check_update("orthogonalize_workspace_bytes", u));
    DBLP_REQUIRE(bytes, DBLP_EINVAL, "orthogonalize_workspace_bytes: null output");
    *bytes = u->batch && u->rows && u->cols ? space_of(u, plan_update(u), nullptr).bytes : 0;
    return DBLP_OK;
}

extern "C" int dblp_orthogonalize(const dblp_orthogonalize_t* u, const void* x, void* out, void* ws, size_t ws_bytes, void* stream)
{
    const char* who = "orthogonalize";
    DBLP_TRY(check_update(who, u));
    DBLP_REQUIRE(u->steps >= 1 && u->steps <= DBLP_ORTHOGONALIZE_STEPS, DBLP_EINVAL, "%s: %u steps (1 to %d)", who, u->steps, DBLP_ORTHOGONALIZE_STEPS);
    DBLP_REQUIRE(u->coefficients, DBLP_EINVAL, "%s: coefficients are null", who);
    for (uint32_t i = 0; i < 3 * u->steps; ++i)
        DBLP_REQUIRE(isfinite(u->coefficients[i]), DBLP_EINVAL, "%s: coefficient %u is not finite", who, i);
    DBLP_REQUIRE(u->eps >= 0.0f && u->eps < INFINITY, DBLP_EINVAL, "%s: eps %g is negative or not finite", who, u->eps);
    DBLP_REQUIRE(isfinite(u->scale), DBLP_EINVAL, "%s: scale is not finite", who);
    if (u->batch == 0 || u->rows == 0 || u->cols == 0) return DBLP_OK;
    DBLP_REQUIRE(x && out, DBLP_EINVAL, "%s: null pointer", who);
    DBLP_REQUIRE((uintptr_t)x % element_bytes(u->x_dtype) == 0 && (uintptr_t)out % element_bytes(u->out_dtype) == 0, DBLP_EALIGN,
                 "%s: a pointer is not aligned to its element type", who);
    const int64_t far = 1ll << 38;
    for (int64_t v : {u->x_batch_stride, u->x_row_stride, u->out_batch_stride, u->out_row_stride})
        DBLP_REQUIRE(v >= 0 && v < far, DBLP_EINVAL, "%s: a stride of %lld", who, (long long)v);
    DBLP_REQUIRE(clear_output(u), DBLP_EINVAL, "%s: rows of the output overlap", who);
    const UpdPlan p = plan_update(u);
    const UpdSpace w = space_of(u, p, ws);
    DBLP_REQUIRE(ws, DBLP_EINVAL, "%s: the workspace is null", who);
    DBLP_REQUIRE(((uintptr_t)ws & 255) == 0, DBLP_EALIGN, "%s: the workspace is not 256-byte aligned", who);
    DBLP_REQUIRE(ws_bytes >= w.bytes, DBLP_ECAPACITY, "%s: workspace of %zu bytes, needs %zu", who, ws_bytes, w.bytes);
    const cudaStream_t s = (cudaStream_t)stream;

    UpdIn in{};
    in.x = source_of(x, u->x_row_stride, u->rows, u->x_dtype);
    in.x.vec = whole(x, u->x_row_stride, u->x_batch_stride, u, u->x_dtype, 16);
    in.each = u->x_batch_stride;
    in.rows = u->rows;
    in.cols = u->cols;
    in.parts = p.parts;
    in.by_row = FastDiv((u->cols + 7) / 8);
    in.squares = w.squares;
    in.eps = u->eps;
    in.out = w.x;
    k_squares<<<dim3(p.parts, u->batch), kUpdThreads, 0, s>>>(in);
    DBLP_LAUNCHED();
    const uint64_t groups = (uint64_t)u->rows * ((u->cols + 15) / 16), blocks = (groups + kUpdThreads - 1) / kUpdThreads;
    DBLP_NEXT(launch_next(k_normalize, dim3((unsigned)(blocks < 1024 ? blocks : 1024), u->batch), kUpdThreads, 0, s, in));

    Words now = w.x, next = w.y;
    for (uint32_t i = 0; i < u->steps; ++i) {
        const float a = u->coefficients[3 * i], b = u->coefficients[3 * i + 1], c = u->coefficients[3 * i + 2];
        const bool both = p.both && (!p.one || i + kLastSteps >= u->steps);
        Words wa = w.a, wb = w.b;
        if (!both) wa.lo = wb.lo = nullptr;
        EpiPoly<true> e{};
        e.out = wa;
        e.alpha = kScaleA / (float)(kScaleX * kScaleX);
        DBLP_TRY(product<true>(gram_product(u, p, now, both), e, w.products, s));
        e.out = wb;
        e.add = wa;
        e.alpha = c / kScaleA;
        e.beta = b;
        DBLP_TRY(product<true>(square_product(u, p, wa, both), e, w.products, s));
        const Product last = step_product(u, p, wb, now, both);
        if (i + 1 < u->steps) {
            DBLP_TRY(product<true>(last, EpiPoly<false>{next, now, 1.0f / kScaleA, a}, w.products, s));
            const Words t = now;
            now = next;
            next = t;
        } else {
            DBLP_TRY(with_type(u->out_dtype, [&](auto t) -> int {
                using O = decltype(t);
                EpiLast<O> f{};
                f.out = rows_of<O>(out, u->out_row_stride, u->rows);
                f.each = u->out_batch_stride;
                f.add = now;
                const float back = u->scale / (float)kScaleX;
                f.alpha = back / kScaleA;
                f.beta = back * a;
                f.aligned = whole(out, u->out_row_stride, u->out_batch_stride, u, u->out_dtype, 32);
                return product<std::is_same<O, __nv_bfloat16>::value>(last, f, w.products, s);
            }));
        }
    }
    return DBLP_OK;
}
