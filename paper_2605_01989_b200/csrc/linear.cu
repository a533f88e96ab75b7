// dblp_linear, dblp_linear_grad: argument checks, the sums of dbias, and the products they are made of (product_kernels.cuh).
#include <math.h>

#include "product.cuh"

namespace dblp {

// ---- dbias: sums of dy's columns -----------------------------------------------------------------------------------------
// A block takes 256 columns and a slice of the rows, eight columns a lane and every eighth row a warp; the slices' sums are
// added in order by a second kernel.
constexpr int kSumThreads = 256;

struct SumArgs {
    Source dy;
    uint32_t rows, cols, slices;
    float* partial;                     // [slices][cols]
    void* out;
    int out_dtype;
    bool accumulate;
};

__global__ void __launch_bounds__(kSumThreads) k_column_sums(const __grid_constant__ SumArgs a)
{
    __shared__ float part[8][32 * 8 + 8];
    after_start();
    const uint32_t lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n = blockIdx.x * 256 + lane * 8;
    const uint32_t per = (a.rows + a.slices - 1) / a.slices, r0 = blockIdx.y * per, r1 = min(a.rows, r0 + per);
    float s[8] = {};
    if (n < a.cols) {
        const uint32_t left = min(8u, a.cols - n);
        const uint16_t* p = (const uint16_t*)a.dy.p + n;
        uint32_t r = r0 + warp;
        if (a.dy.vec && left == 8)
            for (; r + 56 < r1; r += 64) {                      // eight rows in flight a lane
                uint4 q[8];
#pragma unroll
                for (int u = 0; u < 8; ++u) q[u] = *reinterpret_cast<const uint4*>(p + (int64_t)(r + 8 * u) * a.dy.stride);
#pragma unroll
                for (int u = 0; u < 8; ++u) {
                    float t[8];
                    if (a.dy.dtype == DBLP_BF16) {
                        Vec8<__nv_bfloat16> v;
                        v.w = q[u];
                        v.get(t);
                    } else {
                        Vec8<__half> v;
                        v.w = q[u];
                        v.get(t);
                    }
#pragma unroll
                    for (int i = 0; i < 8; ++i) s[i] += t[i];
                }
            }
        for (; r < r1; r += 8) {
            float t[8];
            load8(a.dy, r, n, left, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) s[i] += t[i];
        }
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) part[warp][i * 33 + lane] = s[i];
    __syncthreads();
    const uint32_t c = blockIdx.x * 256 + threadIdx.x, at = (threadIdx.x & 7) * 33 + (threadIdx.x >> 3);
    if (c >= a.cols) return;
    float t = 0.0f;
#pragma unroll
    for (int w = 0; w < 8; ++w) t += part[w][at];
    a.partial[(size_t)blockIdx.y * a.cols + c] = t;
}

// 32 columns a block; eight threads a column take every eighth slice each, then their sums are added in order.
__global__ void __launch_bounds__(256) k_column_join(const __grid_constant__ SumArgs a)
{
    __shared__ float part[8][32];
    wait_before();
    after_start();
    const uint32_t x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.x * 32 + x;
    float t = 0.0f;
    if (c < a.cols)
#pragma unroll 8
        for (uint32_t s = y; s < a.slices; s += 8) t += a.partial[(size_t)s * a.cols + c];
    part[y][x] = t;
    __syncthreads();
    if (y || c >= a.cols) return;
#pragma unroll
    for (int i = 1; i < 8; ++i) t += part[i][x];
    if (a.out_dtype == DBLP_F32) {
        float* p = (float*)a.out + c;
        *p = a.accumulate ? *p + t : t;
    } else if (a.out_dtype == DBLP_BF16) {
        __nv_bfloat16* p = (__nv_bfloat16*)a.out + c;
        *p = from_f32<__nv_bfloat16>(a.accumulate ? to_f32(*p) + t : t);
    } else {
        __half* p = (__half*)a.out + c;
        *p = from_f32<__half>(a.accumulate ? to_f32(*p) + t : t);
    }
}

// At most one slice for every 64 rows begun, as many as give about four blocks a multiprocessor.
static uint32_t sum_slices(uint32_t rows, uint32_t cols)
{
    const uint32_t most = (rows + 63) / 64, want = 4 * kSms / ((cols + 255) / 256) + 1, s = most < want ? most : want;
    return s ? s : 1;
}
static size_t sum_bytes(const dblp_linear_t* l) { return l->out ? ((size_t)sum_slices(l->rows, l->out) * l->out * 4 + 255) & ~(size_t)255 : 0; }

static int column_sums(const dblp_linear_t* l, const dblp_matrix_t* dy, void* dbias, void* ws, cudaStream_t s)
{
    SumArgs a{};
    if (l->rows) a.dy = source_of(dy->data, dy->row_stride, l->rows, l->dtype);
    a.rows = l->rows;
    a.cols = l->out;
    a.slices = sum_slices(l->rows, l->out);
    a.partial = (float*)ws;
    a.out = dbias;
    a.out_dtype = l->bias_dtype;
    a.accumulate = l->flags & DBLP_ACCUMULATE;
    k_column_sums<<<dim3((a.cols + 255) / 256, a.slices), kSumThreads, 0, s>>>(a);
    DBLP_LAUNCHED();
    DBLP_NEXT(launch_next(k_column_join, dim3((a.cols + 31) / 32), 256, 0, s, a));
    return DBLP_OK;
}

// ---- checks --------------------------------------------------------------------------------------------------------------
static int check_linear(const char* who, const dblp_linear_t* l, uint32_t flags)
{
    DBLP_REQUIRE(l, DBLP_EINVAL, "%s: null argument", who);
    DBLP_REQUIRE(l->dtype == DBLP_BF16 || l->dtype == DBLP_F16, DBLP_EINVAL, "%s: dtype %d (bf16 or f16)", who, l->dtype);
    DBLP_REQUIRE(l->out_dtype == l->dtype || l->out_dtype == DBLP_F32, DBLP_EINVAL, "%s: out_dtype %d (dtype or f32)", who, l->out_dtype);
    DBLP_REQUIRE(known_dtype(l->bias_dtype), DBLP_EINVAL, "%s: unknown bias dtype %d", who, l->bias_dtype);
    DBLP_REQUIRE(l->activation >= DBLP_ACT_NONE && l->activation <= DBLP_ACT_SILU, DBLP_EINVAL, "%s: unknown activation %d", who, l->activation);
    DBLP_REQUIRE((l->flags & ~flags) == 0, DBLP_EINVAL, "%s: unknown flags %u", who, l->flags);
    DBLP_REQUIRE(l->rows < (1u << 31) && l->in < (1u << 31) && l->out < (1u << 31), DBLP_ECAPACITY, "%s: 2^31 rows or columns or more", who);
    return DBLP_OK;
}

// rows x cols elements; `either`: the transposed view is allowed too; `output`: no two elements in one place.
static int check_matrix(const char* who, const char* name, const dblp_matrix_t* m, uint32_t rows, uint32_t cols, int dtype, bool either, bool output)
{
    DBLP_REQUIRE(m && m->data, DBLP_EINVAL, "%s: %s is null", who, name);
    DBLP_REQUIRE((uintptr_t)m->data % element_bytes(dtype) == 0, DBLP_EALIGN, "%s: %s is not aligned to its type", who, name);
    const bool by_rows = m->col_stride == 1 || cols <= 1, by_cols = either && (m->row_stride == 1 || rows <= 1);
    DBLP_REQUIRE(by_rows || by_cols, DBLP_EINVAL, "%s: %s has strides %lld and %lld, one has to be 1%s", who, name, (long long)m->row_stride,
                 (long long)m->col_stride, either ? "" : " (that of the columns)");
    const int64_t far = 1ll << 38;
    DBLP_REQUIRE(m->row_stride > -far && m->row_stride < far && m->col_stride > -far && m->col_stride < far, DBLP_EINVAL, "%s: %s has a stride of 2^38 or more", who, name);
    if (output) {
        auto clear = [](int64_t stride, uint32_t n, uint32_t other) { return n <= 1 || stride >= (int64_t)other || stride <= -(int64_t)other; };
        DBLP_REQUIRE((by_rows && clear(m->row_stride, rows, cols)) || (by_cols && clear(m->col_stride, cols, rows)), DBLP_EINVAL,
                     "%s: rows of %s overlap", who, name);
    }
    return DBLP_OK;
}

// w, dw: whether elements of a row are contiguous (else those of a column; a single column may be either)
static bool is_by_rows(const dblp_matrix_t* m, uint32_t cols) { return cols > 1 ? m->col_stride == 1 : m->row_stride != 1; }

static int check_vector(const char* who, const char* name, const void* p, int dtype)
{
    DBLP_REQUIRE((uintptr_t)p % element_bytes(dtype) == 0, DBLP_EALIGN, "%s: %s is not aligned to its type", who, name);
    return DBLP_OK;
}

static int check_space(const char* who, const void* ws, size_t ws_bytes, size_t need)
{
    DBLP_REQUIRE(need == 0 || ws, DBLP_EINVAL, "%s: the workspace is null", who);
    DBLP_REQUIRE(need == 0 || ((uintptr_t)ws & 255) == 0, DBLP_EALIGN, "%s: the workspace is not 256-byte aligned", who);
    DBLP_REQUIRE(ws_bytes >= need, DBLP_ECAPACITY, "%s: workspace of %zu bytes, needs %zu", who, ws_bytes, need);
    return DBLP_OK;
}

// Where a matrix (or a vector, a matrix of one row) lies: `lines` pieces of `bytes` bytes, `step` bytes apart.
struct Extent {
    intptr_t at;
    int64_t lines, bytes;
    __int128 step;
};
static Extent extent_of(const void* p, int64_t stride, uint64_t lines, uint64_t length, int dtype)
{
    const int64_t es = element_bytes(dtype);
    Extent e{(intptr_t)p, lines > 1 && stride != 0 ? (int64_t)lines : 1, (int64_t)length * es, (__int128)stride * es};
    if (e.lines > 1 && e.step < 0) {                            // from its lowest line on
        e.at += (intptr_t)(e.step * (e.lines - 1));
        e.step = -e.step;
    }
    return e;
}
static Extent extent_of(const dblp_matrix_t* m, uint32_t rows, uint32_t cols, int dtype)
{
    return is_by_rows(m, cols) || cols == 1 ? extent_of(m->data, m->row_stride, rows, cols, dtype) : extent_of(m->data, m->col_stride, cols, rows, dtype);
}
// Whether two of them certainly share a byte.  With one step between lines, or a single line on one side, this is exact; lines of
// different steps that start apart are taken to lie between one another.
static bool meet(const Extent& a, const Extent& b)
{
    if (a.at == b.at) return true;
    const __int128 away = (__int128)b.at - a.at, step = a.lines > 1 ? a.step : (b.lines > 1 ? b.step : 1);
    if (a.lines > 1 && b.lines > 1 && a.step != b.step) return false;
    // line j of b and line i of a, k = j - i: they share a byte where -b.bytes < away + k step < a.bytes
    const __int128 low = -b.bytes - away;
    __int128 k = low >= 0 ? low / step + 1 : -((-low - 1) / step);
    if (k < 1 - a.lines) k = 1 - a.lines;
    return k < b.lines && away + k * step < a.bytes;
}
static int check_apart(const char* who, const char* x, const Extent& a, const char* y, const Extent& b)
{
    DBLP_REQUIRE(!meet(a, b), DBLP_EINVAL, "%s: %s lies over %s", who, x, y);
    return DBLP_OK;
}
// what is read element by element where it is written: the same matrix, or apart from it
static int check_same_or_apart(const char* who, const char* x, const dblp_matrix_t* a, const Extent& ea, const char* y, const dblp_matrix_t* b, const Extent& eb)
{
    if (a->data == b->data && ea.lines == eb.lines && (ea.lines == 1 || ea.step == eb.step) && ea.bytes == eb.bytes) return DBLP_OK;
    return check_apart(who, x, ea, y, eb);
}

// The matrix as an operand whose rows are its rows (summed over the columns), or turned: its columns (summed over the rows).
static Operand operand(const dblp_matrix_t* m, uint32_t rows, uint32_t cols, bool turned)
{
    const bool by_rows = is_by_rows(m, cols);
    Operand o{};
    o.p = m->data;
    o.stride = by_rows ? (rows > 1 ? m->row_stride : 0) : (cols > 1 ? m->col_stride : 0);
    o.mn = by_rows == turned;
    return o;
}

static Product product_of(const dblp_linear_t* l, const Operand& a, const Operand& b, uint32_t M, uint32_t N, uint32_t K)
{
    Product p{};
    p.a = a;
    p.b = b;
    p.M = M;
    p.N = N;
    p.K = K;
    p.batch = 1;
    p.dtype = l->dtype;
    p.terms = 1;
    return p;
}

static Product few(Product p)
{
    p.few = true;
    return p;
}

// The three products.  x w, dy w^T, x^T dy (or its transpose, where dw is held that way).
static Product forward_product(const dblp_linear_t* l, const dblp_matrix_t* x, const dblp_matrix_t* w)
{
    return few(product_of(l, operand(x, l->rows, l->in, false), operand(w, l->in, l->out, true), l->rows, l->out, l->in));
}
static Product dx_product(const dblp_linear_t* l, const dblp_matrix_t* dy, const dblp_matrix_t* w)
{
    return few(product_of(l, operand(dy, l->rows, l->out, false), operand(w, l->in, l->out, false), l->rows, l->in, l->out));
}
static Product dw_product(const dblp_linear_t* l, const dblp_matrix_t* dy, const dblp_matrix_t* x, bool by_rows)
{
    const Operand a = operand(x, l->rows, l->in, true), b = operand(dy, l->rows, l->out, true);
    return by_rows ? product_of(l, a, b, l->in, l->out, l->rows) : product_of(l, b, a, l->out, l->in, l->rows);
}

static size_t forward_bytes(const dblp_linear_t* l, const dblp_matrix_t* x, const dblp_matrix_t* w)
{
    return l->rows && l->out && l->in ? product_space(forward_product(l, x, w)) : 0;
}

// One part of the backward pass at a time, all in the same place.
static size_t grad_bytes(const dblp_linear_t* l, const dblp_matrix_t* dy, const dblp_matrix_t* x, const dblp_matrix_t* w)
{
    size_t most = sum_bytes(l);
    if (l->rows && l->in && l->out) {
        const size_t parts[3] = {product_space(dx_product(l, dy, w)), product_space(dw_product(l, dy, x, true)), product_space(dw_product(l, dy, x, false))};
        for (size_t b : parts) most = b > most ? b : most;
    }
    return most;
}

}  // namespace dblp

using namespace dblp;

#define DBLP_TRY(call)                      \
    do {                                    \
        const int rc_ = (call);             \
        if (rc_ != DBLP_OK) return rc_;     \
    } while (0)

extern "C" int dblp_linear_workspace_bytes(const dblp_linear_t* l, const dblp_matrix_t* x, const dblp_matrix_t* w, const dblp_matrix_t* dy,
                                           size_t* fwd_bytes, size_t* grad_bytes_out)
{
    const char* who = "linear_workspace_bytes";
    DBLP_TRY(check_linear(who, l, DBLP_ACCUMULATE));
    if (l->rows && l->in) DBLP_TRY(check_matrix(who, "x", x, l->rows, l->in, l->dtype, false, false));
    if (l->in && l->out) DBLP_TRY(check_matrix(who, "w", w, l->in, l->out, l->dtype, true, false));
    if (dy && l->rows && l->out) DBLP_TRY(check_matrix(who, "dy", dy, l->rows, l->out, l->dtype, false, false));
    const size_t fwd = forward_bytes(l, x, w), grad = dy ? grad_bytes(l, dy, x, w) : 0;
    DBLP_REQUIRE(fwd < 1ull << 62 && grad < 1ull << 62, DBLP_ECAPACITY, "%s: a workspace passes 2^62 bytes", who);
    if (fwd_bytes) *fwd_bytes = fwd;
    if (grad_bytes_out) *grad_bytes_out = grad;
    return DBLP_OK;
}

extern "C" int dblp_linear(const dblp_linear_t* l, const dblp_matrix_t* x, const dblp_matrix_t* w, const void* bias,
                           const dblp_matrix_t* residual, const dblp_matrix_t* pre, const dblp_matrix_t* out, void* ws, size_t ws_bytes,
                           void* stream)
{
    const char* who = "linear";
    DBLP_TRY(check_linear(who, l, 0));
    if (l->rows == 0 || l->out == 0) return DBLP_OK;
    if (l->in) {
        DBLP_TRY(check_matrix(who, "x", x, l->rows, l->in, l->dtype, false, false));
        DBLP_TRY(check_matrix(who, "w", w, l->in, l->out, l->dtype, true, false));
    }
    DBLP_TRY(check_matrix(who, "out", out, l->rows, l->out, l->out_dtype, false, true));
    if (residual) DBLP_TRY(check_matrix(who, "residual", residual, l->rows, l->out, l->out_dtype, false, false));
    if (pre) DBLP_TRY(check_matrix(who, "pre", pre, l->rows, l->out, l->dtype, false, true));
    DBLP_TRY(check_vector(who, "bias", bias, l->bias_dtype));
    DBLP_TRY(check_space(who, ws, ws_bytes, forward_bytes(l, x, w)));
    {                                                           // blocks write while others still read x, w and bias
        const Extent eo = extent_of(out, l->rows, l->out, l->out_dtype), ep = pre ? extent_of(pre, l->rows, l->out, l->dtype) : Extent{};
        if (l->in) {
            const Extent ex = extent_of(x, l->rows, l->in, l->dtype), ew = extent_of(w, l->in, l->out, l->dtype);
            DBLP_TRY(check_apart(who, "out", eo, "x", ex));
            DBLP_TRY(check_apart(who, "out", eo, "w", ew));
            if (pre) DBLP_TRY(check_apart(who, "pre", ep, "x", ex));
            if (pre) DBLP_TRY(check_apart(who, "pre", ep, "w", ew));
        }
        if (bias) DBLP_TRY(check_apart(who, "out", eo, "bias", extent_of(bias, 0, 1, l->out, l->bias_dtype)));
        if (bias && pre) DBLP_TRY(check_apart(who, "pre", ep, "bias", extent_of(bias, 0, 1, l->out, l->bias_dtype)));
        if (pre) DBLP_TRY(check_apart(who, "pre", ep, "out", eo));
        if (residual) {
            const Extent er = extent_of(residual, l->rows, l->out, l->out_dtype);
            DBLP_TRY(check_same_or_apart(who, "out", out, eo, "residual", residual, er));
            if (pre) DBLP_TRY(check_apart(who, "pre", ep, "residual", er));
        }
    }
    const dblp_matrix_t none{nullptr, 1, 1};
    const Product p = l->in ? forward_product(l, x, w) : forward_product(l, &none, &none);
    auto go = [&](auto t, auto o) -> int {
        using T = decltype(t);
        using O = decltype(o);
        EpiLinear<T, O> e{};
        e.out = rows_of<O>(out->data, out->row_stride, l->rows);
        if (residual) e.residual = rows_of<O>(residual->data, residual->row_stride, l->rows);
        if (pre) e.pre = rows_of<T>(pre->data, pre->row_stride, l->rows);
        e.bias = bias;
        e.bias_dtype = l->bias_dtype;
        e.bias_whole = (uintptr_t)bias % 32 == 0;
        e.act = l->activation;
        return run_product<sizeof(O) == 4>(p, e, ws, false, (cudaStream_t)stream);
    };
    if (l->dtype == DBLP_BF16) return l->out_dtype == DBLP_F32 ? go(__nv_bfloat16(), float()) : go(__nv_bfloat16(), __nv_bfloat16());
    return l->out_dtype == DBLP_F32 ? go(__half(), float()) : go(__half(), __half());
}

extern "C" int dblp_linear_grad(const dblp_linear_t* l, const dblp_matrix_t* dy, const dblp_matrix_t* x, const dblp_matrix_t* w,
                                const dblp_matrix_t* residual, const dblp_matrix_t* pre, const dblp_matrix_t* dx, const dblp_matrix_t* dw,
                                void* dbias, void* ws, size_t ws_bytes, void* stream)
{
    const char* who = "linear_grad";
    DBLP_TRY(check_linear(who, l, DBLP_ACCUMULATE));
    DBLP_REQUIRE(!dx || (pre != nullptr) == (l->activation != DBLP_ACT_NONE), DBLP_EINVAL, "%s: dx needs pre with an activation, and only then", who);
    const bool want_dx = dx && l->rows && l->in, want_dw = dw && l->in && l->out, want_db = dbias && l->out;
    const cudaStream_t s = (cudaStream_t)stream;
    if (l->rows && l->out && (want_dx || want_dw || want_db)) DBLP_TRY(check_matrix(who, "dy", dy, l->rows, l->out, l->dtype, false, false));
    if (want_dx) {
        if (l->out) DBLP_TRY(check_matrix(who, "w", w, l->in, l->out, l->dtype, true, false));
        DBLP_TRY(check_matrix(who, "dx", dx, l->rows, l->in, l->dtype, false, true));
        if (residual) DBLP_TRY(check_matrix(who, "residual", residual, l->rows, l->in, l->dtype, false, false));
        if (pre) DBLP_TRY(check_matrix(who, "pre", pre, l->rows, l->in, l->dtype, false, false));
    }
    if (want_dw) {
        if (l->rows) DBLP_TRY(check_matrix(who, "x", x, l->rows, l->in, l->dtype, false, false));
        DBLP_TRY(check_matrix(who, "dw", dw, l->in, l->out, l->out_dtype, true, true));
    }
    if (want_db) DBLP_TRY(check_vector(who, "dbias", dbias, l->bias_dtype));
    const dblp_matrix_t none{nullptr, 1, 1};
    size_t need = want_db ? sum_bytes(l) : 0;
    const Product px = l->out ? dx_product(l, dy ? dy : &none, w ? w : &none) : dx_product(l, &none, &none);
    const bool by_rows = !want_dw || is_by_rows(dw, l->out);
    const Product pw = l->rows ? dw_product(l, dy ? dy : &none, x ? x : &none, by_rows) : dw_product(l, &none, &none, by_rows);
    if (want_dx && l->out) need = max(need, product_space(px));
    if (want_dw && l->rows) need = max(need, product_space(pw));
    DBLP_TRY(check_space(who, ws, ws_bytes, need));
    {                                                           // what a result may lie over: nothing that is read after its first block has written
        Extent out[3], in[5];
        const char *out_name[3], *in_name[5];
        int outs = 0, ins = 0;
        auto output = [&](const char* name, const Extent& e) { out_name[outs] = name; out[outs++] = e; };
        auto input = [&](const char* name, const Extent& e) { in_name[ins] = name; in[ins++] = e; };
        if (l->rows && l->out && (want_dx || want_dw || want_db)) input("dy", extent_of(dy, l->rows, l->out, l->dtype));
        if (want_dx && l->out) input("w", extent_of(w, l->in, l->out, l->dtype));
        const int for_dx = ins;                                 // dx comes last: x, read for dw, may lie under it
        if (want_dw && l->rows) input("x", extent_of(x, l->rows, l->in, l->dtype));
        if (want_dx && residual) input("residual", extent_of(residual, l->rows, l->in, l->dtype));
        if (want_dx && pre) input("pre", extent_of(pre, l->rows, l->in, l->dtype));
        if (want_dw) output("dw", extent_of(dw, l->in, l->out, l->out_dtype));
        if (want_db) output("dbias", extent_of(dbias, 0, 1, l->out, l->bias_dtype));
        for (int i = 0; i < outs; ++i)
            for (int j = 0; j < ins; ++j) DBLP_TRY(check_apart(who, out_name[i], out[i], in_name[j], in[j]));
        if (outs == 2) DBLP_TRY(check_apart(who, "dw", out[0], "dbias", out[1]));
        if (want_dx) {
            const Extent ex = extent_of(dx, l->rows, l->in, l->dtype);
            for (int i = 0; i < outs; ++i) DBLP_TRY(check_apart(who, "dx", ex, out_name[i], out[i]));
            for (int j = 0; j < for_dx; ++j) DBLP_TRY(check_apart(who, "dx", ex, in_name[j], in[j]));
            if (residual) DBLP_TRY(check_same_or_apart(who, "dx", dx, ex, "residual", residual, extent_of(residual, l->rows, l->in, l->dtype)));
            if (pre) DBLP_TRY(check_same_or_apart(who, "dx", dx, ex, "pre", pre, extent_of(pre, l->rows, l->in, l->dtype)));
        }
    }

    // dw before dx: dx may be written over pre or the residual, never over x or dy
    if (want_db) DBLP_TRY(column_sums(l, dy, dbias, ws, s));
    if (want_dw)
        DBLP_TRY(with_type(l->out_dtype, [&](auto t) -> int {
            using O = decltype(t);
            EpiStore<O> e{};
            e.out = rows_of<O>(dw->data, by_rows ? dw->row_stride : dw->col_stride, by_rows ? l->in : l->out);
            e.accumulate = l->flags & DBLP_ACCUMULATE;
            return run_product<sizeof(O) == 4>(pw, e, ws, false, s);
        }));
    if (!want_dx) return DBLP_OK;
    auto go = [&](auto t) -> int {
        using T = decltype(t);
        EpiGradX<T> e{};
        e.out = rows_of<T>(dx->data, dx->row_stride, l->rows);
        if (residual) e.residual = rows_of<T>(residual->data, residual->row_stride, l->rows);
        if (pre) e.pre = rows_of<T>(pre->data, pre->row_stride, l->rows);
        e.act = l->activation;
        return run_product<false>(px, e, ws, false, s);
    };
    return l->dtype == DBLP_BF16 ? go(__nv_bfloat16()) : go(__half());
}
