// dblp_dropout, dblp_dropout_grad: out = [u(i) >= t] * x * 65536 / (65536 - t) [+ residual], u(i) = 16 bits of a Philox
// draw that eight consecutive elements share.
//
// Bound by HBM: 32768 x 6400 fp32 244 us (6.9 TB/s) in bursts, 264 us (6.4) under sustained load, 295 with two 16-byte
// accesses in place of one of 32; 8192 x 1600 bf16 with residual 13.9 us.
// Nothing is kept between forward and backward: the mask costs ten Philox rounds per eight elements (about five
// instructions an element) instead of a byte or bit each to write and read.
#include <math.h>

#include "types.cuh"

namespace dblp {

constexpr int kDropThreads = 256;

struct DropKey {
    uint2 key;
    uint32_t c2, c3;       // purpose | site << 8, step
    uint32_t t;            // dropped iff bits < t
    float inv;             // 65536 / (65536 - t), 0 when everything is dropped
};

__device__ __forceinline__ uint4 drop_draw(const DropKey& k, uint64_t group)
{
    return philox4x32_10(make_uint4((uint32_t)group, (uint32_t)(group >> 32), k.c2, k.c3), k.key);
}

__device__ __forceinline__ float drop_one(const DropKey& k, uint32_t bits, float x)
{
    return bits >= k.t ? __fmul_rn(x, k.inv) : 0.0f;
}

// A thread takes kGroups<T> groups of eight elements of contiguous rows (cols % 8 == 0 and 16-byte aligned rows, or
// everything one row of n elements), all loads before the first draw: one 16-byte load a thread leaves too few bytes in
// flight (32768 x 6400 bf16: 176 us with one group, 153 with two, where DRAM is the bound).  The last group of the one-row form may be short.
template <typename T> constexpr int kGroups = sizeof(T) == 2 ? 2 : 1;

template <typename T, bool RES>
__global__ void __launch_bounds__(kDropThreads)
k_dropout(const T* x, int64_t xs, const T* res, int64_t rs, T* out, int64_t os, uint64_t n, uint32_t groups_per_row, DropKey k)
{
    constexpr int U = kGroups<T>;
    const uint64_t g0 = (uint64_t)blockIdx.x * (kDropThreads * U) + threadIdx.x;
    int64_t xo[U], ro[U], oo[U];
    Vec8<T> vx[U], vr[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint64_t g = g0 + u * kDropThreads, e0 = g * 8;
        xo[u] = ro[u] = oo[u] = (int64_t)e0;
        if (groups_per_row) {
            const uint64_t row = g / groups_per_row, c = (g - row * groups_per_row) * 8;
            xo[u] = (int64_t)row * xs + c; ro[u] = (int64_t)row * rs + c; oo[u] = (int64_t)row * os + c;
        }
        if (e0 + 8 <= n) {
            vx[u].load(x + xo[u]);
            if (RES) vr[u].load(res + ro[u]);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint64_t g = g0 + u * kDropThreads, e0 = g * 8;
        if (e0 >= n) break;
        const uint4 w = drop_draw(k, g);
        const uint32_t b[4] = {w.x, w.y, w.z, w.w};
        if (e0 + 8 <= n) {
            float v[8], r[8];
            vx[u].get(v);
            if (RES) vr[u].get(r);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                v[i] = drop_one(k, i & 1 ? b[i >> 1] >> 16 : b[i >> 1] & 0xFFFFu, v[i]);
                if (RES) v[i] = __fadd_rn(v[i], r[i]);
            }
            vx[u].set(v);
            vx[u].store(out + oo[u]);
        } else {
            for (int i = 0; i < (int)(n - e0); ++i) {
                float y = drop_one(k, (b[i >> 1] >> (i & 1 ? 16 : 0)) & 0xFFFFu, to_f32(x[xo[u] + i]));
                if (RES) y = __fadd_rn(y, to_f32(res[ro[u] + i]));
                out[oo[u] + i] = from_f32<T>(y);
            }
        }
    }
}

// Any strides and widths: one thread per group, element by element.
template <typename T, bool RES>
__global__ void __launch_bounds__(kDropThreads)
k_dropout_any(const T* x, int64_t xs, const T* res, int64_t rs, T* out, int64_t os, uint64_t n, uint32_t cols, DropKey k)
{
    const uint64_t g = (uint64_t)blockIdx.x * kDropThreads + threadIdx.x, e0 = g * 8;
    if (e0 >= n) return;
    const uint4 w = drop_draw(k, g);
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
    uint64_t row = e0 / cols;
    uint32_t col = (uint32_t)(e0 - row * cols);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        if (e0 + i >= n) break;
        float y = drop_one(k, i & 1 ? u[i >> 1] >> 16 : u[i >> 1] & 0xFFFFu, to_f32(x[(int64_t)row * xs + col]));
        if (RES) y = __fadd_rn(y, to_f32(res[(int64_t)row * rs + col]));
        out[(int64_t)row * os + col] = from_f32<T>(y);
        if (++col == cols) { col = 0; ++row; }
    }
}

template <typename T>
static int launch_dropout(const T* x, int64_t xs, const T* res, int64_t rs, T* out, int64_t os, uint64_t rows, uint32_t cols,
                          const DropKey& k, cudaStream_t s)
{
    const uint64_t n = rows * cols, groups = (n + 7) / 8;
    const unsigned grid = (unsigned)((groups + kDropThreads - 1) / kDropThreads), gridv = (grid + kGroups<T> - 1) / kGroups<T>;
    const bool flat = rows == 1 || (xs == cols && os == cols && (!res || rs == cols));
    const bool vec = aligned16(x) && aligned16(out) && (!res || aligned16(res)) &&
                     (flat || (cols % 8 == 0 && xs % 8 == 0 && os % 8 == 0 && (!res || rs % 8 == 0)));
    if (vec) {
        const uint32_t gpr = flat ? 0 : cols / 8;
        if (res) k_dropout<T, true><<<gridv, kDropThreads, 0, s>>>(x, xs, res, rs, out, os, n, gpr, k);
        else k_dropout<T, false><<<gridv, kDropThreads, 0, s>>>(x, xs, res, rs, out, os, n, gpr, k);
    } else {
        if (res) k_dropout_any<T, true><<<grid, kDropThreads, 0, s>>>(x, xs, res, rs, out, os, n, cols, k);
        else k_dropout_any<T, false><<<grid, kDropThreads, 0, s>>>(x, xs, res, rs, out, os, n, cols, k);
    }
    DBLP_LAUNCHED();
    return DBLP_OK;
}

}  // namespace dblp

using namespace dblp;

extern "C" int dblp_dropout(const void* x, int64_t x_stride, const void* residual, int64_t residual_stride, void* out,
                            int64_t out_stride, uint64_t rows, uint32_t cols, int dtype, double p, uint64_t seed, uint32_t step,
                            uint32_t site, void* stream)
{
    DBLP_REQUIRE(known_dtype(dtype), DBLP_EINVAL, "dropout: unknown dtype %d", dtype);
    DBLP_REQUIRE(p >= 0.0 && p <= 1.0, DBLP_EINVAL, "dropout: p = %g outside [0, 1]", p);
    DBLP_REQUIRE(site < (1u << 24), DBLP_EINVAL, "dropout: site %u does not fit in 24 bits", site);
    if (rows == 0 || cols == 0) return DBLP_OK;
    DBLP_REQUIRE(x && out, DBLP_EINVAL, "dropout: null pointer");
    DBLP_REQUIRE(rows <= ((1ull << 41) - 1) / cols, DBLP_ECAPACITY, "dropout: 2^41 elements or more");
    DBLP_REQUIRE(rows == 1 || out_stride >= (int64_t)cols || out_stride <= -(int64_t)cols, DBLP_EINVAL,
                 "dropout: rows of the output overlap (stride %lld, %u columns)", (long long)out_stride, cols);
    const uint64_t es = element_bytes(dtype);
    DBLP_REQUIRE((uintptr_t)x % es == 0 && (uintptr_t)out % es == 0 && (uintptr_t)residual % es == 0, DBLP_EALIGN,
                 "dropout: a pointer is not aligned to its element type");
    DropKey k;
    k.key = make_uint2((uint32_t)seed, (uint32_t)(seed >> 32));
    k.c2 = kStreamDropout | site << 8;
    k.c3 = step;
    k.t = (uint32_t)floor(p * 65536.0);
    k.inv = k.t < 65536u ? (float)(65536.0 / (65536.0 - k.t)) : 0.0f;
    return with_type(dtype, [&](auto tag) -> int {
        using T = decltype(tag);
        return launch_dropout<T>((const T*)x, x_stride, (const T*)residual, residual_stride, (T*)out, out_stride, rows, cols, k,
                                 (cudaStream_t)stream);
    });
}

extern "C" int dblp_dropout_grad(const void* dout, int64_t dout_stride, void* dx, int64_t dx_stride, uint64_t rows, uint32_t cols,
                                 int dtype, double p, uint64_t seed, uint32_t step, uint32_t site, void* stream)
{
    return dblp_dropout(dout, dout_stride, nullptr, 0, dx, dx_stride, rows, cols, dtype, p, seed, step, site, stream);
}
