// What is done with a matrix product's fp32 sums: sixteen consecutive columns of one row at a time, whole 32-byte sectors of a
// 16-bit matrix (two accesses of 16 bytes at a stride of 32 touch every sector twice).
#pragma once

#include "tc.cuh"

namespace dblp {

// A row-major matrix that an epilogue reads or writes.  vec: bytes that an access at a column that is a multiple of sixteen may
// have, 32 or 16; 0 = element by element.
struct Rows {
    void* p;
    int64_t stride;
    int dtype, vec;
    __device__ __forceinline__ explicit operator bool() const { return p != nullptr; }
};
inline Rows rows_of(const void* p, int64_t stride, uint64_t rows, int dtype)
{
    if (rows <= 1) stride = 0;
    const uint64_t at = (uintptr_t)p | (uint64_t)stride * element_bytes(dtype);
    return Rows{(void*)p, stride, dtype, at % 32 == 0 ? 32 : (at % 16 == 0 ? 16 : 0)};
}

inline bool whole(const Rows& r) { return r.p == nullptr || r.vec == 32; }

__device__ __forceinline__ void load32(const void* p, uint32_t* w)
{
    asm volatile("ld.global.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7])
                 : "l"(p)
                 : "memory");
}
__device__ __forceinline__ void store32(void* p, const uint32_t* w)
{
    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]),
                 "r"(w[6]), "r"(w[7])
                 : "memory");
}
// 32 bytes, in one access or two.
__device__ __forceinline__ void load_words(const void* p, int vec, uint32_t* w)
{
    if (vec == 32) {
        load32(p, w);
    } else {
        const uint4 a = ((const uint4*)p)[0], b = ((const uint4*)p)[1];
        w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
    }
}
__device__ __forceinline__ void store_words(void* p, int vec, const uint32_t* w)
{
    if (vec == 32) {
        store32(p, w);
    } else {
        ((uint4*)p)[0] = make_uint4(w[0], w[1], w[2], w[3]);
        ((uint4*)p)[1] = make_uint4(w[4], w[5], w[6], w[7]);
    }
}

// Sixteen elements on their way: as loaded where whole vectors were (in the first eight words those of a 16-bit type), else as
// fp32.  What an epilogue reads is fetched before the sums it belongs to are there.
struct Raw {
    uint32_t w[16];
};
__device__ __forceinline__ void fetch16(const Rows& r, uint32_t m, uint32_t n, uint32_t left, Raw& x)
{
    const int64_t at = (int64_t)m * r.stride + n;
    if (r.vec && left >= 16) {
        const char* p = (const char*)r.p + at * (r.dtype == DBLP_F32 ? 4 : 2);
        load_words(p, r.vec, x.w);
        if (r.dtype == DBLP_F32) load_words(p + 32, r.vec, x.w + 8);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i) {
            float t = 0.0f;
            if (i < left)
                t = r.dtype == DBLP_F32 ? ((const float*)r.p)[at + i]
                                        : (r.dtype == DBLP_BF16 ? to_f32(((const __nv_bfloat16*)r.p)[at + i]) : to_f32(((const __half*)r.p)[at + i]));
            x.w[i] = __float_as_uint(t);
        }
    }
}
template <typename T> __device__ __forceinline__ void widen16(const uint32_t* w, float* x)
{
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float2 f = unpack2<T>(w[i]);
        x[2 * i] = f.x;
        x[2 * i + 1] = f.y;
    }
}
__device__ __forceinline__ void use16(const Rows& r, uint32_t left, const Raw& x, float* t)
{
    if (r.dtype == DBLP_F32 || !r.vec || left < 16) {
#pragma unroll
        for (int i = 0; i < 16; ++i) t[i] = __uint_as_float(x.w[i]);
    } else if (r.dtype == DBLP_BF16) widen16<__nv_bfloat16>(x.w, t);
    else widen16<__half>(x.w, t);
}
template <typename T> __device__ __forceinline__ void store16(T* p, uint32_t left, int vec, const float* x)
{
    if (vec && left >= 16) {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pack2<T>(x[2 * i], x[2 * i + 1]);
        store_words(p, vec, w);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i)
            if (i < left) p[i] = from_f32<T>(x[i]);
    }
}
template <> __device__ __forceinline__ void store16<float>(float* p, uint32_t left, int vec, const float* x)
{
    if (vec && left >= 16) {
        store_words(p, vec, reinterpret_cast<const uint32_t*>(x));
        store_words(p + 8, vec, reinterpret_cast<const uint32_t*>(x) + 8);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 16; ++i)
            if (i < left) p[i] = x[i];
    }
}
__device__ __forceinline__ void store16(const Rows& r, uint32_t m, uint32_t n, uint32_t left, const float* x)
{
    const int64_t at = (int64_t)m * r.stride + n;
    if (r.dtype == DBLP_F32) store16((float*)r.p + at, left, r.vec, x);
    else if (r.dtype == DBLP_BF16) store16((__nv_bfloat16*)r.p + at, left, r.vec, x);
    else store16((__half*)r.p + at, left, r.vec, x);
}

// Eight elements, for the kernels around the products.
__device__ __forceinline__ void load8(const Rows& r, uint32_t m, uint32_t n, uint32_t left, float* x)
{
    const int64_t at = (int64_t)m * r.stride + n;
    auto go = [&](auto tag) {
        using T = decltype(tag);
        const T* p = (const T*)r.p + at;
        if (r.vec && left >= 8) {
            Vec8<T> v;
            v.load(p);
            v.get(x);
        } else {
#pragma unroll
            for (uint32_t i = 0; i < 8; ++i) x[i] = i < left ? to_f32(p[i]) : 0.0f;
        }
    };
    if (r.dtype == DBLP_F32) go(float());
    else if (r.dtype == DBLP_BF16) go(__nv_bfloat16());
    else go(__half());
}

// ---- activations -----------------------------------------------------------------------------------------------------
__device__ __forceinline__ float reciprocal(float x)            // 0 of infinity
{
    float r;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
    return r;
}
// 1 / (1 + e^-x), 0 and 1 at the ends.
__device__ __forceinline__ float logistic(float x) { return reciprocal(1.0f + exp2_fast(-1.4426950408889634f * x)); }

// gelu_tanh(z) = z logistic(2 u), 2 u = sqrt(8 / pi) (z + 0.044715 z^3): the same function without a tanh.
__device__ __forceinline__ float tanh_arg(float z) { return 1.5957691216057308f * z * fmaf(0.044715f * z, z, 1.0f); }

// The normal distribution's integral up to z, and e^(-z^2 / 2), of two values.  With x = |z| / sqrt 2 and t = 1 / (1 + 0.46 x), the tail
// erfc(x) / 2 is e^(-x^2) t P(t): P of degree 7 was fitted here to the least largest relative error over x >= 0 (7e-7), so that far
// tails keep their digits.  (CUDA's erfcf in its place: 8192 x 1600 -> 6400 with bias and gelu 431 us instead of 184.)
__device__ __forceinline__ float2 normal_cdf(float2 z, float2& e)
{
    auto two = [](float x) { return make_float2(x, x); };
    const float2 d = fma2(make_float2(fabsf(z.x), fabsf(z.y)), two(0.32526912f), two(1.0f)), t = make_float2(reciprocal(d.x), reciprocal(d.y));
    const float2 x = mul2(mul2(z, two(-0.72134752f)), z);
    e = make_float2(exp2_fast(x.x), exp2_fast(x.y));
    float2 p = fma2(two(0.0338571332f), t, two(-0.113314494f));
    p = fma2(p, t, two(0.0845952928f));
    p = fma2(p, t, two(0.0263054594f));
    p = fma2(p, t, two(0.0934238359f));
    p = fma2(p, t, two(0.115590952f));
    p = fma2(p, t, two(0.129778638f));
    p = mul2(mul2(fma2(p, t, two(0.129763529f)), t), e);
    const float2 q = fma2(p, two(-1.0f), two(1.0f));
    return make_float2(z.x > 0.0f ? q.x : p.x, z.y > 0.0f ? q.y : p.y);
}

template <int N> __device__ __forceinline__ void activate(int act, float* z)
{
    switch (act) {
    case DBLP_ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] = z[i] < 0.0f ? 0.0f : z[i];
        break;
    case DBLP_ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            float2 e;
            const float2 x = make_float2(z[i], z[i + 1]), y = mul2(x, normal_cdf(x, e));
            z[i] = y.x;
            z[i + 1] = y.y;
        }
        break;
    case DBLP_ACT_GELU_TANH:
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] *= logistic(tanh_arg(z[i]));
        break;
    case DBLP_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i) z[i] *= logistic(z[i]);
        break;
    default: break;
    }
}

// y *= act'(z)
template <int N> __device__ __forceinline__ void activate_grad(int act, const float* z, float* y)
{
    switch (act) {
    case DBLP_ACT_RELU:
#pragma unroll
        for (int i = 0; i < N; ++i) y[i] = z[i] > 0.0f ? y[i] : (z[i] <= 0.0f ? 0.0f : z[i] * y[i]);
        break;
    case DBLP_ACT_GELU:
#pragma unroll
        for (int i = 0; i < N; i += 2) {
            float2 e;
            const float2 x = make_float2(z[i], z[i + 1]), c = normal_cdf(x, e), d = fma2(mul2(x, make_float2(0.39894228f, 0.39894228f)), e, c);
            y[i] *= d.x;
            y[i + 1] *= d.y;
        }
        break;
    case DBLP_ACT_GELU_TANH:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float g = logistic(tanh_arg(z[i])), zz = fminf(z[i] * z[i], 1e12f);        // g (1 - g) is 0 long before
            y[i] *= fmaf(z[i] * g * (1.0f - g), 1.5957691216057308f * fmaf(0.134145f, zz, 1.0f), g);
        }
        break;
    case DBLP_ACT_SILU:
#pragma unroll
        for (int i = 0; i < N; ++i) {
            const float g = logistic(z[i]);
            y[i] *= fmaf(z[i] * g, 1.0f - g, g);
        }
        break;
    default: break;
    }
}

// ---- epilogues -----------------------------------------------------------------------------------------------------------
// v holds the sums of row m, columns n .. n + 15 (left of them inside the matrix) of product b; what `fetch` loaded for them is in f.
struct EpiLinear {                        // out = act(z) + residual, pre = z = v + bias
    Rows out, residual, pre, bias;
    int act;
    bool sectors() const { return whole(out) && whole(residual) && whole(pre); }
    struct Fetched { Raw bias, residual; };
    __device__ __forceinline__ void fetch(uint32_t, uint32_t m, uint32_t n, uint32_t left, Fetched& f) const
    {
        if (bias) fetch16(bias, 0, n, left, f.bias);
        if (residual) fetch16(residual, m, n, left, f.residual);
    }
    __device__ __forceinline__ void apply(uint32_t, uint32_t m, uint32_t n, uint32_t left, const Fetched& f, float* v) const
    {
        float t[16];
        if (bias) {
            use16(bias, left, f.bias, t);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] += t[i];
        }
        if (pre) store16(pre, m, n, left, v);
        activate<16>(act, v);
        if (residual) {
            use16(residual, left, f.residual, t);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] += t[i];
        }
        store16(out, m, n, left, v);
    }
};

struct EpiGradX {                         // dx = (v + residual) act'(pre)
    Rows out, residual, pre;
    int act;
    bool sectors() const { return whole(out) && whole(residual) && whole(pre); }
    struct Fetched { Raw residual, pre; };
    __device__ __forceinline__ void fetch(uint32_t, uint32_t m, uint32_t n, uint32_t left, Fetched& f) const
    {
        if (residual) fetch16(residual, m, n, left, f.residual);
        if (pre) fetch16(pre, m, n, left, f.pre);
    }
    __device__ __forceinline__ void apply(uint32_t, uint32_t m, uint32_t n, uint32_t left, const Fetched& f, float* v) const
    {
        float t[16];
        if (residual) {
            use16(residual, left, f.residual, t);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] += t[i];
        }
        if (pre) {
            use16(pre, left, f.pre, t);
            activate_grad<16>(act, t, v);
        }
        store16(out, m, n, left, v);
    }
};

struct EpiStore {                         // out = v [+ out]
    Rows out;
    bool accumulate;
    bool sectors() const { return whole(out); }
    struct Fetched { Raw out; };
    __device__ __forceinline__ void fetch(uint32_t, uint32_t m, uint32_t n, uint32_t left, Fetched& f) const
    {
        if (accumulate) fetch16(out, m, n, left, f.out);
    }
    __device__ __forceinline__ void apply(uint32_t, uint32_t m, uint32_t n, uint32_t left, const Fetched& f, float* v) const
    {
        if (accumulate) {
            float t[16];
            use16(out, left, f.out, t);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] += t[i];
        }
        store16(out, m, n, left, v);
    }
};

// A matrix in workspace as one or two f16 words an element: value * scale = hi [+ lo].  Batches of `each` elements, rows
// of `stride`, a multiple of sixteen, so that whole groups always fit.
struct Words {
    __half *hi, *lo;
    int64_t each;
    uint32_t stride;
    struct Fetched { uint32_t hi[8], lo[8]; };
    __device__ __forceinline__ int64_t at(uint32_t b, uint32_t m, uint32_t n) const { return b * each + (int64_t)m * stride + n; }
    __device__ __forceinline__ void fetch(uint32_t b, uint32_t m, uint32_t n, Fetched& f) const
    {
        if (!hi) return;
        load32(hi + at(b, m, n), f.hi);
        if (lo) load32(lo + at(b, m, n), f.lo);
    }
    __device__ __forceinline__ void use(const Fetched& f, float* x) const
    {
        widen16<__half>(f.hi, x);
        if (lo) {
            float t[16];
            widen16<__half>(f.lo, t);
#pragma unroll
            for (int i = 0; i < 16; ++i) x[i] += t[i];
        }
    }
    __device__ __forceinline__ void store(uint32_t b, uint32_t m, uint32_t n, const float* x) const
    {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pack2<__half>(x[2 * i], x[2 * i + 1]);
        store32(hi + at(b, m, n), w);
        if (lo) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 t = unpack2<__half>(w[i]);
                w[i] = pack2<__half>(x[2 * i] - t.x, x[2 * i + 1] - t.y);
            }
            store32(lo + at(b, m, n), w);
        }
    }
};

struct EpiPoly {                          // out = alpha v [+ beta add], both in words
    Words out, add;
    float alpha, beta;
    bool sectors() const { return true; }
    using Fetched = Words::Fetched;
    __device__ __forceinline__ void fetch(uint32_t b, uint32_t m, uint32_t n, uint32_t, Fetched& f) const { add.fetch(b, m, n, f); }
    __device__ __forceinline__ void apply(uint32_t b, uint32_t m, uint32_t n, uint32_t, const Fetched& f, float* v) const
    {
        float t[16] = {};
        if (add.hi) add.use(f, t);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = fmaf(beta, t[i], alpha * v[i]);
        out.store(b, m, n, v);
    }
};

struct EpiLast {                          // the caller's out = alpha v + beta add
    Rows out;
    int64_t each;
    Words add;
    float alpha, beta;
    bool sectors() const { return whole(out); }
    using Fetched = Words::Fetched;
    __device__ __forceinline__ void fetch(uint32_t b, uint32_t m, uint32_t n, uint32_t, Fetched& f) const { add.fetch(b, m, n, f); }
    __device__ __forceinline__ void apply(uint32_t b, uint32_t m, uint32_t n, uint32_t left, const Fetched& f, float* v) const
    {
        float t[16];
        add.use(f, t);
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] = fmaf(beta, t[i], alpha * v[i]);
        Rows o = out;
        o.p = (char*)o.p + b * each * (o.dtype == DBLP_F32 ? 4 : 2);
        store16(o, m, n, left, v);
    }
};

}  // namespace dblp
