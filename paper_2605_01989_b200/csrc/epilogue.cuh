// What is done with a matrix product's fp32 sums: eight consecutive columns of one row at a time, so that everything around
// the product is read and written 16 bytes (fp32: 32) a thread.
#pragma once

#include "types.cuh"

namespace dblp {

// A row-major matrix that an epilogue reads or writes.  vec: data and row stride allow 16-byte accesses at columns that
// are multiples of eight.
struct Rows {
    void* p;
    int64_t stride;
    int dtype;
    bool vec;
    __device__ __forceinline__ explicit operator bool() const { return p != nullptr; }
};
inline Rows rows_of(const void* p, int64_t stride, uint64_t rows, int dtype)
{
    if (rows <= 1) stride = 0;
    const int64_t unit = 16 / element_bytes(dtype);
    return Rows{(void*)p, stride, dtype, aligned16(p) && stride % unit == 0};
}

template <typename T> __device__ __forceinline__ void load8(const T* p, uint32_t left, bool vec, float* x)
{
    if (vec && left >= 8) {
        Vec8<T> v;
        v.load(p);
        v.get(x);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i) x[i] = i < left ? to_f32(p[i]) : 0.0f;
    }
}
template <typename T> __device__ __forceinline__ void store8(T* p, uint32_t left, bool vec, const float* x)
{
    if (vec && left >= 8) {
        Vec8<T> v;
        v.set(x);
        v.store(p);
    } else {
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
            if (i < left) p[i] = from_f32<T>(x[i]);
    }
}
__device__ __forceinline__ void load8(const Rows& r, uint32_t m, uint32_t n, uint32_t left, float* x)
{
    const int64_t at = (int64_t)m * r.stride + n;
    if (r.dtype == DBLP_F32) load8((const float*)r.p + at, left, r.vec, x);
    else if (r.dtype == DBLP_BF16) load8((const __nv_bfloat16*)r.p + at, left, r.vec, x);
    else load8((const __half*)r.p + at, left, r.vec, x);
}
__device__ __forceinline__ void store8(const Rows& r, uint32_t m, uint32_t n, uint32_t left, const float* x)
{
    const int64_t at = (int64_t)m * r.stride + n;
    if (r.dtype == DBLP_F32) store8((float*)r.p + at, left, r.vec, x);
    else if (r.dtype == DBLP_BF16) store8((__nv_bfloat16*)r.p + at, left, r.vec, x);
    else store8((__half*)r.p + at, left, r.vec, x);
}

// Eight elements on their way: as loaded where a whole vector was, else as fp32.  What an epilogue reads is fetched for several
// rows before the first is used, so that one latency is paid and not one a row.
struct Raw {
    uint4 a, b;
};
__device__ __forceinline__ void fetch8(const Rows& r, uint32_t m, uint32_t n, uint32_t left, Raw& x)
{
    if (r.vec && left >= 8) {
        const char* p = (const char*)r.p + ((int64_t)m * r.stride + n) * (r.dtype == DBLP_F32 ? 4 : 2);
        x.a = *reinterpret_cast<const uint4*>(p);
        if (r.dtype == DBLP_F32) x.b = *reinterpret_cast<const uint4*>(p + 16);
    } else {
        float t[8];
        load8(r, m, n, left, t);
        x.a = make_uint4(__float_as_uint(t[0]), __float_as_uint(t[1]), __float_as_uint(t[2]), __float_as_uint(t[3]));
        x.b = make_uint4(__float_as_uint(t[4]), __float_as_uint(t[5]), __float_as_uint(t[6]), __float_as_uint(t[7]));
    }
}
template <typename T> __device__ __forceinline__ void widen(const uint4& w, float* x)
{
    Vec8<T> v;
    v.w = w;
    v.get(x);
}
__device__ __forceinline__ void use8(const Rows& r, uint32_t left, const Raw& x, float* t)
{
    if (r.dtype == DBLP_F32 || !r.vec || left < 8) {
        t[0] = __uint_as_float(x.a.x); t[1] = __uint_as_float(x.a.y); t[2] = __uint_as_float(x.a.z); t[3] = __uint_as_float(x.a.w);
        t[4] = __uint_as_float(x.b.x); t[5] = __uint_as_float(x.b.y); t[6] = __uint_as_float(x.b.z); t[7] = __uint_as_float(x.b.w);
    } else if (r.dtype == DBLP_BF16) widen<__nv_bfloat16>(x.a, t);
    else widen<__half>(x.a, t);
}

// ---- activations -----------------------------------------------------------------------------------------------------
// 1 / (1 + e^-x), 0 and 1 at the ends.
__device__ __forceinline__ float logistic(float x) { return __fdividef(1.0f, 1.0f + __expf(-x)); }

// gelu_tanh(z) = z logistic(2 u), 2 u = sqrt(8 / pi) (z + 0.044715 z^3): the same function without a tanh.
__device__ __forceinline__ float tanh_arg(float z) { return 1.5957691216057308f * z * fmaf(0.044715f * z, z, 1.0f); }

__device__ __forceinline__ void activate(int act, float* z)
{
    switch (act) {
    case DBLP_ACT_RELU:
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = z[i] < 0.0f ? 0.0f : z[i];
        break;
    case DBLP_ACT_GELU:
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] = 0.5f * z[i] * erfcf(-0.70710678118654752f * z[i]);
        break;
    case DBLP_ACT_GELU_TANH:
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] *= logistic(tanh_arg(z[i]));
        break;
    case DBLP_ACT_SILU:
#pragma unroll
        for (int i = 0; i < 8; ++i) z[i] *= logistic(z[i]);
        break;
    default: break;
    }
}

// y *= act'(z)
__device__ __forceinline__ void activate_grad(int act, const float* z, float* y)
{
    switch (act) {
    case DBLP_ACT_RELU:
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = z[i] > 0.0f ? y[i] : (z[i] <= 0.0f ? 0.0f : z[i] * y[i]);
        break;
    case DBLP_ACT_GELU:
#pragma unroll
        for (int i = 0; i < 8; ++i)
            y[i] *= fmaf(z[i] * 0.39894228040143268f, __expf(-0.5f * z[i] * z[i]), 0.5f * erfcf(-0.70710678118654752f * z[i]));
        break;
    case DBLP_ACT_GELU_TANH:
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float g = logistic(tanh_arg(z[i])), zz = fminf(z[i] * z[i], 1e12f);        // g (1 - g) is 0 long before
            y[i] *= fmaf(z[i] * g * (1.0f - g), 1.5957691216057308f * fmaf(0.134145f, zz, 1.0f), g);
        }
        break;
    case DBLP_ACT_SILU:
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float g = logistic(z[i]);
            y[i] *= fmaf(z[i] * g, 1.0f - g, g);
        }
        break;
    default: break;
    }
}

// ---- epilogues -----------------------------------------------------------------------------------------------------------
// v holds the sums of row m, columns n .. n + 7 (left of them inside the matrix) of product b; what `fetch` loaded for them is in f.
struct EpiLinear {                        // out = act(z) + residual, pre = z = v + bias
    Rows out, residual, pre, bias;
    int act;
    struct Fetched { Raw bias, residual; };
    __device__ __forceinline__ void fetch(uint32_t, uint32_t m, uint32_t n, uint32_t left, Fetched& f) const
    {
        if (bias) fetch8(bias, 0, n, left, f.bias);
        if (residual) fetch8(residual, m, n, left, f.residual);
    }
    __device__ __forceinline__ void apply(uint32_t, uint32_t m, uint32_t n, uint32_t left, const Fetched& f, float* v) const
    {
        float t[8];
        if (bias) {
            use8(bias, left, f.bias, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
        if (pre) store8(pre, m, n, left, v);
        activate(act, v);
        if (residual) {
            use8(residual, left, f.residual, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
        store8(out, m, n, left, v);
    }
};

struct EpiGradX {                         // dx = (v + residual) act'(pre)
    Rows out, residual, pre;
    int act;
    struct Fetched { Raw residual, pre; };
    __device__ __forceinline__ void fetch(uint32_t, uint32_t m, uint32_t n, uint32_t left, Fetched& f) const
    {
        if (residual) fetch8(residual, m, n, left, f.residual);
        if (pre) fetch8(pre, m, n, left, f.pre);
    }
    __device__ __forceinline__ void apply(uint32_t, uint32_t m, uint32_t n, uint32_t left, const Fetched& f, float* v) const
    {
        float t[8];
        if (residual) {
            use8(residual, left, f.residual, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
        if (pre) {
            use8(pre, left, f.pre, t);
            activate_grad(act, t, v);
        }
        store8(out, m, n, left, v);
    }
};

struct EpiStore {                         // out = v [+ out]
    Rows out;
    bool accumulate;
    struct Fetched { Raw out; };
    __device__ __forceinline__ void fetch(uint32_t, uint32_t m, uint32_t n, uint32_t left, Fetched& f) const
    {
        if (accumulate) fetch8(out, m, n, left, f.out);
    }
    __device__ __forceinline__ void apply(uint32_t, uint32_t m, uint32_t n, uint32_t left, const Fetched& f, float* v) const
    {
        if (accumulate) {
            float t[8];
            use8(out, left, f.out, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
        store8(out, m, n, left, v);
    }
};

// The sums themselves, fp32, one matrix of M x stride per (product, part of the summed dimension): b numbers them.
struct EpiPartial {
    float* p;
    int64_t each;
    uint32_t stride;                      // a multiple of eight
    struct Fetched {};
    __device__ __forceinline__ void fetch(uint32_t, uint32_t, uint32_t, uint32_t, Fetched&) const {}
    __device__ __forceinline__ void apply(uint32_t b, uint32_t m, uint32_t n, uint32_t, const Fetched&, float* v) const
    {
        store8(p + b * each + (int64_t)m * stride + n, 8, true, v);           // rows are padded: whole groups always fit
    }
};

// A matrix in workspace as one or two f16 words an element: value * scale = hi [+ lo].  Batches of `each` elements, rows
// of `stride`, a multiple of eight, so that whole groups always fit.
struct Words {
    __half *hi, *lo;
    int64_t each;
    uint32_t stride;
    struct Fetched { uint4 hi, lo; };
    __device__ __forceinline__ int64_t at(uint32_t b, uint32_t m, uint32_t n) const { return b * each + (int64_t)m * stride + n; }
    __device__ __forceinline__ void fetch(uint32_t b, uint32_t m, uint32_t n, Fetched& f) const
    {
        if (!hi) return;
        f.hi = *reinterpret_cast<const uint4*>(hi + at(b, m, n));
        if (lo) f.lo = *reinterpret_cast<const uint4*>(lo + at(b, m, n));
    }
    __device__ __forceinline__ void use(const Fetched& f, float* x) const
    {
        widen<__half>(f.hi, x);
        if (lo) {
            float t[8];
            widen<__half>(f.lo, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] += t[i];
        }
    }
    __device__ __forceinline__ void store(uint32_t b, uint32_t m, uint32_t n, const float* x) const
    {
        Vec8<__half> v;
        v.set(x);
        v.store(hi + at(b, m, n));
        if (lo) {
            float t[8];
            v.get(t);
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = x[i] - t[i];
            v.set(t);
            v.store(lo + at(b, m, n));
        }
    }
};

struct EpiPoly {                          // out = alpha v [+ beta add], both in words
    Words out, add;
    float alpha, beta;
    using Fetched = Words::Fetched;
    __device__ __forceinline__ void fetch(uint32_t b, uint32_t m, uint32_t n, uint32_t, Fetched& f) const { add.fetch(b, m, n, f); }
    __device__ __forceinline__ void apply(uint32_t b, uint32_t m, uint32_t n, uint32_t, const Fetched& f, float* v) const
    {
        float t[8] = {};
        if (add.hi) add.use(f, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(beta, t[i], alpha * v[i]);
        out.store(b, m, n, v);
    }
};

struct EpiLast {                          // the caller's out = alpha v + beta add
    Rows out;
    int64_t each;
    Words add;
    float alpha, beta;
    using Fetched = Words::Fetched;
    __device__ __forceinline__ void fetch(uint32_t b, uint32_t m, uint32_t n, uint32_t, Fetched& f) const { add.fetch(b, m, n, f); }
    __device__ __forceinline__ void apply(uint32_t b, uint32_t m, uint32_t n, uint32_t left, const Fetched& f, float* v) const
    {
        float t[8];
        add.use(f, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(beta, t[i], alpha * v[i]);
        Rows o = out;
        o.p = (char*)o.p + b * each * (o.dtype == DBLP_F32 ? 4 : 2);
        store8(o, m, n, left, v);
    }
};

}  // namespace dblp
