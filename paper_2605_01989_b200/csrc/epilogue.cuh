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

// ---- epilogues: v holds the sums of row m, columns n .. n + 7 (left of them inside the matrix) of product b -------------------
struct EpiLinear {                        // out = act(z) + residual, pre = z = v + bias
    Rows out, residual, pre, bias;
    int act;
    __device__ __forceinline__ void apply(uint32_t, uint32_t m, uint32_t n, uint32_t left, float* v) const
    {
        float t[8];
        if (bias) {
            load8(bias, 0, n, left, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
        if (pre) store8(pre, m, n, left, v);
        activate(act, v);
        if (residual) {
            load8(residual, m, n, left, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
        store8(out, m, n, left, v);
    }
};

struct EpiGradX {                         // dx = (v + residual) act'(pre)
    Rows out, residual, pre;
    int act;
    __device__ __forceinline__ void apply(uint32_t, uint32_t m, uint32_t n, uint32_t left, float* v) const
    {
        float t[8];
        if (residual) {
            load8(residual, m, n, left, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
        if (pre) {
            load8(pre, m, n, left, t);
            activate_grad(act, t, v);
        }
        store8(out, m, n, left, v);
    }
};

struct EpiStore {                         // out = v [+ out]
    Rows out;
    bool accumulate;
    __device__ __forceinline__ void apply(uint32_t, uint32_t m, uint32_t n, uint32_t left, float* v) const
    {
        if (accumulate) {
            float t[8];
            load8(out, m, n, left, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] += t[i];
        }
        store8(out, m, n, left, v);
    }
};

// A matrix in workspace as one or two f16 words an element: value * scale = hi [+ lo].  Batches of `each` elements, rows
// of `stride`, a multiple of eight.
struct Words {
    __half *hi, *lo;
    int64_t each;
    uint32_t stride;
    __device__ __forceinline__ int64_t at(uint32_t b, uint32_t m, uint32_t n) const { return b * each + (int64_t)m * stride + n; }
    __device__ __forceinline__ void load(uint32_t b, uint32_t m, uint32_t n, uint32_t left, float* x) const
    {
        load8(hi + at(b, m, n), left, true, x);
        if (lo) {
            float t[8];
            load8(lo + at(b, m, n), left, true, t);
#pragma unroll
            for (int i = 0; i < 8; ++i) x[i] += t[i];
        }
    }
    __device__ __forceinline__ void store(uint32_t b, uint32_t m, uint32_t n, uint32_t left, const float* x) const
    {
        store8(hi + at(b, m, n), left, true, x);
        if (lo) {
            float t[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) t[i] = x[i] - __half2float(__float2half_rn(x[i]));
            store8(lo + at(b, m, n), left, true, t);
        }
    }
};

struct EpiPoly {                          // out = alpha v [+ beta add], both in words
    Words out, add;
    float alpha, beta;
    __device__ __forceinline__ void apply(uint32_t b, uint32_t m, uint32_t n, uint32_t left, float* v) const
    {
        float t[8] = {};
        if (add.hi) add.load(b, m, n, left, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(beta, t[i], alpha * v[i]);
        if (out.hi) out.store(b, m, n, left, v);
    }
};

struct EpiLast {                          // the caller's out = alpha v + beta add
    Rows out;
    int64_t each;
    Words add;
    float alpha, beta;
    __device__ __forceinline__ void apply(uint32_t b, uint32_t m, uint32_t n, uint32_t left, float* v) const
    {
        float t[8];
        add.load(b, m, n, left, t);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = fmaf(beta, t[i], alpha * v[i]);
        Rows o = out;
        o.p = (char*)o.p + b * each * (o.dtype == DBLP_F32 ? 4 : 2);
        store8(o, m, n, left, v);
    }
};

}  // namespace dblp
