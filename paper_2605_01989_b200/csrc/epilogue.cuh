// What is done with a matrix product's fp32 sums: sixteen consecutive columns of one row at a time where all matrices allow 32-byte
// accesses (whole sectors of a 16-bit matrix; two accesses of 16 bytes at a stride of 32 touch every sector twice), else one
// element a lane.
#pragma once

#include <type_traits>

#include "tc.cuh"

namespace dblp {

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

// Sixteen elements as they lie in memory.
template <typename T> struct Raw {
    uint32_t w[sizeof(T) * 4];
    __device__ __forceinline__ void load(const T* p)
    {
        load32(p, w);
        if (sizeof(T) == 4) load32((const char*)p + 32, w + (sizeof(T) == 4 ? 8 : 0));
    }
    __device__ __forceinline__ float2 get(int i) const           // elements 2 i and 2 i + 1
    {
        if constexpr (sizeof(T) == 4) return pair(w[2 * i], w[2 * i + 1]);
        else return unpack2<T>(w[i]);
    }
};
// Where sixteen results of a row go: to memory, or into a piece of 32 x 32 in shared memory that one TMA store takes from there.
// (Stores from the lanes, a row each, took 100 cycles an instruction: 32 lines.)  Rows of 64 bytes are laid out as TMA's 64-byte swizzle
// has them, chunk c of row r at c ^ (r / 2 % 4), rows of 128 as its 128-byte swizzle, c ^ (r % 8): no bank conflicts.
struct ToMemory {
    template <typename T> __device__ __forceinline__ void put(int, T* p, const float* x) const;
};
struct ToPiece {
    uint8_t* piece;
    uint32_t first;                       // 0: columns 0 .. 15 of the piece, 16: the others
    template <typename T> __device__ __forceinline__ void put(int output, T*, const float* x) const
    {
        const uint32_t r = threadIdx.x & 31;
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (uint32_t c = 0; c < 4; ++c)
                *reinterpret_cast<float4*>(piece + r * 128 + (((first / 4 + c) ^ (r & 7)) << 4)) = make_float4(x[4 * c], x[4 * c + 1], x[4 * c + 2], x[4 * c + 3]);
        } else {
#pragma unroll
            for (uint32_t c = 0; c < 2; ++c)
                *reinterpret_cast<uint4*>(piece + output * 2048 + r * 64 + (((first / 8 + c) ^ (r >> 1 & 3)) << 4)) =
                    make_uint4(pack2<T>(x[8 * c], x[8 * c + 1]), pack2<T>(x[8 * c + 2], x[8 * c + 3]), pack2<T>(x[8 * c + 4], x[8 * c + 5]),
                               pack2<T>(x[8 * c + 6], x[8 * c + 7]));
        }
    }
};

// A result that TMA can store: null where the epilogue has none.
struct Output {
    void* p;
    int64_t stride, each;                 // rows; products of a batch
    int bytes;                            // of an element
};

template <typename T> __device__ __forceinline__ void store16(T* p, const float* x)
{
    if constexpr (sizeof(T) == 4) {
        store32(p, reinterpret_cast<const uint32_t*>(x));
        store32(p + 8, reinterpret_cast<const uint32_t*>(x) + 8);
    } else {
        uint32_t w[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) w[i] = pack2<T>(x[2 * i], x[2 * i + 1]);
        store32(p, w);
    }
}

template <typename T> __device__ __forceinline__ void ToMemory::put(int, T* p, const float* x) const { store16(p, x); }

// A row-major matrix that an epilogue reads or writes.
template <typename T> struct Rows {
    T* p;
    int64_t stride;
    __device__ __forceinline__ explicit operator bool() const { return p != nullptr; }
    __device__ __forceinline__ T* at(uint32_t m, uint32_t n) const { return p + (int64_t)m * stride + n; }
    __device__ __forceinline__ void add(const Raw<T>& r, float* v) const
    {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 t = add2(make_float2(v[2 * i], v[2 * i + 1]), r.get(i));
            v[2 * i] = t.x;
            v[2 * i + 1] = t.y;
        }
    }
    bool whole() const { return p == nullptr || (((uintptr_t)p | (uint64_t)stride * sizeof(T)) % 32 == 0); }
};
template <typename T> inline Rows<T> rows_of(const void* p, int64_t stride, uint64_t rows) { return Rows<T>{(T*)p, rows <= 1 ? 0 : stride}; }

__device__ __forceinline__ float element(const void* p, int dtype, uint64_t i)
{
    return dtype == DBLP_F32 ? ((const float*)p)[i] : (dtype == DBLP_BF16 ? to_f32(((const __nv_bfloat16*)p)[i]) : to_f32(((const __half*)p)[i]));
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
// tails keep their digits.  (CUDA's erfcf in its place took 431 us for 8192 x 1600 -> 6400 with bias and gelu where this took 184, before
// the epilogue around it was rewritten.)
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

// ---- precision of the sums ------------------------------------------------------------------------------------------------
// The tensor cores' own sums truncate: sums of one sign lose up to 6e-9 of themselves a term (f16; 64 Ki terms: 4e-4).  Where that
// passes an eighth of half a step of the result's type they are taken out every 512 terms and added in fp32.
constexpr uint32_t kAnyTerms = 0xFFFFFFFFu;
template <typename O> constexpr uint32_t run_terms() { return sizeof(O) == 4 ? 0 : (std::is_same<O, __half>::value ? 8192 : 65536); }

// ---- epilogues -----------------------------------------------------------------------------------------------------------
// Of the sums of row m, column n of product b: fetch and apply take columns n .. n + 15, all of them inside (kPadded: or in the
// padding behind a row; kFewRows: A may have few; kMirror: the result
// may equal its transpose and be computed by half; kNothing: the sum may have no terms); fetch1 and apply1 one.  What was fetched is in f.
// In: the operands' type, where A may have few rows.  kTerms: how many terms the tensor cores may add up by themselves.  sectors(): all matrices allow 32-byte accesses.
template <typename T, typename O> struct EpiLinear {            // out = act(z) + residual, pre = z = v + bias
    Rows<O> out, residual;
    Rows<T> pre;
    const void* bias;
    int bias_dtype, act;
    bool bias_whole;                                            // it allows 32-byte accesses (a view of a flat vector may not)
    using In = T;
    static constexpr bool kPadded = false, kFewRows = true, kMirror = false, kNothing = true;
    static constexpr uint32_t kTerms = run_terms<O>();
    bool sectors() const { return out.whole() && residual.whole() && pre.whole(); }
    Output output(int k) const { return k ? Output{out.p, out.stride, 0, (int)sizeof(O)} : Output{pre.p, pre.stride, 0, 2}; }
    struct Fetched { Raw<O> residual; };
    __device__ __forceinline__ void fetch(uint32_t, uint32_t m, uint32_t n, Fetched& f) const
    {
        if (residual) f.residual.load(residual.at(m, n));
    }
    template <typename S> __device__ __forceinline__ void apply(uint32_t, uint32_t m, uint32_t n, const Fetched& f, float* v, const S& to) const
    {
        if (bias && !bias_whole) {                              // the same sixteen for all lanes
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i] += element(bias, bias_dtype, n + i);
        } else if (bias) {
            if (bias_dtype == DBLP_F32) {
                Raw<float> r;
                r.load((const float*)bias + n);
                Rows<float>().add(r, v);
            } else if (bias_dtype == DBLP_BF16) {
                Raw<__nv_bfloat16> r;
                r.load((const __nv_bfloat16*)bias + n);
                Rows<__nv_bfloat16>().add(r, v);
            } else {
                Raw<__half> r;
                r.load((const __half*)bias + n);
                Rows<__half>().add(r, v);
            }
        }
        if (pre) to.put(0, pre.at(m, n), v);
        activate<16>(act, v);
        if (residual) residual.add(f.residual, v);
        to.put(1, out.at(m, n), v);
    }
    __device__ __forceinline__ float2 fetch1(uint32_t, uint32_t m, uint32_t n) const
    {
        return make_float2(bias ? element(bias, bias_dtype, n) : 0.0f, residual ? to_f32(*residual.at(m, n)) : 0.0f);
    }
    __device__ __forceinline__ void apply1(uint32_t, uint32_t m, uint32_t n, float2 f, float x) const
    {
        float v[2] = {bias ? x + f.x : x, 0.0f};
        if (pre) *pre.at(m, n) = from_f32<T>(v[0]);
        activate<2>(act, v);
        *out.at(m, n) = from_f32<O>(residual ? v[0] + f.y : v[0]);
    }
};

template <typename T> struct EpiGradX {                         // dx = (v + residual) act'(pre)
    Rows<T> out, residual, pre;
    int act;
    using In = T;
    static constexpr bool kPadded = false, kFewRows = true, kMirror = false, kNothing = true;
    static constexpr uint32_t kTerms = run_terms<T>();
    bool sectors() const { return out.whole() && residual.whole() && pre.whole(); }
    Output output(int k) const { return k ? Output{out.p, out.stride, 0, 2} : Output{}; }
    struct Fetched { Raw<T> residual, pre; };
    __device__ __forceinline__ void fetch(uint32_t, uint32_t m, uint32_t n, Fetched& f) const
    {
        if (residual) f.residual.load(residual.at(m, n));
        if (pre) f.pre.load(pre.at(m, n));
    }
    template <typename S> __device__ __forceinline__ void apply(uint32_t, uint32_t m, uint32_t n, const Fetched& f, float* v, const S& to) const
    {
        if (residual) residual.add(f.residual, v);
        if (pre) {
            float z[16];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float2 t = f.pre.get(i);
                z[2 * i] = t.x;
                z[2 * i + 1] = t.y;
            }
            activate_grad<16>(act, z, v);
        }
        to.put(1, out.at(m, n), v);
    }
    __device__ __forceinline__ float2 fetch1(uint32_t, uint32_t m, uint32_t n) const
    {
        return make_float2(residual ? to_f32(*residual.at(m, n)) : 0.0f, pre ? to_f32(*pre.at(m, n)) : 0.0f);
    }
    __device__ __forceinline__ void apply1(uint32_t, uint32_t m, uint32_t n, float2 f, float x) const
    {
        float v[2] = {residual ? x + f.x : x, 0.0f};
        if (pre) {
            const float z[2] = {f.y, 0.0f};
            activate_grad<2>(act, z, v);
        }
        *out.at(m, n) = from_f32<T>(v[0]);
    }
};

template <typename O> struct EpiStore {                         // out = v [+ out]
    Rows<O> out;
    bool accumulate;
    static constexpr bool kPadded = false, kFewRows = false, kMirror = false, kNothing = true;
    static constexpr uint32_t kTerms = run_terms<O>();
    bool sectors() const { return out.whole(); }
    Output output(int k) const { return k ? Output{out.p, out.stride, 0, (int)sizeof(O)} : Output{}; }
    struct Fetched { Raw<O> out; };
    __device__ __forceinline__ void fetch(uint32_t, uint32_t m, uint32_t n, Fetched& f) const
    {
        if (accumulate) f.out.load(out.at(m, n));
    }
    template <typename S> __device__ __forceinline__ void apply(uint32_t, uint32_t m, uint32_t n, const Fetched& f, float* v, const S& to) const
    {
        if (accumulate) out.add(f.out, v);
        to.put(1, out.at(m, n), v);
    }
    __device__ __forceinline__ float2 fetch1(uint32_t, uint32_t m, uint32_t n) const
    {
        return make_float2(accumulate ? to_f32(*out.at(m, n)) : 0.0f, 0.0f);
    }
    __device__ __forceinline__ void apply1(uint32_t, uint32_t m, uint32_t n, float2 f, float x) const
    {
        *out.at(m, n) = from_f32<O>(accumulate ? x + f.x : x);
    }
};

// A matrix in workspace as one or two f16 words an element: value * scale = hi [+ lo].  Batches of `each` elements, rows
// of `stride`, a multiple of sixteen, so that whole groups always fit.
struct Words {
    __half *hi, *lo;
    int64_t each;
    uint32_t stride;
    struct Fetched { Raw<__half> hi, lo; };
    __device__ __forceinline__ int64_t at(uint32_t b, uint32_t m, uint32_t n) const { return b * each + (int64_t)m * stride + n; }
    __device__ __forceinline__ void fetch(uint32_t b, uint32_t m, uint32_t n, Fetched& f) const
    {
        if (!hi) return;
        f.hi.load(hi + at(b, m, n));
        if (lo) f.lo.load(lo + at(b, m, n));
    }
    // v = alpha v + beta (the words)
    __device__ __forceinline__ void combine(const Fetched& f, float alpha, float beta, float* v) const
    {
        const float2 a = make_float2(alpha, alpha), b = make_float2(beta, beta);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            float2 t = mul2(make_float2(v[2 * i], v[2 * i + 1]), a);
            if (hi) t = fma2(lo ? add2(f.hi.get(i), f.lo.get(i)) : f.hi.get(i), b, t);
            v[2 * i] = t.x;
            v[2 * i + 1] = t.y;
        }
    }
    __device__ __forceinline__ float value(uint32_t b, uint32_t m, uint32_t n) const
    {
        const int64_t i = at(b, m, n);
        return hi ? to_f32(hi[i]) + (lo ? to_f32(lo[i]) : 0.0f) : 0.0f;
    }
    template <typename S> __device__ __forceinline__ void store(uint32_t b, uint32_t m, uint32_t n, float* x, const S& to) const
    {
        to.put(0, hi + at(b, m, n), x);
        if (!lo) return;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float2 t = unpack2<__half>(pack2<__half>(x[2 * i], x[2 * i + 1]));
            x[2 * i] -= t.x;
            x[2 * i + 1] -= t.y;
        }
        to.put(1, lo + at(b, m, n), x);
    }
};

template <bool SYMMETRIC> struct EpiPoly {                      // out = alpha v [+ beta add], both in words
    Words out, add;
    float alpha, beta;
    static constexpr bool kPadded = true, kFewRows = false, kMirror = SYMMETRIC, kNothing = false;
    static constexpr uint32_t kTerms = run_terms<__half>();
    bool sectors() const { return true; }
    Output output(int k) const { return Output{k ? out.lo : out.hi, out.stride, out.each, 2}; }
    using Fetched = Words::Fetched;
    __device__ __forceinline__ void fetch(uint32_t b, uint32_t m, uint32_t n, Fetched& f) const { add.fetch(b, m, n, f); }
    template <typename S> __device__ __forceinline__ void apply(uint32_t b, uint32_t m, uint32_t n, const Fetched& f, float* v, const S& to) const
    {
        add.combine(f, alpha, beta, v);
        out.store(b, m, n, v, to);
    }
};

template <typename O> struct EpiLast {                          // the caller's out = alpha v + beta add
    Rows<O> out;
    int64_t each;
    Words add;
    float alpha, beta;
    bool aligned;                                               // of all products of the batch
    static constexpr bool kPadded = false, kFewRows = false, kMirror = false, kNothing = false;
    static constexpr uint32_t kTerms = std::is_same<O, __nv_bfloat16>::value ? kAnyTerms : run_terms<O>();     // 32768 at most
    bool sectors() const { return aligned; }
    Output output(int k) const { return k ? Output{out.p, out.stride, each, (int)sizeof(O)} : Output{}; }
    using Fetched = Words::Fetched;
    __device__ __forceinline__ void fetch(uint32_t b, uint32_t m, uint32_t n, Fetched& f) const { add.fetch(b, m, n, f); }
    template <typename S> __device__ __forceinline__ void apply(uint32_t b, uint32_t m, uint32_t n, const Fetched& f, float* v, const S& to) const
    {
        add.combine(f, alpha, beta, v);
        to.put(1, out.at(m, n) + b * each, v);
    }
    __device__ __forceinline__ float2 fetch1(uint32_t b, uint32_t m, uint32_t n) const { return make_float2(add.value(b, m, n), 0.0f); }
    __device__ __forceinline__ void apply1(uint32_t b, uint32_t m, uint32_t n, float2 f, float x) const
    {
        out.at(m, n)[b * each] = from_f32<O>(fmaf(beta, f.x, alpha * x));
    }
};

}  // namespace dblp
