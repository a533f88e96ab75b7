// Element types of the worker-side operators: widening to fp32 and rounding back (to nearest even), one element or a
// group of eight at a time.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace dblp {

constexpr unsigned kSms = 148;                // streaming multiprocessors of the device this library is built for

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f32(__half x) { return __half2float(x); }

template <typename T> __device__ __forceinline__ T from_f32(float x);
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }

// Two values as one 32-bit word, the first in the low half.
template <typename T> __device__ __forceinline__ uint32_t pack2(float a, float b);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float a, float b)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float a, float b)
{
    uint32_t r;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
    return r;
}

template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w)
{
    return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w)
{
    return __half22float2(*reinterpret_cast<const __half2*>(&w));
}

// Eight consecutive elements: one 16-byte vector of a 16-bit type, two of fp32.
template <typename T> struct Vec8 {
    uint4 w;
    __device__ __forceinline__ void load(const T* p) { w = *reinterpret_cast<const uint4*>(p); }
    __device__ __forceinline__ void store(T* p) const { *reinterpret_cast<uint4*>(p) = w; }
    __device__ __forceinline__ void get(float* x) const
    {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2<T>(u[i]);
            x[2 * i] = f.x;
            x[2 * i + 1] = f.y;
        }
    }
    __device__ __forceinline__ void set(const float* x)
    {
        w = make_uint4(pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3]), pack2<T>(x[4], x[5]), pack2<T>(x[6], x[7]));
    }
};
template <> struct Vec8<float> {
    float4 a, b;
    // One 32-byte access where the address allows it (rows of torch tensors do): two of 16 bytes at a stride of 32 touch every
    // sector twice.
    __device__ __forceinline__ void load(const float* p)
    {
        if ((reinterpret_cast<uintptr_t>(p) & 31u) == 0) {
            asm volatile("ld.global.v8.f32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                         : "=f"(a.x), "=f"(a.y), "=f"(a.z), "=f"(a.w), "=f"(b.x), "=f"(b.y), "=f"(b.z), "=f"(b.w)
                         : "l"(p)
                         : "memory");
        } else {
            a = *reinterpret_cast<const float4*>(p);
            b = *reinterpret_cast<const float4*>(p + 4);
        }
    }
    __device__ __forceinline__ void store(float* p) const
    {
        if ((reinterpret_cast<uintptr_t>(p) & 31u) == 0) {
            asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(a.x), "f"(a.y), "f"(a.z), "f"(a.w), "f"(b.x),
                         "f"(b.y), "f"(b.z), "f"(b.w)
                         : "memory");
        } else {
            *reinterpret_cast<float4*>(p) = a;
            *reinterpret_cast<float4*>(p + 4) = b;
        }
    }
    __device__ __forceinline__ void get(float* x) const
    {
        x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w;
        x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
    }
    __device__ __forceinline__ void set(const float* x)
    {
        a = make_float4(x[0], x[1], x[2], x[3]);
        b = make_float4(x[4], x[5], x[6], x[7]);
    }
};

// Division by a launch constant: q = floor(x / d) for every x < 2^32, by a multiply with m = floor(2^32 (2^l - d) / d) + 1
// and a shift, l = ceil(log2 d) (Granlund and Montgomery, "Division by invariant integers using multiplication", 1994).
struct FastDiv {
    uint32_t d, m, s1, s2;
    FastDiv() = default;
    explicit FastDiv(uint32_t div) : d(div)
    {
        uint32_t l = 0;
        while (l < 32 && (1ull << l) < div) ++l;
        m = (uint32_t)(((1ull << 32) * ((1ull << l) - div)) / div + 1);
        s1 = l > 1 ? 1 : l;
        s2 = l > 0 ? l - 1 : 0;
    }
    __device__ __forceinline__ uint32_t div(uint32_t x) const
    {
        const uint32_t t = __umulhi(m, x);
        return (t + ((x - t) >> s1)) >> s2;
    }
};

// Kernels of one call that follow each other: each lets the next one be set up while it still runs (after_start), and waits for
// the one before, results included, as its first step (wait_before).  Every block of every kernel in such a chain does both.
__device__ __forceinline__ void after_start() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }
__device__ __forceinline__ void wait_before() { asm volatile("griddepcontrol.wait;" ::: "memory"); }

template <typename... P, typename... A>
inline cudaError_t launch_next(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t s, A&&... args)
{
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = s;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}

inline int element_bytes(int dtype) { return dtype == DBLP_F32 ? 4 : 2; }
inline bool known_dtype(int dtype) { return dtype == DBLP_F32 || dtype == DBLP_BF16 || dtype == DBLP_F16; }

// Calls f with a value of the C++ type that dtype names.
template <typename F> inline int with_type(int dtype, F&& f)
{
    switch (dtype) {
    case DBLP_F32: return f(float());
    case DBLP_BF16: return f(__nv_bfloat16());
    default: return f(__half());
    }
}

}  // namespace dblp
