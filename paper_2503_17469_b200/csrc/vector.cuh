// Elements of float and bfloat16 buffers in groups of eight, with plain-element fallbacks.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

namespace omni {

constexpr int kGroup = 8;  // elements of a wide access: 16 bytes of bfloat16, 32 of float

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

__device__ __forceinline__ void widen(const uint4 &u, float *f)
{
    const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(w[i] << 16);
        f[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
    }
}
__device__ __forceinline__ uint4 narrow(const float *f)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t *>(&p);
    }
    return {w[0], w[1], w[2], w[3]};
}
// Eight elements at a 16-byte aligned address.
__device__ __forceinline__ void load_group(const float *p, float *f)
{
    const float4 a = *reinterpret_cast<const float4 *>(p), b = *reinterpret_cast<const float4 *>(p + 4);
    f[0] = a.x; f[1] = a.y; f[2] = a.z; f[3] = a.w;
    f[4] = b.x; f[5] = b.y; f[6] = b.z; f[7] = b.w;
}
__device__ __forceinline__ void load_group(const __nv_bfloat16 *p, float *f) { widen(*reinterpret_cast<const uint4 *>(p), f); }
__device__ __forceinline__ void store_group(float *p, const float *f)
{
    *reinterpret_cast<float4 *>(p) = make_float4(f[0], f[1], f[2], f[3]);
    *reinterpret_cast<float4 *>(p + 4) = make_float4(f[4], f[5], f[6], f[7]);
}
__device__ __forceinline__ void store_group(__nv_bfloat16 *p, const float *f) { *reinterpret_cast<uint4 *>(p) = narrow(f); }

// The same for values that nothing reads soon: first to leave L2.
__device__ __forceinline__ void store_streaming(float *p, const float *f)
{
    __stcs(reinterpret_cast<float4 *>(p), make_float4(f[0], f[1], f[2], f[3]));
    __stcs(reinterpret_cast<float4 *>(p + 4), make_float4(f[4], f[5], f[6], f[7]));
}
__device__ __forceinline__ void store_streaming(__nv_bfloat16 *p, const float *f) { __stcs(reinterpret_cast<uint4 *>(p), narrow(f)); }

template <typename I> __device__ __forceinline__ long long load_index(const void *p, unsigned long long i)
{
    return (long long)static_cast<const I *>(p)[i];
}

}  // namespace omni
