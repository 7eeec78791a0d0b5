// What the kernels over rows of a dense [rows, cols] tensor share (softmax, layer norm, embedding): elements to and from 16-byte
// vectors, vectors at any element address, sums and maxima over a group of lanes.
#pragma once
#include "common.h"

#include <math.h>

namespace ngc {

template <typename T> struct SmElem;
template <> struct SmElem<uint16_t> {                  // bf16 bit patterns, 8 per 16 bytes
    static constexpr int E = 8;
    __device__ static void unpack(const uint4 &v, float (&f)[8])
    {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f[2 * j] = __uint_as_float(w[j] << 16);
            f[2 * j + 1] = __uint_as_float(w[j] & 0xFFFF0000u);
        }
    }
    __device__ static uint4 pack(const float (&f)[8])
    {
        return make_uint4(pack_bf16x2_hw(f[0], f[1]), pack_bf16x2_hw(f[2], f[3]), pack_bf16x2_hw(f[4], f[5]),
                          pack_bf16x2_hw(f[6], f[7]));
    }
    __device__ static float load(const uint16_t *p) { return bf16_bits_to_float(*p); }
    __device__ static void store(uint16_t *p, float v) { *p = (uint16_t)(pack_bf16x2_hw(v, 0.f) & 0xFFFFu); }
    // bf16 results carry 8 bits: the hardware exp2 (1 ulp of fp32) is far inside the rounding
    __device__ static float exp_of(float d) { return __builtin_amdgcn_exp2f(d * 1.44269504088896341f); }
};
template <> struct SmElem<float> {
    static constexpr int E = 4;
    __device__ static void unpack(const uint4 &v, float (&f)[4])
    {
        f[0] = __uint_as_float(v.x); f[1] = __uint_as_float(v.y); f[2] = __uint_as_float(v.z); f[3] = __uint_as_float(v.w);
    }
    __device__ static uint4 pack(const float (&f)[4])
    {
        return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
    }
    __device__ static float load(const float *p) { return *p; }
    __device__ static void store(float *p, float v) { *p = v; }
    __device__ static float exp_of(float d) { return expf(d); }
};

template <int GL>
__device__ __forceinline__ float group_max(float v)
{
#pragma unroll
    for (int o = GL / 2; o >= 1; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}
template <int GL>
__device__ __forceinline__ float group_sum(float v)
{
#pragma unroll
    for (int o = GL / 2; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);   // butterfly: every lane ends with the same sum
    return v;
}

// reduction over the NW waves of a workgroup (fixed order); sm holds NW floats
template <int NW>
__device__ __forceinline__ float block_reduce(float v, bool is_max, float *sm)
{
    v = is_max ? group_max<64>(v) : group_sum<64>(v);
    const int wave = threadIdx.x >> 6;
    __syncthreads();                                                     // sm may still be read from the last call
    if ((threadIdx.x & 63) == 0) sm[wave] = v;
    __syncthreads();
    float r = sm[0];
#pragma unroll
    for (int w = 1; w < NW; ++w) r = is_max ? fmaxf(r, sm[w]) : r + sm[w];
    return r;
}

// 16 bytes at any element address
template <typename T>
__device__ __forceinline__ uint4 load16_any(const T *p)
{
    uint4 v;
    __builtin_memcpy(&v, p, 16);
    return v;
}
template <typename T>
__device__ __forceinline__ void store16_any(T *p, uint4 v)
{
    typedef unsigned u32x4_any __attribute__((ext_vector_type(4), aligned(2)));
    const u32x4_any w = {v.x, v.y, v.z, v.w};
    __builtin_nontemporal_store(w, reinterpret_cast<u32x4_any *>(p));
}

// Four elements at any element address as fp32
template <typename T>
__device__ __forceinline__ float4 load4_any(const T *p)
{
    if constexpr (sizeof(T) == 2) {
        uint2 v;
        __builtin_memcpy(&v, p, 8);
        return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16), __uint_as_float(v.y & 0xFFFF0000u));
    } else {
        float4 v;
        __builtin_memcpy(&v, p, 16);
        return v;
    }
}

// Vectors that stay packed over several passes: what was unpacked of them before this point is unpacked again after it instead of being kept
// in registers.
template <int N> __device__ __forceinline__ void keep_packed(uint4 (&v)[N])
{
#pragma unroll
    for (int j = 0; j < N; ++j) asm volatile("" : "+v"(v[j].x), "+v"(v[j].y), "+v"(v[j].z), "+v"(v[j].w));
}

}  // namespace ngc
