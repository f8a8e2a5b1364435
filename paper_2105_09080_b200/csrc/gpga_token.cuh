// What the token-block kernels (embedding lookup, dropout, layer norm) share: activation types, accesses
// to a row in chunks of eight columns, and the dropout mask.  sm_100a only.
#pragma once
#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "gpga_device.cuh"

namespace gpga {

// Sets the text that gpga_last_error(NULL) returns to the calling thread (defined with the C ABI).
int32_t token_error(int32_t code, const char* text) noexcept;

constexpr int kChunk = 8;   // columns per generator call: eight 16-bit halves of its four words

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ void unpack16(uint32_t w, float& lo, float& hi, __nv_bfloat16)
{
    lo = __uint_as_float(w << 16);
    hi = __uint_as_float(w & 0xFFFF0000u);
}
__device__ __forceinline__ void unpack16(uint32_t w, float& lo, float& hi, __half)
{
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&w));
    lo = f.x;
    hi = f.y;
}
__device__ __forceinline__ uint32_t pack16(float lo, float hi, __nv_bfloat16)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t pack16(float lo, float hi, __half)
{
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
}

// The eight columns col .. col + 7 of a row as read from memory.  VEC: 128-bit accesses (the host has
// checked alignment and that d is a multiple of eight).  Otherwise element by element, columns from d on
// read as zero.
template <class T, bool VEC> struct Raw8;
template <class T> struct Raw8<T, true> {
    uint4 w;
    __device__ __forceinline__ void load(const T* row, int col, int) { w = __ldcs(reinterpret_cast<const uint4*>(row + col)); }
    __device__ __forceinline__ void get(float* v) const
    {
        unpack16(w.x, v[0], v[1], T());
        unpack16(w.y, v[2], v[3], T());
        unpack16(w.z, v[4], v[5], T());
        unpack16(w.w, v[6], v[7], T());
    }
};
template <> struct Raw8<float, true> {
    float4 a, b;
    __device__ __forceinline__ void load(const float* row, int col, int)
    {
        a = __ldcs(reinterpret_cast<const float4*>(row + col));
        b = __ldcs(reinterpret_cast<const float4*>(row + col) + 1);
    }
    __device__ __forceinline__ void get(float* v) const
    {
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    }
};
template <class T> struct Raw8<T, false> {
    T e[8];
    __device__ __forceinline__ void load(const T* row, int col, int d)
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) e[j] = col + j < d ? row[col + j] : from_f32<T>(0.f);
    }
    __device__ __forceinline__ void get(float* v) const
    {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = to_f32(e[j]);
    }
};

template <class T, bool VEC>
__device__ __forceinline__ void store8(T* row, int col, int d, const float* v)
{
    if constexpr (!VEC) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (col + j < d) row[col + j] = from_f32<T>(v[j]);
    } else if constexpr (sizeof(T) == 4) {
        __stcs(reinterpret_cast<float4*>(row + col), make_float4(v[0], v[1], v[2], v[3]));
        __stcs(reinterpret_cast<float4*>(row + col) + 1, make_float4(v[4], v[5], v[6], v[7]));
    } else {
        __stcs(reinterpret_cast<uint4*>(row + col), make_uint4(pack16(v[0], v[1], T()), pack16(v[2], v[3], T()),
                                                              pack16(v[4], v[5], T()), pack16(v[6], v[7], T())));
    }
}

// Eight fp32 parameters (a weight row's columns), kept in the caches: every row of a node reads them.
__device__ __forceinline__ void param8(const float* w, int col, int d, bool vec, float* v)
{
    if (vec) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(w + col)), b = __ldg(reinterpret_cast<const float4*>(w + col) + 1);
        v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w;
        v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = col + j < d ? __ldg(w + col + j) : 0.f;
    }
}

// Dropout of one activation tensor: what a launch needs to form any element's mask.
struct DropMask {
    PhiloxKeys keys;
    uint32_t threshold;   // dropped iff the element's 16 bits are below this; 0: no dropout
    float scale;          // 65536 / (65536 - threshold), 0 when everything is dropped
    uint32_t node0;       // global index of local node 0
    uint32_t k, stream;
};

// Dropout of the eight columns of chunk `chunk` (columns 8 chunk .. 8 chunk + 7) of row t of local node i:
// counter (t * chunks + chunk, node, k, stream); column 8 chunk + j owns half j & 1 (low half first) of word j >> 1.
// A dropped element is a selected zero, so that NaN and infinities vanish with it.
__device__ __forceinline__ void drop8(const DropMask& m, uint32_t t, uint32_t i, uint32_t chunks, uint32_t chunk, float* v)
{
    const uint4 w = philox4x32_10(t * chunks + chunk, m.node0 + i, m.k, m.stream, m.keys);
    const uint32_t word[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t bits = (j & 1) ? word[j >> 1] >> 16 : word[j >> 1] & 0xFFFFu;
        v[j] = bits >= m.threshold ? v[j] * m.scale : 0.f;
    }
}

}  // namespace gpga
