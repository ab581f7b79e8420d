// numeric.h -- element types, loads and cross-lane sums of the training
// kernels (score.hip, loss.hip, adamw.hip).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "../../include/smore.h"

namespace smore {

using bf16 = __bf16;
using f16 = _Float16;

// V consecutive elements, at any address that is a multiple of an element's
// size: global loads and stores of 2 to 16 bytes take such addresses on
// gfx950, so rows of odd length keep the wide accesses.
template <class T, int V>
struct Vec {
    T x[V];
};
template <class T, int V>
__device__ __forceinline__ Vec<T, V> load_vec(const T* p)
{
    Vec<T, V> v;
    __builtin_memcpy(&v, p, sizeof(v));
    return v;
}
template <class T, int V>
__device__ __forceinline__ void store_vec(T* p, const Vec<T, V>& v)
{
    __builtin_memcpy(p, &v, sizeof(v));
}

// The first `count` of V elements at p as floats, 0 for the others; none of
// them is read.
template <class T, int V>
__device__ __forceinline__ void load_floats(const T* p, int count, float* out)
{
    if (count >= V) {
        const Vec<T, V> v = load_vec<T, V>(p);
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = (float)v.x[j];
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = j < count ? (float)p[j] : 0.0f;
    }
}
template <class T, int V>
__device__ __forceinline__ void store_floats(T* p, int count, const float* in)
{
    if (count >= V) {
        Vec<T, V> v;
#pragma unroll
        for (int j = 0; j < V; ++j) v.x[j] = (T)in[j];
        store_vec<T, V>(p, v);
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (j < count) p[j] = (T)in[j];
    }
}

// Lane exchanges inside a row of 16 lanes (DPP): with lanes 1 and 2 away in a
// quad, then mirrored in 8 and in 16 lanes.  After all four, every lane of
// the 16 has the combination of all.
template <int CTRL>
__device__ __forceinline__ float dpp(float x)
{
    return __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(x), CTRL, 0xF, 0xF, true));
}
constexpr int DPP_XOR1 = 0xB1, DPP_XOR2 = 0x4E, DPP_MIRROR8 = 0x141, DPP_MIRROR16 = 0x140;

__device__ __forceinline__ float sum16(float x)
{
    x += dpp<DPP_XOR1>(x);
    x += dpp<DPP_XOR2>(x);
    x += dpp<DPP_MIRROR8>(x);
    x += dpp<DPP_MIRROR16>(x);
    return x;
}
__device__ __forceinline__ float sum32(float x)
{
    x = sum16(x);
    return x + __shfl_xor(x, 16);
}
__device__ __forceinline__ float sum64(float x)
{
    x = sum32(x);
    return x + __shfl_xor(x, 32);
}
__device__ __forceinline__ float max64(float x)
{
    x = fmaxf(x, dpp<DPP_XOR1>(x));
    x = fmaxf(x, dpp<DPP_XOR2>(x));
    x = fmaxf(x, dpp<DPP_MIRROR8>(x));
    x = fmaxf(x, dpp<DPP_MIRROR16>(x));
    x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
}

// The outcome of the launches so far.
inline int launched(const char** err)
{
    const hipError_t e = hipGetLastError();
    if (e == hipSuccess) return SMORE_OK;
    *err = hipGetErrorString(e);
    return SMORE_E_HIP;
}

}  // namespace smore
