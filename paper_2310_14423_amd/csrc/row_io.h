// row_io.h -- rows of fp32 or bf16 elements at any alignment of an element, e4m3 codes, and sums over a wavefront (gfx950).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace qsr {

typedef __bf16 bf16_t;

// N consecutive elements of T in one access of at most 16 bytes.  The hardware takes wide global accesses at any address, so the
// type claims no more than its element's alignment; aligned addresses run at full rate all the same.
template <typename T, int N> struct Wide { typedef T vec __attribute__((ext_vector_type(N), aligned(sizeof(T)))); };

template <typename T, int N, bool NT>
__device__ __forceinline__ void load_wide(const T *p, float (&v)[N])
{
    typedef typename Wide<T, N>::vec V;
    const V x = NT ? __builtin_nontemporal_load((const V *)p) : *(const V *)p;
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = (float)x[i];
}
template <typename T, int N, bool NT>
__device__ __forceinline__ void store_wide(T *p, const float (&v)[N])
{
    typedef typename Wide<T, N>::vec V;
    V x;
#pragma unroll
    for (int i = 0; i < N; ++i) x[i] = (T)v[i];
    if (NT) __builtin_nontemporal_store(x, (V *)p);
    else *(V *)p = x;
}
// The first `left` of N elements (left < N; none where it is not positive), the others as `fill`
template <typename T, int N>
__device__ __forceinline__ void load_some(const T *p, int left, float (&v)[N], float fill = 0.f)
{
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = i < left ? (float)p[i] : fill;
}
template <typename T, int N>
__device__ __forceinline__ void store_some(T *p, int left, const float (&v)[N])
{
#pragma unroll
    for (int i = 0; i < N; ++i)
        if (i < left) p[i] = (T)v[i];
}

// elements of T in 16 bytes
template <typename T> constexpr int wide_of() { return 16 / (int)sizeof(T); }

// Four e4m3 codes in a word, to the nearest value (ties to even).  |v| <= 448: the conversion makes NaN of more.
__device__ __forceinline__ uint32_t e4m3_near4(const float *v)
{
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], w, true);
}
constexpr float E4M3_MAX = 448.f, E4M3_TINY = 0.001953125f;         // largest value, smallest above zero (2^-9)

// Sum and maximum over the 64 lanes of a wavefront, in every lane.  fmaxf: NaN gives way to any number.
__device__ __forceinline__ float wave_sum(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
    return v;
}
__device__ __forceinline__ float wave_max(float v)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor(v, o, 64));
    return v;
}

}  // namespace qsr
