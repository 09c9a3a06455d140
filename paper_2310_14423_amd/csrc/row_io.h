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
// The address `bytes` behind p, where p is the same for a wavefront: one register for the distance instead of two for the address
template <typename P> __device__ __forceinline__ P *behind(P *p, uint32_t bytes) { return (P *)((char *)p + bytes); }
template <typename P> __device__ __forceinline__ const P *behind(const P *p, uint32_t bytes) { return (const P *)((const char *)p + bytes); }
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

// A pointer that was read from memory, as one into global memory: the compiler cannot know, and would use flat accesses
template <typename T> __device__ __forceinline__ T *global(T *p) { return (T *)(__attribute__((address_space(1))) T *)(uintptr_t)p; }

// Lanes exchanged within a row of 16 by the data-parallel primitives: after steps 0 to 3 of a sum or maximum every lane has its row's
template <int STEP> __device__ __forceinline__ int row_step(int v)
{
    constexpr int ctrl = STEP == 0 ? 0xB1 : STEP == 1 ? 0x4E : STEP == 2 ? 0x141 : 0x140;   // xor 1, xor 2, half rows mirrored, rows mirrored
    return __builtin_amdgcn_update_dpp(0, v, ctrl, 0xf, 0xf, true);
}
template <int STEP> __device__ __forceinline__ float row_step(float v) { return __int_as_float(row_step<STEP>(__float_as_int(v))); }
__device__ __forceinline__ float lane_of(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }

// Sum and maximum over the 64 lanes of a wavefront, in every lane.  fmaxf: NaN gives way to any number.
__device__ __forceinline__ float wave_sum(float v)
{
    v += row_step<0>(v); v += row_step<1>(v); v += row_step<2>(v); v += row_step<3>(v);
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
// the same in double, whose halves go by the same exchanges
template <int STEP> __device__ __forceinline__ double row_step(double v)
{
    return __hiloint2double(row_step<STEP>(__double2hiint(v)), row_step<STEP>(__double2loint(v)));
}
__device__ __forceinline__ double lane_of(double v, int lane)
{
    return __hiloint2double(__builtin_amdgcn_readlane(__double2hiint(v), lane), __builtin_amdgcn_readlane(__double2loint(v), lane));
}
__device__ __forceinline__ double wave_sum(double v)
{
    v += row_step<0>(v); v += row_step<1>(v); v += row_step<2>(v); v += row_step<3>(v);
    return (lane_of(v, 0) + lane_of(v, 16)) + (lane_of(v, 32) + lane_of(v, 48));
}
__device__ __forceinline__ float wave_max(float v)
{
    v = fmaxf(v, row_step<0>(v)); v = fmaxf(v, row_step<1>(v)); v = fmaxf(v, row_step<2>(v)); v = fmaxf(v, row_step<3>(v));
    return fmaxf(fmaxf(lane_of(v, 0), lane_of(v, 16)), fmaxf(lane_of(v, 32), lane_of(v, 48)));
}
__device__ __forceinline__ uint32_t wave_max(uint32_t v)
{
    v = max(v, (uint32_t)row_step<0>((int)v)); v = max(v, (uint32_t)row_step<1>((int)v));
    v = max(v, (uint32_t)row_step<2>((int)v)); v = max(v, (uint32_t)row_step<3>((int)v));
    const uint32_t a = max((uint32_t)__builtin_amdgcn_readlane((int)v, 0), (uint32_t)__builtin_amdgcn_readlane((int)v, 16));
    const uint32_t b = max((uint32_t)__builtin_amdgcn_readlane((int)v, 32), (uint32_t)__builtin_amdgcn_readlane((int)v, 48));
    return max(a, b);
}
// the high words first, then the low ones of those that have the highest
__device__ __forceinline__ uint64_t wave_max(uint64_t v)
{
    const uint32_t hi = wave_max((uint32_t)(v >> 32)), lo = wave_max((uint32_t)(v >> 32) == hi ? (uint32_t)v : 0u);
    return ((uint64_t)hi << 32) | lo;
}

}  // namespace qsr
