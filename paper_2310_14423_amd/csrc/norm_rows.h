// norm_rows.h -- rows that lie in the registers of a wavefront's or a workgroup's lanes, for the norms (gfx950): how a row is shared out,
// loads, stores and sums.
#pragma once
#include "row_io.h"

namespace qsr {

// A row lies in L = 16, 32 or 64 lanes of a wavefront, or in W wavefronts.  Sum and maximum over all of them.  red: two sets of W words
// that take turns (`turn`): a set is written again behind the next barrier, when all have read it.
template <int L, int W>
__device__ __forceinline__ float group_sum(float v, float (*red)[W], int turn)
{
    if (L == 64) v = wave_sum(v);
    else { v += row_step<0>(v); v += row_step<1>(v); v += row_step<2>(v); v += row_step<3>(v); }
    if (L == 32) v += __shfl_xor(v, 16, 64);
    if (W == 1) return v;
    if ((threadIdx.x & 63) == 0) red[turn & 1][threadIdx.x >> 6] = v;
    __syncthreads();
    float r = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) r += red[turn & 1][i];
    return r;
}
template <int L, int W>
__device__ __forceinline__ float group_max(float v, float (*red)[W], int turn)
{
    if (L == 64) v = wave_max(v);
    else { v = fmaxf(v, row_step<0>(v)); v = fmaxf(v, row_step<1>(v)); v = fmaxf(v, row_step<2>(v)); v = fmaxf(v, row_step<3>(v)); }
    if (L == 32) v = fmaxf(v, __shfl_xor(v, 16, 64));
    if (W == 1) return v;
    if ((threadIdx.x & 63) == 0) red[turn & 1][threadIdx.x >> 6] = v;
    __syncthreads();
    float r = red[turn & 1][0];
#pragma unroll
    for (int i = 1; i < W; ++i) r = fmaxf(r, red[turn & 1][i]);
    return r;
}

// A lane's part of a row of d elements in L W lanes, as it lies in memory: up to NV runs of 16 bytes, L W runs apart, and one of
// the d % E elements behind the whole runs.  A lane without a run loads the last one again, without a branch, and its part is left out
// where it would count: its weight is zero, its square is not added, nothing of it is stored.
template <typename T, int NV> struct Row {
    typename Wide<T, wide_of<T>()>::vec v[NV > 0 ? NV : 1];
    T t;
};
// and in fp32.  NV = 0: rows shorter than a run, d < E.
template <typename T, int NV> struct RowPart { float v[NV > 0 ? NV : 1][wide_of<T>()], t; };

template <typename T, int L, int W, int NV, bool NT>
__device__ __forceinline__ void load_row(const T *p, int lane, int d, Row<T, NV> &r)
{
    constexpr int E = wide_of<T>();
    typedef typename Wide<T, E>::vec V;
    const int runs = d / E;
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const V *const at = (const V *)behind(p, (uint32_t)min(lane + c * L * W, runs - 1) * 16);
        r.v[c] = NT ? __builtin_nontemporal_load(at) : *at;
    }
    r.t = *behind(p, (uint32_t)min(runs * E + lane, d - 1) * (uint32_t)sizeof(T));
}
// Has the compiler forget what it made of a row: it is converted again where it is used again, instead of being held in fp32
template <typename T, int NV>
__device__ __forceinline__ void as_in_memory(Row<T, NV> &r)
{
    typedef int I4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        I4 x = __builtin_bit_cast(I4, r.v[c]);
        asm volatile("" : "+v"(x));
        r.v[c] = __builtin_bit_cast(typename Wide<T, wide_of<T>()>::vec, x);
    }
}
template <typename T, int L, int W, int NV, bool NT>
__device__ __forceinline__ void store_row(T *p, int lane, int d, const RowPart<T, NV> &r)
{
    constexpr int E = wide_of<T>();
    const int runs = d / E, rest = d - runs * E;
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int i = lane + c * L * W;
        if (i < runs) store_wide<T, E, NT>(behind(p, (uint32_t)i * 16), r.v[c]);
    }
    if (lane < rest) p[runs * E + lane] = (T)r.t;
}
// fp32 words (the weight, its gradient) in the lanes of a row of T
template <typename T, int L, int W, int NV>
__device__ __forceinline__ void load_words(const float *p, int lane, int d, RowPart<T, NV> &r)
{
    constexpr int E = wide_of<T>();
    const int runs = d / E, rest = d - runs * E;
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int i = lane + c * L * W;
#pragma unroll
        for (int u = 0; u < E; ++u) r.v[c][u] = 0.f;
        if (i < runs) {
#pragma unroll
            for (int q = 0; q < E; q += 4) {
                float f[4];
                load_wide<float, 4, false>(behind(p, (uint32_t)(i * E + q) * 4), f);
#pragma unroll
                for (int u = 0; u < 4; ++u) r.v[c][q + u] = f[u];
            }
        }
    }
    r.t = lane < rest ? p[runs * E + lane] : 0.f;
}
template <typename T, int L, int W, int NV>
__device__ __forceinline__ void store_words(float *p, int lane, int d, const RowPart<T, NV> &r)
{
    constexpr int E = wide_of<T>();
    const int runs = d / E, rest = d - runs * E;
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int i = lane + c * L * W;
        if (i < runs) {
#pragma unroll
            for (int q = 0; q < E; q += 4) {
                const float f[4] = {r.v[c][q], r.v[c][q + 1], r.v[c][q + 2], r.v[c][q + 3]};
                store_wide<float, 4, false>(behind(p, (uint32_t)(i * E + q) * 4), f);
            }
        }
    }
    if (lane < rest) p[runs * E + lane] = r.t;
}
// Numbers of at most 448 as e4m3 codes
template <typename T, int L, int W, int NV>
__device__ __forceinline__ void store_codes(uint8_t *y, int lane, int d, const RowPart<T, NV> &s)
{
    constexpr int E = wide_of<T>();
    const int runs = d / E, rest = d - runs * E;
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        const int i = lane + c * L * W;
        typedef typename Wide<uint8_t, E>::vec Codes;
        union { uint32_t w[E / 4]; uint8_t b[E]; } code;
#pragma unroll
        for (int g = 0; g < E; g += 4) code.w[g / 4] = e4m3_near4(&s.v[c][g]);
        Codes out;
#pragma unroll
        for (int u = 0; u < E; ++u) out[u] = code.b[u];
        if (i < runs) *(Codes *)behind(y, (uint32_t)i * E) = out;
    }
    if (lane < rest) {
        const float one[4] = {s.t, 0.f, 0.f, 0.f};
        y[runs * E + lane] = (uint8_t)e4m3_near4(one);
    }
}

// f(element of a, the same element of b, c, ...) for all of them
template <typename T, int NV, int W = 0> __device__ __forceinline__ float &at(RowPart<T, NV> &r, int c, int u) { return c < NV ? r.v[c][u] : r.t; }
template <typename T, int NV, int W = 0> __device__ __forceinline__ float at(const Row<T, NV> &r, int c, int u) { return (float)(c < NV ? r.v[c][u] : r.t); }
template <typename T, int NV, typename F, typename... R>
__device__ __forceinline__ void each(F f, R &...r)
{
#pragma unroll
    for (int c = 0; c <= NV; ++c)
#pragma unroll
        for (int u = 0; u < (c < NV ? wide_of<T>() : 1); ++u) f(at<T, NV>(r, c, u)...);
}

// A workgroup has one row at a time (W > 1), or four wavefronts of 64 / L rows each
template <int W> constexpr int rms_threads() { return W == 1 ? 256 : 64 * W; }
template <int L, int W> constexpr int rms_side() { return W == 1 ? 256 / L : 1; }
// A lane's place in its row, and the row's in the workgroup: a number that is the same in a wavefront, and known to be, where L = 64
template <int L, int W> __device__ __forceinline__ int rms_lane() { return W == 1 ? threadIdx.x & (L - 1) : threadIdx.x; }
template <int L, int W> __device__ __forceinline__ int rms_place()
{
    return W > 1 ? 0 : L == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : threadIdx.x / L;
}

constexpr int RMS_MAX_D = 16384;

// How a row of d elements of `size` bytes is shared out: L lanes of W wavefronts
struct RmsPlan { int L, W, side; };
static RmsPlan rms_plan(long long d, int size)
{
    const int half = size == 2 ? 1 : 2;
    RmsPlan q;
    q.L = d <= 128 ? 16 : d <= 256 ? 32 : 64;
    q.W = d <= 512 ? 1 : d <= 1024 ? half : d <= 2048 ? 4 : d <= 4096 ? 4 * half : d <= 8192 ? 8 * half : 16;
    q.side = q.W == 1 ? 256 / q.L : 1;
    return q;
}
// F(T, L, W, NV) for it: sixteen elements to a lane in bf16 where the row is long enough, eight in fp32 (a third row in the backward
// pass would not fit the registers).  us with eight in bf16: 16384 rows of 4096 to e4m3 88 (77.7), 8 x 12608 rows of 768 forward and
// backward 229 (207); with sixteen in fp32, backward: 8192 rows of 4096 106 (94), 4 x 4854 rows of 611 52 (46).  At its limit of 128
// registers the backward pass of the root-mean-square norm keeps 5 or 6 of them in memory with sixteen in bf16, and 18 in fp32 above 8192,
// where a workgroup of 1024 lanes leaves no other choice: 4096 rows of 16384 take 192 us, 5.6 TB/s, and of 8192 93, 5.8.
#define RMS_BY_WIDTH(T, d, F) do { constexpr int E_ = wide_of<T>(); \
    if ((d) < E_) F(T, 16, 1, 0); else if ((d) <= 128) F(T, 16, 1, 8 / E_); else if ((d) <= 256) F(T, 32, 1, 8 / E_); \
    else if ((d) <= 512) F(T, 64, 1, 8 / E_); \
    else if ((d) <= 1024) { if constexpr (sizeof(T) == 2) F(T, 64, 1, 16 / E_); else F(T, 64, 2, 8 / E_); } \
    else if ((d) <= 2048) F(T, 64, 4, 8 / E_); \
    else if ((d) <= 4096) { if constexpr (sizeof(T) == 2) F(T, 64, 4, 16 / E_); else F(T, 64, 8, 8 / E_); } \
    else if ((d) <= 8192) { if constexpr (sizeof(T) == 2) F(T, 64, 8, 16 / E_); else F(T, 64, 16, 8 / E_); } \
    else F(T, 64, 16, 16 / E_); } while (0)

// Workgroups of a worker in the forward pass: one trip each
static long long fwd_groups(long long rows, int side)
{
    const long long need = (rows + side - 1) / side;
    return need < (1 << 20) ? need : 1 << 20;
}
// and in the backward pass: two wavefronts to each of the chip's SIMDs, four in the widest rows and five in narrow ones, which have
// little in flight each, since each workgroup leaves a row of partial sums.  us with four / two: 16384 rows of 2048 61 / 52.5, 8192 fp32 rows of 2048 60 / 52, 2 x 4377 fp32 rows of 903 39.5 / 32.4;
// 4096 rows of 16384 100 / 130.  One, whose sums are the weight's gradient already, for the rows of a few tokens.
static long long back_groups(int K, long long rows, const RmsPlan &q)
{
    if (rows <= 2 * q.side) return 1;
    const long long all = q.L < 64 ? 1280 : q.W == 1 ? 512 : q.W == 16 ? 256 : 2048 / q.W;
    const long long most = (all + K - 1) / K, need = (rows + q.side - 1) / q.side;
    return most < need ? most : need;
}

}  // namespace qsr
