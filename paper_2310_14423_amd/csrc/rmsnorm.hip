// rmsnorm.hip -- root-mean-square norm of rows with the residual's addition, for K workers with a weight each, and its gradients.
//
//   s = x + res (or x);  rstd = 1 / sqrt(mean(s^2) + eps);  y = s rstd w_k
//   h = s rounded to the rows' type, the residual stream behind;  y in the rows' type, or as e4m3 codes with one fp32 scale for each
//   row, scale = max|y| / 448 over the row's finite entries (for a product with scales by rows)
// and backward, from h as it is kept, with u = dy w and dres what comes down the residual stream:
//   dx = rstd (u - h rstd^2 mean(u h)) + dres  (the gradient of x and of res);  dw_k = sum over the worker's rows of dy h rstd
// All arithmetic is fp32; y is taken from s before its rounding, which is in the registers anyway.  rstd is 0 where mean(s^2) + eps is 0
// as a float.
// Bound by memory: every row is read once and lies in the registers of its lanes until both passes over it are done.  bf16, with
// residual: 8 x 12608 rows of 768 93 us, 6.7 TB/s, their gradients 108 us, 5.8 TB/s, and 5 us for the sums of the weights'; 16384 rows of
// 4096 to e4m3 75 us, 6.3 TB/s.  fp32: 3 x 1001 rows of 1003 10.5 us, 4.6 TB/s, gradients 11.2 and 3.8.  Four rows: 2.6 us, latency.
#include <cmath>

#include "qsr_internal.h"
#include "row_io.h"

namespace qsr {

struct RmsArgs {
    const void *x, *res;
    const float *w;
    void *sum, *y;
    float *scale, *rstd;
    long long rows, s_x, s_res, s_sum, s_y;    // rows of a worker; strides from row to row
    long long s_w;                             // and from worker to worker
    int d;
    float eps;
};

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

template <typename T, int L, int W, int NV, bool FP8>
__device__ __forceinline__ void rmsnorm_row(const RmsArgs &a, int k, long long row, int lane, float (*red)[W])
{
    constexpr int E = wide_of<T>();
    Row<T, NV> x, res;
    RowPart<T, NV> s, w;
    load_row<T, L, W, NV, true>((const T *)a.x + row * a.s_x, lane, a.d, x);
    if (a.res != nullptr) load_row<T, L, W, NV, true>((const T *)a.res + row * a.s_res, lane, a.d, res);
    load_words<T, L, W, NV>(a.w + k * a.s_w, lane, a.d, w);
    each<T, NV>([](float &y, float v) { y = v; }, s, x);
    if (a.res != nullptr) each<T, NV>([](float &y, float v) { y += v; }, s, res);
    float q = 0.f;
    const int runs = a.d / E, rest = a.d - runs * E;
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        float part = 0.f;
#pragma unroll
        for (int u = 0; u < E; ++u) part = fmaf(s.v[c][u], s.v[c][u], part);
        q += lane + c * L * W < runs ? part : 0.f;
    }
    q += lane < rest ? s.t * s.t : 0.f;
    if (a.sum != nullptr) store_row<T, L, W, NV, false>((T *)a.sum + row * a.s_sum, lane, a.d, s);
    const float mean = group_sum<L, W>(q, red, 0) / (float)a.d + a.eps;
    const float rstd = mean == 0.f ? 0.f : 1.f / sqrtf(mean);              // a row of zeros without eps: zeros, and no gradient
    if (lane == 0 && a.rstd != nullptr) a.rstd[row] = rstd;
    float top = 0.f;
    each<T, NV>([&](float &y, float &f) {
        y = y * rstd * f;
        if (FP8 && fabsf(y) < INFINITY) top = fmaxf(top, fabsf(y));
    }, s, w);
    if (!FP8) {
        store_row<T, L, W, NV, false>((T *)a.y + row * a.s_y, lane, a.d, s);
        return;
    }
    top = group_max<L, W>(top, red, 1);
    const float scale = top >= 1e-35f ? top * (1.f / E4M3_MAX) : 0.f;      // less would leave the range of floats
    if (lane == 0) a.scale[row] = scale;
    const float f = scale > 0.f ? 1.f / scale : 0.f;
    // a rounding above 448 at most, which still becomes 448; what is not finite becomes NaN
    each<T, NV>([&](float &y) { y *= f; }, s);
    uint8_t *const y = (uint8_t *)a.y + row * a.s_y;
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

template <typename T, int L, int W, int NV, bool FP8>
__global__ __launch_bounds__(rms_threads<W>()) void rmsnorm_kernel(RmsArgs a)
{
    __shared__ float red[2][W];
    constexpr int side = rms_side<L, W>();
    const int k = blockIdx.y, lane = rms_lane<L, W>(), place = rms_place<L, W>();
    for (long long r = (long long)blockIdx.x * side + place; r < a.rows; r += (long long)gridDim.x * side) {
        if (W > 1 && !FP8 && r >= gridDim.x) __syncthreads();          // one set of words a row: it is read before it is written again
        rmsnorm_row<T, L, W, NV, FP8>(a, k, k * a.rows + r, lane, red);
    }
}

struct RmsBackArgs {
    const void *dy, *h;
    const float *w, *rstd;
    const void *dres;
    void *dx;
    float *partial;                            // [K][groups][d]
    long long rows, s_dy, s_h, s_dres, s_dx, s_w;
    int d;
};

// A workgroup takes every gridDim.x-th row (W == 1: four of them at a time) and keeps its part of the weight's gradient in registers.
// The next row's loads are under way, as they lie in memory, while a row is worked on, where w, dw and two rows of three arrays take
// few registers; elsewhere other wavefronts' loads have to do.
template <typename T, int L, int W, int NV>
__global__ __launch_bounds__(rms_threads<W>(), 4) void rmsnorm_back_kernel(RmsBackArgs a)
{
    constexpr int E = wide_of<T>();
    constexpr bool AHEAD = NV * (2 * E + 3 * 2 * 4) <= 40;
    __shared__ float red[2][W];
    __shared__ float side_dw[W == 1 ? 3 * L * (NV * E + 1) : 1];
    constexpr int side = rms_side<L, W>();
    const int k = blockIdx.y, lane = rms_lane<L, W>(), place = rms_place<L, W>();
    const long long step = (long long)gridDim.x * side, last = (k + 1) * a.rows;
    RowPart<T, NV> w, dw;
    load_words<T, L, W, NV>(a.w + k * a.s_w, lane, a.d, w);
    each<T, NV>([](float &x) { x = 0.f; }, dw);
    Row<T, NV> g, h, e = {};
    float rstd = 0.f;
    auto load = [&](long long row) {
        load_row<T, L, W, NV, true>((const T *)a.dy + row * a.s_dy, lane, a.d, g);
        load_row<T, L, W, NV, true>((const T *)a.h + row * a.s_h, lane, a.d, h);
        if (a.dres != nullptr) load_row<T, L, W, NV, true>((const T *)a.dres + row * a.s_dres, lane, a.d, e);
        rstd = a.rstd[row];
    };
    long long row = k * a.rows + (long long)blockIdx.x * side + place;
    if (AHEAD && row < last) load(row);
#pragma unroll 1
    for (int turn = 0; row < last; row += step, ++turn) {
        if (!AHEAD) load(row);
        Row<T, NV> g0 = g, h0 = h, e0 = e;
        const float rs = rstd;
        if (AHEAD) load(min(row + step, last - 1));
        float q = 0.f;
        each<T, NV>([&](float &acc, float f, float y, float x) {
            const float n = x * rs;
            acc = fmaf(y, n, acc);
            q = fmaf(y * f, n, q);
        }, dw, w, g0, h0);
        const float mean = group_sum<L, W>(q, red, turn) / (float)a.d;
        as_in_memory(g0);
        as_in_memory(h0);
        auto dx = [&](float f, float y, float x, float z) { return fmaf(rs, fmaf(-(x * rs), mean, y * f), z); };
        T *const to = (T *)a.dx + row * a.s_dx;
        const int runs = a.d / E, rest = a.d - runs * E;
#pragma unroll
        for (int c = 0; c < NV; ++c) {
            float v[E];
#pragma unroll
            for (int u = 0; u < E; ++u) v[u] = dx(w.v[c][u], (float)g0.v[c][u], (float)h0.v[c][u], (float)e0.v[c][u]);
            const int i = lane + c * L * W;
            if (i < runs) store_wide<T, E, true>(behind(to, (uint32_t)i * 16), v);
        }
        if (lane < rest) to[runs * E + lane] = (T)dx(w.t, (float)g0.t, (float)h0.t, (float)e0.t);
    }
    if (W == 1) {                              // the sums of a wavefront's rows and of the four wavefronts become one, in their order
        const int wave = threadIdx.x >> 6;
#pragma unroll
        for (int o = L; o < 64; o <<= 1) each<T, NV>([&](float &x) { x += __shfl_xor(x, o, 64); }, dw);
        float *const mine = side_dw + (wave > 0 ? wave - 1 : 0) * L * (NV * E + 1) + lane * (NV * E + 1);
        int n = 0;
        if (wave > 0 && (threadIdx.x & 63) < L) each<T, NV>([&](float &x) { mine[n++] = x; }, dw);
        __syncthreads();
        if (threadIdx.x >= L) return;
#pragma unroll
        for (int o = 0; o < 3; ++o) {
            const float *const other = side_dw + (o * L + lane) * (NV * E + 1);
            n = 0;
            each<T, NV>([&](float &x) { x += other[n++]; }, dw);
        }
    }
    store_words<T, L, W, NV>(a.partial + ((long long)k * gridDim.x + blockIdx.x) * a.d, lane, a.d, dw);
}

// dw[k][j] = sum over the parts, in a fixed order: COLS columns and 1024 / COLS runs of parts, four of each in flight, to a workgroup.
// Latency is everything: fewer columns, on more workgroups, where there are few of them.
constexpr int SUM_THREADS = 1024;
template <int COLS>
__global__ __launch_bounds__(SUM_THREADS) void rmsnorm_weight_kernel(const float *__restrict__ partial, int parts, int d, float *__restrict__ dw)
{
    constexpr int RUNS = SUM_THREADS / COLS, WAVES = SUM_THREADS / 64;
    __shared__ float red[WAVES][COLS];
    const int k = blockIdx.y, col = threadIdx.x % COLS, run = threadIdx.x / COLS;
    const int j = blockIdx.x * COLS + col;
    const float *p = partial + (long long)k * parts * d + j;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (j < d)
        for (int i = run; i < parts; i += 4 * RUNS)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u * RUNS < parts) s[u] += p[(long long)(i + u * RUNS) * d];
    float sum = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
    for (int o = COLS; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
    if ((threadIdx.x & 63) < COLS) red[threadIdx.x >> 6][col] = sum;
    __syncthreads();
    if (run != 0 || j >= d) return;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) sum += red[i][col];
    dw[(long long)k * d + j] = sum;
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
// registers the backward pass keeps 5 or 6 of them in memory with sixteen in bf16, and 18 in fp32 above 8192, where a workgroup of 1024
// lanes leaves no other choice: 4096 rows of 16384 take 192 us, 5.6 TB/s, and of 8192 93, 5.8.
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

template <typename T>
static hipError_t launch_rms(const RmsArgs &a, int K, bool fp8, hipStream_t s)
{
#define RMS_FWD(T, L, W, NV) do { const dim3 grid((unsigned)fwd_groups(a.rows, rms_side<L, W>()), (unsigned)K); \
    if (fp8) rmsnorm_kernel<T, L, W, NV, true><<<grid, rms_threads<W>(), 0, s>>>(a); \
    else rmsnorm_kernel<T, L, W, NV, false><<<grid, rms_threads<W>(), 0, s>>>(a); } while (0)
    RMS_BY_WIDTH(T, a.d, RMS_FWD);
#undef RMS_FWD
    return hipGetLastError();
}

template <typename T>
static hipError_t launch_rms_back(RmsBackArgs &a, int K, float *dw, hipStream_t s)
{
    const long long groups = back_groups(K, a.rows, rms_plan(a.d, (int)sizeof(T)));
    if (groups == 1) a.partial = dw;
#define RMS_BACK(T, L, W, NV) rmsnorm_back_kernel<T, L, W, NV><<<dim3((unsigned)groups, (unsigned)K), rms_threads<W>(), 0, s>>>(a)
    RMS_BY_WIDTH(T, a.d, RMS_BACK);
#undef RMS_BACK
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || groups == 1) return e;
    const long long cols = (long long)K * a.d;
    const auto sums = cols >= 256 * 32 ? rmsnorm_weight_kernel<32> : cols >= 256 * 16 ? rmsnorm_weight_kernel<16> : rmsnorm_weight_kernel<8>;
    const int per = cols >= 256 * 32 ? 32 : cols >= 256 * 16 ? 16 : 8;
    sums<<<dim3((unsigned)((a.d + per - 1) / per), (unsigned)K), SUM_THREADS, 0, s>>>(a.partial, (int)groups, a.d, dw);
    return hipGetLastError();
}

}  // namespace qsr

using namespace qsr;

static int finish(hipError_t e)
{
    if (e == hipSuccess) return QSR_OK;
    set_last_hip_error((int)e);
    return QSR_EHIP;
}
static bool off(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) != 0; }
static uintptr_t size_of(int type) { return type == QSR_TYPE_F32 ? 4 : 2; }
static bool sizes_ok(int32_t K, int64_t rows, int64_t d)
{
    return K >= 1 && K <= 65535 && rows >= 0 && rows <= ((long long)1 << 31) && d >= 1;
}

extern "C" int qsr_rmsnorm(const qsr_rmsnorm_args *q, void *stream)
{
    if (!q || !sizes_ok(q->K, q->rows, q->d)) return QSR_EINVAL;
    if (q->type != QSR_TYPE_F32 && q->type != QSR_TYPE_BF16) return QSR_EINVAL;
    const bool fp8 = q->y_type == QSR_TYPE_E4M3;
    if (!fp8 && q->y_type != q->type) return QSR_EINVAL;
    const uintptr_t es = size_of(q->type);
    if (!(std::isfinite(q->eps) && q->eps >= 0.0)) return QSR_EINVAL;
    if (q->d > RMS_MAX_D) return QSR_ELIMIT;
    if (q->rows == 0) return QSR_OK;
    if (!q->x || off(q->x, es) || off(q->residual, es) || !q->weight || off(q->weight, 4) || off(q->sum, es) || !q->y ||
        (!fp8 && off(q->y, es)) || off(q->rstd, 4) || off(q->scale, 4) || (fp8 && !q->scale))
        return QSR_EINVAL;
    if (q->x_stride < q->d || q->y_stride < q->d || (q->residual && q->residual_stride < q->d) || (q->sum && q->sum_stride < q->d) ||
        (q->K > 1 && q->weight_stride < q->d))
        return QSR_EINVAL;
    const RmsArgs a{q->x, q->residual, q->weight, q->sum, q->y, fp8 ? q->scale : nullptr, q->rstd, q->rows, q->x_stride,
                    q->residual_stride, q->sum_stride, q->y_stride, q->weight_stride, (int)q->d, (float)q->eps};
    return finish(q->type == QSR_TYPE_F32 ? launch_rms<float>(a, q->K, fp8, (hipStream_t)stream)
                                          : launch_rms<bf16_t>(a, q->K, fp8, (hipStream_t)stream));
}

extern "C" int qsr_rmsnorm_workspace_bytes(int32_t K, int64_t rows, int64_t d, int32_t type, size_t *bytes)
{
    if (!bytes) return QSR_EINVAL;
    *bytes = 0;
    if (!sizes_ok(K, rows, d) || (type != QSR_TYPE_F32 && type != QSR_TYPE_BF16)) return QSR_EINVAL;
    if (d > RMS_MAX_D) return QSR_ELIMIT;
    const long long groups = back_groups(K, rows, rms_plan(d, (int)size_of(type)));
    *bytes = groups == 1 ? 0 : (size_t)K * (size_t)groups * (size_t)d * sizeof(float);
    return QSR_OK;
}

extern "C" int qsr_rmsnorm_backward(const qsr_rmsnorm_backward_args *q, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!q || !sizes_ok(q->K, q->rows, q->d)) return QSR_EINVAL;
    if (q->type != QSR_TYPE_F32 && q->type != QSR_TYPE_BF16) return QSR_EINVAL;
    const uintptr_t es = size_of(q->type);
    if (!q->weight || off(q->weight, 4) || !q->weight_grad || off(q->weight_grad, 4)) return QSR_EINVAL;
    if (q->rows > 0 && (!q->y_grad || off(q->y_grad, es) || !q->sum || off(q->sum, es) || !q->rstd || off(q->rstd, 4) ||
                        off(q->residual_grad, es) || !q->x_grad || off(q->x_grad, es)))
        return QSR_EINVAL;
    if (q->y_grad_stride < q->d || q->sum_stride < q->d || q->x_grad_stride < q->d ||
        (q->residual_grad && q->residual_grad_stride < q->d) || (q->K > 1 && q->weight_stride < q->d))
        return QSR_EINVAL;
    size_t need = 0;
    const int rc = qsr_rmsnorm_workspace_bytes(q->K, q->rows, q->d, q->type, &need);
    if (rc != QSR_OK) return rc;
    if (need > 0 && (!workspace || off(workspace, 4))) return QSR_EINVAL;
    if (workspace_bytes < need) return QSR_ENOMEM;
    RmsBackArgs a{q->y_grad, q->sum, q->weight, q->rstd, q->residual_grad, q->x_grad, (float *)workspace, q->rows,
                        q->y_grad_stride, q->sum_stride, q->residual_grad_stride, q->x_grad_stride, q->weight_stride, (int)q->d};
    return finish(q->type == QSR_TYPE_F32 ? launch_rms_back<float>(a, q->K, q->weight_grad, (hipStream_t)stream)
                                          : launch_rms_back<bf16_t>(a, q->K, q->weight_grad, (hipStream_t)stream));
}
