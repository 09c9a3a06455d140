// layernorm.hip -- layer norm of rows with the residual's addition, for K workers with a weight and a bias each, and its gradients.
//
//   s = x + res (or x);  mean = mean(s);  rstd = 1 / sqrt(mean((s - mean)^2) + eps);  y = (s - mean) rstd w_k + b_k
//   h = s rounded to the rows' type, the residual stream behind;  y in the rows' type, or as e4m3 codes with one fp32 scale for each
//   row, scale = max|y| / 448 over the row's finite entries
// and backward, from h as it is kept, with n = (h - mean) rstd, u = dy w and dres what comes down the residual stream:
//   dx = rstd (u - mean(u) - n mean(u n)) + dres  (the gradient of x and of res)
//   dw_k = sum over the worker's rows of dy n;  db_k = sum of dy
// All arithmetic is fp32.  The row in the registers is taken about the quotient of its sum, which roundings leave some steps of the floats beside
// the mean; the mean of what remains puts that right, and the deviation is mean(t^2) - mean(t)^2 of the remainders t: rows whose mean is large
// beside their deviation keep it, and rows of equal numbers have none, exactly (their remainders are whole steps j, j < 32, so that sums of j and
// of j^2 over 16384 of them are exact too).  rstd is 0 where the deviation's square + eps is 0 as a float.
// Bound by memory: every row is read once and lies in the registers of its lanes until all passes over it are done, weight and bias are read once a
// workgroup.  bf16, with residual and bias: 8 x 12608 rows of 768 100 us, 6.2 TB/s, their gradients 111 us, 5.6 TB/s, and 5 us for the sums of
// weight's and bias'.  fp32, without either: 3 x 1001 rows of 1003 7.3 us, 3.3 TB/s, gradients 12.2 and 3.9.  To e4m3, from bf16 with residual and
// bias: four rows of 2048 3.3 us, latency; 8192 of 4096 46 us, 5.1 TB/s; 8 x 8192 of 768 65 us, 5.4 TB/s.  2048 rows of 16384 with residual and
// bias: bf16 51 us, 5.3 TB/s, fp32 91 us, 5.9 TB/s; their gradients 83 us, 3.2 TB/s, and 162 us, 3.3 TB/s, at the limit of a lane's registers.
#include <cmath>

#include "norm_rows.h"
#include "qsr_internal.h"

namespace qsr {

template <typename T, int NV, int W = 0> __device__ __forceinline__ float at(const RowPart<T, NV> &r, int c, int u) { return c < NV ? r.v[c][u] : r.t; }

struct LayerArgs {
    const void *x, *res;
    const float *w, *b;
    void *sum, *y;
    float *scale, *mean, *rstd;
    long long rows, s_x, s_res, s_sum, s_y;    // rows of a worker; strides from row to row
    long long s_w, s_b;                        // and from worker to worker
    int d;
    float eps;
};

// How a row of d elements is shared out: L lanes of W wavefronts, sixteen elements to a lane in bf16 where the row is long enough, eight in fp32.
// A row that leaves half of its lanes empty is slower where there is a width between: us, forward and backward, with it / with the next power
// of two, bf16: 15252 rows of 1100 31.9 / 33.0 and 41.7 / 48.5 (but 8192 of 2000 29.4 / 29.4 and 38.9 / 34.5), 3990 of 4204 30.2 / 34.5 and 36.7 /
// 39.6 (but 2943 of 5700 30.4 / 30.7 and 41.4 / 37.6), 1398 of 12000 30.8 / 32.6 and 41.8 / 63.1: twelve wavefronts leave 168 registers to a lane,
// sixteen 128; fp32: 3813 of 2200 29.1 / 28.6 and 32.5 / 37.5.
struct LayerPlan { int L, W, side; };
static LayerPlan layer_plan(long long d, int size)
{
    const long long unit = size == 2 ? 1024 : 512;
    LayerPlan q;
    q.L = d <= 128 ? 16 : d <= 256 ? 32 : 64;
    q.W = d <= 512 || d <= unit ? 1 : d <= 2 * unit ? (size == 2 && d > 1536 ? 4 : 2) : d <= 4 * unit ? 4 : d <= 5 * unit ? 5 : d <= 8 * unit ? 8
                                                                                         : size == 2 && d <= 12 * unit ? 12 : 16;
    q.side = q.W == 1 ? 256 / q.L : 1;
    return q;
}
// F(T, L, W, NV) for it; what no width of a type has is not built
#define LAYER_BY_WIDTH(T, d, F) do { constexpr int E_ = wide_of<T>(), N_ = sizeof(T) == 2 ? 16 / E_ : 8 / E_; \
    if ((d) < E_) F(T, 16, 1, 0); else if ((d) <= 128) F(T, 16, 1, 8 / E_); else if ((d) <= 256) F(T, 32, 1, 8 / E_); \
    else if ((d) <= 512) F(T, 64, 1, 8 / E_); \
    else switch (layer_plan(d, (int)sizeof(T)).W) { \
        case 1: if constexpr (sizeof(T) == 2) F(T, 64, 1, 16 / E_); break; \
        case 2: F(T, 64, 2, N_); break; \
        case 4: if constexpr (sizeof(T) == 2) { if ((d) > 2048) { F(T, 64, 4, 16 / E_); break; } } F(T, 64, 4, 8 / E_); break; \
        case 5: F(T, 64, 5, N_); break; \
        case 8: F(T, 64, 8, N_); break; \
        case 12: if constexpr (sizeof(T) == 2) F(T, 64, 12, 16 / E_); break; \
        default: if constexpr (sizeof(T) == 4) { if ((d) <= 8192) { F(T, 64, 16, 8 / E_); break; } } F(T, 64, 16, 16 / E_); } } while (0)

// Two sums over the lanes of a row with one barrier
template <int L, int W>
__device__ __forceinline__ void group_sums(float &p, float &q, float (*red)[2][W], int turn)
{
    if (W == 1) {
        p = group_sum<L, 1>(p, nullptr, 0);
        q = group_sum<L, 1>(q, nullptr, 0);
        return;
    }
    p = wave_sum(p);
    q = wave_sum(q);
    if ((threadIdx.x & 63) == 0) { red[turn & 1][0][threadIdx.x >> 6] = p; red[turn & 1][1][threadIdx.x >> 6] = q; }
    __syncthreads();
    p = q = 0.f;
#pragma unroll
    for (int i = 0; i < W; ++i) { p += red[turn & 1][0][i]; q += red[turn & 1][1][i]; }
}

// `turn` counts the sums over a group of wavefronts, which take turns at their words
template <typename T, int L, int W, int NV, bool FP8>
__device__ __forceinline__ void layernorm_row(const LayerArgs &a, const RowPart<T, NV> &w, const RowPart<T, NV> &b, long long row, int lane,
                                              float (*red)[W], float (*pair)[2][W], int &turn)
{
    constexpr int E = wide_of<T>();
    Row<T, NV> x, res;
    RowPart<T, NV> s;
    load_row<T, L, W, NV, true>((const T *)a.x + row * a.s_x, lane, a.d, x);
    if (a.res != nullptr) load_row<T, L, W, NV, true>((const T *)a.res + row * a.s_res, lane, a.d, res);
    each<T, NV>([](float &y, float v) { y = v; }, s, x);
    if (a.res != nullptr) each<T, NV>([](float &y, float v) { y += v; }, s, res);
    const int runs = a.d / E, rest = a.d - runs * E;
    // (sums leave the range of floats where their mean does not: by a power of two, whose roundings, of tiny numbers, the second sum puts right)
    constexpr float DOWN = 1.f / 65536.f, UP = 65536.f;
    float q = lane < rest ? s.t * DOWN : 0.f;
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        float part = 0.f;
#pragma unroll
        for (int u = 0; u < E; ++u) part = fmaf(s.v[c][u], DOWN, part);
        q += lane + c * L * W < runs ? part : 0.f;
    }
    if (a.sum != nullptr) store_row<T, L, W, NV, false>((T *)a.sum + row * a.s_sum, lane, a.d, s);
    const float near = group_sum<L, W>(q, red, turn++) / (float)a.d * UP;
    each<T, NV>([&](float &y) { y -= near; }, s);
    float p = lane < rest ? s.t : 0.f;
    q = lane < rest ? s.t * s.t : 0.f;
#pragma unroll
    for (int c = 0; c < NV; ++c) {
        float part = 0.f, squares = 0.f;
#pragma unroll
        for (int u = 0; u < E; ++u) { part += s.v[c][u]; squares = fmaf(s.v[c][u], s.v[c][u], squares); }
        p += lane + c * L * W < runs ? part : 0.f;
        q += lane + c * L * W < runs ? squares : 0.f;
    }
    group_sums<L, W>(p, q, pair, turn++);
    // where squares leave the range of floats, mean(t) is nothing beside them
    const float off = q < INFINITY ? p / (float)a.d : 0.f;
    float var = fmaf(-off, off, q / (float)a.d);
    var = (var < 0.f ? 0.f : var) + a.eps;                                 // (a NaN stays)
    const float rstd = var == 0.f ? 0.f : 1.f / sqrtf(var);                // equal numbers without eps: the bias, and no gradient
    if (lane == 0 && a.mean != nullptr) a.mean[row] = near + off;
    if (lane == 0 && a.rstd != nullptr) a.rstd[row] = rstd;
    each<T, NV>([&](float &y, float f, float g) { y = fmaf((y - off) * rstd, f, g); }, s, w, b);
    if (!FP8) {
        store_row<T, L, W, NV, false>((T *)a.y + row * a.s_y, lane, a.d, s);
        return;
    }
    // (a lane without a run has the last one's numbers without weight and bias: zeros)
    float top = 0.f;
    each<T, NV>([&](float &y) { if (fabsf(y) < INFINITY) top = fmaxf(top, fabsf(y)); }, s);
    top = group_max<L, W>(top, red, turn++);
    const float scale = top >= 1e-35f ? top * (1.f / E4M3_MAX) : 0.f;      // less would leave the range of floats
    if (lane == 0) a.scale[row] = scale;
    const float f = scale > 0.f ? 1.f / scale : 0.f;
    // a rounding above 448 at most, which still becomes 448; what is not finite becomes NaN
    each<T, NV>([&](float &y) { y *= f; }, s);
    store_codes<T, L, W, NV>((uint8_t *)a.y + row * a.s_y, lane, a.d, s);
}

template <typename T, int L, int W, int NV, bool FP8>
__global__ __launch_bounds__(rms_threads<W>()) void layernorm_kernel(LayerArgs a)
{
    __shared__ float red[2][W], pair[2][2][W];
    constexpr int side = rms_side<L, W>();
    const int k = blockIdx.y, lane = rms_lane<L, W>(), place = rms_place<L, W>();
    int turn = 0;
    RowPart<T, NV> w, b;
    load_words<T, L, W, NV>(a.w + k * a.s_w, lane, a.d, w);
    if (a.b != nullptr) load_words<T, L, W, NV>(a.b + k * a.s_b, lane, a.d, b);
    else each<T, NV>([](float &x) { x = 0.f; }, b);
    for (long long r = (long long)blockIdx.x * side + place; r < a.rows; r += (long long)gridDim.x * side)
        layernorm_row<T, L, W, NV, FP8>(a, w, b, k * a.rows + r, lane, red, pair, turn);
}

struct LayerBackArgs {
    const void *dy, *h;
    const float *w, *mean, *rstd;
    const void *dres;
    void *dx;
    float *part_w, *part_b;                    // each workgroup's sums, s_part apart
    long long rows, s_part, s_dy, s_h, s_dres, s_dx, s_w;
    int d;
};

// A workgroup takes every gridDim.x-th row (W == 1: 256 / L of them at a time) and keeps its parts of the gradients of weight and bias in
// registers.  A wavefront may have half of a SIMD's registers (a third and a quarter with twelve and sixteen wavefronts): with a quarter
// the sixteen elements of bf16 rows go to memory and back, 8 x 12608 rows of 768 130 us instead of 116, 8192 rows of 4096 74 instead of
// 56.  With sixteen wavefronts some do: above 12288 columns in bf16 24 bytes of a lane, 100 with a bias, above 8192 in fp32 104 and 172
// (2048 rows of 9001 with a bias 124 us, 2.4 TB/s).  The next row's loads are under way while a row is worked on where that takes few registers, and where a workgroup of five to
// eight wavefronts is alone on its compute unit (4096 rows of 8192 54 us, 60 without; 6 x 1915 of 4204 64, 88 without).
template <typename T, int L, int W, int NV, bool BIAS>
__global__ __launch_bounds__(rms_threads<W>(), W > 8 ? (W + 3) / 4 : 2) void layernorm_back_kernel(LayerBackArgs a)
{
    constexpr int E = wide_of<T>();
    constexpr bool AHEAD = NV * (3 * E + 3 * 2 * 4) <= 48 || (W > 4 && W <= 8 && E == 8);
    __shared__ float red[2][2][W];
    __shared__ float side_sum[W == 1 ? 3 * L * (NV * E + 1) : 1];
    constexpr int side = rms_side<L, W>();
    const int k = blockIdx.y, lane = rms_lane<L, W>(), place = rms_place<L, W>();
    const long long step = (long long)gridDim.x * side, last = (k + 1) * a.rows;
    RowPart<T, NV> w, dw, db;
    load_words<T, L, W, NV>(a.w + k * a.s_w, lane, a.d, w);
    each<T, NV>([](float &x, float &y) { x = 0.f; y = 0.f; }, dw, db);
    Row<T, NV> g, h, e = {};
    float rstd = 0.f, mean = 0.f;
    auto load = [&](long long row) {
        load_row<T, L, W, NV, true>((const T *)a.dy + row * a.s_dy, lane, a.d, g);
        load_row<T, L, W, NV, true>((const T *)a.h + row * a.s_h, lane, a.d, h);
        if (a.dres != nullptr) load_row<T, L, W, NV, true>((const T *)a.dres + row * a.s_dres, lane, a.d, e);
        rstd = a.rstd[row];
        mean = a.mean[row];
    };
    long long row = k * a.rows + (long long)blockIdx.x * side + place;
    if (AHEAD && row < last) load(row);
#pragma unroll 1
    for (int turn = 0; row < last; row += step, ++turn) {
        if (!AHEAD) load(row);
        Row<T, NV> g0 = g, h0 = h, e0 = e;
        const float rs = rstd, mu = mean;
        if (AHEAD) load(min(row + step, last - 1));
        float p = 0.f, q = 0.f;
        each<T, NV>([&](float &acc, float &sum, float f, float y, float x) {
            const float n = (x - mu) * rs, u = y * f;
            acc = fmaf(y, n, acc);
            if (BIAS) sum += y;
            p += u;
            q = fmaf(u, n, q);
        }, dw, db, w, g0, h0);
        group_sums<L, W>(p, q, red, turn);
        p /= (float)a.d;
        q /= (float)a.d;
        as_in_memory(g0);
        as_in_memory(h0);
        auto dx = [&](float f, float y, float x, float z) { return fmaf(rs, fmaf(-((x - mu) * rs), q, y * f - p), z); };
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
    const long long part = ((long long)k * gridDim.x + blockIdx.x) * a.s_part;
#pragma unroll
    for (int kind = 0; kind < (BIAS ? 2 : 1); ++kind) {
        RowPart<T, NV> &sum = kind ? db : dw;
        if (W == 1) {                          // the sums of a wavefront's rows and of the four wavefronts become one, in their order
            const int wave = threadIdx.x >> 6;
#pragma unroll
            for (int o = L; o < 64; o <<= 1) each<T, NV>([&](float &x) { x += __shfl_xor(x, o, 64); }, sum);
            float *const mine = side_sum + (wave > 0 ? wave - 1 : 0) * L * (NV * E + 1) + lane * (NV * E + 1);
            int n = 0;
            if (kind) __syncthreads();         // the weight's have been read
            if (wave > 0 && (threadIdx.x & 63) < L) each<T, NV>([&](float &x) { mine[n++] = x; }, sum);
            __syncthreads();
            if (threadIdx.x < L) {
#pragma unroll
                for (int o = 0; o < 3; ++o) {
                    const float *const other = side_sum + (o * L + lane) * (NV * E + 1);
                    n = 0;
                    each<T, NV>([&](float &x) { x += other[n++]; }, sum);
                }
            }
        }
        if (W > 1 || threadIdx.x < L) store_words<T, L, W, NV>((kind ? a.part_b : a.part_w) + part, lane, a.d, sum);
    }
}

// The gradients of weight and bias: sums over the parts [K][parts][cols], in a fixed order, COLS columns and 1024 / COLS runs of parts, four of
// each in flight, to a workgroup.  The first d columns are the weight's.  Latency is everything: fewer columns, on more workgroups,
// where there are few of them.
constexpr int SUM_THREADS = 1024;
template <int COLS>
__global__ __launch_bounds__(SUM_THREADS) void layernorm_sums_kernel(const float *__restrict__ partial, int parts, int cols, int d, float *__restrict__ dw,
                                                                     float *__restrict__ db)
{
    constexpr int RUNS = SUM_THREADS / COLS, WAVES = SUM_THREADS / 64;
    __shared__ float red[WAVES][COLS];
    const int k = blockIdx.y, col = threadIdx.x % COLS, run = threadIdx.x / COLS;
    const int j = blockIdx.x * COLS + col;
    const float *p = partial + (long long)k * parts * cols + j;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
    if (j < cols)
        for (int i = run; i < parts; i += 4 * RUNS)
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u * RUNS < parts) s[u] += p[(long long)(i + u * RUNS) * cols];
    float sum = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
    for (int o = COLS; o < 64; o <<= 1) sum += __shfl_xor(sum, o, 64);
    if ((threadIdx.x & 63) < COLS) red[threadIdx.x >> 6][col] = sum;
    __syncthreads();
    if (run != 0 || j >= cols) return;
    sum = 0.f;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) sum += red[i][col];
    if (j < d) dw[(long long)k * d + j] = sum;
    else db[(long long)k * d + j - d] = sum;
}

template <typename T>
static hipError_t launch_layer(const LayerArgs &a, int K, bool fp8, hipStream_t s)
{
    // A trip for each workgroup, but for the widest rows, whose weight and bias are as much as a row: one workgroup to a compute unit, and none
    // behind them (us with that / with two / with a trip each: 2048 rows of 16384 55.5 / 57.6 / 60.5, 5 x 1000 of 12000 82 / 83 / 95, and 100
    // with one of each worker more than two make; fp32 with eight elements to a lane, 5 x 596 of 7488, 71 / 69 / 65)
    const long long wide = 256 / K > 1 ? 256 / K : 1;
#define LAYER_FWD(T, L, W, NV) do { const long long trips = fwd_groups(a.rows, rms_side<L, W>()); \
    const dim3 grid((unsigned)(W > 8 && NV * wide_of<T>() == 16 && trips > wide ? wide : trips), (unsigned)K); \
    if (fp8) layernorm_kernel<T, L, W, NV, true><<<grid, rms_threads<W>(), 0, s>>>(a); \
    else layernorm_kernel<T, L, W, NV, false><<<grid, rms_threads<W>(), 0, s>>>(a); } while (0)
    LAYER_BY_WIDTH(T, a.d, LAYER_FWD);
#undef LAYER_FWD
    return hipGetLastError();
}

// Workgroups of a worker in the backward pass, one at least: two wavefronts to each of the chip's SIMDs, four in the widest rows and in narrow ones of bf16,
// which have little in flight (4 x 20000 rows of 200 30.9 us, with two 38.3, with five 36.5; in fp32 30000 of 250 29.1 with four, 26.7 with two),
// and not one more, where each has a place of its own and those behind it would wait for it to end (6 x 1915 rows of 4204 in bf16 63 us, 144 with
// 43 workgroups of a worker instead of 42; 5 x 596 of 7488 in fp32 76, 102 with 52 instead of 51).  Each leaves a row of partial sums, and has
// more than one row where some 160 of them remain: 2 x 455 rows of 1600 in bf16 10.4, 12.2 with a row each; 1000 of 4096 18.3, 22.5; 8 x 1472 of
// 205 9.8, 12.0; but 5 x 171 of 554 8.5 with two, 7.5.  One, whose sums are the gradients already, for the rows of a few tokens.
static long long layer_back_groups(int K, long long rows, long long d, int size)
{
    const LayerPlan q = layer_plan(d, size);
    if (rows <= 2 * q.side) return 1;
    const long long all = (q.L < 64 && size == 2) || q.W == 2 ? 1024 : q.W <= 4 || (q.W == 5 && size == 4) ? 512 : 256;
    const long long most = all / K > 1 ? all / K : 1, trips = (rows + q.side - 1) / q.side, few = q.W == 1 ? 2 : 4;
    const long long own = K * trips / 160, each = own < 1 ? 1 : own < few ? own : few, need = (trips + each - 1) / each;
    return most < need ? most : need;
}

template <typename T>
static hipError_t launch_layer_back(LayerBackArgs &a, int K, float *workspace, float *dw, float *db, hipStream_t s)
{
    const long long groups = layer_back_groups(K, a.rows, a.d, (int)sizeof(T));
    const int cols = a.d * (db != nullptr ? 2 : 1);
    if (groups == 1) { a.part_w = dw; a.part_b = db; a.s_part = a.d; }
    else { a.part_w = workspace; a.part_b = workspace + a.d; a.s_part = cols; }
#define LAYER_BACK(T, L, W, NV) do { const dim3 grid((unsigned)groups, (unsigned)K); \
    if (db != nullptr) layernorm_back_kernel<T, L, W, NV, true><<<grid, rms_threads<W>(), 0, s>>>(a); \
    else layernorm_back_kernel<T, L, W, NV, false><<<grid, rms_threads<W>(), 0, s>>>(a); } while (0)
    LAYER_BY_WIDTH(T, a.d, LAYER_BACK);
#undef LAYER_BACK
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || groups == 1) return e;
    const long long all = (long long)K * cols;
    const auto sums = all >= 256 * 32 ? layernorm_sums_kernel<32> : all >= 256 * 16 ? layernorm_sums_kernel<16> : layernorm_sums_kernel<8>;
    const int per = all >= 256 * 32 ? 32 : all >= 256 * 16 ? 16 : 8;
    sums<<<dim3((unsigned)((cols + per - 1) / per), (unsigned)K), SUM_THREADS, 0, s>>>(workspace, (int)groups, cols, a.d, dw, db);
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

extern "C" int qsr_layernorm(const qsr_layernorm_args *q, void *stream)
{
    if (!q || !sizes_ok(q->K, q->rows, q->d)) return QSR_EINVAL;
    if (q->type != QSR_TYPE_F32 && q->type != QSR_TYPE_BF16) return QSR_EINVAL;
    const bool fp8 = q->y_type == QSR_TYPE_E4M3;
    if (!fp8 && q->y_type != q->type) return QSR_EINVAL;
    const uintptr_t es = size_of(q->type);
    if (!(std::isfinite(q->eps) && q->eps >= 0.0)) return QSR_EINVAL;
    if (q->d > RMS_MAX_D) return QSR_ELIMIT;
    if (q->rows == 0) return QSR_OK;
    if (!q->x || off(q->x, es) || off(q->residual, es) || !q->weight || off(q->weight, 4) || off(q->bias, 4) || off(q->sum, es) || !q->y ||
        (!fp8 && off(q->y, es)) || off(q->mean, 4) || off(q->rstd, 4) || off(q->scale, 4) || (fp8 && !q->scale))
        return QSR_EINVAL;
    if (q->x_stride < q->d || q->y_stride < q->d || (q->residual && q->residual_stride < q->d) || (q->sum && q->sum_stride < q->d) ||
        (q->K > 1 && (q->weight_stride < q->d || (q->bias && q->bias_stride < q->d))))
        return QSR_EINVAL;
    const LayerArgs a{q->x, q->residual, q->weight, q->bias, q->sum, q->y, fp8 ? q->scale : nullptr, q->mean, q->rstd, q->rows, q->x_stride,
                      q->residual_stride, q->sum_stride, q->y_stride, q->weight_stride, q->bias_stride, (int)q->d, (float)q->eps};
    return finish(q->type == QSR_TYPE_F32 ? launch_layer<float>(a, q->K, fp8, (hipStream_t)stream)
                                          : launch_layer<bf16_t>(a, q->K, fp8, (hipStream_t)stream));
}

extern "C" int qsr_layernorm_workspace_bytes(int32_t K, int64_t rows, int64_t d, int32_t type, size_t *bytes)
{
    if (!bytes) return QSR_EINVAL;
    *bytes = 0;
    if (!sizes_ok(K, rows, d) || (type != QSR_TYPE_F32 && type != QSR_TYPE_BF16)) return QSR_EINVAL;
    if (d > RMS_MAX_D) return QSR_ELIMIT;
    const long long groups = layer_back_groups(K, rows, d, (int)size_of(type));
    *bytes = groups == 1 ? 0 : (size_t)K * (size_t)groups * (size_t)(2 * d) * sizeof(float);
    return QSR_OK;
}

extern "C" int qsr_layernorm_backward(const qsr_layernorm_backward_args *q, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!q || !sizes_ok(q->K, q->rows, q->d)) return QSR_EINVAL;
    if (q->type != QSR_TYPE_F32 && q->type != QSR_TYPE_BF16) return QSR_EINVAL;
    const uintptr_t es = size_of(q->type);
    if (!q->weight || off(q->weight, 4) || !q->weight_grad || off(q->weight_grad, 4) || off(q->bias_grad, 4)) return QSR_EINVAL;
    if (q->rows > 0 && (!q->y_grad || off(q->y_grad, es) || !q->sum || off(q->sum, es) || !q->mean || off(q->mean, 4) || !q->rstd ||
                        off(q->rstd, 4) || off(q->residual_grad, es) || !q->x_grad || off(q->x_grad, es)))
        return QSR_EINVAL;
    if (q->y_grad_stride < q->d || q->sum_stride < q->d || q->x_grad_stride < q->d ||
        (q->residual_grad && q->residual_grad_stride < q->d) || (q->K > 1 && q->weight_stride < q->d))
        return QSR_EINVAL;
    size_t need = 0;
    const int rc = qsr_layernorm_workspace_bytes(q->K, q->rows, q->d, q->type, &need);
    if (rc != QSR_OK) return rc;
    if (need > 0 && (!workspace || off(workspace, 4))) return QSR_EINVAL;
    if (workspace_bytes < need) return QSR_ENOMEM;
    LayerBackArgs a{q->y_grad, q->sum, q->weight, q->mean, q->rstd, q->residual_grad, q->x_grad, nullptr, nullptr, q->rows, 0,
                    q->y_grad_stride, q->sum_stride, q->residual_grad_stride, q->x_grad_stride, q->weight_stride, (int)q->d};
    return finish(q->type == QSR_TYPE_F32 ? launch_layer_back<float>(a, q->K, (float *)workspace, q->weight_grad, q->bias_grad, (hipStream_t)stream)
                                          : launch_layer_back<bf16_t>(a, q->K, (float *)workspace, q->weight_grad, q->bias_grad, (hipStream_t)stream));
}
