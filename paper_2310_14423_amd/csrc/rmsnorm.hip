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

#include "norm_rows.h"
#include "qsr_internal.h"

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
    store_codes<T, L, W, NV>((uint8_t *)a.y + row * a.s_y, lane, a.d, s);
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
