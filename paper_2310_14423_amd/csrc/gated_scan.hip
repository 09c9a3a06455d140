// gated_scan.hip -- a gated linear recurrence over sequences, for each channel by itself, and its gradients.
//
//   a_t = sigmoid(f_t), c_t = 1 - a_t = sigmoid(-f_t):   h_t = a_t h'_{t-1} + w_t x_t,   w = c ("complement") or 1 ("plain")
//   h'_{t-1} is h_{t-1}, or 0 where step t is marked as a reset;  h_{-1} = initial or 0
// and backward, with g_t the gradient of h_t from all that follows and e_t = a_t g_t what it leaves to h_{t-1} (0 at a reset):
//   g_t = dh_t + e_{t+1}, e_len = dlast:   dx_t = w_t g_t;   df_t = g_t a_t c_t (h'_{t-1} - x_t), or without x_t in "plain";   dinitial = e_0
// A run of steps is a map h -> A h + H, two of them behind each other are one again: that makes a scan of it.  A wavefront takes
// STEPS steps of 64 lanes' channels into its registers, finds their map, learns from the maps of the wavefronts before it, through LDS, what
// state its own steps begin with, and goes through them once more: x and f are read from memory once.  Where sequences and channels
// give too few workgroups, sequences are cut into parts, whose maps a launch before finds, for which x and f are read a second time.
// Backward, h is not read but made again from the states kept at every STEPS-th step in fp32: 1/4 or 1/8 of the reads of h, and
// nothing of h's rounding in the gradients.
// A reset cuts a map off from what was before: A = -1 stands for that (A is never negative), so that an infinity or a NaN ends there too.
// All arithmetic is fp32.
#include <cmath>

#include "qsr_internal.h"
#include "row_io.h"
#include "tile_grid.h"

namespace qsr {

constexpr int STEPS = QSR_SCAN_STEPS;
constexpr int SCAN_WAVES = 8;                  // wavefronts to a workgroup, where sequences are longer than one of them takes

struct ScanArgs {
    const void *x, *f, *dh;
    void *h, *dx, *df;
    const float *initial;                      // or, backward, the gradient of the last state
    float *last;                               // or, backward, the gradient of the initial state
    float *states;
    const uint8_t *reset;
    const int64_t *lengths;
    float2 *maps;                              // [B][parts + 1][d]: forward, the initial state, then the maps of all parts but the last
    long long s_x, s_f, s_dh, s_h, s_dx, s_df; // from step to step
    long long b_x, b_f, b_dh, b_h, b_dx, b_df; // and from sequence to sequence
    long long tiles;
    int T, d, groups, parts, part_len;
};

// a and c of the gate f.  exp(-|f|) has no overflow, and both come out with the relative precision of a float.
template <typename T> __device__ __forceinline__ void gates(float f, float &a, float &c)
{
    float e, big;
    if constexpr (sizeof(T) == 2) {            // 2^-20 of an error at most, beside the gate's own 2^-9
        e = __builtin_amdgcn_exp2f(-1.44269504f * fabsf(f));
        big = __builtin_amdgcn_rcpf(1.f + e);
    } else {
        e = expf(-fabsf(f));
        const float s = 1.f + e, r = __builtin_amdgcn_rcpf(s);
        big = fmaf(fmaf(-s, r, 1.f), r, r);
    }
    const float small = e * big;
    a = f >= 0.f ? big : small;
    c = f >= 0.f ? small : big;
}

// A map (A, H) behind h
__device__ __forceinline__ float behind_map(float A, float H, float h) { return A < 0.f ? H : fmaf(A, h, H); }

template <typename T, int V> struct Rows { typename Wide<T, V>::vec v[STEPS]; };

// The rows first .. first + n - 1 of a sequence at p (which points at the lane's channels); those behind them again the last one
template <typename T, int V>
__device__ __forceinline__ void load_rows(const T *p, uint32_t at, long long stride, long long first, int n, Rows<T, V> &r)
{
    if (n <= 0) return;
    p += first * stride;
#pragma unroll
    for (int s = 0; s < STEPS; ++s) r.v[s] = *(const typename Wide<T, V>::vec *)behind(p + min(s, n - 1) * stride, at);
}
// without loads of rows that are not there, for few of them
template <typename T, int V>
__device__ __forceinline__ void load_few(const T *p, uint32_t at, long long stride, int n, Rows<T, V> &r)
{
#pragma unroll
    for (int s = 0; s < STEPS; ++s)
        if (s < n) r.v[s] = *(const typename Wide<T, V>::vec *)behind(p + s * stride, at);
}

template <typename T, int V>
__device__ __forceinline__ void store_channels(T *p, uint32_t at, const float (&v)[V], int skip)
{
    if (skip == 0) store_wide<T, V, true>(behind(p, at), v);
    else {
#pragma unroll
        for (int u = 0; u < V; ++u)
            if (u >= skip && skip < V) behind(p, at)[u] = (T)v[u];
    }
}

// A lane's place: V channels from `at`, of which the first `skip` are another lane's (V: all of them)
template <int V> struct Place {
    int b, part, at, skip, len;
    __device__ __forceinline__ bool find(const ScanArgs &a, int lane, int parts)
    {
        const long long id = blockIdx.x + (long long)blockIdx.y * gridDim.x;
        if (id >= a.tiles) return false;
        const long long seq = id / a.groups;
        const int first = ((int)(id - seq * a.groups) * 64 + lane) * V;
        b = (int)(seq / parts);
        part = (int)(seq - (long long)b * parts);
        at = min(first, a.d - V);
        skip = min(first - at, V);
        len = a.T;
        if (a.lengths != nullptr) {
            const long long n = a.lengths[b];
            len = (int)(n < 0 ? 0 : n > a.T ? a.T : n);
        }
        return true;
    }
};

// The marks of steps t .. t + STEPS - 1, a bit each
__device__ __forceinline__ uint32_t marks(const ScanArgs &a, int b, int t, int n, int lane)
{
    if (a.reset == nullptr || n <= 0) return 0;
    const uint8_t m = a.reset[(long long)b * a.T + t + min(lane, n - 1)];
    return (uint32_t)__ballot(m != 0 && lane < n);
}

// Forward, W wavefronts to a workgroup
template <typename T, int V, int W, bool COMP>
__global__ __launch_bounds__(64 * W) void scan_kernel(ScanArgs a)
{
    __shared__ float2 maps[2][W][V][64];
    const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Place<V> q;
    if (!q.find(a, lane, a.parts)) return;
    const T *const px = (const T *)a.x + q.b * a.b_x, *const pf = (const T *)a.f + q.b * a.b_f;
    const uint32_t at = (uint32_t)q.at * (uint32_t)sizeof(T);
    float carry[V];
    if (a.parts > 1) {
        const float2 *const m = a.maps + ((long long)q.b * (a.parts + 1)) * a.d + q.at;
#pragma unroll
        for (int u = 0; u < V; ++u) carry[u] = 0.f;
#pragma unroll 4
        for (int p = 0; p <= q.part; ++p)
#pragma unroll
            for (int u = 0; u < V; ++u) { const float2 f = m[(long long)p * a.d + u]; carry[u] = behind_map(f.x, f.y, carry[u]); }
    } else {
#pragma unroll
        for (int u = 0; u < V; ++u) {
            carry[u] = a.initial != nullptr ? a.initial[(long long)q.b * a.d + q.at + u] : 0.f;
            asm volatile("" : "+v"(carry[u]));             // here before the first barrier: `last` may be the same memory
        }
    }
    const int begin = q.part * a.part_len, end = min(a.T, begin + a.part_len);
    Rows<T, V> rx, rf;
    uint32_t bits = 0;
    auto load = [&](int t0) {
        const int t = t0 + wave * STEPS, n = min(q.len - t, STEPS);
        if (W == 1) { load_few<T, V>(px, at, a.s_x, n, rx); load_few<T, V>(pf, at, a.s_f, n, rf); }
        else { load_rows<T, V>(px, at, a.s_x, t, n, rx); load_rows<T, V>(pf, at, a.s_f, t, n, rf); }
        bits = marks(a, q.b, t, n, lane);
    };
    if (begin < end) load(begin);
    int turn = 0;
#pragma unroll 1
    for (int t0 = begin; t0 < end; t0 += W * STEPS, turn ^= 1) {
        const int t = t0 + wave * STEPS, n = min(q.len - t, STEPS);
        const uint32_t cut = bits;
        float ga[STEPS][V], gb[STEPS][V];
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int u = 0; u < V; ++u) {
                float c;
                gates<T>((float)rf.v[s][u], ga[s][u], c);
                gb[s][u] = COMP ? c * (float)rx.v[s][u] : (float)rx.v[s][u];
                if (s >= n) { ga[s][u] = 1.f; gb[s][u] = 0.f; }            // behind the end the state stays
            }
        if (t0 + W * STEPS < end) load(t0 + W * STEPS);
        float h[V];
        if (W > 1) {
            float A[V], H[V];
#pragma unroll
            for (int u = 0; u < V; ++u) { A[u] = 1.f; H[u] = 0.f; }
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int u = 0; u < V; ++u) {
                    if (cut >> s & 1) H[u] = 0.f;
                    H[u] = fmaf(ga[s][u], H[u], gb[s][u]);
                    A[u] *= ga[s][u];
                }
#pragma unroll
            for (int u = 0; u < V; ++u) maps[turn][wave][u][lane] = make_float2(cut ? -1.f : A[u], H[u]);
            __syncthreads();
#pragma unroll
            for (int w = 0; w < W; ++w)
#pragma unroll
                for (int u = 0; u < V; ++u) {
                    if (w == wave) h[u] = carry[u];
                    const float2 m = maps[turn][w][u][lane];
                    carry[u] = behind_map(m.x, m.y, carry[u]);
                }
        } else {
#pragma unroll
            for (int u = 0; u < V; ++u) h[u] = carry[u];
        }
        if (a.states != nullptr && t < end)
            store_channels<float, V>(a.states + ((long long)q.b * ((a.T + STEPS - 1) / STEPS) + t / STEPS) * a.d, (uint32_t)q.at * 4, h, q.skip);
        T *const ph = (T *)a.h + q.b * a.b_h + t * a.s_h;
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            float y[V];
#pragma unroll
            for (int u = 0; u < V; ++u) {
                if (cut >> s & 1) h[u] = 0.f;
                h[u] = fmaf(ga[s][u], h[u], gb[s][u]);
                y[u] = s < n ? h[u] : 0.f;
            }
            if (t + s < end) store_channels<T, V>(ph + s * a.s_h, at, y, q.skip);
        }
        if (W == 1)
#pragma unroll
            for (int u = 0; u < V; ++u) carry[u] = h[u];
    }
    if (a.last != nullptr && q.part == a.parts - 1 && wave == 0)
        store_channels<float, V>(a.last + (long long)q.b * a.d, (uint32_t)q.at * 4, carry, q.skip);
}

// The maps of parts: a wavefront goes through a run of its part's steps.  Forward: all parts but the last, and the initial state.
// Backward: e before a part from e behind it, all parts but the first.
template <typename T, int V, bool COMP, bool BACK>
__global__ __launch_bounds__(64 * SCAN_WAVES) void scan_maps_kernel(ScanArgs a)
{
    __shared__ float2 maps[SCAN_WAVES][V][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Place<V> q;
    if (!q.find(a, lane, a.parts - 1)) return;
    const int part = BACK ? q.part + 1 : q.part;
    const T *const px = (const T *)(BACK ? a.dh : a.x) + q.b * (BACK ? a.b_dh : a.b_x), *const pf = (const T *)a.f + q.b * a.b_f;
    const long long s_x = BACK ? a.s_dh : a.s_x;
    const uint32_t at = (uint32_t)q.at * (uint32_t)sizeof(T);
    const int each = a.part_len / SCAN_WAVES, begin = part * a.part_len + wave * each, end = min(a.T, begin + each);
    const int trips = begin < end ? (end - begin + STEPS - 1) / STEPS : 0;
    Rows<T, V> rx, rf;
    uint32_t bits = 0;
    auto start_of = [&](int i) { return begin + (BACK ? trips - 1 - i : i) * STEPS; };
    auto load = [&](int t) {
        const int n = min(q.len - t, STEPS);
        load_rows<T, V>(px, at, s_x, t, n, rx);
        load_rows<T, V>(pf, at, a.s_f, t, n, rf);
        bits = marks(a, q.b, t, n, lane);
    };
    float A[V], H[V];
    uint32_t any = 0;
#pragma unroll
    for (int u = 0; u < V; ++u) { A[u] = 1.f; H[u] = 0.f; }
    if (trips > 0) load(start_of(0));
#pragma unroll 1
    for (int i = 0; i < trips; ++i) {
        const int n = min(q.len - start_of(i), STEPS);
        const uint32_t cut = bits;
        const Rows<T, V> x = rx, f = rf;
        if (i + 1 < trips) load(start_of(i + 1));
        any |= cut;
#pragma unroll
        for (int o = 0; o < STEPS; ++o) {
            const int s = BACK ? STEPS - 1 - o : o;
            if (s < n) {
#pragma unroll
                for (int u = 0; u < V; ++u) {
                    float ga, c;
                    gates<T>((float)f.v[s][u], ga, c);
                    const float v = (float)x.v[s][u];
                    if (BACK) {
                        H[u] = ga * (v + H[u]);
                        if (cut >> s & 1) H[u] = 0.f;
                    } else {
                        if (cut >> s & 1) H[u] = 0.f;
                        H[u] = fmaf(ga, H[u], COMP ? c * v : v);
                    }
                    A[u] *= ga;
                }
            }
        }
    }
#pragma unroll
    for (int u = 0; u < V; ++u) maps[wave][u][lane] = make_float2(any ? -1.f : A[u], H[u]);
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int u = 0; u < V; ++u) { A[u] = 1.f; H[u] = 0.f; }
#pragma unroll
    for (int i = 0; i < SCAN_WAVES; ++i)
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const float2 m = maps[BACK ? SCAN_WAVES - 1 - i : i][u][lane];
            H[u] = behind_map(m.x, m.y, H[u]);
            A[u] = m.x < 0.f || A[u] < 0.f ? -1.f : A[u] * m.x;
        }
    float2 *const m = a.maps + ((long long)q.b * (a.parts + 1)) * a.d + q.at;
#pragma unroll
    for (int u = 0; u < V; ++u)
        if (u >= q.skip) {
            m[(long long)(BACK ? part : part + 1) * a.d + u] = make_float2(A[u], H[u]);
            if (!BACK && part == 0) m[u] = make_float2(-1.f, a.initial != nullptr ? a.initial[(long long)q.b * a.d + q.at + u] : 0.f);
        }
}

// Backward, W wavefronts to a workgroup, from the end
template <typename T, int V, int W, bool COMP>
__global__ __launch_bounds__(64 * W, 2) void scan_back_kernel(ScanArgs a)
{
    __shared__ float2 maps[2][W][V][64];
    const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Place<V> q;
    if (!q.find(a, lane, a.parts)) return;
    const T *const px = (const T *)a.x + q.b * a.b_x, *const pf = (const T *)a.f + q.b * a.b_f, *const pg = (const T *)a.dh + q.b * a.b_dh;
    const float *const ps = a.states + (long long)q.b * ((a.T + STEPS - 1) / STEPS) * a.d + q.at;
    const uint32_t at = (uint32_t)q.at * (uint32_t)sizeof(T);
    float carry[V];
#pragma unroll
    for (int u = 0; u < V; ++u) carry[u] = a.initial != nullptr ? a.initial[(long long)q.b * a.d + q.at + u] : 0.f;
    if (a.parts > 1) {
        const float2 *const m = a.maps + ((long long)q.b * (a.parts + 1)) * a.d + q.at;
#pragma unroll 4
        for (int p = a.parts - 1; p > q.part; --p)
#pragma unroll
            for (int u = 0; u < V; ++u) { const float2 f = m[(long long)p * a.d + u]; carry[u] = behind_map(f.x, f.y, carry[u]); }
    }
    const int begin = q.part * a.part_len, end = min(a.T, begin + a.part_len);
    const int trips = begin < end ? (end - begin + W * STEPS - 1) / (W * STEPS) : 0;
    Rows<T, V> rx, rf, rg;
    float rs[V] = {};
    uint32_t bits = 0;
    auto load = [&](int t0) {
        const int t = t0 + wave * STEPS, n = min(q.len - t, STEPS);
        if (W == 1) {
            load_few<T, V>(px, at, a.s_x, n, rx);
            load_few<T, V>(pf, at, a.s_f, n, rf);
            load_few<T, V>(pg, at, a.s_dh, n, rg);
        } else {
            load_rows<T, V>(px, at, a.s_x, t, n, rx);
            load_rows<T, V>(pf, at, a.s_f, t, n, rf);
            load_rows<T, V>(pg, at, a.s_dh, t, n, rg);
        }
        if (n > 0)
#pragma unroll
            for (int u = 0; u < V; ++u) rs[u] = ps[(long long)(t / STEPS) * a.d + u];
        bits = marks(a, q.b, t, n, lane);
    };
    if (trips > 0) load(begin + (trips - 1) * W * STEPS);
    int turn = 0;
#pragma unroll 1
    for (int i = trips - 1; i >= 0; --i, turn ^= 1) {
        const int t = begin + i * W * STEPS + wave * STEPS, n = min(q.len - t, STEPS);
        const uint32_t cut = bits;
        float ga[STEPS][V], gc[STEPS][V], h[V];
        const Rows<T, V> x = rx, g = rg;
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int u = 0; u < V; ++u) {
                gates<T>((float)rf.v[s][u], ga[s][u], gc[s][u]);
                if (s >= n) ga[s][u] = 1.f;
            }
#pragma unroll
        for (int u = 0; u < V; ++u) h[u] = rs[u];
        if (i > 0) load(begin + (i - 1) * W * STEPS);
        float e[V];
        if (W > 1) {
            float A[V], H[V];
#pragma unroll
            for (int u = 0; u < V; ++u) { A[u] = 1.f; H[u] = 0.f; }
#pragma unroll
            for (int s = STEPS - 1; s >= 0; --s)
#pragma unroll
                for (int u = 0; u < V; ++u) {
                    H[u] = ga[s][u] * (H[u] + (s < n ? (float)g.v[s][u] : 0.f));
                    if (cut >> s & 1) H[u] = 0.f;
                    A[u] *= ga[s][u];
                }
#pragma unroll
            for (int u = 0; u < V; ++u) maps[turn][wave][u][lane] = make_float2(cut ? -1.f : A[u], H[u]);
            __syncthreads();
#pragma unroll
            for (int w = W - 1; w >= 0; --w)
#pragma unroll
                for (int u = 0; u < V; ++u) {
                    if (w == wave) e[u] = carry[u];
                    const float2 m = maps[turn][w][u][lane];
                    carry[u] = behind_map(m.x, m.y, carry[u]);
                }
        } else {
#pragma unroll
            for (int u = 0; u < V; ++u) e[u] = carry[u];
        }
        float before[STEPS][V];
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int u = 0; u < V; ++u) {
                if (cut >> s & 1) h[u] = 0.f;
                before[s][u] = h[u];
                const float v = (float)x.v[s][u];
                h[u] = fmaf(ga[s][u], h[u], COMP ? gc[s][u] * v : v);
            }
        T *const pdx = (T *)a.dx + q.b * a.b_dx + t * a.s_dx, *const pdf = (T *)a.df + q.b * a.b_df + t * a.s_df;
#pragma unroll
        for (int s = STEPS - 1; s >= 0; --s) {
            float dx[V], df[V];
#pragma unroll
            for (int u = 0; u < V; ++u) {
                if (s < n) {
                    const float v = (float)x.v[s][u], grad = (float)g.v[s][u] + e[u];
                    dx[u] = COMP ? gc[s][u] * grad : grad;
                    e[u] = ga[s][u] * grad;
                    df[u] = e[u] * gc[s][u] * (COMP ? before[s][u] - v : before[s][u]);
                    if (cut >> s & 1) e[u] = 0.f;
                } else dx[u] = df[u] = 0.f;
            }
            if (t + s < end) {
                store_channels<T, V>(pdx + s * a.s_dx, at, dx, q.skip);
                store_channels<T, V>(pdf + s * a.s_df, at, df, q.skip);
            }
        }
        if (W == 1)
#pragma unroll
            for (int u = 0; u < V; ++u) carry[u] = e[u];
    }
    if (a.last != nullptr && q.part == 0 && wave == 0)
        store_channels<float, V>(a.last + (long long)q.b * a.d, (uint32_t)q.at * 4, carry, q.skip);
}

// ---------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------
// Channels of a lane: four bytes of them, one where there are not as many
static int scan_channels(int type, long long d) { return type == QSR_TYPE_BF16 && d >= 2 ? 2 : 1; }

struct ScanPlan { int waves, parts, part_len; long long groups; };
static ScanPlan scan_plan(long long B, long long T, long long d, int type)
{
    ScanPlan p;
    const int V = scan_channels(type, d);
    p.groups = (d + 64 * V - 1) / (64 * V);
    p.waves = T <= STEPS ? 1 : SCAN_WAVES;
    p.parts = 1;
    const long long trip = (long long)p.waves * STEPS, trips = (T + trip - 1) / trip, have = B * p.groups;
    if (have < 256 && trips >= 8) {
        long long want = (512 + have - 1) / have;
        if (want > trips / 4) want = trips / 4;
        const long long each = (trips + want - 1) / want;
        p.parts = (int)((trips + each - 1) / each);
        p.part_len = (int)(each * trip);
    } else p.part_len = (int)(trips * trip < T ? T : trips * trip);
    return p;
}

template <typename T, int V, bool COMP>
static hipError_t launch_scan(ScanArgs &a, const ScanPlan &p, long long B, bool back, hipStream_t s)
{
    a.groups = (int)p.groups;
    a.parts = p.parts;
    a.part_len = p.part_len;
    if (p.parts > 1) {
        a.tiles = B * (p.parts - 1) * p.groups;
        const TileGrid g = tile_grid(a.tiles, 64 * SCAN_WAVES);
        if (g.x == 0) return hipErrorInvalidConfiguration;
        if (back) scan_maps_kernel<T, V, COMP, true><<<dim3(g.x, g.y), 64 * SCAN_WAVES, 0, s>>>(a);
        else scan_maps_kernel<T, V, COMP, false><<<dim3(g.x, g.y), 64 * SCAN_WAVES, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    a.tiles = B * p.parts * p.groups;
    const TileGrid g = tile_grid(a.tiles, 64 * p.waves);
    if (g.x == 0) return hipErrorInvalidConfiguration;
    const dim3 grid(g.x, g.y);
    if (p.waves == 1) {
        if (back) scan_back_kernel<T, V, 1, COMP><<<grid, 64, 0, s>>>(a);
        else scan_kernel<T, V, 1, COMP><<<grid, 64, 0, s>>>(a);
    } else {
        if (back) scan_back_kernel<T, V, SCAN_WAVES, COMP><<<grid, 64 * SCAN_WAVES, 0, s>>>(a);
        else scan_kernel<T, V, SCAN_WAVES, COMP><<<grid, 64 * SCAN_WAVES, 0, s>>>(a);
    }
    return hipGetLastError();
}
static hipError_t launch_scan(ScanArgs &a, int type, int input, long long B, bool back, hipStream_t s)
{
    const ScanPlan p = scan_plan(B, a.T, a.d, type);
    const bool comp = input == QSR_SCAN_COMPLEMENT;
    if (type == QSR_TYPE_F32) return comp ? launch_scan<float, 1, true>(a, p, B, back, s) : launch_scan<float, 1, false>(a, p, B, back, s);
    if (scan_channels(type, a.d) == 2) return comp ? launch_scan<bf16_t, 2, true>(a, p, B, back, s) : launch_scan<bf16_t, 2, false>(a, p, B, back, s);
    return comp ? launch_scan<bf16_t, 1, true>(a, p, B, back, s) : launch_scan<bf16_t, 1, false>(a, p, B, back, s);
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
static bool scan_sizes_ok(int64_t B, int64_t T, int64_t d, int32_t type)
{
    return (type == QSR_TYPE_F32 || type == QSR_TYPE_BF16) && B >= 0 && T >= 0 && d >= 1;
}
static bool scan_limits_ok(int64_t B, int64_t T, int64_t d)
{
    return B < ((int64_t)1 << 31) && T <= ((int64_t)1 << 30) && d <= ((int64_t)1 << 28) &&
           B * ((d + 63) / 64) < ((int64_t)1 << 36);
}
// Rows of d elements, `step` from step to step and `seq` from sequence to sequence.  written: no two of them share an element.
static bool strides_ok(int64_t B, int64_t T, int64_t d, int64_t seq, int64_t step, bool written)
{
    if ((T > 1 && step < d) || (B > 1 && seq < d)) return false;
    if (!written || T <= 1 || B <= 1) return true;
    return seq / step >= T ? true : seq >= (T - 1) * step + d || step >= (B - 1) * seq + d;
}

extern "C" int qsr_gated_scan_workspace_bytes(int64_t batch, int64_t steps, int64_t d, int32_t type, size_t *bytes)
{
    if (!bytes) return QSR_EINVAL;
    *bytes = 0;
    if (!scan_sizes_ok(batch, steps, d, type)) return QSR_EINVAL;
    if (!scan_limits_ok(batch, steps, d)) return QSR_ELIMIT;
    if (batch == 0) return QSR_OK;
    const ScanPlan p = scan_plan(batch, steps, d, type);
    *bytes = p.parts > 1 ? (size_t)batch * (size_t)(p.parts + 1) * (size_t)d * sizeof(float2) : 0;
    return QSR_OK;
}

extern "C" int qsr_gated_scan(const qsr_gated_scan_args *q, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!q || !scan_sizes_ok(q->batch, q->steps, q->d, q->type)) return QSR_EINVAL;
    if (q->input != QSR_SCAN_COMPLEMENT && q->input != QSR_SCAN_PLAIN) return QSR_EINVAL;
    if (!scan_limits_ok(q->batch, q->steps, q->d)) return QSR_ELIMIT;
    const uintptr_t es = q->type == QSR_TYPE_F32 ? 4 : 2;
    if (q->batch == 0 || (q->steps == 0 && !q->last)) return QSR_OK;
    if (off(q->initial, 4) || off(q->last, 4) || off(q->states, 4) || off(q->lengths, 8)) return QSR_EINVAL;
    if (q->steps > 0 && (!q->x || off(q->x, es) || !q->gate || off(q->gate, es) || !q->h || off(q->h, es))) return QSR_EINVAL;
    if (!strides_ok(q->batch, q->steps, q->d, q->x_batch_stride, q->x_stride, false) ||
        !strides_ok(q->batch, q->steps, q->d, q->gate_batch_stride, q->gate_stride, false) ||
        !strides_ok(q->batch, q->steps, q->d, q->h_batch_stride, q->h_stride, true))
        return QSR_EINVAL;
    size_t need = 0;
    const int rc = qsr_gated_scan_workspace_bytes(q->batch, q->steps, q->d, q->type, &need);
    if (rc != QSR_OK) return rc;
    if (need > 0 && (!workspace || off(workspace, 8))) return QSR_EINVAL;
    if (workspace_bytes < need) return QSR_ENOMEM;
    ScanArgs a{};
    a.x = q->x; a.f = q->gate; a.h = q->h;
    a.initial = q->initial; a.last = q->last; a.states = q->states;
    a.reset = q->reset; a.lengths = q->lengths; a.maps = (float2 *)workspace;
    a.s_x = q->x_stride; a.s_f = q->gate_stride; a.s_h = q->h_stride;
    a.b_x = q->x_batch_stride; a.b_f = q->gate_batch_stride; a.b_h = q->h_batch_stride;
    a.T = (int)q->steps; a.d = (int)q->d;
    return finish(launch_scan(a, q->type, q->input, q->batch, false, (hipStream_t)stream));
}

extern "C" int qsr_gated_scan_backward(const qsr_gated_scan_backward_args *q, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!q || !scan_sizes_ok(q->batch, q->steps, q->d, q->type)) return QSR_EINVAL;
    if (q->input != QSR_SCAN_COMPLEMENT && q->input != QSR_SCAN_PLAIN) return QSR_EINVAL;
    if (!scan_limits_ok(q->batch, q->steps, q->d)) return QSR_ELIMIT;
    const uintptr_t es = q->type == QSR_TYPE_F32 ? 4 : 2;
    if (q->batch == 0 || (q->steps == 0 && !q->initial_grad)) return QSR_OK;
    if (off(q->last_grad, 4) || off(q->initial_grad, 4) || off(q->lengths, 8)) return QSR_EINVAL;
    if (q->steps > 0 && (!q->h_grad || off(q->h_grad, es) || !q->x || off(q->x, es) || !q->gate || off(q->gate, es) || !q->states ||
                         off(q->states, 4) || !q->x_grad || off(q->x_grad, es) || !q->gate_grad || off(q->gate_grad, es)))
        return QSR_EINVAL;
    if (!strides_ok(q->batch, q->steps, q->d, q->x_batch_stride, q->x_stride, false) ||
        !strides_ok(q->batch, q->steps, q->d, q->gate_batch_stride, q->gate_stride, false) ||
        !strides_ok(q->batch, q->steps, q->d, q->h_grad_batch_stride, q->h_grad_stride, false) ||
        !strides_ok(q->batch, q->steps, q->d, q->x_grad_batch_stride, q->x_grad_stride, true) ||
        !strides_ok(q->batch, q->steps, q->d, q->gate_grad_batch_stride, q->gate_grad_stride, true))
        return QSR_EINVAL;
    size_t need = 0;
    const int rc = qsr_gated_scan_workspace_bytes(q->batch, q->steps, q->d, q->type, &need);
    if (rc != QSR_OK) return rc;
    if (need > 0 && (!workspace || off(workspace, 8))) return QSR_EINVAL;
    if (workspace_bytes < need) return QSR_ENOMEM;
    ScanArgs a{};
    a.x = q->x; a.f = q->gate; a.dh = q->h_grad; a.dx = q->x_grad; a.df = q->gate_grad;
    a.initial = q->last_grad; a.last = q->initial_grad; a.states = (float *)q->states;
    a.reset = q->reset; a.lengths = q->lengths; a.maps = (float2 *)workspace;
    a.s_x = q->x_stride; a.s_f = q->gate_stride; a.s_dh = q->h_grad_stride; a.s_dx = q->x_grad_stride; a.s_df = q->gate_grad_stride;
    a.b_x = q->x_batch_stride; a.b_f = q->gate_batch_stride; a.b_dh = q->h_grad_batch_stride;
    a.b_dx = q->x_grad_batch_stride; a.b_df = q->gate_grad_batch_stride;
    a.T = (int)q->steps; a.d = (int)q->d;
    return finish(launch_scan(a, q->type, q->input, q->batch, true, (hipStream_t)stream));
}
