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
// Backward, h is not read but made again from the states kept at every STEPS-th step in fp32: 1/8 of the reads of h in bf16, 1/16 in fp32, and
// nothing of h's rounding in the gradients.
// A reset cuts a map off from what was before: A = -1 stands for that (A is never negative), so that an infinity or a NaN ends there too.
// Without one a channel that has met an infinity stays infinite or becomes NaN (a map whose A is too small for a float makes NaN of it).
// All arithmetic is fp32.
// Rows are addressed as buffers (what is the same for a wavefront stays in scalar registers: forward a fifth fewer vector instructions than with
// pointers, 85 -> 76 us below).  Bound by memory at 64 x 1024 steps of 1024 in bf16: forward 74 us, 5.7 TB/s, backward 150 us, 4.6 TB/s with one
// workgroup of eight wavefronts to a compute unit (190 registers a lane; at 128 they go to memory and back, 230 us).  32768 steps of 2048 on
// 512 workgroups: maps 44 us, 6.0 TB/s, and 65 us; 2 x 16384 of 768 19 + 33 us, backward 18 + 49.  fp32, 13 sequences of up to 1001
// steps of 1003: 26 and 38 us, from memory 37 and 49, the time of the longest one: all of 1001 steps take 41 and 52, with 1024 channels, whose
// rows are whole lines, 35 and 49 (208 workgroups, one to a compute unit, whose tiles follow each other).  Four single steps of 2048: 3 us, latency.
// What the second read costs could be saved by workgroups that wait for each other's maps while they hold their steps in registers; that
// was not tried.  Thirds and quarters of the sequence at a time, so that the second read is from the last-level cache, are slower than the
// whole (32768 steps of 2048 131 us, 141 and 152).
#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "qsr_internal.h"
#include "row_io.h"
#include "tile_grid.h"

namespace qsr {

constexpr int STEPS = QSR_SCAN_STEPS;
constexpr int WAVES = 8, MANY_WAVES = 16;      // wavefronts to a workgroup, where sequences have steps for as many

struct ScanArgs {
    const void *x, *f, *dh;
    void *h, *dx, *df;
    const float *initial;                      // or, backward, the gradient of the last state
    float *last;                               // or, backward, the gradient of the initial state
    float *states;
    const uint8_t *reset;
    const int64_t *lengths;
    float2 *maps;                              // [B][parts + 1][d]: forward, the initial state, then the maps of all parts but the last
    long long b_x, b_f, b_dh, b_h, b_dx, b_df; // from sequence to sequence
    int s_x, s_f, s_dh, s_h, s_dx, s_df;       // and from step to step, in bytes
    long long tiles;
    int T, d, groups, parts, part_len;
    bool near;                                 // neighbouring channels on one die
};

// exp(-x) for 0 <= x.  In fp32 what the argument to the base 2 loses to rounding, x units of the result, is put back; beside a gate in bf16,
// whose own rounding is 2^-9 of it, that is nothing.
template <typename T> __device__ __forceinline__ float exp_minus(float x)
{
    constexpr float L = 1.44269504f, L_REST = 1.92596303e-8f, LN2 = 0.693147181f;         // log2(e) = L + L_REST
    if constexpr (sizeof(T) == 2) return __builtin_amdgcn_exp2f(-L * x);
    const float y = __builtin_elementwise_minimum(x, 200.f), t = L * y, rest = fmaf(L_REST, y, fmaf(L, y, -t)), e = __builtin_amdgcn_exp2f(-t);
    return fmaf(e, -LN2 * rest, e);
}
// The larger and the smaller one of a = sigmoid(f) and c = 1 - a.  The smaller one has the relative precision of the exponential, and the
// larger one is 1 less it, with a rounding of half a unit: a state remembers thousands of steps through gates near 1, and an error of the
// reciprocal there would add up.  a is the larger one where f has no sign.  Infinite gates are exact, a NaN stays.
template <typename T> __device__ __forceinline__ void gates(float f, float &big, float &small)
{
    const float e = exp_minus<T>(fabsf(f));
    small = e * __builtin_amdgcn_rcpf(1.f + e);
    big = 1.f - small;
}
template <typename T> __device__ __forceinline__ void gates_of(float f, float &a, float &c)
{
    float big, small;
    gates<T>(f, big, small);               // (a NaN in both)
    a = f >= 0.f ? big : small;
    c = f >= 0.f ? small : big;
}
// Both in one number: the smaller one, with a's place in the sign
template <typename T> __device__ __forceinline__ float gates_in_one(float f) { float big, small; gates<T>(f, big, small); return copysignf(small, f); }
__device__ __forceinline__ float a_of(float v) { return __float_as_int(v) >= 0 ? 1.f - v : -v; }
__device__ __forceinline__ float c_of(float v) { return __float_as_int(v) >= 0 ? v : 1.f + v; }

// A map (A, H) behind h
__device__ __forceinline__ float behind_map(float A, float H, float h) { return A < 0.f ? H : fmaf(A, h, H); }

// A lane's V channels in a word (V = 1 in bf16: half of one)
template <typename T, int V> __device__ __forceinline__ float channel(uint32_t w, int u)
{
    if constexpr (sizeof(T) == 4) return __uint_as_float(w);
    else return __uint_as_float(u == 0 ? w << 16 : w & 0xffff0000u);
}
template <typename T, int V> __device__ __forceinline__ uint32_t word_of(const float (&v)[V])
{
    if constexpr (sizeof(T) == 4) return __float_as_uint(v[0]);
    else {
        typedef bf16_t Two __attribute__((ext_vector_type(2)));
        const Two two = {(bf16_t)v[0], (bf16_t)v[V - 1]};
        return __builtin_bit_cast(uint32_t, two);
    }
}

// Rows of a sequence as a buffer: what is the same for a wavefront (where the rows are, how far apart) stays out of its lanes' registers
// and instructions.  2^31 bytes from a tile's first row on; an offset of NOWHERE is outside, and its store is dropped.
constexpr uint32_t NOWHERE = 0x80000000u;
typedef __amdgpu_buffer_rsrc_t Rows;
__device__ __forceinline__ Rows rows_at(const void *base, long long seq, int t, int step)
{
    return __builtin_amdgcn_make_buffer_rsrc((char *)const_cast<void *>(base) + seq + (long long)t * step, 0, NOWHERE, 0x00020000);
}
template <typename T, int V> __device__ __forceinline__ uint32_t load_word(Rows r, uint32_t at, int row)
{
    if constexpr (V * sizeof(T) == 2) return __builtin_amdgcn_raw_buffer_load_b16(r, (int)at, row, 0);
    else return __builtin_amdgcn_raw_buffer_load_b32(r, (int)at, row, 0);
}
// The first n of STEPS rows; zeros for the others
template <typename T, int V>
__device__ __forceinline__ void load_rows(Rows r, uint32_t at, int step, int n, uint32_t (&w)[STEPS])
{
    if (n >= STEPS) {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) w[s] = load_word<T, V>(r, at, s * step);
    } else {
#pragma unroll
        for (int s = 0; s < STEPS; ++s) {
            w[s] = 0;
            if (s < n) w[s] = load_word<T, V>(r, at, s * step);
        }
    }
}

// A lane's place: V channels from `at`, of which the first `skip` are another lane's (V: all of them)
template <typename T, int V> struct Place {
    int b, part, at, skip, len;
    uint32_t in, out, half;                    // offsets in a row: for loads, for stores of all V channels, and of the last one alone
    bool halves;                               // some lane of the wavefront has that
    __device__ __forceinline__ bool find(const ScanArgs &a, int lane, int parts)
    {
        long long id = blockIdx.x + (long long)blockIdx.y * gridDim.x;
        if (a.near) {                          // workgroups go to the eight dies in turn
            const long long each = (a.tiles + 7) / 8, nth = id / 8;
            id = nth < each ? id % 8 * each + nth : a.tiles;
        }
        if (id >= a.tiles) return false;
        const long long seq = id / a.groups;
        const int first = ((int)(id - seq * a.groups) * 64 + lane) * V;
        b = (int)(seq / parts);
        part = (int)(seq - (long long)b * parts);
        at = min(first, a.d - V);
        skip = min(first - at, V);
        in = (uint32_t)at * (uint32_t)sizeof(T);
        out = skip == 0 ? in : NOWHERE;
        half = skip == 1 && V == 2 ? in + (uint32_t)sizeof(T) : NOWHERE;
        halves = V == 2 && __ballot(skip == 1) != 0;
        len = a.T;
        if (a.lengths != nullptr) {
            const long long n = a.lengths[b];
            len = (int)(n < 0 ? 0 : n > a.T ? a.T : n);
        }
        return true;
    }
    // STREAM: lines that are written as a whole and need not stay
    template <bool STREAM> __device__ __forceinline__ void store(Rows r, int row, const float (&v)[V]) const
    {
        constexpr int NT = STREAM ? 2 : 0;
        const uint32_t w = word_of<T, V>(v);
        if constexpr (V * sizeof(T) == 2) __builtin_amdgcn_raw_buffer_store_b16((uint16_t)w, r, (int)out, row, NT);
        else {
            __builtin_amdgcn_raw_buffer_store_b32(w, r, (int)out, row, NT);
            if (V == 2 && halves) __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(w >> 16), r, (int)half, row, NT);
        }
    }
    // fp32 numbers of one row of d
    __device__ __forceinline__ void store_floats(float *row, const float (&v)[V]) const
    {
#pragma unroll
        for (int u = 0; u < V; ++u)
            if (u >= skip) row[at + u] = v[u];
    }
};

// The marks of steps t .. t + n - 1, a bit each
__device__ __forceinline__ uint32_t marks(const ScanArgs &a, int b, int t, int n, int lane)
{
    if (a.reset == nullptr || n <= 0) return 0;
    const uint8_t m = a.reset[(long long)b * a.T + t + min(lane, n - 1)];
    return (uint32_t)__ballot(m != 0 && lane < n);
}

// f(true) where a tile ends early or has marks, f(false) where every step is as the others
template <typename F> __device__ __forceinline__ void by_tile(bool plain, F f)
{
    if (plain) f(std::integral_constant<bool, false>());
    else f(std::integral_constant<bool, true>());
}

// Behind the `count` maps first, first + step, ... of parts: a wavefront joins a run of them, and all of them the wavefronts' through `words`
template <int V, int W>
__device__ __forceinline__ void behind_parts(const float2 *m, long long d, int first, int step, int count, int wave, int lane, float2 (&words)[W][V][64],
                                             float (&carry)[V])
{
    const int each = (count + W - 1) / W, from = min(count, wave * each), end = min(count, from + each);
    float A[V], H[V];
#pragma unroll
    for (int u = 0; u < V; ++u) { A[u] = 1.f; H[u] = 0.f; }
#pragma unroll 8
    for (int i = from; i < end; ++i)
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const float2 f = m[(long long)(first + i * step) * d + u];
            H[u] = behind_map(f.x, f.y, H[u]);
            A[u] = f.x < 0.f || A[u] < 0.f ? -1.f : A[u] * f.x;
        }
#pragma unroll
    for (int u = 0; u < V; ++u) words[wave][u][lane] = make_float2(A[u], H[u]);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < W; ++w)
#pragma unroll
        for (int u = 0; u < V; ++u) { const float2 f = words[w][u][lane]; carry[u] = behind_map(f.x, f.y, carry[u]); }
}

// Forward, W wavefronts to a workgroup
template <typename T, int V, int W, bool COMP, bool STREAM>
__global__ __launch_bounds__(64 * W, 4) void scan_kernel(ScanArgs a)
{
    __shared__ float2 maps[2][W][V][64];
    const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Place<T, V> q;
    if (!q.find(a, lane, a.parts)) return;
    float carry[V];
    if (a.parts > 1) {
#pragma unroll
        for (int u = 0; u < V; ++u) carry[u] = 0.f;
        behind_parts<V, W>(a.maps + ((long long)q.b * (a.parts + 1)) * a.d + q.at, a.d, 0, 1, q.part + 1, wave, lane, maps[1], carry);
    } else {
#pragma unroll
        for (int u = 0; u < V; ++u) {
            carry[u] = a.initial != nullptr ? a.initial[(long long)q.b * a.d + q.at + u] : 0.f;
            asm volatile("" : "+v"(carry[u]));             // here before the first barrier: `last` may be the same memory
        }
    }
    const int begin = q.part * a.part_len, end = min(a.T, begin + a.part_len);
    uint32_t rx[STEPS], rf[STEPS], bits = 0;
    auto load = [&](int t0) {
        const int t = t0 + wave * STEPS, n = min(q.len - t, STEPS);
        load_rows<T, V>(rows_at(a.x, q.b * a.b_x, t, a.s_x), q.in, a.s_x, n, rx);
        load_rows<T, V>(rows_at(a.f, q.b * a.b_f, t, a.s_f), q.in, a.s_f, n, rf);
        bits = marks(a, q.b, t, n, lane);
    };
    int turn = 0;
#pragma unroll 1
    for (int t0 = begin; t0 < end; t0 += W * STEPS, turn ^= 1) {
        const int t = t0 + wave * STEPS, n = min(q.len - t, STEPS);
        load(t0);
        const uint32_t cut = bits;
        float ga[STEPS][V], gb[STEPS][V], A[V], H[V], h[V];
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int u = 0; u < V; ++u) {
                float c;
                const float x = channel<T, V>(rx[s], u);
                gates_of<T>(channel<T, V>(rf[s], u), ga[s][u], c);
                gb[s][u] = COMP ? c * x : x;
            }
        if (n < STEPS) {                       // behind the end the state stays
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int u = 0; u < V; ++u)
                    if (s >= n) { ga[s][u] = 1.f; gb[s][u] = 0.f; }
        }
#pragma unroll
        for (int u = 0; u < V; ++u) { A[u] = 1.f; H[u] = 0.f; }
        if (W > 1) {
            by_tile(cut == 0, [&](auto marked) {
#pragma unroll
                for (int s = 0; s < STEPS; ++s)
#pragma unroll
                    for (int u = 0; u < V; ++u) {
                        if (marked() && (cut >> s & 1)) H[u] = 0.f;
                        H[u] = fmaf(ga[s][u], H[u], gb[s][u]);
                        A[u] *= ga[s][u];
                    }
            });
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
        if (t < end) {
            if (a.states != nullptr) q.store_floats(a.states + ((long long)q.b * ((a.T + STEPS - 1) / STEPS) + t / STEPS) * a.d, h);
            const Rows rh = rows_at(a.h, q.b * a.b_h, t, a.s_h);
            by_tile(cut == 0 && n >= STEPS, [&](auto marked) {
#pragma unroll
                for (int s = 0; s < STEPS; ++s) {
                    float y[V];
#pragma unroll
                    for (int u = 0; u < V; ++u) {
                        if (marked() && (cut >> s & 1)) h[u] = 0.f;
                        h[u] = fmaf(ga[s][u], h[u], gb[s][u]);
                        y[u] = !marked() || s < n ? h[u] : 0.f;
                    }
                    if (!marked() || t + s < end) q.template store<STREAM>(rh, s * a.s_h, y);
                }
            });
        }
        if (W == 1)
#pragma unroll
            for (int u = 0; u < V; ++u) carry[u] = h[u];
    }
    if (a.last != nullptr && q.part == a.parts - 1 && wave == 0) q.store_floats(a.last + (long long)q.b * a.d, carry);
}

// One step of every sequence: a thread has V channels of one.  Of a sequence without steps x and gate are not read, as with more steps.
template <typename T, int V, bool COMP>
__global__ __launch_bounds__(256) void scan_step_kernel(ScanArgs a)
{
    const long long id = (blockIdx.x + (long long)blockIdx.y * gridDim.x) * 256 + threadIdx.x, each = (a.d + V - 1) / V;
    if (id >= a.tiles) return;
    const long long b = id / each;
    const int first = (int)(id - b * each) * V, at = min(first, a.d - V), skip = first - at;
    typedef typename Wide<T, V>::vec Vec;
    const bool live = a.lengths == nullptr || a.lengths[b] > 0, cut = a.reset != nullptr && a.reset[b] != 0;
    Vec x = (Vec)((T)0.f), f = x;
    if (live) {
        x = *(const Vec *)((const char *)a.x + b * a.b_x + at * (long long)sizeof(T));
        f = *(const Vec *)((const char *)a.f + b * a.b_f + at * (long long)sizeof(T));
    }
    float h[V], y[V];
#pragma unroll
    for (int u = 0; u < V; ++u) h[u] = a.initial != nullptr ? a.initial[b * a.d + at + u] : 0.f;
    T *const to = (T *)((char *)a.h + b * a.b_h) + at;
#pragma unroll
    for (int u = 0; u < V; ++u) {
        if (u < skip) continue;
        if (a.states != nullptr) a.states[b * a.d + at + u] = h[u];
        float ga, gc;
        gates_of<T>((float)f[u], ga, gc);
        const float v = (float)x[u];
        y[u] = fmaf(ga, cut ? 0.f : h[u], COMP ? gc * v : v);
        to[u] = (T)(live ? y[u] : 0.f);
        if (a.last != nullptr) a.last[b * a.d + at + u] = live ? y[u] : h[u];
    }
}

// The maps of parts: a wavefront goes through a run of its part's steps, from its end.  Forward: all parts but the last, and the initial
// state.  Backward: e before a part from e behind it, all parts but the first; COMP makes no difference.
template <typename T, int V, bool COMP, bool BACK>
__global__ __launch_bounds__(64 * WAVES) void scan_maps_kernel(ScanArgs a)
{
    __shared__ float2 maps[WAVES][V][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Place<T, V> q;
    if (!q.find(a, lane, a.parts - 1)) return;
    const int part = BACK ? q.part + 1 : q.part;
    const void *const vx = BACK ? a.dh : a.x;
    const long long b_x = q.b * (BACK ? a.b_dh : a.b_x);
    const int s_x = BACK ? a.s_dh : a.s_x;
    const int each = a.part_len / WAVES, begin = part * a.part_len + wave * each, end = min(a.T, begin + each);
    const int trips = begin < end ? (end - begin + STEPS - 1) / STEPS : 0;
    uint32_t rx[STEPS], rf[STEPS], bits = 0, any = 0;
    // Forward, a part's first steps are read last: the launch behind begins with them, and finds them in the last-level cache
    auto start_of = [&](int i) { return begin + (BACK ? i : trips - 1 - i) * STEPS; };
    auto load = [&](int t) {
        const int n = min(q.len - t, STEPS);
        load_rows<T, V>(rows_at(vx, b_x, t, s_x), q.in, s_x, n, rx);
        load_rows<T, V>(rows_at(a.f, q.b * a.b_f, t, a.s_f), q.in, a.s_f, n, rf);
        bits = marks(a, q.b, t, n, lane);
    };
    float A[V], H[V];
#pragma unroll
    for (int u = 0; u < V; ++u) { A[u] = 1.f; H[u] = 0.f; }
#pragma unroll 1
    for (int i = 0; i < trips; ++i) {
        const int n = min(q.len - start_of(i), STEPS);
        load(start_of(i));
        const uint32_t cut = bits;
        float ga[STEPS][V], gb[STEPS][V], P[V], E[V];
#pragma unroll
        for (int s = 0; s < STEPS; ++s)
#pragma unroll
            for (int u = 0; u < V; ++u) {
                float c;
                const float x = channel<T, V>(rx[s], u);
                gates_of<T>(channel<T, V>(rf[s], u), ga[s][u], c);
                gb[s][u] = BACK || !COMP ? x : c * x;
            }
        if (n < STEPS) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int u = 0; u < V; ++u)
                    if (s >= n) { ga[s][u] = 1.f; gb[s][u] = 0.f; }
        }
#pragma unroll
        for (int u = 0; u < V; ++u) { P[u] = 1.f; E[u] = 0.f; }
        // the map of these steps
        by_tile(cut == 0, [&](auto marked) {
#pragma unroll
            for (int o = 0; o < STEPS; ++o) {
                const int s = BACK ? STEPS - 1 - o : o;
#pragma unroll
                for (int u = 0; u < V; ++u) {
                    if (!BACK && marked() && (cut >> s & 1)) E[u] = 0.f;
                    E[u] = BACK ? ga[s][u] * (gb[s][u] + E[u]) : fmaf(ga[s][u], E[u], gb[s][u]);
                    if (BACK && marked() && (cut >> s & 1)) E[u] = 0.f;
                    P[u] *= ga[s][u];
                }
            }
        });
        // in front of (forward, from the end) or behind (backward, from the start, where later steps come first) those before
#pragma unroll
        for (int u = 0; u < V; ++u) {
            H[u] = any ? H[u] : fmaf(A[u], E[u], H[u]);
            A[u] *= P[u];
        }
        any |= cut;
    }
#pragma unroll
    for (int u = 0; u < V; ++u) maps[wave][u][lane] = make_float2(any ? -1.f : A[u], H[u]);
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int u = 0; u < V; ++u) { A[u] = 1.f; H[u] = 0.f; }
#pragma unroll
    for (int i = 0; i < WAVES; ++i)
#pragma unroll
        for (int u = 0; u < V; ++u) {
            const float2 m = maps[BACK ? WAVES - 1 - i : i][u][lane];
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
template <typename T, int V, int W, bool COMP, bool STREAM>
__global__ __launch_bounds__(64 * W, 2) void scan_back_kernel(ScanArgs a)
{
    __shared__ float2 maps[2][W][V][64];
    const int lane = threadIdx.x & 63, wave = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Place<T, V> q;
    if (!q.find(a, lane, a.parts)) return;
    float carry[V];
#pragma unroll
    for (int u = 0; u < V; ++u) carry[u] = a.initial != nullptr ? a.initial[(long long)q.b * a.d + q.at + u] : 0.f;
    if (a.parts > 1)
        behind_parts<V, W>(a.maps + ((long long)q.b * (a.parts + 1)) * a.d + q.at, a.d, a.parts - 1, -1, a.parts - 1 - q.part, wave, lane, maps[1], carry);
    const int begin = q.part * a.part_len, end = min(a.T, begin + a.part_len);
    const int trips = begin < end ? (end - begin + W * STEPS - 1) / (W * STEPS) : 0;
    uint32_t rx[STEPS], rf[STEPS], rg[STEPS], bits = 0;
    float rs[V] = {};
    auto load = [&](int t0) {
        const int t = t0 + wave * STEPS, n = min(q.len - t, STEPS);
        load_rows<T, V>(rows_at(a.f, q.b * a.b_f, t, a.s_f), q.in, a.s_f, n, rf);
        load_rows<T, V>(rows_at(a.x, q.b * a.b_x, t, a.s_x), q.in, a.s_x, n, rx);
        load_rows<T, V>(rows_at(a.dh, q.b * a.b_dh, t, a.s_dh), q.in, a.s_dh, n, rg);
        if (n > 0) {
            const float *const row = a.states + ((long long)q.b * ((a.T + STEPS - 1) / STEPS) + t / STEPS) * a.d + q.at;
#pragma unroll
            for (int u = 0; u < V; ++u) rs[u] = row[u];
        }
        bits = marks(a, q.b, t, n, lane);
    };
    if (trips > 0) load(begin + (trips - 1) * W * STEPS);
    int turn = 0;
#pragma unroll 1
    for (int i = trips - 1; i >= 0; --i, turn ^= 1) {
        const int t = begin + i * W * STEPS + wave * STEPS, n = min(q.len - t, STEPS);
        const uint32_t cut = bits;
        uint32_t x[STEPS], g[STEPS];
        float v[STEPS][V], before[STEPS][V], h[V], e[V];
#pragma unroll
        for (int u = 0; u < V; ++u) h[u] = rs[u];
        // the gates, and the states before each step
        by_tile(cut == 0, [&](auto marked) {
#pragma unroll
            for (int s = 0; s < STEPS; ++s) {
                x[s] = rx[s];
                g[s] = rg[s];
#pragma unroll
                for (int u = 0; u < V; ++u) {
                    v[s][u] = gates_in_one<T>(channel<T, V>(rf[s], u));
                    if (marked() && (cut >> s & 1)) h[u] = 0.f;
                    before[s][u] = h[u];
                    const float y = channel<T, V>(x[s], u);
                    h[u] = fmaf(a_of(v[s][u]), h[u], COMP ? c_of(v[s][u]) * y : y);
                }
            }
        });
        if (i > 0) load(begin + (i - 1) * W * STEPS);
        if (n < STEPS) {                       // behind the end: a = 1, and no gradients (g is 0)
#pragma unroll
            for (int s = 0; s < STEPS; ++s)
#pragma unroll
                for (int u = 0; u < V; ++u)
                    if (s >= n) v[s][u] = 0.f;
        }
        if (W > 1) {
            float A[V], H[V];
#pragma unroll
            for (int u = 0; u < V; ++u) { A[u] = 1.f; H[u] = 0.f; }
            by_tile(cut == 0, [&](auto marked) {
#pragma unroll
                for (int s = STEPS - 1; s >= 0; --s)
#pragma unroll
                    for (int u = 0; u < V; ++u) {
                        const float ga = a_of(v[s][u]);
                        H[u] = ga * (H[u] + channel<T, V>(g[s], u));
                        if (marked() && (cut >> s & 1)) H[u] = 0.f;
                        A[u] *= ga;
                    }
            });
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
        if (t < end) {
            const Rows rdx = rows_at(a.dx, q.b * a.b_dx, t, a.s_dx), rdf = rows_at(a.df, q.b * a.b_df, t, a.s_df);
            by_tile(cut == 0 && n >= STEPS, [&](auto marked) {
#pragma unroll
                for (int s = STEPS - 1; s >= 0; --s) {
                    float dx[V], df[V];
#pragma unroll
                    for (int u = 0; u < V; ++u) {
                        const float ga = a_of(v[s][u]), gc = c_of(v[s][u]), grad = channel<T, V>(g[s], u) + e[u];
                        dx[u] = COMP ? gc * grad : grad;
                        const float down = ga * grad;
                        df[u] = down * gc * (COMP ? before[s][u] - channel<T, V>(x[s], u) : before[s][u]);
                        e[u] = marked() && (cut >> s & 1) ? 0.f : down;
                        if (marked() && s >= n) { dx[u] = df[u] = 0.f; }
                    }
                    if (!marked() || t + s < end) {
                        q.template store<STREAM>(rdx, s * a.s_dx, dx);
                        q.template store<STREAM>(rdf, s * a.s_df, df);
                    }
                }
            });
        }
        if (W == 1)
#pragma unroll
            for (int u = 0; u < V; ++u) carry[u] = e[u];
    }
    if (a.last != nullptr && q.part == 0 && wave == 0) q.store_floats(a.last + (long long)q.b * a.d, carry);
}

// ---------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------
// Channels of a lane: four bytes of them, or one where a wavefront has them all, where there are not as many workgroups as compute units with all
// tiles apart, and where enough workgroups take at most half as many rounds again with one, which are shorter.  us with one / two, forward and
// backward: 300 x 500 steps of 64 channels 24.8 / 31.1 and 37.9 / 49.6; 8 x 512 of 512 9.3 / 11.6 and 10.6 / 13.5; rounds 1 and 1: 16 x 1024 of 1024
// 29.3 / 35.4 and 43.4 / 49.8, 13 x 1001 of 1003 27.3 / 37.9 and 43.3 / 53.2, 64 x 1000 of 160 25.3 / 33.1 and 38.7 / 44.0; 2 and 2: 100 x 1000 of 320
// 51.5 / 63.3 and 80.8 / 97.5; 3 and 2: 64 x 500 of 700 37.0 / 42.0 and 67.7 / 68.7; but 2 and 1: 24 x 700 of 1024 35.1 / 29.6 and 56.2 / 44.7; too few
// workgroups: 8 x 1024 of 1024 24.0 / 19.4 and 32.3 / 26.7.
static int scan_channels(int type, long long B, long long T, long long d)
{
    if (type != QSR_TYPE_BF16 || d <= 64) return 1;
    if (T < 2) return 2;
    const long long ones = B * ((d + 63) / 64), twos = B * ((d + 127) / 128), tiles = ones * ((T + WAVES * STEPS - 1) / (WAVES * STEPS));
    return tiles <= 256 || (twos >= 96 && 2 * ((ones + 255) / 256) <= 3 * ((twos + 255) / 256)) ? 1 : 2;
}

// A workgroup has all steps of 64 lanes' channels, or a part of them.  Parts cost a second read of two of three to five arrays and a
// launch; they are taken where workgroups are too few otherwise.
// What a trip of a workgroup costs, in tenths of its time: 10 without parts and 14 with them, a part's start 3, the second launch 8; the maps of
// the parts before, which each part joins, count a little.  Workgroups run 512 at a time forward and 256 backward with two channels a lane; with
// one, more of them fit (56 registers of a lane forward, 128 backward in "plain"), which the rule does not count.  us without parts / with them,
// bf16 and two channels of a lane, forward and backward: 8 x 512 steps of 512 channels 17.0 / 12.5 and 26.5 / 14.9; 9 x 7000 of 700 243 / 100 and
// 356 / 150; 32768 steps of 2048 942 / 111, of 64 948 / 12.4 and 1513 / 14.1.  With 128 workgroups and more forward and 192 backward the second
// read costs what is won (16 x 1024 steps of 1024, forward: 37 with parts, 32.3 with sixteen wavefronts to a workgroup, which fill the chip's SIMDs
// up to 512 workgroups; from there on eight are faster, 76 against 80 at 64 x 1024 steps of 1024).  Short sequences have no more wavefronts than
// they can use, since a workgroup that waits for a place waits for idle ones too: us with / with eight or sixteen, bf16, 1000 x 30 steps of 512 23
// / 48 and 38 / 110, 40 x 30 of 1000 5.0 / 15.5 and 6.5 / 15.6, 40 x 100 of 1024 8.4 / 15.8 forward.  Sixteen that have all steps at once are
// faster than parts, 7.1 against 7.8 for 4 x 250 of 1000; with two trips they are not, 11.2 against 9.4 for 512 of 4096.
struct ScanPlan { int channels, waves, parts, part_len; long long groups; };
static ScanPlan scan_plan(long long B, long long T, long long d, int type, bool back)
{
    ScanPlan p;
    const int V = p.channels = scan_channels(type, B, T, d);
    p.groups = (d + 64 * V - 1) / (64 * V);
    p.parts = 1;
    const long long have = B * p.groups, slots = back ? 256 : 512, few = back ? 192 : 128;
    const bool many = !back && T > WAVES * STEPS && have < 512 && (have >= few || T <= MANY_WAVES * STEPS);
    p.waves = T <= STEPS ? 1 : T <= 2 * STEPS ? 2 : T <= 4 * STEPS ? 4 : many ? MANY_WAVES : WAVES;
    const long long trip = (long long)p.waves * STEPS, trips = (T + trip - 1) / trip;
    long long each = trips, best = 10 * trips;
    for (int round = 1; have < few && p.waves == WAVES && trips > 1 && round <= 4; ++round) {
        const long long most = round * slots / have;           // more parts in as many rounds cost less
        if (most < 2) continue;
        const long long e = (trips + most - 1) / most, n = (trips + e - 1) / e, cost = (have * n + slots - 1) / slots * (14 * e + 3) + n / 32 + 8;
        if (n > 1 && cost < best) { best = cost; each = e; }
    }
    if (trips > 0) p.parts = (int)((trips + each - 1) / each);
    p.part_len = (int)(each * trip);
    return p;
}

template <typename T, int V, bool COMP, bool STREAM>
static void launch_back(const ScanArgs &a, const ScanPlan &p, dim3 grid, hipStream_t s)
{
    if (p.waves == 1) scan_back_kernel<T, V, 1, COMP, STREAM><<<grid, 64, 0, s>>>(a);
    else if (p.waves == 2) scan_back_kernel<T, V, 2, COMP, STREAM><<<grid, 128, 0, s>>>(a);
    else if (p.waves == 4) scan_back_kernel<T, V, 4, COMP, STREAM><<<grid, 256, 0, s>>>(a);
    else scan_back_kernel<T, V, WAVES, COMP, STREAM><<<grid, 64 * WAVES, 0, s>>>(a);
}
template <typename T, int V, bool COMP, bool STREAM>
static void launch_forward(const ScanArgs &a, const ScanPlan &p, dim3 grid, hipStream_t s)
{
    if (p.waves == 1) scan_kernel<T, V, 1, COMP, STREAM><<<grid, 64, 0, s>>>(a);
    else if (p.waves == 2) scan_kernel<T, V, 2, COMP, STREAM><<<grid, 128, 0, s>>>(a);
    else if (p.waves == 4) scan_kernel<T, V, 4, COMP, STREAM><<<grid, 256, 0, s>>>(a);
    else if (p.waves == WAVES) scan_kernel<T, V, WAVES, COMP, STREAM><<<grid, 64 * WAVES, 0, s>>>(a);
    else scan_kernel<T, V, MANY_WAVES, COMP, STREAM><<<grid, 64 * MANY_WAVES, 0, s>>>(a);
}
// Whole lines to a wavefront's part of a row.  Then what is written streams past the caches.  Otherwise neighbouring parts share lines, which
// are read and written as a whole where both parts are on one die, in its cache; there, what is written does not stream, but for
// forward passes with lengths.  us with / without neighbours on one die, forward and backward: fp32, 2 x 4000 steps of 3001 100 / 116 and
// 144 / 170, 13 x 1001 of 1003 39 / 48 and 62 / 77, with lengths 40 / 43 and 54 / 68; 64 x 1024 of 1024 in bf16, whole lines, 79 / 76 and
// 163 / 152.  Streamed / not: whole lines as the last 76 / 90 and 151 / 156; the fp32 ones 41 / 39 and 70 / 62, with lengths 30 / 40 and 58 / 54.
static bool lines(const void *p, long long seq, int step) { return (((uintptr_t)p | (uintptr_t)seq | (uintptr_t)step) & 127) == 0; }

template <typename T, int V, bool COMP>
static hipError_t launch_scan(ScanArgs &a, const ScanPlan &p, long long B, bool back, hipStream_t s)
{
    if (a.T == 1 && !back) {
        a.tiles = B * ((a.d + V - 1) / V);
        const TileGrid g = tile_grid((a.tiles + 255) / 256, 256);
        if (g.x == 0) return hipErrorInvalidConfiguration;
        scan_step_kernel<T, V, COMP><<<dim3(g.x, g.y), 256, 0, s>>>(a);
        return hipGetLastError();
    }
    a.groups = (int)p.groups;
    a.parts = p.parts;
    a.part_len = p.part_len;
    if (p.parts > 1) {
        a.tiles = B * (p.parts - 1) * p.groups;
        a.near = !(lines(a.f, a.b_f, a.s_f) && (back ? lines(a.dh, a.b_dh, a.s_dh) : lines(a.x, a.b_x, a.s_x)));
        const TileGrid g = tile_grid((a.tiles + 7) / 8 * 8, 64 * WAVES);
        if (g.x == 0) return hipErrorInvalidConfiguration;
        if (back) scan_maps_kernel<T, V, false, true><<<dim3(g.x, g.y), 64 * WAVES, 0, s>>>(a);
        else scan_maps_kernel<T, V, COMP, false><<<dim3(g.x, g.y), 64 * WAVES, 0, s>>>(a);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const bool in = lines(a.f, a.b_f, a.s_f) && lines(a.x, a.b_x, a.s_x) && (!back || lines(a.dh, a.b_dh, a.s_dh));
    const bool out = back ? lines(a.dx, a.b_dx, a.s_dx) && lines(a.df, a.b_df, a.s_df) : lines(a.h, a.b_h, a.s_h);
    a.near = !(in && out);
    a.tiles = B * p.parts * p.groups;
    const TileGrid g = tile_grid((a.tiles + 7) / 8 * 8, 64 * p.waves);
    if (g.x == 0) return hipErrorInvalidConfiguration;
    const dim3 grid(g.x, g.y);
    if (back) {
        if (out) launch_back<T, V, COMP, true>(a, p, grid, s);
        else launch_back<T, V, COMP, false>(a, p, grid, s);
    } else {
        if (out || a.lengths != nullptr) launch_forward<T, V, COMP, true>(a, p, grid, s);
        else launch_forward<T, V, COMP, false>(a, p, grid, s);
    }
    return hipGetLastError();
}
static hipError_t launch_scan(ScanArgs &a, int type, int input, long long B, bool back, hipStream_t s)
{
    const ScanPlan p = scan_plan(B, a.T, a.d, type, back);
    const bool comp = input == QSR_SCAN_COMPLEMENT;
    if (type == QSR_TYPE_F32) return comp ? launch_scan<float, 1, true>(a, p, B, back, s) : launch_scan<float, 1, false>(a, p, B, back, s);
    if (p.channels == 2) return comp ? launch_scan<bf16_t, 2, true>(a, p, B, back, s) : launch_scan<bf16_t, 2, false>(a, p, B, back, s);
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
constexpr int64_t MOST_STRIDE = 1 << 24;       // elements from step to step: a tile's rows lie within 2^31 bytes
static bool steps_near(int64_t T, std::initializer_list<int64_t> strides)
{
    for (int64_t s : strides)
        if (T > 1 && s > MOST_STRIDE) return false;
    return true;
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
    const int f = scan_plan(batch, steps, d, type, false).parts, b = scan_plan(batch, steps, d, type, true).parts, parts = f > b ? f : b;
    *bytes = parts > 1 ? (size_t)batch * (size_t)(parts + 1) * (size_t)d * sizeof(float2) : 0;
    return QSR_OK;
}

extern "C" int qsr_gated_scan(const qsr_gated_scan_args *q, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!q || !scan_sizes_ok(q->batch, q->steps, q->d, q->type)) return QSR_EINVAL;
    if (q->input != QSR_SCAN_COMPLEMENT && q->input != QSR_SCAN_PLAIN) return QSR_EINVAL;
    if (!scan_limits_ok(q->batch, q->steps, q->d)) return QSR_ELIMIT;
    const int64_t es = q->type == QSR_TYPE_F32 ? 4 : 2;
    if (q->batch == 0 || (q->steps == 0 && !q->last)) return QSR_OK;
    if (off(q->initial, 4) || off(q->last, 4) || off(q->states, 4) || off(q->lengths, 8)) return QSR_EINVAL;
    if (q->steps > 0 && (!q->x || off(q->x, es) || !q->gate || off(q->gate, es) || !q->h || off(q->h, es))) return QSR_EINVAL;
    if (!strides_ok(q->batch, q->steps, q->d, q->x_batch_stride, q->x_stride, false) ||
        !strides_ok(q->batch, q->steps, q->d, q->gate_batch_stride, q->gate_stride, false) ||
        !strides_ok(q->batch, q->steps, q->d, q->h_batch_stride, q->h_stride, true))
        return QSR_EINVAL;
    if (!steps_near(q->steps, {q->x_stride, q->gate_stride, q->h_stride})) return QSR_ELIMIT;
    size_t need = 0;
    const int rc = qsr_gated_scan_workspace_bytes(q->batch, q->steps, q->d, q->type, &need);
    if (rc != QSR_OK) return rc;
    if (need > 0 && (!workspace || off(workspace, 8))) return QSR_EINVAL;
    if (workspace_bytes < need) return QSR_ENOMEM;
    // a workgroup may write its part of `last` before another one has read the same place as another channel's or sequence's initial state
    const uintptr_t first = (uintptr_t)q->initial, last = (uintptr_t)q->last, apart = first < last ? last - first : first - last;
    if (first != 0 && last != 0 && apart != 0 && apart < (uintptr_t)q->batch * (uintptr_t)q->d * 4) return QSR_EINVAL;
    ScanArgs a{};
    a.x = q->x; a.f = q->gate; a.h = q->h;
    a.initial = q->initial; a.last = q->last; a.states = q->states;
    a.reset = q->reset; a.lengths = q->lengths; a.maps = (float2 *)workspace;
    auto step = [&](int64_t n) { return q->steps > 1 ? (int)(n * es) : 0; };               // in bytes
    auto seq = [&](int64_t n) { return q->batch > 1 ? n * es : 0; };
    a.s_x = step(q->x_stride); a.s_f = step(q->gate_stride); a.s_h = step(q->h_stride);
    a.b_x = seq(q->x_batch_stride); a.b_f = seq(q->gate_batch_stride); a.b_h = seq(q->h_batch_stride);
    a.T = (int)q->steps; a.d = (int)q->d;
    return finish(launch_scan(a, q->type, q->input, q->batch, false, (hipStream_t)stream));
}

extern "C" int qsr_gated_scan_backward(const qsr_gated_scan_backward_args *q, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!q || !scan_sizes_ok(q->batch, q->steps, q->d, q->type)) return QSR_EINVAL;
    if (q->input != QSR_SCAN_COMPLEMENT && q->input != QSR_SCAN_PLAIN) return QSR_EINVAL;
    if (!scan_limits_ok(q->batch, q->steps, q->d)) return QSR_ELIMIT;
    const int64_t es = q->type == QSR_TYPE_F32 ? 4 : 2;
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
    if (!steps_near(q->steps, {q->x_stride, q->gate_stride, q->h_grad_stride, q->x_grad_stride, q->gate_grad_stride})) return QSR_ELIMIT;
    size_t need = 0;
    const int rc = qsr_gated_scan_workspace_bytes(q->batch, q->steps, q->d, q->type, &need);
    if (rc != QSR_OK) return rc;
    if (need > 0 && (!workspace || off(workspace, 8))) return QSR_EINVAL;
    if (workspace_bytes < need) return QSR_ENOMEM;
    ScanArgs a{};
    a.x = q->x; a.f = q->gate; a.dh = q->h_grad; a.dx = q->x_grad; a.df = q->gate_grad;
    a.initial = q->last_grad; a.last = q->initial_grad; a.states = (float *)q->states;
    a.reset = q->reset; a.lengths = q->lengths; a.maps = (float2 *)workspace;
    auto step = [&](int64_t n) { return q->steps > 1 ? (int)(n * es) : 0; };
    auto seq = [&](int64_t n) { return q->batch > 1 ? n * es : 0; };
    a.s_x = step(q->x_stride); a.s_f = step(q->gate_stride); a.s_dh = step(q->h_grad_stride);
    a.s_dx = step(q->x_grad_stride); a.s_df = step(q->gate_grad_stride);
    a.b_x = seq(q->x_batch_stride); a.b_f = seq(q->gate_batch_stride); a.b_dh = seq(q->h_grad_batch_stride);
    a.b_dx = seq(q->x_grad_batch_stride); a.b_df = seq(q->gate_grad_batch_stride);
    a.T = (int)q->steps; a.d = (int)q->d;
    return finish(launch_scan(a, q->type, q->input, q->batch, true, (hipStream_t)stream));
}
