// token_logprobs.hip -- log probabilities of given tokens from rows of logits, with the entropy and the best alternatives, and the
// gradient with respect to the logits.
//
//   z = x / T;  lse = log sum_j exp z_j;  logp = z_token - lse;  H = lse - sum_j p_j z_j;  alternatives: the `top` largest z_j - lse,
//   the lower index first where they tie
//   dx_j = 1/T [ a (delta_{j,token} - p_j) - b p_j (log p_j + H) ]   for a = d/dlogp and b = d/dH
// A row that is masked as a whole (all -inf) has lse = logp = -inf, H = 0 and no gradient.  A token outside 0..V-1 stands for none:
// logp = 0 and no gradient from it.
//
// One pass over the logits: every lane keeps the largest logit m it has seen, s = sum 2^t and w = sum t 2^t with t = (x - m) c,
// c = log2 e / T, rescaled where m grows; H = log s - ln 2 w / s.  s and w are double, a trip of logits a term (take): 1 - p of a token
// that is nearly certain is what is left of s beside one.  m starts at the lowest float, not at -inf, so that masked entries
// (t = -inf) are zeros and never NaN.  x - m is taken before the scaling: c x - c m in one product-sum would shift the row by the
// rounding of c m, and a token that is certain would not have logp = H = 0.  The wide loads of a trip are in flight together and
// share one comparison with m.
// Alternatives without a second pass over the row: a lane's largest logit is at hand, and the few lanes that can hold alternatives have
// their logits looked at again, from the caches (find_top).
//
// What bounds it: many rows, the memory, and close behind it the arithmetic (an exponential, at a quarter of the rate, and eight other
// instructions a logit).  8192 bf16 rows of 32768: 100 us, 5.4 TB/s (98 with float sums); 1001 fp32 rows of 50021 with 5 alternatives
// 41 us, 4.9 TB/s (39.5).  Few rows: chains of latencies, 4 bf16 rows of 131072 with 8 alternatives 6.8 us and 5.3 for the join.
#include <cmath>

#include "qsr_internal.h"
#include "row_io.h"

namespace qsr {

constexpr float LOWEST = -3.402823466e38f, LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int LP_MAX_TOP = 64;                 // alternatives: the lanes of a wavefront

// A logit and its place as one number that orders them: the larger logit, then the lower index, is larger.  NaN counts as -inf;
// 0 is smaller than any.
__device__ __forceinline__ uint64_t lp_key(float x, uint32_t index)
{
    x = x == x ? x + 0.f : -INFINITY;          // -0 and 0 are equal
    const uint32_t b = __float_as_uint(x);
    return ((uint64_t)(b ^ ((b >> 31) ? 0xFFFFFFFFu : 0x80000000u)) << 32) | (uint32_t)~index;
}
__device__ __forceinline__ float key_value(uint64_t key)
{
    const uint32_t b = (uint32_t)(key >> 32);
    return __uint_as_float(b ^ ((b >> 31) ? 0x80000000u : 0xFFFFFFFFu));
}
__device__ __forceinline__ uint32_t key_index(uint64_t key) { return ~(uint32_t)key; }
// m: the largest logit (the lowest float at least); s, w: see above
struct Stat { float m; double s, w; };
__device__ __forceinline__ void rescale(Stat &a, float m, float c)
{
    const float d = fmaxf((a.m - m) * c, -1000.f), f = __builtin_amdgcn_exp2f(d);
    a.w = (double)f * fma((double)d, a.s, a.w);
    a.s *= (double)f;
    a.m = m;
}
// A trip's logits, whose sums are one term of the lane's sums in double: beside a token that is nearly certain every other term is less
// than half a unit of s as a float, and one after the other they would all be lost.  s in chains of at most four, so that a trip loses
// little either.  A masked entry's 2^t is 0, and its t 2^t is 0 too and not 0 * -inf (2^-1000 is 0 already).
template <int N>
__device__ __forceinline__ void take(Stat &a, const float *x, float c)
{
    constexpr int CHAINS = N < 4 ? N : 4;
    static_assert(CHAINS == 1 || CHAINS == 4, "");
    float s[CHAINS], w;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const float t = (x[i] - a.m) * c, e = __builtin_amdgcn_exp2f(t), u = fmaxf(t, -1000.f);
        s[i % CHAINS] = i < CHAINS ? e : s[i % CHAINS] + e;
        w = i == 0 ? e * u : fmaf(e, u, w);
    }
    if constexpr (CHAINS == 4) s[0] = (s[0] + s[1]) + (s[2] + s[3]);
    a.s += (double)s[0];
    a.w += (double)w;
}
__device__ __forceinline__ Stat wave_merge(Stat a, float c)
{
    rescale(a, wave_max(a.m), c);
    a.s = wave_sum(a.s);
    a.w = wave_sum(a.w);
    return a;
}
// The wavefronts' sums, one to a lane
template <int W>
__device__ __forceinline__ Stat merge_all(const Stat *p, float c)
{
    const int lane = threadIdx.x & 63;
    Stat a = {LOWEST, 0.0, 0.0};
    if (lane < W) a = p[lane];
    return wave_merge(a, c);
}

struct LpArgs {
    const void *x;
    const int64_t *tokens;
    long long rows, stride;
    int V, top, splits, part;                  // part: elements of a split, whole runs of 16 bytes
    float inv_t;
    float *logp, *entropy, *lse, *stats, *top_logp;
    int32_t *top_id;
    Stat *parts;                               // [rows][splits]
    uint64_t *keys;                            // [rows][splits][top]
};

// What a row's sums come to: ls = log sum e^((x - m)/T).  Log probabilities are taken from x - m: lse alone, as a float, has lost ls
// where the logits are large (a row of masks of the lowest value has p = 1/V like any row of equal logits).  For the same reason
// `stats` keeps m and ls for the backward pass.
struct Done { float m, ls, entropy; bool empty; };
__device__ __forceinline__ Done lp_done(const Stat &st)
{
    const float s = (float)st.s, rest = (float)(st.s - (double)s);             // (rest: where one token is certain, much of log s)
    Done r;
    r.m = st.m;
    r.empty = st.s == 0.0;
    r.ls = r.empty ? -INFINITY : logf(s) + rest / s;
    r.entropy = r.empty ? 0.f : r.ls - LN2 * ((float)st.w / s);
    return r;
}
__device__ __forceinline__ float lp_of(const LpArgs &a, const Done &r, float x)
{
    return r.empty ? -INFINITY : fmaf(x - r.m, a.inv_t, -r.ls);
}
__device__ __forceinline__ void lp_alternative(const LpArgs &a, long long row, int place, uint64_t key, const Done &r)
{
    a.top_logp[row * a.top + place] = lp_of(a, r, key_value(key));
    a.top_id[row * a.top + place] = (int32_t)key_index(key);
}
__device__ __forceinline__ long long lp_token(const LpArgs &a, long long row)
{
    const long long t = a.tokens != nullptr ? a.tokens[row] : -1;
    return t >= 0 && t < a.V ? t : -1;
}
template <typename T>
__device__ __forceinline__ void lp_row(const LpArgs &a, long long row, const Done &r)
{
    if (a.lse != nullptr) a.lse[row] = r.empty ? -INFINITY : fmaf(r.m, a.inv_t, r.ls);
    if (a.stats != nullptr) { a.stats[2 * row] = r.m; a.stats[2 * row + 1] = r.ls; }
    if (a.entropy != nullptr) a.entropy[row] = r.entropy;
    if (a.logp == nullptr) return;
    const long long token = lp_token(a, row);
    a.logp[row] = token < 0 ? 0.f : lp_of(a, r, (float)((const T *)a.x)[row * a.stride + token]);
}

// The runs of a split: `head` elements up to the first 16-byte boundary, whole runs, and what is left.  Lane i takes head element i,
// runs i, i + threads, ..., and element i of the rest, in ascending order.
struct Runs { int head, n, tail; };
template <typename T>
__device__ __forceinline__ Runs runs_of(const T *p, int count)
{
    constexpr int E = wide_of<T>();
    Runs r;
    r.head = min(count, (int)((16 - ((uintptr_t)p & 15)) & 15) / (int)sizeof(T));
    r.n = (count - r.head) / E;
    r.tail = count - r.head - r.n * E;
    return r;
}

// A part of a row in a workgroup's hands: where it begins in the row, its runs, and the LDS words of the search for alternatives
template <typename T> struct Part { const T *p, *body, *rest; int j0, count; Runs q; };
template <int THREADS> struct Search {
    float group[64], bound;                    // the largest logit of each of 64 groups of lanes
    unsigned short owner[THREADS];
    static constexpr int LIST = THREADS > 64 ? 1024 : 256;                     // logits from the bound on that fit
    uint64_t list[LIST], best[LP_MAX_TOP];
    int owners, listed;
};
template <int G> __device__ __forceinline__ float group_most(float v)
{
    if (G >= 2) v = fmaxf(v, row_step<0>(v));
    if (G >= 4) v = fmaxf(v, row_step<1>(v));
    if (G >= 8) v = fmaxf(v, row_step<2>(v));
    return v;
}

// The top-th largest of 64 numbers, by taking the largest away until that many are gone; for many by counting how many are larger.
__device__ __forceinline__ float top_bound(const float *group, int top)
{
    float v = group[threadIdx.x & 63];
    if (top <= 12) {
        for (int gone = 0;;) {
            const float most = wave_max(v);
            const bool is = v == most;
            gone += __popcll(__ballot(is));
            if (gone >= top || most == -INFINITY) return most;
            v = is ? -INFINITY : v;
        }
    }
    int above = 0;
    for (int i = 0; i < 64; ++i) above += group[i] > v ? 1 : 0;
    return -wave_max(above < top ? -v : -INFINITY);
}

// The `top` largest keys of a part to se.best, 0 where it has fewer elements.  mine: the lane's largest logit, -inf if all are masked.
// The `top`-th largest of 64 groups' maxima is a bound: that many logits reach it, and only lanes whose own maximum does have any that
// do.  Their logits alone are looked at again, shared out among all lanes, and those from the bound on are put in order.  Entries of
// -inf are left out of this; where too few others are there, the first of them follow.  More than the list holds (many equal logits, or
// few tokens left by masks of the lowest value, which then are the bound) are found by `top` passes over the part: 1001 fp32 rows of
// 50021 with 5 alternatives 277 us, 36 with masks of -inf or few masks.
template <typename T, int THREADS>
__device__ __forceinline__ void find_top(const Part<T> &a, float mine, int top, Search<THREADS> &se)
{
    constexpr int E = wide_of<T>(), G = THREADS / 64;
    const int tid = threadIdx.x, lane = tid & 63;
    const float most = group_most<G>(mine);
    if (tid % G == 0) se.group[tid / G] = most;
    if (tid < top) se.best[tid] = 0;
    if (tid == 0) se.owners = se.listed = 0;
    __syncthreads();
    if (tid < 64) {                            // one wavefront: the chip's arithmetic is as short as its bandwidth here
        const float b = top_bound(se.group, top);
        if (tid == 0) se.bound = b;
    }
    __syncthreads();
    const float bound = se.bound;
    if (mine >= bound && mine > -INFINITY) se.owner[atomicAdd(&se.owners, 1)] = (unsigned short)tid;
    __syncthreads();
    const int cols = (a.q.n + THREADS - 1) / THREADS + 2;                      // a lane's runs, and its elements of head and rest
    const int shift = 32 - __builtin_clz(cols - 1), items = se.owners << shift;
    auto add = [&](float x, int j) {
        if (x >= bound && x > -INFINITY) {
            const int slot = atomicAdd(&se.listed, 1);
            if (slot < se.LIST) se.list[slot] = lp_key(x, a.j0 + j);
        }
    };
    for (int i = tid; i < items; i += THREADS) {
        const int owner = se.owner[i >> shift], col = i & ((1 << shift) - 1), run = (col - 1) * THREADS + owner;
        if (col >= cols) continue;
        if (col == 0) { if (owner < a.q.head) add((float)a.p[owner], owner); }
        else if (col == cols - 1) { if (owner < a.q.tail) add((float)a.rest[owner], a.q.head + a.q.n * E + owner); }
        else if (run < a.q.n) {
            float x[E];
            load_wide<T, E, false>(a.body + (long long)run * E, x);
#pragma unroll
            for (int u = 0; u < E; ++u) add(x[u], a.q.head + run * E + u);
        }
    }
    __syncthreads();
    const int n = se.listed;
    if (n <= se.LIST) {
        for (int i = tid; i < n; i += THREADS) {
            const uint64_t key = se.list[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += se.list[j] > key ? 1 : 0;
            if (rank < top) se.best[rank] = key;
        }
        if (n < top && tid < 64)               // masked entries (and NaN): at most n of the first n + top are others
            for (int j0 = 0, have = n; j0 < a.count && have < top; j0 += 64) {
                const int j = j0 + lane;
                const float x = j < a.count ? (float)a.p[j] : 0.f;
                const bool masked = j < a.count && !(x > -INFINITY);
                const uint64_t mask = __ballot(masked);
                const int place = have + __popcll(mask & ((1ull << lane) - 1));
                if (masked && place < top) se.best[place] = lp_key(x, a.j0 + j);
                have += __popcll(mask);
            }
    } else {
        // many equal ones: one after the other, each the largest key below the one before
        uint64_t last = ~0ull;
        for (int place = 0; place < top; ++place) {
            uint64_t key = 0;
            for (int j = tid; j < a.count; j += THREADS) {
                const uint64_t other = lp_key((float)a.p[j], a.j0 + j);
                if (other < last && other > key) key = other;
            }
            key = wave_max(key);
            __syncthreads();
            if (lane == 0) se.list[tid >> 6] = key;
            __syncthreads();
            for (int i = 0; i < THREADS / 64; ++i) key = se.list[i] > key ? se.list[i] : key;
            if (tid == 0) se.best[place] = key;
            last = key;
        }
    }
    __syncthreads();
}

// One workgroup to a split of a row
template <typename T, int THREADS, bool TOP>
__global__ __launch_bounds__(THREADS, 8) void token_logprobs_kernel(LpArgs a)
{
    constexpr int E = wide_of<T>(), W = THREADS / 64, U = (TOP ? 8 : 16) / E;      // (with alternatives sixteen logits of a trip would cost registers)
    __shared__ Stat red[W];
    __shared__ Search<TOP ? THREADS : 1> se;
    const int tid = threadIdx.x;
    const float c = a.inv_t * LOG2E;
    for (long long row = blockIdx.y; row < a.rows; row += gridDim.y) {
        Part<T> part;
        part.j0 = blockIdx.x * a.part;
        part.count = min(a.V - part.j0, a.part);
        part.p = (const T *)a.x + row * a.stride + part.j0;
        const Runs q = part.q = runs_of(part.p, part.count);
        part.body = part.p + q.head;
        part.rest = part.body + q.n * E;
        Stat st = {LOWEST, 0.0, 0.0};
        auto seen = [&](float top) {
            if (top > st.m) rescale(st, top, c);
        };
        auto one = [&](float x) {
            seen(x);
            take<1>(st, &x, c);
        };
        if (tid < q.head) one((float)part.p[tid]);
        int i = tid;
        for (; i + (U - 1) * THREADS < q.n; i += U * THREADS) {
            typedef typename Wide<T, E>::vec V;
            V raw[U];
#pragma unroll
            for (int v = 0; v < U; ++v) raw[v] = *(const V *)(part.body + (long long)(i + v * THREADS) * E);
            if (!TOP) __builtin_amdgcn_sched_barrier(0);       // or the second load waits for the first: 8192 bf16 rows of 32768 take 2 to 4 us more of 100 then
            float x[U * E];
#pragma unroll
            for (int v = 0; v < U; ++v)
#pragma unroll
                for (int u = 0; u < E; ++u) x[v * E + u] = (float)raw[v][u];
            float top = x[0];
#pragma unroll
            for (int u = 1; u < U * E; ++u) top = fmaxf(top, x[u]);
            seen(top);
            take<U * E>(st, x, c);
        }
        for (; i < q.n; i += THREADS) {
            float x[E];
            load_wide<T, E, false>(part.body + (long long)i * E, x);
            float top = x[0];
#pragma unroll
            for (int u = 1; u < E; ++u) top = fmaxf(top, x[u]);
            seen(top);
            take<E>(st, x, c);
        }
        if (tid < q.tail) one((float)part.rest[tid]);
        const float mine = st.s == 0.0 ? -INFINITY : st.m;                     // (its own largest has 2^0 in s)
        st = wave_merge(st, c);
        if (W > 1) {
            if ((tid & 63) == 0) red[tid >> 6] = st;
            __syncthreads();
            st = merge_all<W>(red, c);
        }
        const bool alone = a.splits == 1;
        Done r = {};
        if (alone) {
            r = lp_done(st);
            if (tid == 0) lp_row<T>(a, row, r);
        } else if (tid == 0) a.parts[row * a.splits + blockIdx.x] = st;
        if constexpr (TOP) {
            find_top<T, THREADS>(part, mine, a.top, se);
            if (tid < a.top) {
                if (alone) lp_alternative(a, row, tid, se.best[tid], r);
                else a.keys[(row * a.splits + blockIdx.x) * a.top + tid] = se.best[tid];
            }
        }
        __syncthreads();                       // the LDS words serve the next row
    }
}

// Rows that were split: a wavefront joins a row's parts.  Alternatives: each lane holds the largest key not yet taken of each of its
// splits, whose lists are sorted and lie in LDS; `top` times the largest of all lanes is taken.
constexpr int LP_MAX_SPLITS = 256;
template <typename T>
__global__ __launch_bounds__(64) void token_logprobs_join_kernel(LpArgs a)
{
    constexpr int S = LP_MAX_SPLITS / 64;
    extern __shared__ uint64_t keys[];         // [splits][top]
    const int lane = threadIdx.x, n = a.splits * a.top;
    const float c = a.inv_t * LOG2E;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        Stat st = {LOWEST, 0.0, 0.0}, mine[S];
        for (int i = lane; i < n; i += 8 * 64) {                   // eight loads in flight
            uint64_t key[8];
#pragma unroll
            for (int u = 0; u < 8; ++u) key[u] = a.keys[row * n + min(i + u * 64, n - 1)];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                if (i + u * 64 < n) keys[i + u * 64] = key[u];
        }
        float m = LOWEST;
#pragma unroll
        for (int i = 0; i < S; ++i) {
            mine[i] = lane + i * 64 < a.splits ? a.parts[row * a.splits + lane + i * 64] : st;
            m = fmaxf(m, mine[i].m);
        }
        m = wave_max(m);
        st.m = m;
#pragma unroll
        for (int i = 0; i < S; ++i) { rescale(mine[i], m, c); st.s += mine[i].s; st.w += mine[i].w; }
        st.s = wave_sum(st.s);
        st.w = wave_sum(st.w);
        const Done r = lp_done(st);
        if (lane == 0) lp_row<T>(a, row, r);
        __syncthreads();
        int at[S];
        uint64_t head[S];
#pragma unroll
        for (int i = 0; i < S; ++i) {
            at[i] = (lane + i * 64) * a.top;
            head[i] = at[i] < n ? keys[at[i]] : 0;
        }
        for (int t = 0; t < a.top; ++t) {
            uint64_t most = head[0];
#pragma unroll
            for (int i = 1; i < S; ++i) most = head[i] > most ? head[i] : most;
            most = wave_max(most);
#pragma unroll
            for (int i = 0; i < S; ++i)
                if (head[i] == most) head[i] = ++at[i] < (lane + i * 64 + 1) * a.top ? keys[at[i]] : 0;
            if (lane == 0) lp_alternative(a, row, t, most, r);
        }
        __syncthreads();
    }
}

struct LpBackArgs {
    const void *x;
    const int64_t *tokens;
    const float *stats, *entropy, *dlogp, *dent;
    void *dx;
    long long rows, s_x, s_dx;
    int V, part;
    double inv_t;
};

// dx_j = 1/T p_j (-a - b (log p_j + H)), and a/T more at the token.  Bound by memory: a read and a write of each logit.  A lane has four
// loads in flight, the last of a row again where it has fewer: 8192 bf16 rows of 32768 158 us, 6.8 TB/s (168 with one).
template <typename T, int THREADS>
__global__ __launch_bounds__(THREADS) void token_logprobs_back_kernel(LpBackArgs q)
{
    constexpr int E = wide_of<T>();
    const int j0 = blockIdx.x * q.part, count = min(q.V - j0, q.part);
    for (long long row = blockIdx.y; row < q.rows; row += gridDim.y) {
        const T *const p = (const T *)q.x + row * q.s_x + j0;
        T *const d = (T *)q.dx + row * q.s_dx + j0;
        const long long token = q.tokens != nullptr ? q.tokens[row] : -1;
        const bool has = token >= 0 && token < q.V;
        const float m = q.stats[2 * row], ls = q.stats[2 * row + 1], a = has && q.dlogp != nullptr ? q.dlogp[row] : 0.f, b = q.dent != nullptr ? q.dent[row] : 0.f;
        const float H = b != 0.f ? q.entropy[row] : 0.f;
        const bool empty = ls == -INFINITY;
        const int at = has ? (int)(token - j0) : -1;
        const float inv_t = (float)q.inv_t, base = (float)((-a - (double)b * H) * q.inv_t), slope = (float)(-b * q.inv_t), extra = (float)(a * q.inv_t);
        auto grad = [&](float x, int j) {
            const float lp = fmaf(x - m, inv_t, -ls);
            const float e = __builtin_amdgcn_exp2f(lp * LOG2E);
            const float g = empty ? 0.f : e * fmaf(slope, fmaxf(lp, -1000.f), base);
            return j == at && !empty ? g + extra : g;
        };
        const Runs r = runs_of(p, count);
        if ((int)threadIdx.x < r.head) d[threadIdx.x] = (T)grad((float)p[threadIdx.x], threadIdx.x);
        for (int i = threadIdx.x; i < r.n; i += 4 * THREADS) {
            float x[4][E];
#pragma unroll
            for (int v = 0; v < 4; ++v) load_wide<T, E, true>(p + r.head + (long long)min(i + v * THREADS, r.n - 1) * E, x[v]);
#pragma unroll
            for (int v = 0; v < 4; ++v) {
                const int run = i + v * THREADS;
                if (run >= r.n) break;
#pragma unroll
                for (int u = 0; u < E; ++u) x[v][u] = grad(x[v][u], r.head + run * E + u);
                store_wide<T, E, true>(d + r.head + (long long)run * E, x[v]);
            }
        }
        const int t0 = r.head + r.n * E + threadIdx.x;
        if ((int)threadIdx.x < r.tail) d[t0] = (T)grad((float)p[t0], t0);
    }
}

// How a row is shared out: workgroups of 64 lanes for short rows, 256 for longer ones and wherever rows are many (8192 bf16 rows of
// 32768 100 us, 106 with 512), 512 for long rows that one workgroup each just about fills the chip with (512 fp32 rows of 50020 19.0 us,
// 22.6 with 256).  Long rows too few to fill the chip are split, down to a run for each of 256 lanes, and joined by a second launch;
// from eight runs for each of 512 lanes on, as a shorter row takes no longer whole (one of 16000 in bf16 5.1 us either way).
struct LpPlan { int threads, splits, part; };
static LpPlan lp_plan(long long rows, long long V, int E, int top)
{
    LpPlan q;
    q.threads = V <= 64 * E * 4 ? 64 : V <= 256 * E * 8 || rows >= 2048 ? 256 : 512;
    q.splits = 1;
    if (V > 512 * E * 8 && rows < 512) {
        const long long want = (1024 + rows - 1) / rows, most = (V + 256 * E - 1) / (256 * E);
        q.splits = (int)(want < most ? want : most);
        if (q.splits > LP_MAX_SPLITS) q.splits = LP_MAX_SPLITS;
        if (q.splits * top > 4096) q.splits = 4096 / top;            // the joining wavefront's LDS: 32 KiB
        if (q.splits > 1) q.threads = 256;
    }
    q.part = (int)((V + q.splits - 1) / q.splits + E - 1) / E * E;
    q.splits = (int)((V + q.part - 1) / q.part);
    return q;
}

template <typename T, int THREADS>
static hipError_t launch_lp(const LpArgs &a, hipStream_t s)
{
    const dim3 grid((unsigned)a.splits, (unsigned)(a.rows < 65535 ? a.rows : 65535));
    if (a.top > 0) token_logprobs_kernel<T, THREADS, true><<<grid, THREADS, 0, s>>>(a);
    else token_logprobs_kernel<T, THREADS, false><<<grid, THREADS, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.splits == 1) return e;
    token_logprobs_join_kernel<T><<<(unsigned)(a.rows < 65535 ? a.rows : 65535), 64, (size_t)a.splits * a.top * sizeof(uint64_t), s>>>(a);
    return hipGetLastError();
}
template <typename T>
static hipError_t launch_lp(const LpArgs &a, int threads, hipStream_t s)
{
    return threads == 64 ? launch_lp<T, 64>(a, s) : threads == 256 ? launch_lp<T, 256>(a, s) : launch_lp<T, 512>(a, s);
}

template <typename T>
static hipError_t launch_lp_back(LpBackArgs &q, hipStream_t s)
{
    constexpr int E = wide_of<T>();
    const bool small = q.V <= 64 * E * 8;
    q.part = small ? (q.V + E - 1) / E * E : 256 * E * 4;
    const dim3 grid((unsigned)((q.V + q.part - 1) / q.part), (unsigned)(q.rows < 65535 ? q.rows : 65535));
    if (small) token_logprobs_back_kernel<T, 64><<<grid, 64, 0, s>>>(q);
    else token_logprobs_back_kernel<T, 256><<<grid, 256, 0, s>>>(q);
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
static bool type_ok(int type) { return type == QSR_TYPE_F32 || type == QSR_TYPE_BF16; }
static uintptr_t size_of(int type) { return type == QSR_TYPE_F32 ? 4 : 2; }
static bool sizes_ok(int64_t rows, int64_t V) { return rows >= 0 && rows <= ((long long)1 << 31) && V >= 1 && V <= (1 << 30); }

// 1 / T as a float; of use where log2(e) / T is one as well
static bool inverse(double temperature, float &inv_t)
{
    if (!(std::isfinite(temperature) && temperature > 0.0)) return false;
    inv_t = (float)(1.0 / temperature);
    return inv_t > 0.f && inv_t * LOG2E < INFINITY;
}

extern "C" int qsr_token_logprobs_workspace_bytes(int64_t rows, int64_t vocab, int32_t type, int32_t top, size_t *bytes)
{
    if (!bytes) return QSR_EINVAL;
    *bytes = 0;
    if (!sizes_ok(rows, vocab) || !type_ok(type) || top < 0 || top > vocab) return QSR_EINVAL;
    if (top > LP_MAX_TOP) return QSR_ELIMIT;
    if (rows == 0) return QSR_OK;
    const LpPlan p = lp_plan(rows, vocab, 16 / (int)size_of(type), top);
    if (p.splits > 1) *bytes = (size_t)rows * p.splits * ((size_t)top * sizeof(uint64_t) + sizeof(Stat));
    return QSR_OK;
}

extern "C" int qsr_token_logprobs(const qsr_token_logprobs_args *q, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!q) return QSR_EINVAL;
    size_t need = 0;
    const int rc = qsr_token_logprobs_workspace_bytes(q->rows, q->vocab, q->type, q->top, &need);
    if (rc != QSR_OK) return rc;
    float inv_t;
    if (!inverse(q->temperature, inv_t) || q->stride < q->vocab) return QSR_EINVAL;
    if (q->rows == 0) return QSR_OK;
    if (!q->logits || off(q->logits, size_of(q->type)) || off(q->tokens, 8) || off(q->logp, 4) || off(q->entropy, 4) || off(q->lse, 4) || off(q->stats, 4))
        return QSR_EINVAL;
    if (q->logp && !q->tokens) return QSR_EINVAL;
    if (q->top > 0 && (!q->top_logp || !q->top_id || off(q->top_logp, 4) || off(q->top_id, 4))) return QSR_EINVAL;
    if (need > 0 && (!workspace || off(workspace, 8))) return QSR_EINVAL;
    if (workspace_bytes < need) return QSR_ENOMEM;
    const LpPlan p = lp_plan(q->rows, q->vocab, 16 / (int)size_of(q->type), q->top);
    uint64_t *const keys = (uint64_t *)workspace;
    const LpArgs a{q->logits, q->tokens, q->rows, q->stride, (int)q->vocab, q->top, p.splits, p.part, inv_t, q->logp, q->entropy,
                   q->lse, q->stats, q->top_logp, q->top_id, (Stat *)(keys + (p.splits > 1 ? q->rows * p.splits * q->top : 0)), keys};
    return finish(q->type == QSR_TYPE_F32 ? launch_lp<float>(a, p.threads, (hipStream_t)stream)
                                          : launch_lp<bf16_t>(a, p.threads, (hipStream_t)stream));
}

extern "C" int qsr_token_logprobs_backward(const qsr_token_logprobs_backward_args *q, void *stream)
{
    if (!q || !sizes_ok(q->rows, q->vocab) || !type_ok(q->type)) return QSR_EINVAL;
    float inv_t;
    if (!inverse(q->temperature, inv_t) || q->stride < q->vocab || q->grad_stride < q->vocab) return QSR_EINVAL;
    if (q->rows == 0) return QSR_OK;
    const uintptr_t es = size_of(q->type);
    if (!q->logits || off(q->logits, es) || !q->grad || off(q->grad, es) || off(q->tokens, 8) || !q->stats || off(q->stats, 4) ||
        off(q->entropy, 4) || off(q->logp_grad, 4) || off(q->entropy_grad, 4))
        return QSR_EINVAL;
    if ((q->logp_grad && !q->tokens) || (q->entropy_grad && !q->entropy)) return QSR_EINVAL;
    LpBackArgs a{q->logits, q->tokens, q->stats, q->entropy, q->logp_grad, q->entropy_grad, q->grad, q->rows, q->stride, q->grad_stride,
                 (int)q->vocab, 0, 1.0 / q->temperature};
    return finish(q->type == QSR_TYPE_F32 ? launch_lp_back<float>(a, (hipStream_t)stream) : launch_lp_back<bf16_t>(a, (hipStream_t)stream));
}
