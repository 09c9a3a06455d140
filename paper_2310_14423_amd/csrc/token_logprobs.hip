// token_logprobs.hip -- log probabilities of given tokens from rows of logits, with the entropy and the best alternatives, and the
// gradient with respect to the logits.
//
//   z = x / T;  lse = log sum_j exp z_j;  logp = z_token - lse;  H = lse - sum_j p_j z_j;  alternatives: the `top` largest z_j - lse,
//   the lower index first where they tie
//   dx_j = 1/T [ a (delta_{j,token} - p_j) - b p_j (log p_j + H) ]   for a = d/dlogp and b = d/dH
// A row that is masked as a whole (all -inf) has lse = logp = -inf, H = 0 and no gradient.  A token outside 0..V-1 stands for none:
// logp = 0 and no gradient from it.
//
// One pass over the logits: every lane keeps the largest logit m it has seen, s = sum e^((x - m)/T) and w = sum of t e^.. with
// t = (x - m)/T in units of log 2, rescaled where m grows; H = ln 2 (log2 s - w / s).  m starts at the lowest float, not at -inf,
// so that masked entries (x - m = -inf) are zeros and never NaN.  x - m is taken before the scaling: one product-sum with a rounded
// m / T would shift all exponents of a row by its rounding.
// Alternatives without a second pass: a lane also keeps its largest logit and where it was.  The `top` largest of these lane
// maxima are a bound: nothing below the last of them is an alternative, and the only lanes with anything above it are their owners.
// Those `top` lanes' logits alone are read again, from the caches.
#include <cmath>

#include "qsr_internal.h"
#include "row_io.h"

namespace qsr {

constexpr float LOWEST = -3.402823466e38f, LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;
constexpr int LP_MAX_TOP = 64;                 // alternatives: the lanes of a wavefront
constexpr int LP_LIST = 1024;                  // logits above the bound that fit LDS

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
__device__ __forceinline__ uint64_t key_xor(uint64_t v, int o)
{
    return ((uint64_t)(uint32_t)__shfl_xor((int)(v >> 32), o, 64) << 32) | (uint32_t)__shfl_xor((int)(uint32_t)v, o, 64);
}

struct Stat { float m, s, w; };
__device__ __forceinline__ void merge(Stat &a, const Stat &b, float c)
{
    const float m = fmaxf(a.m, b.m);
    // no further down than 2^-1000: a sum of zeros times -inf would be NaN
    const float da = fmaxf((a.m - m) * c, -1000.f), db = fmaxf((b.m - m) * c, -1000.f);
    const float fa = __builtin_amdgcn_exp2f(da), fb = __builtin_amdgcn_exp2f(db);
    const float s = fa * a.s + fb * b.s;
    a.w = fa * fmaf(da, a.s, a.w) + fb * fmaf(db, b.s, b.w);
    a.s = s; a.m = m;
}
__device__ __forceinline__ Stat wave_merge(Stat a, float c)
{
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
        const Stat b = {__shfl_xor(a.m, o, 64), __shfl_xor(a.s, o, 64), __shfl_xor(a.w, o, 64)};
        merge(a, b, c);
    }
    return a;
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

// Log probabilities are taken from x - m: lse alone, as a float, has lost log s where the logits are large (a row of masks of the
// lowest value has p = 1/V like any row of equal logits).  For the same reason `stats` keeps m and log s for the backward pass.
__device__ __forceinline__ float lp_of(const LpArgs &a, const Stat &st, float x)
{
    return st.s == 0.f ? -INFINITY : fmaf(-LN2, __log2f(st.s), (x - st.m) * a.inv_t);
}
__device__ __forceinline__ void lp_result(const LpArgs &a, long long row, const Stat &st)
{
    const float ls = LN2 * __log2f(st.s);
    const bool empty = st.s == 0.f;
    if (a.lse != nullptr) a.lse[row] = empty ? -INFINITY : fmaf(st.m, a.inv_t, ls);
    if (a.stats != nullptr) { a.stats[2 * row] = st.m; a.stats[2 * row + 1] = ls; }
    if (a.entropy != nullptr) a.entropy[row] = empty ? 0.f : fmaf(-LN2, st.w / st.s, ls);
}
__device__ __forceinline__ void lp_alternative(const LpArgs &a, long long row, int place, uint64_t key, const Stat &st)
{
    a.top_logp[row * a.top + place] = lp_of(a, st, key_value(key));
    a.top_id[row * a.top + place] = (int32_t)key_index(key);
}
__device__ __forceinline__ long long lp_token(const LpArgs &a, long long row)
{
    const long long t = a.tokens != nullptr ? a.tokens[row] : -1;
    return t >= 0 && t < a.V ? t : -1;
}
template <typename T>
__device__ __forceinline__ void lp_row(const LpArgs &a, long long row, const Stat &st)
{
    lp_result(a, row, st);
    if (a.logp == nullptr) return;
    const long long token = lp_token(a, row);
    a.logp[row] = token < 0 ? 0.f : lp_of(a, st, (float)((const T *)a.x)[row * a.stride + token]);
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

// The `top` largest keys among n in LDS, by counting how many are larger, to out[0..top) in LDS.  Keys other than 0 differ.
template <int THREADS>
__device__ __forceinline__ void rank_keys(const uint64_t *in, int n, int top, uint64_t *out)
{
    for (int i = threadIdx.x; i < n; i += THREADS) {
        const uint64_t key = in[i];
        int rank = 0;
        for (int j = 0; j < n; ++j) rank += in[j] > key ? 1 : 0;
        if (rank < top && key != 0) out[rank] = key;
    }
}

// One workgroup to a split of a row.  best: the top largest keys of the split (0 where there are fewer elements).
template <typename T, int THREADS, bool TOP>
__global__ __launch_bounds__(THREADS) void token_logprobs_kernel(LpArgs a)
{
    constexpr int E = wide_of<T>(), W = THREADS / 64;
    __shared__ Stat red[W];
    __shared__ uint64_t cand[TOP ? W * LP_MAX_TOP : 1], list[TOP ? LP_LIST : 1], best[TOP ? LP_MAX_TOP : 1];
    __shared__ int listed;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const float c = a.inv_t * LOG2E;
    const int j0 = blockIdx.x * a.part, count = min(a.V - j0, a.part);
    for (long long row = blockIdx.y; row < a.rows; row += gridDim.y) {
        const T *const p = (const T *)a.x + row * a.stride + j0;
        const Runs q = runs_of(p, count);
        const T *const body = p + q.head, *const rest = body + q.n * E;
        Stat st = {LOWEST, 0.f, 0.f};
        float big = -INFINITY;
        int big_at = -1;                       // -1: head, run, n: rest
        bool any = false;
        auto take = [&](float x, int at) {
            if (x > st.m) { const Stat one = {x, 0.f, 0.f}; merge(st, one, c); }
            const float t = (x - st.m) * c, e = __builtin_amdgcn_exp2f(t);
            st.s += e;
            st.w = fmaf(e, fmaxf(t, -1000.f), st.w);
            if (TOP && (!any || x > big)) { big = fmaxf(x, -INFINITY); big_at = at; any = true; }     // (NaN: -inf)
        };
        if (tid < q.head) take((float)p[tid], -1);
        for (int i = tid; i < q.n; i += THREADS) {
            float x[E];
            load_wide<T, E, false>(body + (long long)i * E, x);
            float top = x[0];
#pragma unroll
            for (int u = 1; u < E; ++u) top = fmaxf(top, x[u]);
            if (top > st.m) { const Stat one = {top, 0.f, 0.f}; merge(st, one, c); }
#pragma unroll
            for (int u = 0; u < E; ++u) {
                const float t = (x[u] - st.m) * c, e = __builtin_amdgcn_exp2f(t);
                st.s += e;
                st.w = fmaf(e, fmaxf(t, -1000.f), st.w);
            }
            if (TOP && (!any || top > big)) { big = fmaxf(top, -INFINITY); big_at = i; any = true; }
        }
        if (tid < q.tail) take((float)rest[tid], q.n);
        st = wave_merge(st, c);
        if (W > 1) {
            if (lane == 0) red[wave] = st;
            __syncthreads();
            st = red[0];
#pragma unroll
            for (int i = 1; i < W; ++i) merge(st, red[i], c);
        }
        const bool alone = a.splits == 1;
        if (tid == 0) {
            if (alone) lp_row<T>(a, row, st);
            else a.parts[row * a.splits + blockIdx.x] = st;
        }
        if (TOP) {
            // the lane's largest: the first element of its run that has it
            uint64_t key = 0;
            if (any) {
                if (big_at < 0) key = lp_key(big, j0 + tid);
                else if (big_at == q.n) key = lp_key(big, j0 + q.head + q.n * E + tid);
                else {
#pragma unroll
                    for (int u = 0; u < E; ++u) {
                        const uint64_t other = lp_key((float)body[(long long)big_at * E + u], j0 + q.head + big_at * E + u);
                        key = other > key ? other : key;
                    }
                }
            }
            if (tid < a.top) best[tid] = 0;
            if (tid == 0) listed = 0;
            // a wavefront's `top` largest lane maxima, sorted by compare and exchange
#pragma unroll
            for (int size = 2; size <= 64; size <<= 1)
#pragma unroll
                for (int o = size >> 1; o > 0; o >>= 1) {
                    const uint64_t other = key_xor(key, o);
                    const bool up = (lane & size) == 0, low = (lane & o) == 0;      // descending runs where `up`
                    const bool more = other > key;
                    key = (up == low) == more ? other : key;
                }
            if (lane < a.top) cand[wave * a.top + lane] = key;
            __syncthreads();
            rank_keys<THREADS>(cand, W * a.top, a.top, best);
            __syncthreads();
            // the owners' elements from the bound on
            const uint64_t bound = best[a.top - 1];
            const int cols = (q.n + THREADS - 1) / THREADS + 2;                      // a lane's runs, and its head and rest
            for (int i = tid; i < cols * a.top; i += THREADS) {
                const uint64_t own = best[i / cols];
                if (own == 0) continue;
                const int at = (int)key_index(own) - j0;                             // the owner, from where its largest is
                const int owner = at < q.head ? at : at < q.head + q.n * E ? ((at - q.head) / E) % THREADS : at - q.head - q.n * E;
                const int col = i % cols;
                auto add = [&](float x, int j) {
                    const uint64_t k2 = lp_key(x, j0 + j);
                    if (k2 >= bound) {
                        const int slot = atomicAdd(&listed, 1);
                        if (slot < LP_LIST) list[slot] = k2;
                    }
                };
                if (col == 0) { if (owner < q.head) add((float)p[owner], owner); }
                else if (col == cols - 1) { if (owner < q.tail) add((float)rest[owner], q.head + q.n * E + owner); }
                else {
                    const int run = (col - 1) * THREADS + owner;
                    if (run < q.n) {
                        float x[E];
                        load_wide<T, E, false>(body + (long long)run * E, x);
#pragma unroll
                        for (int u = 0; u < E; ++u) add(x[u], q.head + run * E + u);
                    }
                }
            }
            __syncthreads();
            const int n = listed;
            if (n <= LP_LIST) {
                __syncthreads();
                rank_keys<THREADS>(list, n, a.top, best);
            } else {
                // more of them than fit: one after the other, each the largest below the one before
                uint64_t last = ~0ull;
                for (int place = 0; place < a.top; ++place) {
                    uint64_t most = 0;
                    for (int j = tid; j < count; j += THREADS) {
                        const uint64_t k2 = lp_key((float)p[j], j0 + j);
                        if (k2 < last && k2 > most) most = k2;
                    }
#pragma unroll
                    for (int o = 32; o > 0; o >>= 1) { const uint64_t other = key_xor(most, o); most = other > most ? other : most; }
                    __syncthreads();
                    if (lane == 0) cand[wave] = most;
                    __syncthreads();
                    for (int i = 0; i < W; ++i) most = cand[i] > most ? cand[i] : most;
                    if (tid == 0) best[place] = most;
                    last = most;
                }
            }
            __syncthreads();
            if (tid < a.top) {
                if (alone) lp_alternative(a, row, tid, best[tid], st);
                else a.keys[(row * a.splits + blockIdx.x) * a.top + tid] = best[tid];
            }
        }
        __syncthreads();                       // the LDS words serve the next row
    }
}

// Rows that were split: a wavefront joins a row's parts.  Alternatives: each lane keeps the largest key not yet taken of its splits,
// whose lists are sorted; `top` times the largest of all lanes is taken.
constexpr int LP_MAX_SPLITS = 256;
template <typename T>
__global__ __launch_bounds__(64) void token_logprobs_join_kernel(LpArgs a)
{
    constexpr int S = LP_MAX_SPLITS / 64;
    const int lane = threadIdx.x;
    const float c = a.inv_t * LOG2E;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        Stat st = {LOWEST, 0.f, 0.f};
        for (int i = lane; i < a.splits; i += 64) merge(st, a.parts[row * a.splits + i], c);
        st = wave_merge(st, c);
        if (lane == 0) lp_row<T>(a, row, st);
        const uint64_t *const keys = a.keys + row * a.splits * a.top;
        uint64_t head[S];
        int place[S];
#pragma unroll
        for (int i = 0; i < S; ++i) {
            place[i] = 0;
            head[i] = a.top > 0 && lane + i * 64 < a.splits ? keys[(lane + i * 64) * a.top] : 0;
        }
        for (int t = 0; t < a.top; ++t) {
            uint64_t most = head[0];
#pragma unroll
            for (int i = 1; i < S; ++i) most = head[i] > most ? head[i] : most;
#pragma unroll
            for (int o = 32; o > 0; o >>= 1) { const uint64_t other = key_xor(most, o); most = other > most ? other : most; }
#pragma unroll
            for (int i = 0; i < S; ++i)
                if (head[i] == most && most != 0) head[i] = ++place[i] < a.top ? keys[(lane + i * 64) * a.top + place[i]] : 0;
            if (lane == 0) lp_alternative(a, row, t, most, st);
        }
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

// dx_j = 1/T p_j (-a - b (log p_j + H)), and a/T more at the token.  Bound by memory: a read and a write of each logit.
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
        for (int i = threadIdx.x; i < r.n; i += THREADS) {
            float x[E];
            load_wide<T, E, true>(p + r.head + (long long)i * E, x);
#pragma unroll
            for (int u = 0; u < E; ++u) x[u] = grad(x[u], r.head + i * E + u);
            store_wide<T, E, true>(d + r.head + (long long)i * E, x);
        }
        const int t0 = r.head + r.n * E + threadIdx.x;
        if ((int)threadIdx.x < r.tail) d[t0] = (T)grad((float)p[t0], t0);
    }
}

// How a row is shared out: workgroups of 64 lanes for short rows, 256 and 512 for longer ones; rows too few to fill the chip are split.
struct LpPlan { int threads, splits, part; };
static LpPlan lp_plan(long long rows, long long V, int E)
{
    LpPlan q;
    q.threads = V <= 64 * E * 4 ? 64 : V <= 256 * E * 8 ? 256 : 512;
    q.splits = 1;
    if (q.threads > 64) {
        const long long want = (1024 + rows - 1) / rows, most = (V + q.threads * E * 2 - 1) / (q.threads * E * 2);
        q.splits = (int)(rows >= 512 ? 1 : want < most ? want : most);
        if (q.splits > LP_MAX_SPLITS) q.splits = LP_MAX_SPLITS;
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
    token_logprobs_join_kernel<T><<<(unsigned)(a.rows < 65535 ? a.rows : 65535), 64, 0, s>>>(a);
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

extern "C" int qsr_token_logprobs_workspace_bytes(int64_t rows, int64_t vocab, int32_t type, int32_t top, size_t *bytes)
{
    if (!bytes) return QSR_EINVAL;
    *bytes = 0;
    if (!sizes_ok(rows, vocab) || !type_ok(type) || top < 0 || top > vocab) return QSR_EINVAL;
    if (top > LP_MAX_TOP) return QSR_ELIMIT;
    if (rows == 0) return QSR_OK;
    const LpPlan p = lp_plan(rows, vocab, 16 / (int)size_of(type));
    if (p.splits > 1) *bytes = (size_t)rows * p.splits * ((size_t)top * sizeof(uint64_t) + sizeof(Stat));
    return QSR_OK;
}

extern "C" int qsr_token_logprobs(const qsr_token_logprobs_args *q, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!q) return QSR_EINVAL;
    size_t need = 0;
    const int rc = qsr_token_logprobs_workspace_bytes(q->rows, q->vocab, q->type, q->top, &need);
    if (rc != QSR_OK) return rc;
    if (!(std::isfinite(q->temperature) && q->temperature > 0.0)) return QSR_EINVAL;
    const float inv_t = (float)(1.0 / q->temperature);
    if (!(inv_t > 0.f && inv_t < INFINITY) || q->stride < q->vocab) return QSR_EINVAL;
    if (q->rows == 0) return QSR_OK;
    if (!q->logits || off(q->logits, size_of(q->type)) || off(q->tokens, 8) || off(q->logp, 4) || off(q->entropy, 4) || off(q->lse, 4) || off(q->stats, 4))
        return QSR_EINVAL;
    if (q->logp && !q->tokens) return QSR_EINVAL;
    if (q->top > 0 && (!q->top_logp || !q->top_id || off(q->top_logp, 4) || off(q->top_id, 4))) return QSR_EINVAL;
    if (need > 0 && (!workspace || off(workspace, 8))) return QSR_EINVAL;
    if (workspace_bytes < need) return QSR_ENOMEM;
    const LpPlan p = lp_plan(q->rows, q->vocab, 16 / (int)size_of(q->type));
    uint64_t *const keys = (uint64_t *)workspace;
    const LpArgs a{q->logits, q->tokens, q->rows, q->stride, (int)q->vocab, q->top, p.splits, p.part, inv_t, q->logp, q->entropy,
                   q->lse, q->stats, q->top_logp, q->top_id, (Stat *)(keys + (p.splits > 1 ? q->rows * p.splits * q->top : 0)), keys};
    return finish(q->type == QSR_TYPE_F32 ? launch_lp<float>(a, p.threads, (hipStream_t)stream)
                                          : launch_lp<bf16_t>(a, p.threads, (hipStream_t)stream));
}

extern "C" int qsr_token_logprobs_backward(const qsr_token_logprobs_backward_args *q, void *stream)
{
    if (!q || !sizes_ok(q->rows, q->vocab) || !type_ok(q->type)) return QSR_EINVAL;
    if (!(std::isfinite(q->temperature) && q->temperature > 0.0)) return QSR_EINVAL;
    const float inv_t = (float)(1.0 / q->temperature);
    if (!(inv_t > 0.f && inv_t < INFINITY) || q->stride < q->vocab || q->grad_stride < q->vocab) return QSR_EINVAL;
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
