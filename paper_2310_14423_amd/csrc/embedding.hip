// embedding.hip -- rows of K workers' tables by tokens, scaled, and the gradient of the tables.
//
//   y_i = scale E_k[t_i];   dE_k[v] = scale * (sum of dy_i over the worker's tokens with t_i = v)  (+ what was there)
// A token outside 0..V-1 stands for none: zeros, and no gradient.
// The gradient's sums are made in a fixed order and without atomics.  The worker's tokens are sorted with their places by a stable radix
// sort, so that a row's terms lie side by side in the order of their places.  The sorted list is cut into chunks of equal length, however
// often a token comes: a chunk's sums go to their rows, but for a sum that other chunks have a part in, which is kept aside and joined by a
// second launch in the chunks' order.  Few tokens are sorted, summed and joined in LDS, by one launch whose workgroups share the table's
// rows.  Rows that no token names are cleared beside the sort, or where the list does not hold them.  All sums are fp32; a row is scaled,
// and rounded, once.
// Bound by memory: rows are read once and written once, the table is cleared once.  8 x 8192 tokens, the first rows frequent, over 32768 rows of 768,
// rows in bf16, the table's gradient in fp32: 141 us for the sort and the clearing, 5.7 TB/s, 45 for the sums, 9.5 for what several chunks
// share; lookup 29 us.  30011 tokens over 50021 rows of 1003 in fp32, added to what is there: 30 us for the sort (four launches, latency),
// 42 and 7.3; lookup 28.  4 x 1024 tokens over 512 rows of 128: 6.0 us in one launch, a chain of latencies; lookup 2.5.
#include <cmath>

#include "qsr_internal.h"
#include "row_io.h"

namespace qsr {

constexpr int EMBED_THREADS = 256;

struct LookupArgs {
    const void *table;
    const int64_t *tokens;
    void *y;
    long long N, V, s_table, s_worker, s_y;
    int d, lanes;              // lanes to a row: a power of two up to EMBED_THREADS
    float scale;
};

// The elements of a run that starts at column `first` of d, or E from the row's end where it would end behind it: the run's last E - `skip`
struct Run { int at, skip; };
__device__ __forceinline__ Run run_of(int first, int d, int E) { const int at = min(first, d - E); return {at, first - at}; }

template <typename T, int E>
__device__ __forceinline__ void store_run(T *p, const float (&v)[E], int skip)
{
    if (skip == 0) store_wide<T, E, sizeof(T) * E <= 16>(p, v);           // (two accesses of a lane leave lines to be joined in the cache)
    else {
#pragma unroll
        for (int u = 0; u < E; ++u)
            if (u >= skip) p[u] = (T)v[u];
    }
}

template <typename TI, typename TO, int E>
__global__ __launch_bounds__(EMBED_THREADS) void embedding_kernel(LookupArgs a)
{
    const int lane = threadIdx.x & (a.lanes - 1), place = threadIdx.x / a.lanes, side = EMBED_THREADS / a.lanes, k = blockIdx.y;
    for (long long row = (long long)blockIdx.x * side + place; row < a.N; row += (long long)gridDim.x * side) {
        const long long tok = a.tokens[k * a.N + row];
        const bool has = tok >= 0 && tok < a.V;
        const TI *const from = (const TI *)a.table + k * a.s_worker + (has ? tok : 0) * a.s_table;
        TO *const to = (TO *)a.y + (k * a.N + row) * a.s_y;
        for (int first = lane * E; first < a.d; first += a.lanes * E) {
            const Run r = run_of(first, a.d, E);
            float v[E];
            load_wide<TI, E, false>(from + r.at, v);
#pragma unroll
            for (int u = 0; u < E; ++u) v[u] = has ? v[u] * a.scale : 0.f;
            store_run<TO, E>(to + r.at, v, r.skip);
        }
    }
}

// ---------------------------------------------------------------------------------------------------
// tokens in order
// ---------------------------------------------------------------------------------------------------
constexpr int DIGITS = 512;                    // at most, of a pass of the sort
constexpr int SORT_SMALL = 16384;              // tokens of a worker that one workgroup sorts in LDS
constexpr int SORT_THREADS = 512, SMALL_THREADS = 1024;

// Tables that are cleared beside a sort by one workgroup: by workgroups behind those that sort, `groups` to a worker with `rows` rows each
struct Clear {
    char *out;
    long long V, s_row, s_worker, groups;      // in bytes
    int row, rows, lanes;
};

struct SortArgs {
    Clear clear;
    int K;
    const int64_t *tokens;                     // first pass: these, and places as they come
    const uint32_t *keys_in;
    const int *place_in;
    uint32_t *keys;                            // [K][N]
    int *place;
    int *counts;                               // [K][blocks][DIGITS]
    long long N, V, per;                       // tokens to a workgroup: whole rounds
    int shift, bits, passes;
};

// The nth workgroup's rows of worker k: 16 bytes to a lane, the last of a row's ending with it
__device__ __forceinline__ void clear_rows(const Clear &c, int k, long long nth)
{
    typedef typename Wide<uint16_t, 8>::vec Bytes16;
    const long long v0 = nth * c.rows;
    const int lane = threadIdx.x & (c.lanes - 1), rows = (int)min((long long)c.rows, c.V - v0);
    for (int i = threadIdx.x / c.lanes; i < rows; i += blockDim.x / c.lanes) {
        char *const to = c.out + k * c.s_worker + (v0 + i) * c.s_row;
        if (c.row < 16) {
            for (int b = 2 * lane; b < c.row; b += 2 * c.lanes) *(uint16_t *)(to + b) = 0;
        } else
            for (int b = 16 * lane; b < c.row; b += 16 * c.lanes) __builtin_nontemporal_store((Bytes16)(0), (Bytes16 *)(to + min(b, c.row - 16)));
    }
}

// V stands for none and comes last
__device__ __forceinline__ uint32_t key_of(long long tok, long long V) { return tok >= 0 && tok < V ? (uint32_t)tok : (uint32_t)V; }
__device__ __forceinline__ uint32_t sort_key(const SortArgs &a, int k, long long i)
{
    return a.tokens != nullptr ? key_of(a.tokens[k * a.N + i], a.V) : a.keys_in[k * a.N + i];
}

// How many lanes of the wavefront that take part and lie before this one have its digit, and how many have it in all
__device__ __forceinline__ void same_digit(uint32_t digit, bool in, int bits, int &before, int &all)
{
    const uint64_t there = __ballot(in);
    uint32_t lo = (uint32_t)there, hi = (uint32_t)(there >> 32);
#pragma unroll
    for (int b = 0; b < 9; ++b)
        if (b < bits) {
            const uint32_t own = (uint32_t)((int32_t)(digit << (31 - b)) >> 31);           // all ones where the bit is one
            const uint64_t one = __ballot(own != 0);
            lo &= ~(own ^ (uint32_t)one);
            hi &= ~(own ^ (uint32_t)(one >> 32));
        }
    before = (int)__builtin_amdgcn_mbcnt_hi(hi, __builtin_amdgcn_mbcnt_lo(lo, 0));
    all = __popc(lo) + __popc(hi);
}

// counts[digit], digit < DIGITS, to the sums over all digits before.  Every thread has to be here.
template <int THREADS>
__device__ __forceinline__ void sums_before(int *counts, int *waves)
{
    constexpr int EACH = (DIGITS + THREADS - 1) / THREADS;
    const int tid = threadIdx.x, lane = tid & 63;
    int c[EACH], sum = 0;
#pragma unroll
    for (int i = 0; i < EACH; ++i) { c[i] = tid * EACH + i < DIGITS ? counts[tid * EACH + i] : 0; sum += c[i]; }
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) { const int v = __shfl_up(upto, o, 64); upto += lane >= o ? v : 0; }
    if (lane == 63) waves[tid >> 6] = upto;
    __syncthreads();
    int base = upto - sum;
    for (int w = 0; w < (tid >> 6); ++w) base += waves[w];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (tid * EACH + i < DIGITS) counts[tid * EACH + i] = base;
        base += c[i];
    }
    __syncthreads();
}

// What a wavefront's lanes have read and written in LDS stays before what they read and write behind this: LDS takes a wavefront's accesses in
// their order, so that the compiler alone has to keep to it, and no instruction is needed
__device__ __forceinline__ void wave_in_order()
{
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}

// A wavefront's next EACH * 64 keys, of which `left` are there: each one's place among those of its digit, from `count` on, which goes on.
// (No atomics: the keys of frequent tokens would wait for each other.)
template <int EACH>
__device__ __forceinline__ void rank_keys(const uint32_t (&key)[EACH], int left, int shift, int bits, int *count, int (&rank)[EACH])
{
    const int lane = threadIdx.x & 63;
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        if (i * 64 >= left) break;
        const bool in = i * 64 + lane < left;
        const uint32_t digit = (key[i] >> shift) & ((1u << bits) - 1);
        int before, all;
        same_digit(digit, in, bits, before, all);
        const int here = count[digit];
        rank[i] = here + before;
        wave_in_order();
        if (in && before == 0) count[digit] = here + all;
        wave_in_order();
    }
}

constexpr int SORT_EACH = 4, SORT_WAVES = SORT_THREADS / 64, SORT_ROUND = SORT_THREADS * SORT_EACH;

// Each digit's number in a workgroup's tokens
__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(SortArgs a)
{
    __shared__ int count[SORT_WAVES][DIGITS];
    const int k = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
#pragma unroll
    for (int w = 0; w < SORT_WAVES; ++w) count[w][tid] = 0;
    __syncthreads();
    const long long start = blockIdx.x * a.per, stop = min(a.N, start + a.per);
    for (long long from = start + wave * (SORT_EACH * 64); from < stop; from += SORT_ROUND) {
        const int left = (int)min(stop - from, (long long)SORT_EACH * 64);
        uint32_t key[SORT_EACH];
        int rank[SORT_EACH];
#pragma unroll
        for (int i = 0; i < SORT_EACH; ++i) key[i] = sort_key(a, k, from + min(i * 64 + lane, left - 1));
        rank_keys<SORT_EACH>(key, left, a.shift, a.bits, count[wave], rank);
    }
    __syncthreads();
    int sum = 0;
#pragma unroll
    for (int w = 0; w < SORT_WAVES; ++w) sum += count[w][tid];
    a.counts[((long long)k * gridDim.x + blockIdx.x) * DIGITS + tid] = sum;
}

// A workgroup moves its tokens in rounds, in which each wavefront has a run of them; DIGITS = SORT_THREADS: a thread has a digit
__global__ __launch_bounds__(SORT_THREADS) void sort_move_kernel(SortArgs a)
{
    static_assert(DIGITS == SORT_THREADS, "a thread has a digit");
    __shared__ int start[DIGITS], to[SORT_WAVES][DIGITS], sums[SORT_WAVES];
    const int k = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const long long begin = blockIdx.x * a.per, stop = min(a.N, begin + a.per);
    const int *const c = a.counts + (long long)k * gridDim.x * DIGITS + tid;
    int total = 0, next = 0;
#pragma unroll 16
    for (unsigned b = 0; b < gridDim.x; ++b) {
        const int n = c[b * DIGITS];
        total += n;
        next += b < blockIdx.x ? n : 0;
    }
    start[tid] = total;
    __syncthreads();
    sums_before<SORT_THREADS>(start, sums);
    next += start[tid];                        // where this digit's next one goes
    for (long long round = begin; round < stop; round += SORT_ROUND) {
        const long long from = round + wave * (SORT_EACH * 64);
        const int left = (int)max(0ll, min(stop - from, (long long)SORT_EACH * 64));
        uint32_t key[SORT_EACH];
        int place[SORT_EACH], rank[SORT_EACH];
        if (left > 0)
#pragma unroll
            for (int i = 0; i < SORT_EACH; ++i) {
                const long long j = from + min(i * 64 + lane, left - 1);
                key[i] = sort_key(a, k, j);
                place[i] = a.tokens != nullptr ? (int)j : a.place_in[k * a.N + j];
            }
#pragma unroll
        for (int w = 0; w < SORT_WAVES; ++w) to[w][tid] = 0;
        __syncthreads();
        rank_keys<SORT_EACH>(key, left, a.shift, a.bits, to[wave], rank);
        __syncthreads();
#pragma unroll
        for (int w = 0; w < SORT_WAVES; ++w) { const int n = to[w][tid]; to[w][tid] = next; next += n; }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < SORT_EACH; ++i)
            if (i * 64 + lane < left) {
                const long long at = k * a.N + to[wave][(key[i] >> a.shift) & ((1u << a.bits) - 1)] + rank[i];
                a.keys[at] = key[i];
                a.place[at] = place[i];
            }
        __syncthreads();
    }
}

// Few tokens: all passes in LDS.  A pass takes a wavefront's run of the list into registers before it is written again.
template <int MOST>
__global__ __launch_bounds__(SMALL_THREADS) void sort_small_kernel(SortArgs a)
{
    constexpr int WAVES = SMALL_THREADS / 64, EACH = MOST / SMALL_THREADS;
    __shared__ uint32_t keys[MOST];
    __shared__ uint16_t place[MOST];
    __shared__ int start[DIGITS], to[WAVES][DIGITS], sums[WAVES];
    if (blockIdx.x >= (unsigned)a.K) {
        const long long nth = blockIdx.x - (unsigned)a.K, k = nth / a.clear.groups;
        clear_rows(a.clear, (int)k, nth - k * a.clear.groups);
        return;
    }
    const int k = blockIdx.x, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63, N = (int)a.N;
    const int run = (N + SMALL_THREADS - 1) / SMALL_THREADS * 64, from = min(N, wave * run), left = min(N - from, run);
    uint32_t key[EACH];
    int at[EACH], rank[EACH];
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
        const int j = i * 64 + lane;
        key[i] = j < left ? key_of(a.tokens[(long long)k * N + from + j], a.V) : 0;
        at[i] = from + j;
    }
    for (int pass = 0; pass < a.passes; ++pass) {
        const int shift = pass * a.bits;
        for (int i = tid; i < WAVES * DIGITS; i += SMALL_THREADS) (&to[0][0])[i] = 0;
        __syncthreads();
        rank_keys<EACH>(key, left, shift, a.bits, to[wave], rank);
        __syncthreads();
        int n[WAVES], all = 0;
        if (tid < DIGITS) {
#pragma unroll
            for (int w = 0; w < WAVES; ++w) { n[w] = to[w][tid]; all += n[w]; }
            start[tid] = all;
        }
        __syncthreads();
        sums_before<SMALL_THREADS>(start, sums);
        if (tid < DIGITS) {
            int here = start[tid];
#pragma unroll
            for (int w = 0; w < WAVES; ++w) { to[w][tid] = here; here += n[w]; }
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < EACH; ++i)
            if (i * 64 + lane < left) {
                const int j = to[wave][(key[i] >> shift) & ((1u << a.bits) - 1)] + rank[i];
                keys[j] = key[i];
                place[j] = (uint16_t)at[i];
            }
        __syncthreads();
        if (pass + 1 < a.passes) {
#pragma unroll
            for (int i = 0; i < EACH; ++i) {
                const int j = min(from + i * 64 + lane, N - 1);
                key[i] = keys[j];
                at[i] = place[j];
            }
        }
    }
    for (int i = tid; i < N; i += SMALL_THREADS) {
        a.keys[(long long)k * N + i] = keys[i];
        a.place[(long long)k * N + i] = place[i];
    }
}

// ---------------------------------------------------------------------------------------------------
// sums of the sorted rows
// ---------------------------------------------------------------------------------------------------
struct GradArgs {
    const void *dy;
    const uint32_t *keys;
    const int *place;
    void *out;
    float *parts;                              // [K][chunks][2][d]: of a chunk's first sum, which began before it, and of its last, which goes on
    long long N, V, chunks, s_dy, s_out, s_worker;
    long long chunk_groups;                    // workgroups with chunks; those behind clear rows
    int d, lanes, chunk, clear_rows, clear_lanes;
    float scale;
    bool add;
};

// Elements of a store that clears: 16 bytes, in rows of E elements at least
constexpr int clear_elements(int E, int size) { return E < 16 / size ? E : 16 / size; }

template <typename TO, int E>
__device__ __forceinline__ void finish_run(const GradArgs &a, int k, uint32_t v, const Run &r, const float (&sum)[E])
{
    TO *const to = (TO *)a.out + k * a.s_worker + (long long)v * a.s_out + r.at;
    float x[E];
#pragma unroll
    for (int u = 0; u < E; ++u) x[u] = a.scale * sum[u];
    if (a.add) {
        float old[E];
        load_wide<TO, E, false>(to, old);
#pragma unroll
        for (int u = 0; u < E; ++u) x[u] += old[u];
    }
    store_run<TO, E>(to, x, r.skip);
}

// The first place in the worker's sorted keys that holds v or more
__device__ __forceinline__ long long first_of(const uint32_t *keys, long long from, long long N, uint32_t v)
{
    long long lo = from, hi = N;
    while (lo < hi) {
        const long long mid = (lo + hi) >> 1;
        if (keys[mid] < v) lo = mid + 1;
        else hi = mid;
    }
    return lo;
}

constexpr int CHUNK_MOST = 32;                 // tokens to a chunk
template <typename TI, typename TO, int E>
__global__ __launch_bounds__(EMBED_THREADS) void embedding_sums_kernel(GradArgs a)
{
    __shared__ uint32_t skey[EMBED_THREADS / 16 * CHUNK_MOST];
    __shared__ int splace[EMBED_THREADS / 16 * CHUNK_MOST];
    const int k = blockIdx.y, lane = threadIdx.x & (a.lanes - 1), place = threadIdx.x / a.lanes, side = EMBED_THREADS / a.lanes;
    const uint32_t *const keys = a.keys + k * a.N;
    if ((long long)blockIdx.x >= a.chunk_groups) {
        if (blockIdx.z != 0) return;
        const long long v0 = ((long long)blockIdx.x - a.chunk_groups) * a.clear_rows, rows = min((long long)a.clear_rows, a.V - v0);
        for (int i = threadIdx.x; i < rows; i += EMBED_THREADS) {
            const long long at = first_of(keys, 0, a.N, (uint32_t)(v0 + i));
            skey[i] = at < a.N && keys[at] == (uint32_t)(v0 + i);
        }
        __syncthreads();
        // 16 bytes to a lane, as many rows side by side as the workgroup's lanes hold
        constexpr int C = clear_elements(E, (int)sizeof(TO));
        const float zero[C] = {};
        for (int i = threadIdx.x / a.clear_lanes; i < rows; i += EMBED_THREADS / a.clear_lanes) {
            if (skey[i]) continue;
            TO *const to = (TO *)a.out + k * a.s_worker + (v0 + i) * a.s_out;
            for (int c = (threadIdx.x & (a.clear_lanes - 1)) * C; c < a.d; c += a.clear_lanes * C) store_wide<TO, C, true>(to + min(c, a.d - C), zero);
        }
        return;
    }
    const int first = ((int)blockIdx.z * a.lanes + lane) * E;
    const Run run = run_of(min(first, a.d - 1), a.d, E);
    const long long c0 = (long long)blockIdx.x * side * a.chunk;
    for (int i = threadIdx.x; i < side * a.chunk; i += EMBED_THREADS) {
        const bool in = c0 + i < a.N;
        skey[i] = in ? keys[c0 + i] : (uint32_t)a.V;
        splace[i] = in ? a.place[k * a.N + c0 + i] : 0;
    }
    __syncthreads();
    const long long chunk = (long long)blockIdx.x * side + place, from = chunk * a.chunk;
    if (first >= a.d || from >= a.N) return;
    const uint32_t *const ck = skey + place * a.chunk;
    const int *const cp = splace + place * a.chunk;
    const uint32_t none = (uint32_t)a.V;
    uint32_t cur = ck[0];
    if (cur == none) return;
    bool begun = from > 0 && keys[from - 1] == cur;                        // the first sum began before this chunk
    float sum[E] = {};
    const TI *const dy = (const TI *)a.dy + k * a.N * a.s_dy + run.at;
    float *const parts = a.parts + (k * a.chunks + chunk) * 2 * a.d + run.at;
    for (int i = 0; i < a.chunk; i += 8) {
        typename Wide<TI, E>::vec v[8];
#pragma unroll
        for (int u = 0; u < 8; ++u) v[u] = __builtin_nontemporal_load((const typename Wide<TI, E>::vec *)(dy + cp[i + u] * a.s_dy));
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const uint32_t key = ck[i + u];
            if (key != cur) {
                if (cur != none) {
                    if (begun) store_run<float, E>(parts, sum, run.skip);
                    else finish_run<TO, E>(a, k, cur, run, sum);
                }
                begun = false;
                cur = key;
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] = 0.f;
            }
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += (float)v[u][e];
        }
    }
    if (cur == none) return;
    const bool on = from + a.chunk < a.N && keys[from + a.chunk] == cur;
    if (begun) store_run<float, E>(parts, sum, run.skip);
    else if (on) store_run<float, E>(parts + a.d, sum, run.skip);
    else finish_run<TO, E>(a, k, cur, run, sum);
}

// A sum that goes on behind the chunk in which it begins: its parts, every fourth to a wavefront, in their order.  One workgroup to a chunk,
// most of which have nothing to do, and 64 E columns.
template <typename TO, int E>
__global__ __launch_bounds__(EMBED_THREADS) void embedding_join_kernel(GradArgs a)
{
    constexpr int WAVES = EMBED_THREADS / 64;
    __shared__ float red[WAVES][64][E + 1];
    const int k = blockIdx.y, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const uint32_t *const keys = a.keys + k * a.N;
    const long long chunk = blockIdx.x, from = chunk * a.chunk, end = from + a.chunk;
    if (end >= a.N) return;
    // all of these at once: most chunks have nothing here, and then it is their latency that counts.  Chunk + 1 + i has no other token
    // if its last is v, since the list is in order; the last chunk of the sum is the one behind those.
    const uint32_t before = keys[max(from, 1ll) - 1], start = keys[from], v = keys[end - 1], next = keys[end];
    auto whole = [&](long long i) { const long long e = end + (i + lane + 1) * a.chunk; return e <= a.N && keys[min(e, a.N) - 1] == v; };
    bool mine = whole(0);
    if (v == (uint32_t)a.V || next != v || (start == v && from > 0 && before == v)) return;
    long long count = 0;
    for (;;) {
        const uint64_t others = ~__ballot(mine);
        if (others != 0) { count += __ffsll((unsigned long long)others) - 1; break; }
        count += 64;
        mine = whole(count);
    }
    // behind `count` whole chunks one more has a part, unless it begins with another token or is not there
    const long long behind = end + count * a.chunk;
    const long long last = chunk + count + (behind < a.N && keys[behind] == v ? 1 : 0);       // chunk + 1 .. last: first sums of theirs
    const int first = ((int)blockIdx.z * 64 + lane) * E;
    const Run run = run_of(min(first, a.d - 1), a.d, E);
    const float *const parts = a.parts + (k * a.chunks + chunk) * 2 * a.d + run.at;
    float sum[E] = {};
    for (long long i = wave; i <= last - chunk; i += 8 * WAVES) {
        float x[8][E];
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            const long long j = min(i + u * WAVES, last - chunk);
            load_wide<float, E, false>(j == 0 ? parts + a.d : parts + 2 * j * a.d, x[u]);
        }
#pragma unroll
        for (int u = 0; u < 8; ++u)
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += i + u * WAVES <= last - chunk ? x[u][e] : 0.f;
    }
#pragma unroll
    for (int e = 0; e < E; ++e) red[wave][lane][e] = sum[e];
    __syncthreads();
    if (wave != 0 || first >= a.d) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w)
#pragma unroll
        for (int e = 0; e < E; ++e) sum[e] += red[w][lane][e];
    finish_run<TO, E>(a, k, v, run, sum);
}

// ---------------------------------------------------------------------------------------------------
// few tokens: all of it in one launch
// ---------------------------------------------------------------------------------------------------
constexpr int DIRECT_TOKENS = 2048, DIRECT_ROWS = 64;      // of a worker; of the table, to a workgroup

struct DirectArgs {
    const void *dy;
    const int64_t *tokens;
    void *out;
    long long V, s_dy, s_out, s_worker;
    int N, d, lanes, rows;                     // rows of the table to a workgroup
    float scale;
    bool add;
};

// A workgroup has some rows of the table and L * E columns.  It goes through all tokens of the worker, each wavefront through a run of
// them, sorts those that are its own in LDS, gives each group of lanes the same number of them, and joins the sums that several groups have a part in.
template <typename TI, typename TO, int E>
__global__ __launch_bounds__(EMBED_THREADS) void embedding_direct_kernel(DirectArgs a)
{
    constexpr int WAVES = EMBED_THREADS / 64, RUN = DIRECT_TOKENS / WAVES;
    __shared__ uint32_t found[WAVES][RUN], list[DIRECT_TOKENS];            // a row's number among the workgroup's, and a place
    __shared__ int to[WAVES][DIRECT_ROWS], start[DIRECT_ROWS + 1];
    __shared__ float parts[EMBED_THREADS * E];
    const int k = blockIdx.y, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
    const long long v0 = (long long)blockIdx.x * a.rows;
    const int rows = (int)min((long long)a.rows, a.V - v0);
    to[wave][lane] = 0;
    const int run = (a.N + EMBED_THREADS - 1) / EMBED_THREADS * 64, from = min(a.N, wave * run), end = min(a.N, from + run);
    int mine = 0;
    long long tok[RUN / 64];                   // all of them on their way at once
#pragma unroll
    for (int i = 0; i < RUN / 64; ++i)
        if (from + i * 64 < end) tok[i] = a.tokens[(long long)k * a.N + min(from + i * 64 + lane, end - 1)];
#pragma unroll
    for (int i = 0; i < RUN / 64; ++i) {
        const int j = from + i * 64 + lane;
        if (from + i * 64 >= end) break;
        const long long row = tok[i] - v0;
        const bool in = j < end && row >= 0 && row < rows;
        const uint64_t mask = __ballot(in);
        if (in) {
            found[wave][mine + __popcll(mask & ((1ull << lane) - 1))] = (uint32_t)row << 16 | (uint32_t)j;
            atomicAdd(&to[wave][row], 1);
        }
        mine += __popcll(mask);
    }
    __syncthreads();
    if (wave == 0) {                           // DIRECT_ROWS = 64: a lane to a row
        int n[WAVES], all = 0;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) { n[w] = to[w][lane]; all += n[w]; }
        int upto = all;
#pragma unroll
        for (int o = 1; o < 64; o <<= 1) { const int v = __shfl_up(upto, o, 64); upto += lane >= o ? v : 0; }
        int at = upto - all;
        start[lane] = at;
        if (lane == 63) start[64] = upto;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) { to[w][lane] = at; at += n[w]; }
    }
    __syncthreads();
    for (int i = 0; i < mine; i += 64) {
        const bool in = i + lane < mine;
        const uint32_t entry = found[wave][min(i + lane, mine - 1)], row = entry >> 16;
        int before, all;
        same_digit(row, in, 6, before, all);
        const int at = to[wave][row];
        if (in) list[at + before] = entry;
        wave_in_order();
        if (in && before == 0) to[wave][row] = at + all;
        wave_in_order();
    }
    __syncthreads();
    const int groups = EMBED_THREADS / a.lanes, group = tid / a.lanes, place = tid & (a.lanes - 1), M = start[64], each = (M + groups - 1) / groups;
    const int first = ((int)blockIdx.z * a.lanes + place) * E;
    const Run r = run_of(min(first, a.d - 1), a.d, E);
    const bool in = first < a.d;
    auto write = [&](int row, const float (&sum)[E]) {
        TO *const p = (TO *)a.out + k * a.s_worker + (v0 + row) * a.s_out + r.at;
        float x[E];
#pragma unroll
        for (int u = 0; u < E; ++u) x[u] = a.scale * sum[u];
        if (a.add) {
            float old[E];
            load_wide<TO, E, false>(p, old);
#pragma unroll
            for (int u = 0; u < E; ++u) x[u] += old[u];
        }
        store_run<TO, E>(p, x, r.skip);
    };
    const int c0 = min(M, group * each), c1 = min(M, c0 + each);
    float sum[E] = {};
    int cur = -1;
    bool begun = false, on = false;
    float *const own = parts + tid * E;        // of the first sum, where it began before
    if (in && c0 < c1) {
        const TI *const dy = (const TI *)a.dy + (long long)k * a.N * a.s_dy + r.at;
        cur = (int)(list[c0] >> 16);
        begun = c0 > 0 && (int)(list[c0 - 1] >> 16) == cur;
        for (int i = c0; i < c1; i += 8) {
            typename Wide<TI, E>::vec v[8];
#pragma unroll
            for (int u = 0; u < 8; ++u)
                v[u] = __builtin_nontemporal_load((const typename Wide<TI, E>::vec *)(dy + (long long)(list[min(i + u, c1 - 1)] & 0xffff) * a.s_dy));
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (i + u >= c1) break;
                const int row = (int)(list[i + u] >> 16);
                if (row != cur) {
                    if (begun) {
#pragma unroll
                        for (int e = 0; e < E; ++e) own[e] = sum[e];
                    } else write(cur, sum);
                    begun = false;
                    cur = row;
#pragma unroll
                    for (int e = 0; e < E; ++e) sum[e] = 0.f;
                }
#pragma unroll
                for (int e = 0; e < E; ++e) sum[e] += (float)v[u][e];
            }
        }
        on = !begun && c1 < M && (int)(list[c1] >> 16) == cur;
        if (begun) {
#pragma unroll
            for (int e = 0; e < E; ++e) own[e] = sum[e];
        } else if (!on) write(cur, sum);
    }
    __syncthreads();
    if (!in) return;
    if (on) {                                  // the row's other parts, in their order
        const int last = (start[cur + 1] - 1) / each;
        for (int g = group + 1; g <= last; ++g)
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += parts[(g * a.lanes + place) * E + e];
        write(cur, sum);
    }
    if (a.add) return;
    const float zero[E] = {};
    for (int row = group; row < rows; row += groups)
        if (start[row] == start[row + 1]) store_run<TO, E>((TO *)a.out + k * a.s_worker + (v0 + row) * a.s_out + r.at, zero, r.skip);
}

// ---------------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------------
constexpr long long EMBED_MOST = 1ll << 27;    // tokens of a worker

// Elements of a lane: 16 bytes of the wider of what is read and what is written, so that what is written streams in whole lines (8 x 8192
// tokens over 32768 rows of 768, rows in bf16, the table's gradient in fp32: 222 us a pass, lookup included, 239 with 32 bytes of a lane to write)
template <typename TI, typename TO> constexpr int lane_elements() { return wide_of<TI>() < wide_of<TO>() ? wide_of<TI>() : wide_of<TO>(); }

static int lanes_for(long long d, int E)
{
    const long long runs = (d + E - 1) / E;
    int L = 16;
    while (L < EMBED_THREADS && L < runs) L <<= 1;
    return L;
}

// Rows of the table to a workgroup that goes through all tokens: as many as make some thousand workgroups
static int direct_rows(long long K, long long V)
{
    const long long rows = (K * V + 1023) / 1024;
    return (int)(rows > DIRECT_ROWS ? DIRECT_ROWS : rows);
}
// Few tokens with little in their rows, and not too many workgroups that read all of the tokens: one launch.  A workgroup with several rows
// of the table may have a third of all tokens, if the first rows are the frequent ones.  us with one launch / with a sort: 4 x 1024
// tokens over 512 rows of 128 in bf16 5.6 / 15.1, 64 over 200000 of 64 8.5 / 12.2, 8 x 1000 over 100 of 700 in fp32 9.3 / 19.1, 2000 over 16 of 512
// in bf16 10.8 / 12.8; but 2000 over 2 of 512 45 / 14, 2048, the first rows frequent, over 32768 of 512 40 / 17, 8 x 2048 over 200000 of 64 80 / 48.
static bool direct(long long K, long long N, long long V, long long d, int size)
{
    if (N < 1 || N > DIRECT_TOKENS) return false;
    const long long rows = direct_rows(K, V), bytes = N * d * size;
    if (bytes > (rows > 1 ? 1 << 19 : 1 << 21) || bytes * rows > V * (1 << 17)) return false;
    return K * ((V + rows - 1) / rows) * N * 8 <= (1 << 27);
}

// How the tokens of K workers are sorted and summed, and where what lies in the workspace
struct GradPlan {
    int passes, bits, chunk;
    long long blocks, per, chunks;
    size_t keys[2], place[2], counts, parts, bytes;
};
static GradPlan grad_plan(int K, long long N, long long V, long long d, int E)
{
    GradPlan p;
    int bits = 1;
    while (bits < 32 && ((uint64_t)V >> bits) != 0) ++bits;                // V itself is a key
    p.passes = (bits + 8) / 9;
    p.bits = (bits + p.passes - 1) / p.passes;
    p.per = SORT_ROUND;
    while ((N + p.per - 1) / p.per > 128) p.per *= 2;
    // One pass of many workgroups takes less than that of one from 8192 tokens on (16384 of 400 rows of 64, sums included 23.5 us, 27.8), two of them
    // do not (16384 of 100000 rows of 1024 80, 59)
    p.blocks = N <= (p.passes > 1 ? SORT_SMALL : SORT_SMALL / 2) ? 0 : (N + p.per - 1) / p.per;
    const long long waves = (long long)K * ((N + CHUNK_MOST - 1) / CHUNK_MOST) * ((d + 64 * E - 1) / (64 * E));
    p.chunk = waves < 2048 ? 8 : CHUNK_MOST;
    p.chunks = (N + p.chunk - 1) / p.chunk;
    size_t at = 0;
    auto take = [&](size_t n) { const size_t here = at; at += (n + 255) / 256 * 256; return here; };
    const size_t list = (size_t)K * (size_t)N * 4;
    for (int i = 0; i < (p.blocks ? 2 : 1); ++i) { p.keys[i] = take(list); p.place[i] = take(list); }
    if (!p.blocks) { p.keys[1] = p.keys[0]; p.place[1] = p.place[0]; }
    p.counts = take((size_t)K * (size_t)p.blocks * DIGITS * 4);
    p.parts = take((size_t)K * (size_t)p.chunks * 2 * (size_t)d * 4);
    p.bytes = N > 0 ? at : 0;
    return p;
}

template <typename TI, typename TO, int E>
static hipError_t launch_sums(GradArgs &a, const GradPlan &p, int K, bool cleared, hipStream_t s)
{
    a.lanes = lanes_for(a.d, E);
    const int side = EMBED_THREADS / a.lanes, slices = (int)((a.d + (long long)a.lanes * E - 1) / ((long long)a.lanes * E));
    a.chunk_groups = (p.chunks + side - 1) / side;
    // some 128 KiB to a workgroup that clears, and a row to each of its threads at most
    const long long row = (long long)a.d * (long long)sizeof(TO), rows = (131072 + row - 1) / row;
    a.clear_rows = (int)(rows < EMBED_THREADS ? rows : EMBED_THREADS);
    a.clear_lanes = lanes_for(a.d, clear_elements(E, (int)sizeof(TO)));
    const long long clears = a.add || cleared ? 0 : (a.V + a.clear_rows - 1) / a.clear_rows;
    if (a.chunk_groups + clears > 0)
        embedding_sums_kernel<TI, TO, E><<<dim3((unsigned)(a.chunk_groups + clears), (unsigned)K, (unsigned)slices), EMBED_THREADS, 0, s>>>(a);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || p.chunks < 2) return e;
    constexpr int J = E < 4 ? 1 : 4;
    embedding_join_kernel<TO, J><<<dim3((unsigned)(p.chunks - 1), (unsigned)K, (unsigned)((a.d + 64 * J - 1) / (64 * J))), EMBED_THREADS, 0, s>>>(a);
    return hipGetLastError();
}

template <typename TI, typename TO, int E>
static hipError_t launch_direct(DirectArgs &a, int K, hipStream_t s)
{
    a.lanes = lanes_for(a.d, E);
    const dim3 grid((unsigned)((a.V + a.rows - 1) / a.rows), (unsigned)K, (unsigned)((a.d + (long long)a.lanes * E - 1) / ((long long)a.lanes * E)));
    embedding_direct_kernel<TI, TO, E><<<grid, EMBED_THREADS, 0, s>>>(a);
    return hipGetLastError();
}

template <typename TI, typename TO>
static hipError_t launch_lookup(LookupArgs &a, int K, hipStream_t s)
{
    constexpr int E = lane_elements<TI, TO>();
    a.lanes = lanes_for(a.d, a.d < E ? 1 : E);
    const long long side = EMBED_THREADS / a.lanes, trips = (a.N + side - 1) / side;
    const dim3 grid((unsigned)(trips < (1 << 20) ? trips : 1 << 20), (unsigned)K);
    if (a.d < E) embedding_kernel<TI, TO, 1><<<grid, EMBED_THREADS, 0, s>>>(a);
    else embedding_kernel<TI, TO, E><<<grid, EMBED_THREADS, 0, s>>>(a);
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
static bool is_type(int t) { return t == QSR_TYPE_F32 || t == QSR_TYPE_BF16; }
static uintptr_t size_of(int type) { return type == QSR_TYPE_F32 ? 4 : 2; }
static bool sizes_ok(int32_t K, int64_t N, int64_t V, int64_t d)
{
    return K >= 1 && K <= 65535 && N >= 0 && V >= 1 && V < ((int64_t)1 << 31) && d >= 1 && d <= ((int64_t)1 << 22);
}
// elements of a run: 16 bytes of the rows that are read, or one in rows that are shorter
static int run_elements(int type, int64_t d)
{
    const int E = type == QSR_TYPE_F32 ? 4 : 8;
    return d < E ? 1 : E;
}

// Whether n rows of `len` bytes, `stride` apart from `at` on, share memory with K tables of V rows of `row` bytes, `step` apart, `worker` from
// table to table.  Rows between the table's, as far apart as those, share none; others that begin and end within a table are taken to.
typedef __int128 Bytes;                        // (strides are whatever the caller gave)
static bool shares(const void *at, Bytes n, Bytes stride, Bytes len, const void *table, int K, Bytes worker, Bytes V, Bytes step, Bytes row)
{
    const Bytes p = (Bytes)(uintptr_t)at, t = (Bytes)(uintptr_t)table, extent = (V - 1) * step + row;
    if (n == 1) stride = step;
    auto apart = [&](Bytes from, Bytes to) { return p >= to || p + (n - 1) * stride + len <= from; };
    if (apart(t, t + (K - 1) * worker + extent)) return false;
    for (int k = 0; k < K; ++k) {
        const Bytes from = t + k * worker, to = from + extent;
        if (apart(from, to)) continue;
        const Bytes i = p + len > from ? 0 : (from - p - len) / stride + 1;                // the first row that ends behind `from`
        if (i >= n || p + i * stride >= to) continue;
        const Bytes within = ((p - from) % step + step) % step;
        if (stride != step || within < row || within + len > step) return true;
    }
    return false;
}

extern "C" int qsr_embedding(const qsr_embedding_args *q, void *stream)
{
    if (!q || !sizes_ok(q->K, q->tokens_each, q->vocab, q->d) || !is_type(q->type) || !is_type(q->y_type)) return QSR_EINVAL;
    if (!std::isfinite((float)q->scale)) return QSR_EINVAL;
    if (q->tokens_each > EMBED_MOST) return QSR_ELIMIT;
    if (q->tokens_each == 0) return QSR_OK;
    if (!q->table || off(q->table, size_of(q->type)) || !q->tokens || off(q->tokens, 8) || !q->y || off(q->y, size_of(q->y_type))) return QSR_EINVAL;
    if (q->table_stride < q->d || q->y_stride < q->d || (q->K > 1 && q->worker_stride < q->d)) return QSR_EINVAL;
    LookupArgs a{q->table, q->tokens, q->y, q->tokens_each, q->vocab, q->table_stride, q->worker_stride, q->y_stride, (int)q->d, 0, (float)q->scale};
    const hipStream_t s = (hipStream_t)stream;
    const bool wide = q->y_type == QSR_TYPE_F32;
    return finish(q->type == QSR_TYPE_F32 ? (wide ? launch_lookup<float, float>(a, q->K, s) : launch_lookup<float, bf16_t>(a, q->K, s))
                                          : (wide ? launch_lookup<bf16_t, float>(a, q->K, s) : launch_lookup<bf16_t, bf16_t>(a, q->K, s)));
}

extern "C" int qsr_embedding_workspace_bytes(int32_t K, int64_t tokens_each, int64_t vocab, int64_t d, int32_t type, size_t *bytes)
{
    if (!bytes) return QSR_EINVAL;
    *bytes = 0;
    if (!sizes_ok(K, tokens_each, vocab, d) || !is_type(type)) return QSR_EINVAL;
    if (tokens_each > EMBED_MOST) return QSR_ELIMIT;
    if (!direct(K, tokens_each, vocab, d, (int)size_of(type))) *bytes = grad_plan(K, tokens_each, vocab, d, run_elements(type, d)).bytes;
    return QSR_OK;
}

extern "C" int qsr_embedding_backward(const qsr_embedding_backward_args *q, void *workspace, size_t workspace_bytes, void *stream)
{
    if (!q || !sizes_ok(q->K, q->tokens_each, q->vocab, q->d) || !is_type(q->type) || !is_type(q->grad_type)) return QSR_EINVAL;
    if (!std::isfinite((float)q->scale) || (q->accumulate != 0 && q->accumulate != 1)) return QSR_EINVAL;
    if (!q->grad || off(q->grad, size_of(q->grad_type)) || q->grad_stride < q->d) return QSR_EINVAL;
    if (q->K > 1 && q->worker_stride < (q->vocab - 1) * q->grad_stride + q->d) return QSR_EINVAL;
    if (q->tokens_each > 0 && (!q->y_grad || off(q->y_grad, size_of(q->type)) || !q->tokens || off(q->tokens, 8) || q->y_grad_stride < q->d))
        return QSR_EINVAL;
    size_t need = 0;
    const int rc = qsr_embedding_workspace_bytes(q->K, q->tokens_each, q->vocab, q->d, q->type, &need);
    if (rc != QSR_OK) return rc;
    if (need > 0 && (!workspace || off(workspace, 16))) return QSR_EINVAL;
    if (workspace_bytes < need) return QSR_ENOMEM;
    // rows of the table are cleared or written before all of y_grad and tokens has been read
    const Bytes es = (Bytes)size_of(q->type), gs = (Bytes)size_of(q->grad_type), tokens = (Bytes)q->K * q->tokens_each, apart = q->K > 1 ? gs * q->worker_stride : 0;
    if (tokens > 0 && (shares(q->y_grad, tokens, es * q->y_grad_stride, es * q->d, q->grad, q->K, apart, q->vocab, gs * q->grad_stride, gs * q->d) ||
                       shares(q->tokens, 1, 8, 8 * tokens, q->grad, q->K, apart, q->vocab, gs * q->grad_stride, gs * q->d)))
        return QSR_EINVAL;
    const hipStream_t s = (hipStream_t)stream;
    const int K = q->K, E = run_elements(q->type, q->d);
    const long long N = q->tokens_each;
    const bool wide = q->grad_type == QSR_TYPE_F32;
#define EMBED_BY_TYPE(F) (q->type == QSR_TYPE_F32 ? (wide ? F(float, float) : F(float, bf16_t)) : (wide ? F(bf16_t, float) : F(bf16_t, bf16_t)))
    if (direct(K, N, q->vocab, q->d, (int)size_of(q->type))) {
        DirectArgs a{q->y_grad, q->tokens, q->grad, q->vocab, q->y_grad_stride, q->grad_stride, q->worker_stride, (int)N, (int)q->d, 0,
                     direct_rows(K, q->vocab), (float)q->scale, q->accumulate != 0};
#define EMBED_DIRECT(TI, TO) (E == 1 ? launch_direct<TI, TO, 1>(a, K, s) : launch_direct<TI, TO, lane_elements<TI, TO>()>(a, K, s))
        return finish(EMBED_BY_TYPE(EMBED_DIRECT));
#undef EMBED_DIRECT
    }
    const GradPlan p = grad_plan(K, N, q->vocab, q->d, E);
    char *const ws = (char *)workspace;
    int done = 0;                              // which of the two lists holds the result
    // A sort by one workgroup leaves most of the chip idle, which clears the tables meanwhile, though some rows are written again then.  us with
    // that / with rows cleared that a search in the list does not find: 16384 tokens over 100000 rows of 1024 in bf16 59 / 87, 8 x 8192 over
    // 32768 of 768 in fp32 197 / 213, all tokens equally likely 199 / 198.  The launches of a sort by many are too short for it: 32768
    // tokens over 50000 rows of 4096 in fp32 371 / 308.
    const bool cleared = p.blocks == 0 && N > 0 && !q->accumulate;
    if (N > 0) {
        SortArgs a{};
        a.tokens = q->tokens;
        a.keys = (uint32_t *)(ws + p.keys[0]);
        a.place = (int *)(ws + p.place[0]);
        a.counts = (int *)(ws + p.counts);
        a.N = N;
        a.V = q->vocab;
        a.per = p.per;
        a.bits = p.bits;
        a.passes = p.passes;
        a.K = K;
        if (cleared) {
            Clear &c = a.clear;
            const long long es = (long long)size_of(q->grad_type);
            c.out = (char *)q->grad;
            c.V = q->vocab;
            c.row = (int)(q->d * es);
            c.s_row = q->grad_stride * es;
            c.s_worker = K > 1 ? q->worker_stride * es : 0;
            c.rows = 131072 / c.row > 1 ? 131072 / c.row : 1;
            c.lanes = lanes_for(c.row, c.row < 16 ? 2 : 16);
            c.groups = (c.V + c.rows - 1) / c.rows;
        }
        hipError_t e = hipSuccess;
        if (p.blocks == 0) {
            const dim3 grid((unsigned)(K + K * a.clear.groups));
            if (N <= SORT_SMALL / 4) sort_small_kernel<SORT_SMALL / 4><<<grid, SMALL_THREADS, 0, s>>>(a);
            else sort_small_kernel<SORT_SMALL><<<grid, SMALL_THREADS, 0, s>>>(a);
            e = hipGetLastError();
        }
        for (int pass = 0; p.blocks > 0 && pass < p.passes && e == hipSuccess; ++pass) {
            done = pass & 1;
            a.keys = (uint32_t *)(ws + p.keys[done]);
            a.place = (int *)(ws + p.place[done]);
            if (pass > 0) { a.tokens = nullptr; a.keys_in = (uint32_t *)(ws + p.keys[done ^ 1]); a.place_in = (int *)(ws + p.place[done ^ 1]); }
            a.shift = pass * p.bits;
            const dim3 grid((unsigned)p.blocks, (unsigned)K);
            sort_count_kernel<<<grid, SORT_THREADS, 0, s>>>(a);
            e = hipGetLastError();
            if (e == hipSuccess) sort_move_kernel<<<grid, SORT_THREADS, 0, s>>>(a);
            if (e == hipSuccess) e = hipGetLastError();
        }
        if (e != hipSuccess) return finish(e);
    }
    GradArgs a{q->y_grad, (const uint32_t *)(ws + p.keys[done]), (const int *)(ws + p.place[done]), q->grad, (float *)(ws + p.parts), N, q->vocab, p.chunks,
               q->y_grad_stride, q->grad_stride, q->worker_stride, 0, (int)q->d, 0, p.chunk, 0, 0, (float)q->scale, q->accumulate != 0};
#define EMBED_SUMS(TI, TO) (E == 1 ? launch_sums<TI, TO, 1>(a, p, K, cleared, s) : launch_sums<TI, TO, lane_elements<TI, TO>()>(a, p, K, cleared, s))
    return finish(EMBED_BY_TYPE(EMBED_SUMS));
#undef EMBED_SUMS
#undef EMBED_BY_TYPE
}
