// adamw_tensors.hip -- AdamW over a list of tensors in one launch, for K workers, with the moments in 32 or in 8 bits.
//
// For a model of a caller's own, whose parameters are many tensors.  Tensor i holds n_i elements for each worker (rows of any stride).
// One step, n = t + 1:
//   g <- coef_k g                               (clip_norm: coef_k = min(1, c / (||g_k|| + 1e-6)), the norm over all tensors of worker k)
//   m <- m + (1 - beta1)(g - m);  v <- v + (1 - beta2)(g^2 - v);  r = sqrt(v)
//   theta <- theta - [eta lambda_i theta + eta/(1 - beta1^n) m / (r / sqrt(1 - beta2^n) + eps)]
// with the arithmetic of the [K][P] update (opt_elem.h) where the moments are fp32: the same bits.  Where they are held in 8 bits
// every operation that leads to a code is rounded by itself, in the order of the formulas and with no fused ones: a last bit decides
// now and then which of two codes a moment becomes, and so the codes are those of any fp32 implementation of this comment.
// Parameters are fp32: steps are smaller than half a unit of a bf16 parameter.  A copy of the new parameters in bf16, rounded to
// nearest, is written on request.
//
// Moments in 8 bits: each 256 consecutive elements of a worker's tensor are a block with one fp32 scale, a lane of a wavefront holds
// four of them.  m and r (the root: half of v's range of exponents) are e4m3 codes of value * (1 / top * 448), top = max|value| over
// the block's finite values, with the scale top * (1 / 448); a value that is not finite becomes NaN and spoils no other.  Blocks whose
// top is below 1e-35 are stored as zeros: the factor would leave the range of floats.
// Rounding is stochastic (v_cvt_sr_fp8_f32): up with the probability of the part of a step that is left.  An iteration moves r by a
// relative (1 - beta2)/2 = 5e-4, less than a hundredth of a code's step (1/16 to 1/8 of the value): to nearest it would never move.
// A root above zero does not become zero (the smallest code instead): m / r of the next step stays bounded.
// The random words: a 32-bit multiply-xorshift mix (constants from C. Wellons' search for mixes of low bias) of the element's index,
// counted over the padded blocks of all tensors (modulo 2^32), and the step's key; 16 bits for each of the two moments.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <new>
#include <vector>

#include "opt_elem.h"
#include "qsr_internal.h"
#include "row_io.h"

namespace qsr {

constexpr int AT_BLOCK = 256;                  // elements that share a scale
constexpr int AT_SPAN = 2;                     // blocks of a wavefront's trip (four: 900 against 869 us for 2 x 85e6 with fp32 moments)

struct AtTensor {
    float *param;
    const void *grad;
    void *m, *v;
    float *m_scale, *v_scale;
    bf16_t *copy;
    long long n, s_param, s_grad, s_state, s_scale, s_copy;   // elements, and strides from worker to worker
    double decay;
    long long first;                           // blocks of the tensors before this one
};
struct AtChunk { int tensor, block; };         // a trip's first block
struct AtStep { double eta; float step, rsq, c1, c2, eps; uint32_t key; };

// 16 random bits for either moment: index counts the worker's elements over all tensors, padded to blocks
// (plus the worker's number times an odd constant)
__device__ __forceinline__ uint32_t at_word(uint32_t index, uint32_t key)
{
    uint32_t x = index ^ key;
    x ^= x >> 16; x *= 0x21F0AAADu;
    x ^= x >> 15; x *= 0x735A2D97u;
    return x ^ (x >> 15);
}

// A trip's rows, as pointers to its first element
template <typename G> struct AtRows {
    float *th;
    const G *g;
    bf16_t *copy;
    __device__ __forceinline__ AtRows(const AtTensor &t, long long k, long long e)
        : th(global(t.param) + k * t.s_param + e), g(global((const G *)t.grad) + k * t.s_grad + e),
          copy(t.copy != nullptr ? global(t.copy) + k * t.s_copy + e : nullptr) {}
};

// FULL: the trip's elements are all there.  Otherwise `left` are, of which a lane may have four, some or none in each block.
template <typename T, bool FULL>
__device__ __forceinline__ void at_load(const T *p, long long left, float (&v)[4])
{
    if (FULL || left >= 4) load_wide<T, 4, true>(p, v);
    else load_some(p, (int)left, v);
}
template <typename T, bool FULL>
__device__ __forceinline__ void at_store(T *p, long long left, const float (&v)[4])
{
    if (FULL || left >= 4) store_wide<T, 4, true>(p, v);
    else store_some(p, (int)left, v);
}

template <typename G, bool FULL>
__device__ __forceinline__ void at_trip_f32(const AtTensor &t, const AtStep &st, long long k, long long e0, float gs)
{
    const int lane = threadIdx.x;
    const AtRows<G> q(t, k, e0);
    float *const m = global((float *)t.m) + k * t.s_state + e0, *const v = global((float *)t.v) + k * t.s_state + e0;
    const float etalam = (float)(st.eta * t.decay);
    float a[AT_SPAN][4], b[AT_SPAN][4], c[AT_SPAN][4], d[AT_SPAN][4];
#pragma unroll
    for (int u = 0; u < AT_SPAN; ++u) {
        const int i = u * AT_BLOCK + lane * 4;
        const long long left = t.n - e0 - i;
        at_load<float, FULL>(q.th + i, left, a[u]);
        at_load<float, FULL>(m + i, left, c[u]);
        at_load<float, FULL>(v + i, left, d[u]);
        at_load<G, FULL>(q.g + i, left, b[u]);
    }
#pragma unroll
    for (int u = 0; u < AT_SPAN; ++u) {
        const int i = u * AT_BLOCK + lane * 4;
        const long long left = t.n - e0 - i;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            adamw_elem(a[u][j], b[u][j] * gs, c[u][j], d[u][j], etalam, st.step, st.rsq, st.c1, st.c2, st.eps);
        at_store<float, FULL>(q.th + i, left, a[u]);
        at_store<float, FULL>(m + i, left, c[u]);
        at_store<float, FULL>(v + i, left, d[u]);
        if (q.copy != nullptr) at_store<bf16_t, FULL>(q.copy + i, left, a[u]);
    }
}

// The square root, rounded to nearest where x >= 2^-96 (an ulp below that), by trying the neighbours of the instruction's result:
// x lies above s (s + ulp) where s + ulp is nearer, and not above s (s - ulp) where s - ulp is
__device__ __forceinline__ float root(float x)
{
    const float s = __builtin_amdgcn_sqrtf(x);
    const float lo = __int_as_float(__float_as_int(s) - 1), hi = __int_as_float(__float_as_int(s) + 1);
    float r = fmaf(-lo, s, x) <= 0.f ? lo : s;
    r = fmaf(-hi, s, x) > 0.f ? hi : r;
    return r;
}
// One element with 8-bit moments: m, the root r of v, and theta.  What leads to a code is rounded operation by operation; the step
// itself is not held to that (a reciprocal within an ulp).
__device__ __forceinline__ void adamw_rounded(float &th, float g, float &m, float &r, float etalam, const AtStep &st)
{
    {
#pragma clang fp contract(off)
        const float v = r * r;
        m = m + st.c1 * (g - m);
        r = root(v + st.c2 * (g * g - v));
    }
    th = th - fmaf(etalam, th, st.step * m * __builtin_amdgcn_rcpf(fmaf(r, st.rsq, st.eps)));
}
__device__ __forceinline__ float finite_or_zero(float x) { return fabsf(x) < INFINITY ? x : 0.f; }

// The codes of four elements, x * factor to the value below or above; ROOTS: what is not zero does not become zero
template <bool FINITE, bool ROOTS>
__device__ __forceinline__ uint32_t at_codes(const float (&x)[4], float factor, const uint32_t (&word)[4])
{
    int code = 0;
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        y[j] = x[j] * factor;
        // the factor's rounding may take the largest value past 448, which could round to NaN; what is not finite shall become NaN
        y[j] = __builtin_amdgcn_fmed3f(y[j], ROOTS ? E4M3_TINY : -E4M3_MAX, E4M3_MAX);
        if (ROOTS) y[j] = x[j] > 0.f ? y[j] : 0.f;
        if (!FINITE && !(fabsf(x[j]) < INFINITY)) y[j] = NAN;
    }
    code = __builtin_amdgcn_cvt_sr_fp8_f32(y[0], ROOTS ? word[0] << 16 : word[0] & 0xFFFF0000u, code, 0);
    code = __builtin_amdgcn_cvt_sr_fp8_f32(y[1], ROOTS ? word[1] << 16 : word[1] & 0xFFFF0000u, code, 1);
    code = __builtin_amdgcn_cvt_sr_fp8_f32(y[2], ROOTS ? word[2] << 16 : word[2] & 0xFFFF0000u, code, 2);
    code = __builtin_amdgcn_cvt_sr_fp8_f32(y[3], ROOTS ? word[3] << 16 : word[3] & 0xFFFF0000u, code, 3);
    return (uint32_t)code;
}

// Lane 2u + s < 2 AT_SPAN holds what belongs to block u of the trip and to m (s = 0) or r (s = 1): the scales, and the divisions
// behind the factors, are one for all blocks.
template <typename G, bool FULL>
__device__ __forceinline__ void at_trip_fp8(const AtTensor &t, const AtStep &st, long long k, long long e0, float gs)
{
    const int lane = threadIdx.x;
    const AtRows<G> q(t, k, e0);
    uint8_t *const mc = global((uint8_t *)t.m) + k * t.s_state + e0, *const vc = global((uint8_t *)t.v) + k * t.s_state + e0;
    const float etalam = (float)(st.eta * t.decay);
    const int blocks = FULL ? AT_SPAN : min(AT_SPAN, (int)((t.n - e0 + AT_BLOCK - 1) / AT_BLOCK));
    float *const sc = (lane & 1 ? global(t.v_scale) : global(t.m_scale)) + k * t.s_scale + e0 / AT_BLOCK + (lane >> 1);
    const bool holds = lane < 2 * blocks;
    float a[AT_SPAN][4], b[AT_SPAN][4], c[AT_SPAN][4], d[AT_SPAN][4];
    uint32_t cm[AT_SPAN], cv[AT_SPAN];
    const float scale0 = holds ? *sc : 0.f;
#pragma unroll
    for (int u = 0; u < AT_SPAN; ++u) {
        const int i = u * AT_BLOCK + lane * 4;
        const long long left = t.n - e0 - i;
        at_load<float, FULL>(q.th + i, left, a[u]);
        at_load<G, FULL>(q.g + i, left, b[u]);
        // rows of codes are whole blocks: no part of one is missing
        cm[u] = cv[u] = 0;
        if (u < blocks) {
            cm[u] = __builtin_nontemporal_load((const uint32_t *)(mc + i));
            cv[u] = __builtin_nontemporal_load((const uint32_t *)(vc + i));
        }
    }
    uint32_t top[2 * AT_SPAN];
#pragma unroll
    for (int u = 0; u < AT_SPAN; ++u) {
        const int i = u * AT_BLOCK + lane * 4;
        const long long left = t.n - e0 - i;
        const float ms = lane_of(scale0, 2 * u), vs = lane_of(scale0, 2 * u + 1);
        typedef float f2 __attribute__((ext_vector_type(2)));
        const f2 m01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)cm[u], false), m23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)cm[u], true);
        const f2 v01 = __builtin_amdgcn_cvt_pk_f32_fp8((int)cv[u], false), v23 = __builtin_amdgcn_cvt_pk_f32_fp8((int)cv[u], true);
        c[u][0] = m01.x * ms; c[u][1] = m01.y * ms; c[u][2] = m23.x * ms; c[u][3] = m23.y * ms;
        d[u][0] = v01.x * vs; d[u][1] = v01.y * vs; d[u][2] = v23.x * vs; d[u][3] = v23.y * vs;
        uint32_t tm = 0, tv = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            adamw_rounded(a[u][j], b[u][j] * gs, c[u][j], d[u][j], etalam, st);
            if (!FULL && j >= left) c[u][j] = d[u][j] = 0.f;
            tm = max(tm, __float_as_uint(c[u][j]) & 0x7FFFFFFFu);
            tv = max(tv, __float_as_uint(d[u][j]) & 0x7FFFFFFFu);
        }
        at_store<float, FULL>(q.th + i, left, a[u]);
        if (q.copy != nullptr) at_store<bf16_t, FULL>(q.copy + i, left, a[u]);
        top[2 * u] = wave_max(tm);
        top[2 * u + 1] = wave_max(tv);
    }
    // as whole numbers, magnitudes order like floats, with infinities and NaN above: then the largest of the others is looked for
    uint32_t most = top[0];
#pragma unroll
    for (int u = 1; u < 2 * AT_SPAN; ++u) most = max(most, top[u]);
    const bool finite = most < 0x7F800000u;
    if (!finite) {
#pragma unroll
        for (int u = 0; u < AT_SPAN; ++u) {
            float tm = 0.f, tv = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                tm = fmaxf(tm, fabsf(finite_or_zero(c[u][j])));
                tv = fmaxf(tv, finite_or_zero(d[u][j]));
            }
            top[2 * u] = __float_as_uint(wave_max(tm));
            top[2 * u + 1] = __float_as_uint(wave_max(tv));
        }
    }
    uint32_t mine = 0;
#pragma unroll
    for (int u = 0; u < 2 * AT_SPAN; ++u) mine = lane == u ? top[u] : mine;
    const float largest = __uint_as_float(mine);
    const bool some = largest >= 1e-35f;
    const float factor = some ? 1.f / largest * E4M3_MAX : 0.f;
    if (holds) *sc = some ? largest * (1.f / E4M3_MAX) : 0.f;
    const uint32_t index = (uint32_t)((t.first * AT_BLOCK) + e0 + lane * 4) + (uint32_t)k * 0x9E3779B9u;
#pragma unroll
    for (int u = 0; u < AT_SPAN; ++u) {
        const float fm = lane_of(factor, 2 * u), fv = lane_of(factor, 2 * u + 1);
        uint32_t word[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) word[j] = at_word(index + u * AT_BLOCK + j, st.key);
        const uint32_t nm = finite ? at_codes<true, false>(c[u], fm, word) : at_codes<false, false>(c[u], fm, word);
        const uint32_t nv = finite ? at_codes<true, true>(d[u], fv, word) : at_codes<false, true>(d[u], fv, word);
        if (u < blocks) {
            const int i = u * AT_BLOCK + lane * 4;
            __builtin_nontemporal_store(nm, (uint32_t *)(mc + i));
            __builtin_nontemporal_store(nv, (uint32_t *)(vc + i));
        }
    }
}

// How a worker's factor comes to the update: from `coef`, or, where its partial sums of squares are at most one to a lane (nb > 0),
// from these, added up by every wavefront in the same order; the first one leaves factor and norm in coef for those who ask.  A norm
// that is infinite makes the factor 0; one that is no number clips nothing (factor 1), as in clip_coef_kernel.
struct AtClip { float *coef; const double *partial; int nb, K; float max_norm; };
__device__ __forceinline__ float at_factor(const AtClip &c, int k)
{
    if (c.coef == nullptr) return 1.f;
    if (c.nb == 0) return c.coef[k];
    double sum = (int)threadIdx.x < c.nb ? c.partial[(long long)k * c.nb + threadIdx.x] : 0.0;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o, 64);
    const double norm = sqrt(sum), f = (double)c.max_norm / (norm + 1e-6);
    const float factor = f < 1.0 ? (float)f : 1.0f;
    if (blockIdx.x == 0 && threadIdx.x == 0) { c.coef[k] = factor; c.coef[c.K + k] = (float)norm; }
    return factor;
}

// Workgroups go to the chip's 8 dies in turn, each with an L2 of its own.  With 8-bit moments 64 trips in a row are one die's, so that
// their scales' and chunks' cache lines are fetched once and not by every die: 1.80 against 1.87 ms for 8 x 85e6 elements with bf16
// gradients (runs of 16: 1.93, 32: 1.93, 256: 1.81).  With fp32 moments, which have no scales, it only scatters: 0.885 against 0.878 ms.
__device__ __forceinline__ unsigned at_trip(unsigned block, unsigned n)
{
    constexpr unsigned DIES = 8, RUN = 64;
    if ((block | (DIES * RUN - 1)) >= n) return block;                         // the last, incomplete group
    return (block & ~(DIES * RUN - 1)) + (block % DIES) * RUN + block / DIES % RUN;
}

// Bound by memory.  With 85e6 elements a worker:
//   fp32 moments and gradients, 2 workers: 28 bytes an element, 0.72-0.74 ms, 6.4-6.6 TB/s; clipped, 0.11 ms before it for the norm
//   8-bit moments, bf16 gradients and copies, 8 workers: 16.03 bytes an element, 1.80 ms, 6.1 TB/s
// (a large copy reaches 5.4 TB/s, with one byte written for each one read).  The arithmetic of roots, random words and codes hides
// behind the loads of the other 31 wavefronts of a CU: 49 registers a lane.
// A wavefront is a workgroup: a block's largest value needs no LDS and no barrier.
template <typename G, bool FP8>
__global__ __launch_bounds__(64) void adamw_tensors_kernel(const AtTensor *__restrict__ list, const AtChunk *__restrict__ chunks,
                                                           AtStep st, AtClip clip)
{
    const AtChunk ch = chunks[FP8 ? at_trip(blockIdx.x, gridDim.x) : blockIdx.x];
    const AtTensor &t = list[ch.tensor];
    const long long k = blockIdx.y, e0 = (long long)ch.block * AT_BLOCK;
    const float gs = at_factor(clip, blockIdx.y);
    const bool full = t.n - e0 >= AT_SPAN * AT_BLOCK;
    if (FP8) {
        if (full) at_trip_fp8<G, true>(t, st, k, e0, gs);
        else at_trip_fp8<G, false>(t, st, k, e0, gs);
    } else {
        if (full) at_trip_f32<G, true>(t, st, k, e0, gs);
        else at_trip_f32<G, false>(t, st, k, e0, gs);
    }
}

// Sum of squares of a span of blocks of a tensor, for each worker: partial[k][span].  Squares and sums are double, in a fixed order: a
// gradient's square may leave the range of floats (from 1.8e19 on), and a norm that is lost there is one that nothing is clipped by.
// Bound by memory, four loads of a lane in flight, double or not: 109 us for 2 x 85e6 fp32, 6.2 TB/s.
constexpr int AT_NORM_THREADS = 256;
struct AtSpan { int tensor, block, blocks; };
template <typename G>
__global__ __launch_bounds__(AT_NORM_THREADS) void tensors_sqnorm_kernel(const AtTensor *__restrict__ list, const AtSpan *__restrict__ spans,
                                                                         double *__restrict__ partial)
{
    __shared__ double red[AT_NORM_THREADS / 64];
    const AtSpan sp = spans[blockIdx.x];
    const AtTensor t = list[sp.tensor];
    const int k = blockIdx.y;
    const G *const g = global((const G *)t.grad) + k * t.s_grad;
    const long long e0 = (long long)sp.block * AT_BLOCK, e1 = min(t.n, e0 + (long long)sp.blocks * AT_BLOCK);
    double s[4] = {0.0, 0.0, 0.0, 0.0};
    constexpr int U = 4, STEP = AT_NORM_THREADS * 4;
    long long e = e0 + threadIdx.x * 4;
    for (; e + (U - 1) * STEP + 4 <= e1; e += U * STEP) {
        float x[U][4];
#pragma unroll
        for (int u = 0; u < U; ++u) load_wide<G, 4, false>(g + e + u * STEP, x[u]);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[i] = fma((double)x[u][i], (double)x[u][i], s[i]);
    }
    for (; e < e1; e += STEP) {
        float x[4];
        if (e1 - e >= 4) load_wide<G, 4, false>(g + e, x);
        else load_some(g + e, (int)(e1 - e), x);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = fma((double)x[i], (double)x[i], s[i]);
    }
    double acc = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) acc += __shfl_xor(acc, o, 64);
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = acc;
    __syncthreads();
    if (threadIdx.x == 0) partial[(long long)k * gridDim.x + blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

// The gradients' addresses, which change where a backward pass allocates them anew: carried in the kernel's arguments, so that the
// exchange is a launch like any other, in the stream's order.
constexpr int AT_PTRS = 256;
struct AtPtrs { const void *p[AT_PTRS]; };
__global__ __launch_bounds__(AT_PTRS) void tensors_set_grads_kernel(AtTensor *list, AtPtrs ptrs, int first, int n)
{
    if ((int)threadIdx.x < n) list[first + threadIdx.x].grad = ptrs.p[threadIdx.x];
}

}  // namespace qsr

using namespace qsr;

struct qsr_adamw {
    int device, K, n, grad_bf16, fp8;
    double beta1, beta2;
    float eps, clip;
    uint64_t seed;
    long long chunks, spans;
    AtTensor *d_list;
    AtChunk *d_chunks;
    AtSpan *d_spans;
    double *d_partial;
    float *d_coef;                             // [K] factors, then [K] norms
};

#define HIP_TRY(expr)                                    \
    do {                                                 \
        hipError_t e_ = (expr);                          \
        if (e_ != hipSuccess) {                          \
            set_last_hip_error((int)e_);                 \
            return QSR_EHIP;                             \
        }                                                \
    } while (0)

static bool unaligned(const void *p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) != 0; }

// Two tensors of the list that share memory of one kind (in the first worker's rows): two wavefronts would update the same elements at
// once.  of: where a tensor's memory begins and how many bytes a row of it has.
struct AtRange { uintptr_t at, bytes; };
template <typename F> static bool shared(const qsr_adamw_config *c, F of)
{
    std::vector<AtRange> ranges;
    ranges.reserve((size_t)c->n_tensors);
    for (int i = 0; i < c->n_tensors; ++i) {
        const AtRange r = of(c->tensors[i]);
        if (r.at) ranges.push_back(r);
    }
    std::sort(ranges.begin(), ranges.end(), [](const AtRange &x, const AtRange &y) { return x.at < y.at; });
    for (size_t i = 1; i < ranges.size(); ++i)
        if (ranges[i].at - ranges[i - 1].at < ranges[i - 1].bytes) return true;
    return false;
}

extern "C" int qsr_adamw_validate(const qsr_adamw_config *c, const char **why)
{
    const char *w = nullptr;
    auto finite_ge0 = [](double x) { return std::isfinite(x) && x >= 0.0; };
    if (!c) w = "cfg is NULL";
    else if (c->K < 1 || c->K > 65535) w = "K";
    else if (c->n_tensors < 1 || c->n_tensors > (1 << 20) || !c->tensors) w = "tensors";
    else if (c->grad_type != QSR_TYPE_F32 && c->grad_type != QSR_TYPE_BF16) w = "grad_type";
    else if (c->state_type != QSR_TYPE_F32 && c->state_type != QSR_TYPE_E4M3) w = "state_type";
    else if (!(finite_ge0(c->beta1) && c->beta1 < 1.0 && finite_ge0(c->beta2) && c->beta2 < 1.0)) w = "beta1/beta2";
    else if (!(std::isfinite(c->eps) && c->eps >= 1.2e-38)) w = "eps";          // a normal float: its reciprocal is finite
    else if (!finite_ge0(c->clip_norm) || c->clip_norm > 1e38 || (c->clip_norm > 0.0 && c->clip_norm < 1e-37)) w = "clip_norm";
    const bool fp8 = !w && c->state_type == QSR_TYPE_E4M3;
    const uintptr_t ga = !w && c->grad_type == QSR_TYPE_BF16 ? 2 : 4;
    long long blocks = 0;
    for (int i = 0; !w && i < c->n_tensors; ++i) {
        const qsr_tensor &t = c->tensors[i];
        if (t.n < 1 || t.n > ((long long)1 << 34)) { w = "a tensor's n"; break; }
        const long long nb = (t.n + AT_BLOCK - 1) / AT_BLOCK;
        blocks += nb;
        const bool many = c->K > 1;
        if (!t.param || unaligned(t.param, 4) || !t.grad || unaligned(t.grad, ga)) w = "a tensor's param/grad";
        else if (!t.m || !t.v || unaligned(t.m, 4) || unaligned(t.v, 4)) w = "a tensor's m/v";
        else if (fp8 && (!t.m_scale || !t.v_scale || unaligned(t.m_scale, 4) || unaligned(t.v_scale, 4))) w = "a tensor's m_scale/v_scale";
        else if (t.copy && unaligned(t.copy, 2)) w = "a tensor's copy";
        else if (many && (t.param_stride < t.n || t.grad_stride < t.n || (t.copy && t.copy_stride < t.n))) w = "a tensor's param_stride/grad_stride/copy_stride";
        else if (many && !fp8 && t.state_stride < t.n) w = "a tensor's state_stride";
        else if (many && fp8 && (t.state_stride < nb * AT_BLOCK || t.state_stride % 4 != 0 || t.scale_stride < nb)) w = "a tensor's state_stride/scale_stride";
        else if (!finite_ge0(t.weight_decay)) w = "a tensor's weight_decay";
    }
    if (!w && blocks > ((long long)1 << 26)) w = "tensors (above 2^34 elements together)";     // the grid's limit of 2^32 threads
    if (!w) {
        try {
            auto numbers = [](const void *p, long long n, int size) { return AtRange{(uintptr_t)p, (uintptr_t)n * (uintptr_t)size}; };
            auto padded = [](long long n) { return (n + AT_BLOCK - 1) / AT_BLOCK * AT_BLOCK; };
            auto state = [&](const void *p, long long n) { return fp8 ? numbers(p, padded(n), 1) : numbers(p, n, 4); };
            auto scales = [&](const void *p, long long n) { return fp8 ? numbers(p, padded(n) / AT_BLOCK, 4) : AtRange{0, 0}; };
            if (shared(c, [&](const qsr_tensor &t) { return numbers(t.param, t.n, 4); })) w = "a tensor's param (given twice)";
            else if (shared(c, [&](const qsr_tensor &t) { return state(t.m, t.n); })) w = "a tensor's m (given twice)";
            else if (shared(c, [&](const qsr_tensor &t) { return state(t.v, t.n); })) w = "a tensor's v (given twice)";
            else if (shared(c, [&](const qsr_tensor &t) { return numbers(t.copy, t.n, 2); })) w = "a tensor's copy (given twice)";
            else if (shared(c, [&](const qsr_tensor &t) { return scales(t.m_scale, t.n); })) w = "a tensor's m_scale (given twice)";
            else if (shared(c, [&](const qsr_tensor &t) { return scales(t.v_scale, t.n); })) w = "a tensor's v_scale (given twice)";
        } catch (...) {
            w = "tensors (the host's memory does not hold their addresses)";
        }
    }
    if (why) *why = w ? w : "ok";
    return w ? QSR_EINVAL : QSR_OK;
}

static void free_adamw(qsr_adamw *a)
{
    if (!a) return;
    if (a->d_list) (void)hipFree(a->d_list);
    if (a->d_chunks) (void)hipFree(a->d_chunks);
    if (a->d_spans) (void)hipFree(a->d_spans);
    if (a->d_partial) (void)hipFree(a->d_partial);
    if (a->d_coef) (void)hipFree(a->d_coef);
    delete a;
}

static int init_adamw(qsr_adamw *a, const qsr_adamw_config *c)
{
    HIP_TRY(hipGetDevice(&a->device));
    hipDeviceProp_t prop;
    HIP_TRY(hipGetDeviceProperties(&prop, a->device));
    if (std::strncmp(prop.gcnArchName, "gfx950", 6) != 0) return QSR_ENOGPU;
    std::vector<AtTensor> list((size_t)c->n_tensors);
    std::vector<AtChunk> chunks;
    std::vector<AtSpan> spans;
    long long blocks = 0;
    for (int i = 0; i < c->n_tensors; ++i) {
        const qsr_tensor &t = c->tensors[i];
        list[i] = AtTensor{t.param, t.grad, t.m, t.v, t.m_scale, t.v_scale, (bf16_t *)t.copy, t.n, t.param_stride, t.grad_stride,
                           t.state_stride, t.scale_stride, t.copy_stride, t.weight_decay, blocks};
        const long long nb = (t.n + AT_BLOCK - 1) / AT_BLOCK;
        for (long long b = 0; b < nb; b += AT_SPAN) chunks.push_back(AtChunk{i, (int)b});
        blocks += nb;
    }
    a->chunks = (long long)chunks.size();
    HIP_TRY(hipMalloc((void **)&a->d_list, list.size() * sizeof(AtTensor)));
    HIP_TRY(hipMalloc((void **)&a->d_chunks, chunks.size() * sizeof(AtChunk)));
    HIP_TRY(hipMemcpy(a->d_list, list.data(), list.size() * sizeof(AtTensor), hipMemcpyHostToDevice));
    HIP_TRY(hipMemcpy(a->d_chunks, chunks.data(), chunks.size() * sizeof(AtChunk), hipMemcpyHostToDevice));
    if (a->clip > 0.f) {
        // spans of 64 blocks, longer where that would leave more than 4096 partial sums to a worker
        const long long per = blocks / 4096 > 64 ? (blocks + 4095) / 4096 : 64;
        for (int i = 0; i < c->n_tensors; ++i) {
            const long long nb = (c->tensors[i].n + AT_BLOCK - 1) / AT_BLOCK;
            for (long long b = 0; b < nb; b += per) spans.push_back(AtSpan{i, (int)b, (int)(nb - b < per ? nb - b : per)});
        }
        a->spans = (long long)spans.size();
        HIP_TRY(hipMalloc((void **)&a->d_spans, spans.size() * sizeof(AtSpan)));
        HIP_TRY(hipMemcpy(a->d_spans, spans.data(), spans.size() * sizeof(AtSpan), hipMemcpyHostToDevice));
        HIP_TRY(hipMalloc((void **)&a->d_partial, (size_t)a->K * spans.size() * sizeof(double)));
        HIP_TRY(hipMalloc((void **)&a->d_coef, 2 * (size_t)a->K * sizeof(float)));
    }
    return QSR_OK;
}

extern "C" int qsr_adamw_init(const qsr_adamw_config *cfg, qsr_adamw **out)
{
    if (!out) return QSR_EINVAL;
    *out = nullptr;
    int rc = qsr_adamw_validate(cfg, nullptr);
    if (rc != QSR_OK) return rc;
    qsr_adamw *a = new (std::nothrow) qsr_adamw();
    if (!a) return QSR_ENOMEM;
    a->K = cfg->K; a->n = cfg->n_tensors;
    a->grad_bf16 = cfg->grad_type == QSR_TYPE_BF16; a->fp8 = cfg->state_type == QSR_TYPE_E4M3;
    a->beta1 = cfg->beta1; a->beta2 = cfg->beta2; a->eps = (float)cfg->eps; a->clip = (float)cfg->clip_norm;
    a->seed = cfg->seed;
    try {
        rc = init_adamw(a, cfg);
    } catch (...) {                            // the host's tables did not fit its memory
        rc = QSR_ENOMEM;
    }
    if (rc != QSR_OK) { free_adamw(a); return rc; }
    *out = a;
    return QSR_OK;
}

// The step's key: high half of a 64-bit mix (splitmix64: Steele, Lea, Flood, OOPSLA 2014) of the seed and the number of the step
static uint32_t step_key(uint64_t seed, long long t)
{
    uint64_t z = seed + (uint64_t)(t + 1) * 0x9E3779B97F4A7C15ull;
    z = (z ^ (z >> 30)) * 0xBF58476D1CE4E5B9ull;
    z = (z ^ (z >> 27)) * 0x94D049BB133111EBull;
    return (uint32_t)((z ^ (z >> 31)) >> 32);
}

extern "C" int qsr_adamw_step(qsr_adamw *a, int64_t t, double eta, void *stream)
{
    if (!a || t < 0 || t == INT64_MAX || !std::isfinite(eta) || eta < 0.0) return QSR_EINVAL;
    hipStream_t s = (hipStream_t)stream;
    AtClip clip{nullptr, nullptr, 0, a->K, a->clip};
    const unsigned K = (unsigned)a->K;
    if (a->clip > 0.f) {
        if (a->grad_bf16) tensors_sqnorm_kernel<bf16_t><<<dim3((unsigned)a->spans, K), AT_NORM_THREADS, 0, s>>>(a->d_list, a->d_spans, a->d_partial);
        else tensors_sqnorm_kernel<float><<<dim3((unsigned)a->spans, K), AT_NORM_THREADS, 0, s>>>(a->d_list, a->d_spans, a->d_partial);
        HIP_TRY(hipGetLastError());
        clip.coef = a->d_coef;
        clip.partial = a->d_partial;
        if (a->spans <= 64) clip.nb = (int)a->spans;
        else HIP_TRY(launch_clip_finish(a->d_partial, a->K, (int)a->spans, a->clip, a->d_coef, a->d_coef + a->K, s));
    }
    const double n = (double)(t + 1);
    AtStep st;
    st.eta = eta;
    st.step = (float)(eta / (1.0 - std::pow(a->beta1, n)));
    st.rsq = (float)(1.0 / std::sqrt(1.0 - std::pow(a->beta2, n)));
    st.c1 = (float)(1.0 - a->beta1); st.c2 = (float)(1.0 - a->beta2); st.eps = a->eps;
    st.key = step_key(a->seed, t);
    const dim3 grid((unsigned)a->chunks, K);
    if (a->fp8 && a->grad_bf16) adamw_tensors_kernel<bf16_t, true><<<grid, 64, 0, s>>>(a->d_list, a->d_chunks, st, clip);
    else if (a->fp8) adamw_tensors_kernel<float, true><<<grid, 64, 0, s>>>(a->d_list, a->d_chunks, st, clip);
    else if (a->grad_bf16) adamw_tensors_kernel<bf16_t, false><<<grid, 64, 0, s>>>(a->d_list, a->d_chunks, st, clip);
    else adamw_tensors_kernel<float, false><<<grid, 64, 0, s>>>(a->d_list, a->d_chunks, st, clip);
    HIP_TRY(hipGetLastError());
    return QSR_OK;
}

extern "C" int qsr_adamw_set_grads(qsr_adamw *a, const void *const *grads, int32_t n, void *stream)
{
    if (!a || !grads || n != a->n) return QSR_EINVAL;
    for (int i = 0; i < n; ++i)
        if (!grads[i] || unaligned(grads[i], a->grad_bf16 ? 2 : 4)) return QSR_EINVAL;
    for (int first = 0; first < n; first += AT_PTRS) {
        AtPtrs p;
        const int m = n - first < AT_PTRS ? n - first : AT_PTRS;
        for (int i = 0; i < AT_PTRS; ++i) p.p[i] = i < m ? grads[first + i] : nullptr;
        tensors_set_grads_kernel<<<1, AT_PTRS, 0, (hipStream_t)stream>>>(a->d_list, p, first, m);
        HIP_TRY(hipGetLastError());
    }
    return QSR_OK;
}

extern "C" int qsr_adamw_clip(qsr_adamw *a, const float **coef, const float **norm)
{
    if (!a) return QSR_EINVAL;
    if (!a->d_coef) return QSR_ESTATE;
    if (coef) *coef = a->d_coef;
    if (norm) *norm = a->d_coef + a->K;
    return QSR_OK;
}

extern "C" int qsr_adamw_destroy(qsr_adamw *a)
{
    if (!a) return QSR_EINVAL;
    int now = a->device;
    (void)hipGetDevice(&now);
    (void)hipSetDevice(a->device);
    (void)hipDeviceSynchronize();
    free_adamw(a);
    (void)hipSetDevice(now);
    return QSR_OK;
}
