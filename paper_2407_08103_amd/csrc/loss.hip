// Scoring and training under a constraint: the log-probability of given tokens under the softmax
// over the tokens that a state allows, its gradient, the clipped policy loss with a KL term, and the
// preference loss of paired sequences, for gfx950.
//
// Row i has logits z, allowed set A, token t and c = 1 / temperature.  With m the largest z in A
// and s = sum over A of exp((z_j - m) c):
//     lp = (z_t - m) c - ln s            p_j = exp((z_j - m) c) / s  in A, 0 elsewhere
//     d lp / d z_j = c ([j = t] - p_j)
// and every loss is a function of the rows' lp, so its gradient is that row times d loss / d lp.
// All sums are held in binary32 (those over the rows of a sequence, and over all rows, in binary64),
// and a gradient is rounded once, to the type of the logits.
//
// A row "takes part" if its token is in A, its logit is a number above -inf, lp is above -inf in
// binary32 (a logit of the type's lowest value may be further below m than that) and the row's
// weight is not zero.  What the others report follows, but for an lp that overflows, from the token
// alone (0: no token was chosen; -inf: probability zero), so that their logits are not read.
#include "tdfa_internal.h"

#include <cmath>

namespace tdfa {
namespace {

constexpr int kThreads = 256;
constexpr float kLog2e = 1.44269504088896341f;
constexpr float kLn2 = 0.693147180559945309f;
constexpr float kLowest = -3.402823466e38f;

// Logits are read and gradients written in groups of 16 bytes.
template <int DTYPE> struct Elem { using type = float; static constexpr int kGroup = 4; };
template <> struct Elem<TDFA_BF16> { using type = uint16_t; static constexpr int kGroup = 8; };

__device__ __forceinline__ float to_f32(float x) { return x; }
__device__ __forceinline__ float to_f32(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ void store_rounded(float* p, float x) { *p = x; }
__device__ __forceinline__ void store_rounded(uint16_t* p, float x)
{
    const __bf16 r = (__bf16)x;                              // nearest even
    *p = __builtin_bit_cast(uint16_t, r);
}
__device__ __forceinline__ uint32_t rounded_pair(float lo, float hi)
{
    typedef __bf16 pair __attribute__((ext_vector_type(2)));
    const pair r = {(__bf16)lo, (__bf16)hi};
    return __builtin_bit_cast(uint32_t, r);
}

template <int DTYPE>
__device__ __forceinline__ void unpack(uint4 x, float (&z)[Elem<DTYPE>::kGroup])
{
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (DTYPE == TDFA_F32) {
            z[k] = __uint_as_float(w[k]);
        } else {
            z[2 * k] = __uint_as_float(w[k] << 16);
            z[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
        }
    }
}

template <int DTYPE>
__device__ __forceinline__ uint4 pack(const float (&g)[Elem<DTYPE>::kGroup])
{
    if constexpr (DTYPE == TDFA_F32) return make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
    else return make_uint4(rounded_pair(g[0], g[1]), rounded_pair(g[2], g[3]), rounded_pair(g[4], g[5]), rounded_pair(g[6], g[7]));
}

template <int DTYPE> constexpr uint32_t kNegInf = DTYPE == TDFA_F32 ? 0xFF800000u : 0xFF80FF80u;

// What is known about a row before its logits are read.
struct Row {
    const uint32_t* bits;      // its state's allowed bits, or NULL: every token is allowed
    int32_t token;
    bool live;                 // takes part, unless lp overflows
    float lp;                  // of a row that does not
    float z;                   // the token's logit, of a row that does
};

template <int DTYPE>
__device__ __forceinline__ Row row_of(const TokenRows& a, int64_t i)
{
    using E = typename Elem<DTYPE>::type;
    Row r = {nullptr, a.tokens[i], false, 0.0f, 0.0f};
    if (r.token == TDFA_NO_TOKEN || (a.weights && a.weights[i] == 0.0f)) return r;
    r.lp = -INFINITY;
    if (r.token < 0 || r.token >= a.n_tokens) return r;
    if (a.allow) {
        const int32_t q = a.states[i];
        if (q < 0 || q >= a.n_states) return r;
        r.bits = a.allow + (int64_t)q * a.row_words;
        if (!(r.bits[r.token >> 5] >> (r.token & 31) & 1)) return r;
    }
    r.z = to_f32(static_cast<const E*>(a.logits)[i * a.row_stride + r.token]);
    r.live = r.z > -INFINITY;                                // neither -inf nor NaN
    return r;
}

__device__ __forceinline__ bool allowed(const uint32_t* bits, int32_t t)
{
    return !bits || (bits[t >> 5] >> (t & 31) & 1);
}

// The allowed bits of group g, from bit 0 on.
template <int DTYPE>
__device__ __forceinline__ uint32_t group_bits(const uint32_t* bits, int32_t g)
{
    const uint8_t* b = reinterpret_cast<const uint8_t*>(bits);
    if constexpr (DTYPE == TDFA_F32) return (uint32_t)(b[g >> 1] >> ((g & 1) * 4)) & 15u;
    else return b[g];
}

// Masks of four 16-bit elements by their four allowed bits: an entry of 8 bytes per bit pattern.  16 entries lie in 32
// different banks, so that lanes never wait for one another.
__device__ __forceinline__ void fill_masks(uint2 (&masks)[16])
{
    const uint32_t n = threadIdx.x;
    if (n < 16) masks[n] = make_uint2((n & 1 ? 0xFFFFu : 0u) | (n & 2 ? 0xFFFF0000u : 0u), (n & 4 ? 0xFFFFu : 0u) | (n & 8 ? 0xFFFF0000u : 0u));
}

// -inf in place of the elements that are not allowed.
template <int DTYPE>
__device__ __forceinline__ uint4 keep_allowed(uint4 x, uint32_t bits, const uint2 (&masks)[16])
{
    constexpr uint32_t none = kNegInf<DTYPE>;
    if constexpr (DTYPE == TDFA_F32) {
        return make_uint4(bits & 1 ? x.x : none, bits & 2 ? x.y : none, bits & 4 ? x.z : none, bits & 8 ? x.w : none);
    } else {
        const uint2 a = masks[bits & 15], b = masks[bits >> 4];
        return make_uint4((x.x & a.x) | (none & ~a.x), (x.y & a.y) | (none & ~a.y), (x.z & b.x) | (none & ~b.x), (x.w & b.y) | (none & ~b.y));
    }
}

// Groups g0 + threadIdx.x + k NT of a row, k < U, with -inf where a token is not allowed or the row is at an end; groups
// without an allowed token are not fetched.
template <int DTYPE, int NT, int U, bool BITS>
__device__ __forceinline__ void fetch(const uint4* row, const uint32_t* bits, int32_t g0, int32_t n_groups, const uint2 (&masks)[16], uint4 (&x)[U])
{
    constexpr uint32_t none = kNegInf<DTYPE>;
    uint32_t b[U];
    const int32_t g = g0 + (int32_t)threadIdx.x;
    if constexpr (BITS) {
#pragma unroll
        for (int k = 0; k < U; ++k) b[k] = g + k * NT < n_groups ? group_bits<DTYPE>(bits, g + k * NT) : 0u;
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
        x[k] = make_uint4(none, none, none, none);
        if (BITS ? b[k] != 0 : g + k * NT < n_groups) x[k] = row[g + k * NT];
    }
    if constexpr (BITS) {
#pragma unroll
        for (int k = 0; k < U; ++k) x[k] = keep_allowed<DTYPE>(x[k], b[k], masks);
    }
}

template <int DTYPE, int U, bool EXACT>
__device__ __forceinline__ float sum_of(const uint4 (&x)[U], float ref, float c2)
{
    float s[2] = {0.0f, 0.0f};
#pragma unroll
    for (int k = 0; k < U; ++k) {
        float z[Elem<DTYPE>::kGroup];
        unpack<DTYPE>(x[k], z);
#pragma unroll
        for (int j = 0; j < Elem<DTYPE>::kGroup; ++j) {
            const float e = __builtin_amdgcn_exp2f((z[j] - ref) * c2);
            s[j & 1] += EXACT && z[j] != z[j] ? 0.0f : e;
        }
    }
    return s[0] + s[1];
}

template <int DTYPE, int U>
__device__ __forceinline__ float max_of(const uint4 (&x)[U], float m)
{
#pragma unroll
    for (int k = 0; k < U; ++k) {
        float z[Elem<DTYPE>::kGroup];
        unpack<DTYPE>(x[k], z);
#pragma unroll
        for (int j = 0; j < Elem<DTYPE>::kGroup; ++j) m = fmaxf(m, z[j]);          // a NaN is passed over
    }
    return m;
}

// The element behind the last whole group that belongs to this thread, -inf if there is none.
template <int DTYPE>
__device__ __forceinline__ float last_element(const TokenRows& a, const typename Elem<DTYPE>::type* row, const uint32_t* bits)
{
    const int32_t t = a.n_tokens / Elem<DTYPE>::kGroup * Elem<DTYPE>::kGroup + (int32_t)threadIdx.x;
    return t < a.n_tokens && allowed(bits, t) ? to_f32(row[t]) : -INFINITY;
}

__device__ __forceinline__ float wave_sum(float s)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d);
    return s;
}
__device__ __forceinline__ float wave_max(float m)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) m = fmaxf(m, __shfl_xor(m, d));
    return m;
}
// Sum (MAX: maximum) over the workgroup, in every thread and in one order.  Two barriers.
template <int NT, bool MAX>
__device__ __forceinline__ float block_reduce(float v, float (&part)[NT / 64])
{
    v = MAX ? wave_max(v) : wave_sum(v);
    if constexpr (NT > 64) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
        __syncthreads();
        v = part[0];
#pragma unroll
        for (int w = 1; w < NT / 64; ++w) v = MAX ? fmaxf(v, part[w]) : v + part[w];
    }
    return v;
}

// A sum of exponentials relative to `ref` that has neither overflowed nor met a NaN, and has the token's own term in it.
__device__ __forceinline__ bool usable(float s) { return s >= 0.5f && s < 3.0e38f; }

// ln s in binary64 from the logarithm of the significand in binary32: off by 2^-25 or so whatever s is, where the rounding of
// a binary32 logarithm of 10 would be 2^-21.
__device__ __forceinline__ double ln_of(float s)
{
    int e;
    const float m = frexpf(s, &e);
    return (double)e * 0.69314718055994530942 + (double)logf(m);
}

// The fallback's sum may be any (NaN where an allowed logit is +inf).
struct Scored {
    float ls;        // ln s
    double lp;
};
__device__ __forceinline__ Scored score(float z, float ref, float s, float inv_t)
{
    const double ls = ln_of(s);
    return {(float)ls, (double)(z - ref) * (double)inv_t - ls};
}

// Sum of the exponentials of a row relative to its largest logit, NaN passed over: what a row takes whose sum relative to its own
// token is not usable.  Sets *ref to that logit.
template <int DTYPE, int NT, int U, bool BITS>
__device__ __forceinline__ float careful_sum(const uint4* row4, const uint32_t* bits, int32_t n_groups, float last, float c2, float* ref,
                                          const uint2 (&masks)[16], float (&part)[NT / 64])
{
    uint4 x[U];
    float m = fmaxf(kLowest, last);
    for (int32_t g = 0; g < n_groups; g += NT * U) {
        fetch<DTYPE, NT, U, BITS>(row4, bits, g, n_groups, masks, x);
        m = max_of<DTYPE, U>(x, m);
    }
    m = block_reduce<NT, true>(m, part);
    float s = last == last ? __builtin_amdgcn_exp2f((last - m) * c2) : 0.0f;
    for (int32_t g = 0; g < n_groups; g += NT * U) {
        fetch<DTYPE, NT, U, BITS>(row4, bits, g, n_groups, masks, x);
        s += sum_of<DTYPE, U, true>(x, m, c2);
    }
    *ref = m;
    return block_reduce<NT, false>(s, part);
}

// One workgroup per row: its log-probability and its statistics {ref, ln s}; {0, +inf} for a row that takes no part.
// The sum is taken relative to the row's own token, ref = z_t, so that no maximum has to be known and lp = -ln s; where that
// overflows (lp below -87) or a NaN is met, the row is read again, for the largest logit and the sum relative to it.
template <int DTYPE, int NT, int U, bool BITS>
__global__ void __launch_bounds__(NT) token_stats_kernel(TokenRows a, float* logprobs, float2* stats, float* zeros, double* exact)
{
    using E = typename Elem<DTYPE>::type;
    __shared__ float s_part[NT / 64];
    __shared__ uint2 s_masks[16];
    const float c2 = a.inv_t * kLog2e;
    const int32_t n_groups = a.n_tokens / Elem<DTYPE>::kGroup;
    if (BITS && DTYPE == TDFA_BF16) {
        fill_masks(s_masks);
        __syncthreads();
    }
    for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
        const Row r = row_of<DTYPE>(a, i);
        if (threadIdx.x == 0 && zeros) zeros[i] = 0.0f;
        if (!r.live) {
            if (threadIdx.x == 0) {
                logprobs[i] = r.lp;
                if (stats) stats[i] = make_float2(0.0f, INFINITY);
            }
            continue;
        }
        const E* row = static_cast<const E*>(a.logits) + i * a.row_stride;
        const uint4* row4 = reinterpret_cast<const uint4*>(row);
        const float last = last_element<DTYPE>(a, row, r.bits);
        float ref = r.z, s = __builtin_amdgcn_exp2f((last - ref) * c2);
        uint4 x[U];
        for (int32_t g = 0; g < n_groups; g += NT * U) {
            fetch<DTYPE, NT, U, BITS>(row4, r.bits, g, n_groups, s_masks, x);
            s += sum_of<DTYPE, U, false>(x, ref, c2);
        }
        s = block_reduce<NT, false>(s, s_part);
        if (!usable(s)) s = careful_sum<DTYPE, NT, 2, BITS>(row4, r.bits, n_groups, last, c2, &ref, s_masks, s_part);
        if (threadIdx.x == 0) {
            const Scored q = score(r.z, ref, s, a.inv_t);
            const float lp = (float)q.lp;
            logprobs[i] = lp;
            if (stats) stats[i] = lp == -INFINITY ? make_float2(0.0f, INFINITY) : make_float2(ref, q.ls);
            if (exact) exact[i] = q.lp;
        }
    }
}

// grad[i][j] = down[i] c ([j = t] - p_j) over A, 0 elsewhere; 0 throughout in a row that takes no part.  A workgroup
// takes NT U groups of one row; the last of a row takes the elements behind the last whole group too.
template <int DTYPE, int NT, int U, bool BITS>
__global__ void __launch_bounds__(NT) token_grad_kernel(TokenRows a, const float2* stats, const float* down, void* grad, int64_t grad_stride, int32_t parts)
{
    using E = typename Elem<DTYPE>::type;
    constexpr int G = Elem<DTYPE>::kGroup;
    __shared__ uint2 s_masks[16];
    if (BITS && DTYPE == TDFA_BF16) {
        fill_masks(s_masks);
        __syncthreads();
    }
    const float c2 = a.inv_t * kLog2e;
    const int32_t n_groups = a.n_tokens / G;
    for (int64_t w = blockIdx.x; w < a.rows * parts; w += gridDim.x) {
        const int64_t i = w / parts;
        const int32_t part = (int32_t)(w - i * parts);
        const Row r = row_of<DTYPE>(a, i);
        const float2 st = stats[i];
        const float d = r.live && st.y != INFINITY ? down[i] * a.inv_t : 0.0f;
        const E* row = static_cast<const E*>(a.logits) + i * a.row_stride;
        E* out = static_cast<E*>(grad) + i * grad_stride;
        uint4* out4 = reinterpret_cast<uint4*>(out);
        const int32_t g0 = part * (NT * U), g = g0 + (int32_t)threadIdx.x;
        const int32_t behind = n_groups * G + (int32_t)threadIdx.x;
        if (d == 0.0f) {
#pragma unroll
            for (int k = 0; k < U; ++k)
                if (g + k * NT < n_groups) out4[g + k * NT] = make_uint4(0, 0, 0, 0);
            if (part == parts - 1 && behind < a.n_tokens) store_rounded(out + behind, 0.0f);
            continue;
        }
        const float k2 = -st.y * kLog2e;
        const float last = part == parts - 1 ? last_element<DTYPE>(a, row, r.bits) : -INFINITY;
        uint4 x[U];
        fetch<DTYPE, NT, U, BITS>(reinterpret_cast<const uint4*>(row), r.bits, g0, n_groups, s_masks, x);
#pragma unroll
        for (int k = 0; k < U; ++k) {
            float z[G];
            unpack<DTYPE>(x[k], z);
#pragma unroll
            for (int j = 0; j < G; ++j) {
                const float p = __builtin_amdgcn_exp2f(fmaf(z[j] - st.x, c2, k2));
                z[j] = z[j] == z[j] ? -d * p : 0.0f;
            }
            if (g + k * NT < n_groups) out4[g + k * NT] = pack<DTYPE>(z);
        }
        if (part == parts - 1 && behind < a.n_tokens)
            store_rounded(out + behind, last == last ? -d * __builtin_amdgcn_exp2f(fmaf(last - st.x, c2, k2)) : 0.0f);
        // the token's own element, by the thread that has just written its group
        if (r.token / G == n_groups ? part == parts - 1 && behind == r.token : r.token / G >= g0 && r.token / G < g0 + NT * U && (r.token / G - g) % NT == 0)
            store_rounded(out + r.token, d - d * __builtin_amdgcn_exp2f(fmaf(r.z - st.x, c2, k2)));
    }
}

// The policy term of one row from its log-probability: the loss (without the weight) and d loss / d lp.
__device__ __forceinline__ void policy_term(const PolicyArgs& p, int64_t i, float lp, float* each, float* down)
{
    const float adv = p.advantages[i];
    const float ratio = expf(lp - p.old_logprobs[i]);
    const float free = ratio * adv;
    const float clipped = fminf(fmaxf(ratio, p.clip_low), p.clip_high) * adv;
    // NaN (an infinite ratio and no advantage) stays NaN
    *each = clipped < free ? -clipped : -free;
    *down = clipped < free ? 0.0f : -free;
    if (p.ref_logprobs) {
        const float d = p.ref_logprobs[i] - lp, e = expm1f(d);
        *each += p.kl_coef * (e - d);
        *down -= p.kl_coef * e;
    }
}

// One workgroup per row, one pass after the other: the sum, the row's term, the gradient.  The logits of the second pass come from
// the caches, which hold what the workgroups in flight have read.
template <int DTYPE, int NT, int U, bool BITS>
__global__ void __launch_bounds__(NT, 2048 / 64 / 4) policy_row_kernel(TokenRows a, PolicyArgs p, float* logprobs, float* each, void* grad, int64_t grad_stride)
{
    using E = typename Elem<DTYPE>::type;
    constexpr int G = Elem<DTYPE>::kGroup;
    __shared__ float s_part[NT / 64];
    __shared__ uint2 s_masks[16];
    __shared__ float s_d, s_k2;
    const float c2 = a.inv_t * kLog2e;
    const int32_t n_groups = a.n_tokens / G;
    if (BITS && DTYPE == TDFA_BF16) {
        fill_masks(s_masks);
        __syncthreads();
    }
    for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
        const Row r = row_of<DTYPE>(a, i);
        const E* row = static_cast<const E*>(a.logits) + i * a.row_stride;
        const uint4* row4 = reinterpret_cast<const uint4*>(row);
        float d = 0.0f, k2 = 0.0f, ref = r.z, last = -INFINITY;
        if (r.live) {
            last = last_element<DTYPE>(a, row, r.bits);
            float s = __builtin_amdgcn_exp2f((last - ref) * c2);
            uint4 x[U];
            for (int32_t g = 0; g < n_groups; g += NT * U) {
                fetch<DTYPE, NT, U, BITS>(row4, r.bits, g, n_groups, s_masks, x);
                s += sum_of<DTYPE, U, false>(x, ref, c2);
            }
            s = block_reduce<NT, false>(s, s_part);
            if (!usable(s)) s = careful_sum<DTYPE, NT, 2, BITS>(row4, r.bits, n_groups, last, c2, &ref, s_masks, s_part);
            if (threadIdx.x < 64) {
                const Scored q = score(r.z, ref, s, a.inv_t);
                const float lp = (float)q.lp;
                float e = 0.0f;
                if (lp != -INFINITY) {
                    policy_term(p, i, lp, &e, &d);
                    const float w = a.weights ? a.weights[i] : 1.0f;
                    e *= w;
                    d *= w * a.inv_t;
                }
                if (threadIdx.x == 0) {
                    logprobs[i] = lp;
                    each[i] = e;
                    s_d = d;
                    s_k2 = -q.ls * kLog2e;
                }
            }
            __syncthreads();
            d = s_d;
            k2 = s_k2;
        } else if (threadIdx.x == 0) {
            logprobs[i] = r.lp;
            each[i] = 0.0f;
        }
        if (!grad) continue;
        E* out = static_cast<E*>(grad) + i * grad_stride;
        uint4* out4 = reinterpret_cast<uint4*>(out);
        const int32_t behind = n_groups * G + (int32_t)threadIdx.x;
        if (d == 0.0f) {
            for (int32_t g = threadIdx.x; g < n_groups; g += NT) out4[g] = make_uint4(0, 0, 0, 0);
            if (behind < a.n_tokens) store_rounded(out + behind, 0.0f);
            continue;
        }
        // the part of the row that was read last first
        for (int32_t g0 = (n_groups - 1) / (NT * U) * (NT * U); g0 >= 0; g0 -= NT * U) {
            uint4 x[U];
            fetch<DTYPE, NT, U, BITS>(row4, r.bits, g0, n_groups, s_masks, x);
            const int32_t g = g0 + (int32_t)threadIdx.x;
#pragma unroll
            for (int k = 0; k < U; ++k) {
                float z[G];
                unpack<DTYPE>(x[k], z);
#pragma unroll
                for (int j = 0; j < G; ++j) {
                    const float e = __builtin_amdgcn_exp2f(fmaf(z[j] - ref, c2, k2));
                    z[j] = z[j] == z[j] ? -d * e : 0.0f;
                }
                if (g + k * NT < n_groups) out4[g + k * NT] = pack<DTYPE>(z);
            }
        }
        if (behind < a.n_tokens) store_rounded(out + behind, last == last ? -d * __builtin_amdgcn_exp2f(fmaf(last - ref, c2, k2)) : 0.0f);
        // the token's own element, by the thread that has written its group
        if (r.token / G == n_groups ? behind == r.token : r.token / G % NT == (int32_t)threadIdx.x)
            store_rounded(out + r.token, d - d * __builtin_amdgcn_exp2f(fmaf(r.z - ref, c2, k2)));
    }
}

// loss = scale * the sum of each, by one workgroup, in an order that depends on nothing but n.
template <typename F>
__global__ void __launch_bounds__(1024) loss_sum_kernel(const F* each, int64_t n, double scale, float* loss)
{
    __shared__ double s_part[16];
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += 1024) sum += (double)each[i];
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int w = 1; w < 16; ++w) sum += s_part[w];
        *loss = (float)(sum * scale);
    }
}

// One workgroup per pair: the two rewards, the pair's loss, and d loss / d lp of every row of the pair.
__global__ void __launch_bounds__(kThreads)
pair_kernel(PairArgs p, int64_t rows, const double* exact, const float2* stats, float* down, double* each)
{
    __shared__ double s_part[kThreads / 64];
    __shared__ double s_reward[2];
    for (int64_t k = blockIdx.x; k < p.n_pairs; k += gridDim.x) {
        int64_t from[2], to[2];
        for (int side = 0; side < 2; ++side) {
            // a sequence that reaches outside the rows is cut there
            from[side] = max((int64_t)p.begin[2 * k + side], (int64_t)0);
            to[side] = min((int64_t)p.begin[2 * k + side + 1], rows);
            double sum = 0.0;
            for (int64_t i = from[side] + threadIdx.x; i < to[side]; i += kThreads)
                if (stats[i].y != INFINITY) sum += exact[i] - (double)p.ref_logprobs[i];
#pragma unroll
            for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
            __syncthreads();
            if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = sum;
            __syncthreads();
            if (threadIdx.x == 0) {
                for (int w = 1; w < kThreads / 64; ++w) sum += s_part[w];
                s_reward[side] = (double)p.beta * sum;
                p.rewards[2 * k + side] = (float)s_reward[side];
            }
        }
        __syncthreads();
        const double gap = s_reward[0] - s_reward[1], eps = p.smoothing;
        // softplus(x) = max(x, 0) + log1p(exp(-|x|))
        const double tail = log1p(exp(-fabs(gap)));
        if (threadIdx.x == 0) each[k] = (1.0 - eps) * (fmax(-gap, 0.0) + tail) + eps * (fmax(gap, 0.0) + tail);
        if (down) {
            const double slope = (eps / (1.0 + exp(-gap)) - (1.0 - eps) / (1.0 + exp(gap))) * (double)p.beta / (double)p.n_pairs;
            for (int side = 0; side < 2; ++side)
                for (int64_t i = from[side] + threadIdx.x; i < to[side]; i += kThreads) down[i] = (float)(side ? -slope : slope);
        }
    }
}

unsigned blocks_for(int64_t n) { return (unsigned)(n < 1 << 20 ? n : 1 << 20); }

template <int DTYPE, bool BITS>
int stats_launch(const TokenRows& a, float* logprobs, float2* stats, float* zeros, double* exact, hipStream_t stream)
{
    const int32_t n_groups = a.n_tokens / Elem<DTYPE>::kGroup;
    if (n_groups <= 512) token_stats_kernel<DTYPE, 64, 8, BITS><<<blocks_for(a.rows), 64, 0, stream>>>(a, logprobs, stats, zeros, exact);
    else if (n_groups <= 4096) token_stats_kernel<DTYPE, 256, 8, BITS><<<blocks_for(a.rows), 256, 0, stream>>>(a, logprobs, stats, zeros, exact);
    else token_stats_kernel<DTYPE, 1024, 8, BITS><<<blocks_for(a.rows), 1024, 0, stream>>>(a, logprobs, stats, zeros, exact);
    TDFA_HIP(hipGetLastError());
    return TDFA_OK;
}

// zeros: [rows] set to zero on the way, exact: [rows] receives lp in binary64 for rows that take part; or NULL.
int stats_of(const TokenRows& a, float* logprobs, float2* stats, float* zeros, double* exact, hipStream_t stream)
{
    if (a.dtype == TDFA_F32) return a.allow ? stats_launch<TDFA_F32, true>(a, logprobs, stats, zeros, exact, stream) : stats_launch<TDFA_F32, false>(a, logprobs, stats, zeros, exact, stream);
    return a.allow ? stats_launch<TDFA_BF16, true>(a, logprobs, stats, zeros, exact, stream) : stats_launch<TDFA_BF16, false>(a, logprobs, stats, zeros, exact, stream);
}

template <int DTYPE, bool BITS>
int grad_launch(const TokenRows& a, const float2* stats, const float* down, void* grad, int64_t grad_stride, hipStream_t stream)
{
    const int32_t n_groups = a.n_tokens / Elem<DTYPE>::kGroup;
    if (n_groups <= 256) {
        token_grad_kernel<DTYPE, 64, 4, BITS><<<blocks_for(a.rows), 64, 0, stream>>>(a, stats, down, grad, grad_stride, 1);
    } else {
        const int32_t parts = (n_groups + 256 * 4 - 1) / (256 * 4);
        token_grad_kernel<DTYPE, 256, 4, BITS><<<blocks_for(a.rows * parts), 256, 0, stream>>>(a, stats, down, grad, grad_stride, parts);
    }
    TDFA_HIP(hipGetLastError());
    return TDFA_OK;
}

}  // namespace

int launch_token_logprobs(const TokenRows& a, float* logprobs, float* stats, void* workspace, hipStream_t stream)
{
    (void)workspace;
    if (a.rows == 0) return TDFA_OK;
    return stats_of(a, logprobs, reinterpret_cast<float2*>(stats), nullptr, nullptr, stream);
}

int launch_token_grad(const TokenRows& a, const float* stats, const float* down, void* grad, int64_t grad_stride, hipStream_t stream)
{
    if (a.rows == 0) return TDFA_OK;
    const float2* st = reinterpret_cast<const float2*>(stats);
    if (a.dtype == TDFA_F32)
        return a.allow ? grad_launch<TDFA_F32, true>(a, st, down, grad, grad_stride, stream) : grad_launch<TDFA_F32, false>(a, st, down, grad, grad_stride, stream);
    return a.allow ? grad_launch<TDFA_BF16, true>(a, st, down, grad, grad_stride, stream) : grad_launch<TDFA_BF16, false>(a, st, down, grad, grad_stride, stream);
}

// Workspace: double [n_pairs] losses of the pairs, double [rows] lp or float [rows] losses, float2 [rows] statistics,
// float [rows] d loss / d lp.
int64_t loss_workspace(int64_t rows, int64_t n_pairs) { return 8 * n_pairs + 20 * rows; }

template <int DTYPE, bool BITS>
static int policy_launch(const TokenRows& a, const PolicyArgs& p, float* logprobs, float* each, void* grad, int64_t grad_stride, hipStream_t stream)
{
    const int32_t n_groups = a.n_tokens / Elem<DTYPE>::kGroup;
    if (n_groups <= 256) policy_row_kernel<DTYPE, 64, 4, BITS><<<blocks_for(a.rows), 64, 0, stream>>>(a, p, logprobs, each, grad, grad_stride);
    else if (n_groups <= 4096) policy_row_kernel<DTYPE, 256, 4, BITS><<<blocks_for(a.rows), 256, 0, stream>>>(a, p, logprobs, each, grad, grad_stride);
    else policy_row_kernel<DTYPE, 1024, 4, BITS><<<blocks_for(a.rows), 1024, 0, stream>>>(a, p, logprobs, each, grad, grad_stride);
    TDFA_HIP(hipGetLastError());
    return TDFA_OK;
}

int launch_policy_loss(const TokenRows& a, const PolicyArgs& p, float* loss, float* logprobs, void* grad, int64_t grad_stride, void* workspace,
                       hipStream_t stream)
{
    float* each = static_cast<float*>(workspace);
    if (a.rows) {
        const int rc = a.dtype == TDFA_F32 ? (a.allow ? policy_launch<TDFA_F32, true>(a, p, logprobs, each, grad, grad_stride, stream)
                                                      : policy_launch<TDFA_F32, false>(a, p, logprobs, each, grad, grad_stride, stream))
                                           : (a.allow ? policy_launch<TDFA_BF16, true>(a, p, logprobs, each, grad, grad_stride, stream)
                                                      : policy_launch<TDFA_BF16, false>(a, p, logprobs, each, grad, grad_stride, stream));
        if (rc != TDFA_OK) return rc;
    }
    loss_sum_kernel<float><<<1, 1024, 0, stream>>>(each, a.rows, 1.0, loss);
    TDFA_HIP(hipGetLastError());
    return TDFA_OK;
}

int launch_preference_loss(const TokenRows& a, const PairArgs& p, float* loss, float* logprobs, void* grad, int64_t grad_stride, void* workspace,
                           hipStream_t stream)
{
    double* each = static_cast<double*>(workspace);
    double* exact = each + p.n_pairs;
    float2* stats = reinterpret_cast<float2*>(exact + a.rows);
    float* down = reinterpret_cast<float*>(stats + a.rows);
    int rc = TDFA_OK;
    if (a.rows) {
        rc = stats_of(a, logprobs, stats, down, exact, stream);             // rows of no sequence keep a slope of zero
        if (rc != TDFA_OK) return rc;
    }
    if (p.n_pairs) {
        pair_kernel<<<blocks_for(p.n_pairs), kThreads, 0, stream>>>(p, a.rows, exact, stats, down, each);
        TDFA_HIP(hipGetLastError());
    }
    loss_sum_kernel<double><<<1, 1024, 0, stream>>>(each, p.n_pairs, p.n_pairs ? 1.0 / (double)p.n_pairs : 0.0, loss);
    TDFA_HIP(hipGetLastError());
    if (grad && a.rows) rc = launch_token_grad(a, reinterpret_cast<const float*>(stats), down, grad, grad_stride, stream);
    return rc;
}

}  // namespace tdfa
