// Scoring and training under a constraint: the log-probability of given tokens under the softmax
// over the tokens that a state allows, its gradient, the clipped policy loss with a KL term, and the
// preference loss of paired sequences, for gfx950.
//
// Row i has logits z, allowed set A, token t and c = 1 / temperature.  With m the largest z in A
// and s = sum over A of exp((z_j - m) c):
//     lp = (z_t - m) c - ln s            p_j = exp((z_j - m) c) / s  in A, 0 elsewhere
//     d lp / d z_j = c ([j = t] - p_j)
// and every loss is a function of the rows' lp, so its gradient is that row times d loss / d lp.  Where p_t is near 1, as
// in a state that allows one token, s and p_t do not tell how near: the sums leave the token's own term out, o = the sum of
// the others relative to it gives ln s = ln(1 + o), and 1 - p_t is worked out by itself.
// All sums are held in binary32 (those over the rows of a sequence, and over all rows, in binary64),
// and a gradient is rounded once, to the type of the logits.
//
// A row "takes part" if its token is in A, its logit is a number above -inf, lp is above -inf in
// binary32 (a logit of the type's lowest value may be further below m than that) and the row's
// weight is not zero.  Of the others one without a token or of weight 0 reports 0 and is not read, any
// other -inf.
#include "rows_device.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace tdfa {
namespace {

constexpr int kThreads = 256;
// What the kernels are handed.  A launch whose arguments take at most 112 bytes, and whose kernel asks for nothing else (the size of its
// grid, say), costs the host 2.6 us, a larger one 3.3; so strides are in units of 16 bytes, rows are numbered by the workgroups of a grid
// that has no others, and what a call keeps of a row lies together.  A workgroup does one thing and ends: a loop over rows would
// have the compiler keep every group's address and bounds in registers from one row to the next.
struct RowArgs {
    const uint32_t* allow;     // or NULL: every token is allowed
    const void* logits;
    const int32_t* states;
    const int32_t* tokens;
    uint32_t stride16;
    int32_t n_states, n_tokens;
    float inv_t;
};
// What a loss keeps of a row between its launches.
struct RowWork {
    double value;              // preference loss: lp; policy loss: the row's part of the loss
    float2 stats;
    float down;                // d loss / d lp
    float scale;               // exp(-ls)
};
// Log-probabilities and statistics for the caller, or for the preference loss.
struct ScoreArgs : RowArgs {
    float* logprobs;
    float2* stats;             // or NULL
};
struct PairScoreArgs : RowArgs {
    float* logprobs;
    RowWork* work;
};
// What a row of the policy loss has beside its logits.
struct PolicyTerms : RowArgs {
    const float* old_logprobs;
    const float* ref_logprobs;
    const float* advantages;
    const float* weights;
    float* logprobs;
    float clip_low, clip_high, kl_coef;
    uint32_t grad_stride16;
};
struct PolicyScoreArgs : PolicyTerms {
    RowWork* work;
};
struct PolicyRowArgs : PolicyTerms {
    void* grad;
};
static_assert(sizeof(PolicyScoreArgs) <= 112 && sizeof(PolicyRowArgs) <= 112, "see above");

// What is known about a row before its logits are read.
struct Row {
    const uint32_t* bits;      // its state's allowed bits, or NULL: every token is allowed
    int32_t token;
    bool read;                 // its logits have to be read: the token is one, the state is a row of the table, the weight is not zero
    float lp;                  // of a row that is not read
};

// (i is the same in all lanes of a wavefront.)  The loads do not wait for one another: what there is none of is read from the tokens,
// and all three values are wanted before any of them is looked at.
__device__ __forceinline__ Row row_of(const RowArgs& a, const float* weights, uint32_t i)
{
    int32_t token = a.tokens[i], q = (a.allow ? a.states : a.tokens)[i];
    int32_t w = (weights ? reinterpret_cast<const int32_t*>(weights) : a.tokens)[i];
    asm volatile("" : "+v"(token), "+v"(q), "+v"(w));
    token = __builtin_amdgcn_readfirstlane(token);
    q = __builtin_amdgcn_readfirstlane(q);
    w = __builtin_amdgcn_readfirstlane(w);
    Row r = {nullptr, token, false, 0.0f};
    if (token == TDFA_NO_TOKEN || (weights && __int_as_float(w) == 0.0f)) return r;
    r.lp = -INFINITY;
    if (token < 0 || token >= a.n_tokens || (a.allow && (q < 0 || q >= a.n_states))) return r;
    if (a.allow) r.bits = bits_of(a.allow, q, a.n_tokens);
    r.read = true;                                         // (and lp is -inf if the token turns out not to be allowed)
    return r;
}

// The logit of a row's token, -inf if it is not allowed or NaN: the row takes part if it is above -inf (unless lp overflows).
template <typename E>
__device__ __forceinline__ float token_logit(const Row& r, const E* row)
{
    uint32_t word = r.bits ? r.bits[r.token >> 5] : 0xFFFFFFFFu;
    float z = to_f32(row[r.token]);
    asm volatile("" : "+v"(word), "+v"(z));                // both are on their way before either is looked at
    word = __builtin_amdgcn_readfirstlane(word);
    z = __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(z)));
    return (word >> (r.token & 31) & 1) && z == z ? z : -INFINITY;
}

// Where a row's token lies among the groups g0 + n + k NT that thread n takes: in the k-th of one thread, whose mask has its element's bits
// (the others' is empty); k = -1: in none of them.
struct Own {
    int32_t k, j;              // element j of the group
    bool mine;
    uint4 mask;
};
template <int DTYPE, int NT, int U>
__device__ __forceinline__ Own own_of(int32_t token, int32_t g0)
{
    constexpr int G = Elem<DTYPE>::kGroup;
    const int32_t at = token / G - g0, j = token & (G - 1), word = DTYPE == TDFA_F32 ? j : j >> 1;
    const bool mine = (int32_t)threadIdx.x == (at & (NT - 1));
    const uint32_t m = !mine ? 0u : DTYPE == TDFA_F32 ? 0xFFFFFFFFu : j & 1 ? 0xFFFF0000u : 0xFFFFu;
    return {(uint32_t)at < (uint32_t)(NT * U) ? at / NT : -1, j, mine, make_uint4(word == 0 ? m : 0, word == 1 ? m : 0, word == 2 ? m : 0, word == 3 ? m : 0)};
}
// Takes the token's own element out of the group, as if it were not allowed.
template <int DTYPE, bool BITS>
__device__ __forceinline__ void leave_own(const Own& own, uint4& x, uint32_t& b)
{
    if constexpr (BITS) b &= ~((own.mine ? 1u : 0u) << own.j);
    else x = where(own.mask, kNegInf<DTYPE>, x);
}

// Sum of 2^(z c2 + nb), nb = -ref c2 rounded: the rounding moves all terms, the token's own among them, by the same factor.
template <int DTYPE>
__device__ __forceinline__ void add_group(uint4 x, float c2, float nb, float (&s)[2])
{
    float z[Elem<DTYPE>::kGroup];
    unpack<DTYPE>(x, z);
#pragma unroll
    for (int j = 0; j < Elem<DTYPE>::kGroup; ++j) s[j & 1] += __builtin_amdgcn_exp2f(fmaf(z[j], c2, nb));
}
// The same with differences taken first and NaN passed over (fmaxf with a number does).
template <int DTYPE>
__device__ __forceinline__ void add_group_careful(uint4 x, float c2, float ref, float& s)
{
    float z[Elem<DTYPE>::kGroup];
    unpack<DTYPE>(x, z);
#pragma unroll
    for (int j = 0; j < Elem<DTYPE>::kGroup; ++j) s += __builtin_amdgcn_exp2f((fmaxf(z[j], -INFINITY) - ref) * c2);
}
// Over fetched groups, but for the token's own element.  Bit k of `some`: the wavefront has another allowed token in its k-th groups.
template <int DTYPE, int NT, int U, bool BITS>
__device__ __forceinline__ void add_groups(uint4 (&x)[U], uint32_t (&b)[U], int32_t g0, int32_t n_groups, const uint2 (&masks)[16], int32_t token, float c2,
                                           float nb, float (&s)[2], uint32_t& some)
{
    const Own own = own_of<DTYPE, NT, U>(token, g0);
    some = 0;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        if (k == own.k) leave_own<DTYPE, BITS>(own, x[k], b[k]);
        if (!settle<DTYPE, BITS>(x[k], b[k], g0 + (int32_t)threadIdx.x + k * NT, n_groups, masks)) continue;
        some |= 1u << k;
        add_group<DTYPE>(x[k], c2, nb, s);
        next_group();
    }
}

// The same relative to the largest logit that the thread has met, m: a running maximum, and a sum that is scaled where it moves, four groups
// at a time so that sums do not wait for all loads.  Exponents are z c2 - m c2 with m c2 rounded (SAFE: differences taken first and NaN
// passed over, which takes half as many instructions again).
template <int DTYPE, int NT, int U, bool BITS, bool SAFE>
__device__ __forceinline__ void add_groups_running(uint4 (&x)[U], uint32_t (&b)[U], int32_t g0, int32_t n_groups, const uint2 (&masks)[16], int32_t token,
                                                   float c2, float& m, float (&s)[2], uint32_t& some)
{
    static_assert(U % 4 == 0);
    const Own own = own_of<DTYPE, NT, U>(token, g0);
    some = 0;
#pragma unroll
    for (int k0 = 0; k0 < U; k0 += 4) {
        float top = m;
#pragma unroll
        for (int k = k0; k < k0 + 4; ++k) {
            if (k == own.k) leave_own<DTYPE, BITS>(own, x[k], b[k]);
            if (!settle<DTYPE, BITS>(x[k], b[k], g0 + (int32_t)threadIdx.x + k * NT, n_groups, masks)) continue;
            some |= 1u << k;
            top = max_group<DTYPE>(x[k], top);
            next_group();
        }
        const float nb = offset_of(top, c2), scale = rescale<SAFE>(m, top, c2);
        s[0] *= scale;
        s[1] *= scale;
        m = top;
#pragma unroll
        for (int k = k0; k < k0 + 4; ++k) {
            if (!(some >> k & 1)) continue;
            if constexpr (SAFE) add_group_careful<DTYPE>(x[k], c2, m, s[0]);
            else add_group<DTYPE>(x[k], c2, nb, s);
            next_group();
        }
    }
}

// Whether a row's own term and the sum of the others, both relative to about its own logit, are what they should be: not so where the
// exponents overflowed or a NaN was met.
__device__ __forceinline__ bool usable(float own, float others) { return own >= 0.25f && own <= 4.0f && others < 3.0e38f; }

// ln(own + others) in binary64.  The sum is a significand between sqrt(1/2) and sqrt(2) and an exponent, so that the binary32 logarithm
// is off by 2^-25 or so whatever the sum is (the rounding of a binary32 logarithm of 10 would be 2^-21) and keeps its bits where the sum
// is near 1; what its rounding has lost, all of `others` where they are small beside an own term of 1, is added to first order.
__device__ __forceinline__ double ln_total(float own, float others)
{
    const float s = own + others, t = s - own, lost = (own - (s - t)) + (others - t);
    int e = __builtin_amdgcn_frexp_expf(s);
    float m = __builtin_amdgcn_frexp_mantf(s);
    if (m < 0.70710678f) {
        m += m;
        e -= 1;
    }
    return 0.69314718055994530942 * ((double)e + (double)__builtin_amdgcn_logf(m)) + (double)(lost * __builtin_amdgcn_rcpf(s));
}

// What a row's sum gives: p_j = exp((z_j - ref) c - ls), ls >= 0, exp(-ls), 1 - p_t, and lp.
struct Scored {
    float ref, ls, scale, rest;
    double lp;
};
// The statistics of a row as they are handed on: {ref, ls}, {ref, -ls} of a row that was summed with care and may hold NaN or have a
// reference other than its token's logit, {0, +inf} of a row that takes no part.
__device__ __forceinline__ float2 stats_of_row(Scored q, bool careful)
{
    return (float)q.lp == -INFINITY ? make_float2(0.0f, INFINITY) : make_float2(q.ref, careful ? -q.ls : q.ls);
}
// The row's own term, 2^(z c2 + nb) with the rounding of nb in it as in all others.
__device__ __forceinline__ float own_term(float z, float c2, float nb) { return __builtin_amdgcn_exp2f(fmaf(z, c2, nb)); }
// From the row's own term and the sum of the others, both relative to `ref` (the sum is NaN where an allowed logit is +inf).
__device__ __forceinline__ Scored score(float z, float ref, float own, float others, float inv_t)
{
    const double ls = ln_total(own, others), lp = ((double)z - (double)ref) * (double)inv_t - ls;
    // a sum beyond 2^126 has no normal reciprocal; own's share of it is zero
    const float scale = __builtin_amdgcn_rcpf(own + others);
    return {ref, fabsf((float)ls), scale, others < own ? others * scale : 1.0f - own * scale, lp > 0.0 ? 0.0 : lp};
}

// Sum of the exponentials of a row relative to its largest logit, NaN passed over and the token's own left out: what a row takes whose
// sum relative to its own token's logit z is not usable.  Sets *ref to the largest logit.
template <int DTYPE, int NT, int U, bool BITS>
__device__ __forceinline__ float careful_sum(const RowBuffers& row, int32_t n_groups, int32_t token, float z, float last, float c2, float* ref,
                                             const uint2 (&masks)[16], float (&part)[NT / 64])
{
    uint4 x[U];
    uint32_t b[U];
    float m = fmaxf(fmaxf(kLowest, z), last);
    for (int32_t g = 0; g < n_groups; g += NT * U) {
        fetch<DTYPE, NT, U, BITS>(row, g, n_groups, x, b);
#pragma unroll
        for (int k = 0; k < U; ++k)
            if (settle<DTYPE, BITS>(x[k], b[k], g + (int32_t)threadIdx.x + k * NT, n_groups, masks)) m = max_group<DTYPE>(x[k], m);
    }
    m = block_reduce<NT, true>(m, part);
    float s = __builtin_amdgcn_exp2f((fmaxf(last, -INFINITY) - m) * c2);
    for (int32_t g = 0; g < n_groups; g += NT * U) {
        fetch<DTYPE, NT, U, BITS>(row, g, n_groups, x, b);
        const Own own = own_of<DTYPE, NT, U>(token, g);
#pragma unroll
        for (int k = 0; k < U; ++k) {
            if (k == own.k) leave_own<DTYPE, BITS>(own, x[k], b[k]);
            if (settle<DTYPE, BITS>(x[k], b[k], g + (int32_t)threadIdx.x + k * NT, n_groups, masks)) add_group_careful<DTYPE>(x[k], c2, m, s);
        }
    }
    *ref = m;
    return block_reduce<NT, false>(s, part);
}

// What the sums of a row are taken relative to.  In 16 bits its own token's logit: no maximum is needed, and what the exponents lose where
// that is far below the largest (2^-24 of the distance) the rounding of the gradients hides.  In fp32 it would show: gradients of a
// token 10 below the largest were off by 6e-7 of themselves and 80 below by 4e-6, and are by 1e-7 whatever the token, so there a
// running maximum is kept.
template <int DTYPE> constexpr bool kRelativeToMax = DTYPE == TDFA_F32;

struct PolicyRow {
    float old, ref, adv, w;
};
__device__ __forceinline__ PolicyRow policy_row(const PolicyTerms& a, uint32_t i)
{
    return {a.old_logprobs[i], a.ref_logprobs ? a.ref_logprobs[i] : 0.0f, a.advantages[i], a.weights ? a.weights[i] : 1.0f};
}
__device__ __forceinline__ PolicyRow policy_row(const RowArgs&, uint32_t) { return {}; }
__device__ __forceinline__ const float* weights_of(const PolicyTerms& a) { return a.weights; }
__device__ __forceinline__ const float* weights_of(const RowArgs&) { return nullptr; }

// The term of a row from its log-probability: the loss and d loss / d lp.
__device__ __forceinline__ void policy_term(float clip_low, float clip_high, float kl_coef, bool kl, PolicyRow v, float lp, float* each, float* down)
{
    const float ratio = expf(lp - v.old);
    const float free = ratio * v.adv;
    const float clipped = fminf(fmaxf(ratio, clip_low), clip_high) * v.adv;
    // NaN (an infinite ratio and no advantage) stays NaN
    float e = clipped < free ? -clipped : -free, s = clipped < free ? 0.0f : -free;
    if (kl) {
        const float d = v.ref - lp, m = expm1f(d);
        e += kl_coef * (m - d);
        s -= kl_coef * m;
    }
    *each = v.w * e;
    *down = v.w * s;
}

// What is made of a row's sum (one thread): of a row that takes no part, and of one that does unless lp overflows.
__device__ __forceinline__ void leave_out(const ScoreArgs& a, uint32_t i, float lp)
{
    a.logprobs[i] = lp;
    if (a.stats) a.stats[i] = make_float2(0.0f, INFINITY);
}
__device__ __forceinline__ void leave_out(const PairScoreArgs& a, uint32_t i, float lp)
{
    a.logprobs[i] = lp;
    a.work[i] = {0.0, make_float2(0.0f, INFINITY), 0.0f, 0.0f};
}
__device__ __forceinline__ void leave_out(const PolicyScoreArgs& a, uint32_t i, float lp)
{
    a.logprobs[i] = lp;
    a.work[i] = {0.0, make_float2(0.0f, INFINITY), 0.0f, 0.0f};
}
__device__ __forceinline__ void finish(const ScoreArgs& a, uint32_t i, Scored q, bool careful, PolicyRow)
{
    a.logprobs[i] = (float)q.lp;
    if (a.stats) a.stats[i] = stats_of_row(q, careful);
}
__device__ __forceinline__ void finish(const PairScoreArgs& a, uint32_t i, Scored q, bool careful, PolicyRow)
{
    a.logprobs[i] = (float)q.lp;
    a.work[i] = {q.lp, stats_of_row(q, careful), 0.0f, q.scale};              // rows of no sequence keep a slope of zero
}
__device__ __forceinline__ void finish(const PolicyScoreArgs& a, uint32_t i, Scored q, bool careful, PolicyRow v)
{
    const float lp = (float)q.lp;
    float e = 0.0f, d = 0.0f;
    if (lp != -INFINITY) policy_term(a.clip_low, a.clip_high, a.kl_coef, a.ref_logprobs, v, lp, &e, &d);
    a.logprobs[i] = lp;
    a.work[i] = {(double)e, stats_of_row(q, careful), d, q.scale};
}

// One workgroup per row.  In 16 bits the sum is taken relative to the row's own token, ref = z_t, so that no maximum has to be known, terms
// are added as they arrive, and lp = -ln(1 + the sum of the others); where that overflows (lp below -87) or a NaN is met, the row is read
// again, for the largest logit and the sum relative to it.  In fp32 lanes keep a running maximum.  Bound by the memory where there are
// many rows: 2,900 rows of 128,256 tokens in bf16, on changing inputs, 83 us, of which 0.53 of the 128-byte lines hold an allowed token
// (394 MB, 4.7 TB/s; torch's maximum over the rows of a matrix reads 4.9 to 5.2), 2,047 of 32,003 in fp32 27 us (126 MB, 4.6 TB/s); by one
// compute unit's stream of a long row where there are few (256 KB in 7.4 us, about 40 GB/s whatever is in flight); by the chain token, bits,
// logits in short ones (2.6 us).
template <typename A, int DTYPE, int NT, int U, bool BITS>
__global__ void __launch_bounds__(NT, 8) token_stats_kernel(A a)
{
    constexpr bool kMax = kRelativeToMax<DTYPE>;
    __shared__ float s_part[NT / 64], s_running[2][NT / 64];
    __shared__ uint2 s_masks[16];
    const uint32_t i = blockIdx.x;
    const Row r = row_of(a, weights_of(a), i);
    const PolicyRow v = policy_row(a, i);
    const float c2 = a.inv_t * kLog2e;
    const int32_t n_groups = a.n_tokens / Elem<DTYPE>::kGroup;
    if (BITS && DTYPE == TDFA_BF16) {
        fill_masks(s_masks);
        __syncthreads();
    }
    const auto* row = row_at<DTYPE>(a.logits, i, a.stride16);
    if (!r.read) {
        if (threadIdx.x == 0) leave_out(a, i, r.lp);
        return;
    }
    // the first bits are on their way together with the token's logit
    const RowBuffers buf = row_buffers<DTYPE>(row, r.bits, n_groups);
    uint32_t b[U];
    fetch_bits<DTYPE, NT, U, BITS>(buf, 0, b);
    const float z = token_logit(r, row), last = last_element<DTYPE>(a.n_tokens, row, r.bits, r.token);
    if (z == -INFINITY) {
        if (threadIdx.x == 0) leave_out(a, i, r.lp);
        return;
    }
    float m = kMax ? fmaxf(z, last) : z;
    const float nb = offset_of(m, c2);
    float sum[2] = {__builtin_amdgcn_exp2f(fmaf(last, c2, nb)), 0.0f};
    for (int32_t g = 0; g < n_groups; g += NT * U) {
        uint4 x[U];
        uint32_t some;
        if (g) fetch_bits<DTYPE, NT, U, BITS>(buf, g, b);
        fetch_groups<DTYPE, NT, U, BITS>(buf, g, n_groups, x, b);
        if constexpr (kMax) add_groups_running<DTYPE, NT, U, BITS, false>(x, b, g, n_groups, s_masks, r.token, c2, m, sum, some);
        else add_groups<DTYPE, NT, U, BITS>(x, b, g, n_groups, s_masks, r.token, c2, nb, sum, some);
    }
    float own = 1.0f, s, ref = z;
    if constexpr (kMax) {
        s = sum_of_running<NT, false>(m, sum[0] + sum[1], c2, &ref, s_running);
    } else {
        s = block_reduce<NT, false>(sum[0] + sum[1], s_part);
        own = own_term(z, c2, nb);
        s *= __builtin_amdgcn_rcpf(own);
    }
    const bool careful = !usable(own, s);
    if (careful) s = careful_sum<DTYPE, NT, 2, BITS>(buf, n_groups, r.token, z, last, c2, &ref, s_masks, s_part);
    own = kMax || careful ? __builtin_amdgcn_exp2f((z - ref) * c2) : 1.0f;
    if (threadIdx.x == 0) finish(a, i, score(z, ref, own, s, a.inv_t), kMax || careful, v);
}

// The largest logit and the sum relative to it of a part of a row without the token's own; {kLowest, 0}: of none.
struct Part {
    float m, s;
};

// One workgroup per part of `span` groups of a row: few long rows are shared out, and every part finds a reference of its own (its largest
// logit: lanes keep a running maximum and sum, which begin at no logit of the row, so with differences taken first).  Bound by the memory: 300 rows of 256,000 tokens in fp32, half of whose lines are read
// (0.15 GB), on changing inputs 28 us (5.3 TB/s).
template <int DTYPE, int NT, int U, bool BITS>
__global__ void __launch_bounds__(NT) part_stats_kernel(RowArgs a, const float* weights, Part* out, int32_t parts, int32_t span)
{
    __shared__ float s_running[2][NT / 64];
    __shared__ uint2 s_masks[16];
    const uint32_t i = blockIdx.x / (uint32_t)parts;
    const int32_t part = (int32_t)(blockIdx.x - i * (uint32_t)parts);
    const Row r = row_of(a, weights, i);
    if (!r.read) return;
    const float c2 = a.inv_t * kLog2e;
    const int32_t n_groups = a.n_tokens / Elem<DTYPE>::kGroup;
    if (BITS && DTYPE == TDFA_BF16) {
        fill_masks(s_masks);
        __syncthreads();
    }
    const auto* row = row_at<DTYPE>(a.logits, i, a.stride16);
    const int32_t end = min(n_groups, (part + 1) * span);
    const RowBuffers buf = row_buffers<DTYPE>(row, r.bits, end);
    // fmaxf with a number passes over a NaN
    const float last = part == parts - 1 ? fmaxf(last_element<DTYPE>(a.n_tokens, row, r.bits, r.token), -INFINITY) : -INFINITY;
    float m = fmaxf(kLowest, last), s[2] = {__builtin_amdgcn_exp2f((last - m) * c2), 0.0f};
    for (int32_t g = part * span; g < end; g += NT * U) {
        uint4 x[U];
        uint32_t b[U], some;
        fetch<DTYPE, NT, U, BITS>(buf, g, end, x, b);
        add_groups_running<DTYPE, NT, U, BITS, true>(x, b, g, end, s_masks, r.token, c2, m, s, some);
    }
    float top;
    const float sum = sum_of_running<NT, true>(m, s[0], c2, &top, s_running);
    if (threadIdx.x == 0) out[blockIdx.x] = {top, sum};
}

// A wavefront per row joins its parts, at most 64.  Bound by its chain of reads (4.8 us).
template <typename A, int DTYPE>
__global__ void __launch_bounds__(kThreads) join_parts_kernel(A a, const Part* in, int32_t parts, uint32_t rows)
{
    const uint32_t i = blockIdx.x * (kThreads / 64) + threadIdx.x / 64;
    if (i >= rows) return;
    const int lane = threadIdx.x & 63;
    const Row r = row_of(a, weights_of(a), i);
    const PolicyRow v = policy_row(a, i);
    const float z = r.read ? token_logit(r, row_at<DTYPE>(a.logits, i, a.stride16)) : -INFINITY;
    if (z == -INFINITY) {
        if (lane == 0) leave_out(a, i, r.lp);
        return;
    }
    const float c2 = a.inv_t * kLog2e;
    const Part mine = lane < parts ? in[(int64_t)i * parts + lane] : Part{kLowest, 0.0f};
    const float top = fmaxf(wave_max(mine.m), z), s = wave_sum(mine.s * __builtin_amdgcn_exp2f((mine.m - top) * c2));
    if (lane == 0) finish(a, i, score(z, top, __builtin_amdgcn_exp2f((z - top) * c2), s, a.inv_t), true, v);
}

// What a row's gradient is made of: g_j = -d p_j, but d (1 - p_t) at the token.
struct Slope {
    float d, ref;
    float k;                   // 16 bits: p_j = 2^((z_j - ref) c2 + k), fp32: -d p_j = k 2^((z_j - ref) c2), which keeps exponents of likely tokens small
    float fold;                // 16 bits: |d| p_j = 2^(z_j c2 + fold), or NaN: not to be taken
};
// 1 - exp(lp), by its series (off by 2^-26 of itself) where it is small.
__device__ __forceinline__ float rest_from(float lp)
{
    const float near = fmaf(lp, fmaf(lp, fmaf(lp, fmaf(lp, fmaf(lp, fmaf(lp, 1.0f / 5040.0f, 1.0f / 720.0f), 1.0f / 120.0f), 1.0f / 24.0f), 1.0f / 6.0f), 0.5f), 1.0f);
    return lp > -0.35f ? -lp * near : 1.0f - __builtin_amdgcn_exp2f(lp * kLog2e);
}
// fold takes two roundings instead of a subtraction and a product per element: of ref c2, up to 2^10 here, and of its sum with k and
// log2 |d|, which may pass that (k and a small slope add up to -126 each).  They are 2^-15 and 2^-14 of the exponent at most, 2^-13.8 of p,
// next to a rounding of the result by up to 2^-8.  Careful rows (a NaN among the logits) do without.
template <int DTYPE>
__device__ __forceinline__ Slope slope_of(float d, float ref, float ls, float scale, float c2, bool careful)
{
    if constexpr (DTYPE == TDFA_F32) {
        return {d, ref, -d * scale, 0.0f};
    } else {
        const float k = -ls * kLog2e, nb = -ref * c2;
        const bool folds = !careful && fabsf(nb) < 1024.0f;
        return {d, ref, k, folds ? nb + (k + __builtin_amdgcn_logf(fabsf(d))) : __uint_as_float(0x7FC00000u)};
    }
}

__device__ __forceinline__ Slope shared_by_wave(Slope q) { return {shared_by_wave(q.d), shared_by_wave(q.ref), shared_by_wave(q.k), shared_by_wave(q.fold)}; }

// Gradient of one element other than the token's own.
template <int DTYPE>
__device__ __forceinline__ float gradient_of(float z, Slope q, float c2)
{
    const float g = DTYPE == TDFA_F32 ? q.k * __builtin_amdgcn_exp2f((z - q.ref) * c2) : -q.d * __builtin_amdgcn_exp2f(fmaf(z - q.ref, c2, q.k));
    return z == z ? g : 0.0f;
}
// Gradient of one group, the token's own element among the others.
template <int DTYPE>
__device__ __forceinline__ uint4 gradient_of(uint4 x, bool some, Slope q, float c2, bool folds, uint32_t sign)
{
    constexpr int G = Elem<DTYPE>::kGroup;
    if (!some) return make_uint4(0, 0, 0, 0);
    float z[G];
    unpack<DTYPE>(x, z);
    if (folds) {
#pragma unroll
        for (int j = 0; j < G; ++j) z[j] = __builtin_amdgcn_exp2f(fmaf(z[j], c2, q.fold));
        const uint4 y = pack<DTYPE>(z);
        return make_uint4(y.x ^ sign, y.y ^ sign, y.z ^ sign, y.w ^ sign);
    }
#pragma unroll
    for (int j = 0; j < G; ++j) z[j] = gradient_of<DTYPE>(z[j], q, c2);
    return pack<DTYPE>(z);
}

// What the gradients of all groups of a row share.
template <int DTYPE>
struct Writer {
    Slope q;
    float c2;
    bool folds;
    uint32_t sign;
    __device__ __forceinline__ Writer(Slope q, float c2)
        : q(q), c2(c2), folds(DTYPE == TDFA_BF16 && q.fold == q.fold), sign(q.d > 0.0f ? 0x80008000u : 0u) {}
    // some: the wavefront has an allowed token in its groups; here: the token's own is in one of them, and its gradient is y.
    __device__ __forceinline__ void write(__amdgpu_buffer_rsrc_t out, int32_t g, uint4 x, bool some, bool here, uint4 mask, float y) const
    {
        x = gradient_of<DTYPE>(x, some, q, c2, folds, sign);
        if (here) x = where(mask, DTYPE == TDFA_F32 ? __float_as_uint(y) : rounded_pair(y, y), x);
        set_group(out, g, x);
        next_group();
    }
};
// Where the gradient of a row comes from: statistics and slopes that the caller gives; those that the launches before have left; or the pairs
// of a preference loss of few rows, whose slopes each workgroup works out.  The losses are summed by the first workgroup of the last two.
struct GivenGradArgs : RowArgs {
    const float2* stats;
    const float* down;
    void* grad;
    uint32_t grad_stride16;
    int32_t parts;
};
struct WorkGradArgs : RowArgs {
    const RowWork* work;
    const double* each;        // the losses, `step` apart
    float* loss;
    void* grad;
    uint32_t grad_stride16, n;
    int32_t parts, step, mean;
};
struct PairArgsOnCard {        // of a preference loss
    const float* ref_logprobs;
    const int32_t* begin;
    float* rewards;
    int32_t n_pairs, rows;
    float beta, smoothing;
};
struct FewPairsGradArgs {
    const uint32_t* allow;
    const void* logits;
    const int32_t* states;
    const int32_t* tokens;
    const RowWork* work;
    void* grad;
    float* loss;
    PairArgsOnCard pairs;
    uint32_t stride16, grad_stride16;
    int32_t n_tokens;
    float inv_t;
};
static_assert(sizeof(FewPairsGradArgs) <= 112 && sizeof(WorkGradArgs) <= 112, "the arguments of a launch that costs the host little");

// Sums of lp - ref over the rows of the two sequences of pair k, as far as `lane` of `width` lanes has them.  A sequence that reaches
// outside the rows is cut there.
__device__ __forceinline__ void add_pair(const PairArgsOnCard& p, const RowWork* work, int64_t k, int lane, int width, double (&sum)[2])
{
    const int32_t b0 = p.begin[2 * k], b1 = p.begin[2 * k + 1], b2 = p.begin[2 * k + 2];
#pragma unroll
    for (int side = 0; side < 2; ++side) {
        const int64_t from = max(side ? b1 : b0, 0), to = min(side ? b2 : b1, p.rows);
        for (int64_t i = from + lane; i < to; i += width) {
            const double lp = work[i].value, ref = (double)p.ref_logprobs[i];
            if (work[i].stats.y != INFINITY) sum[side] += lp - ref;
        }
    }
}
// softplus(x) = max(x, 0) + log1p(exp(-|x|)); binary32 from the difference of the rewards on.  A gap may be infinite (a reference that gives
// a token probability zero), which a side of weight zero has nothing of.
__device__ __forceinline__ float pair_loss(const PairArgsOnCard& p, float gap)
{
    const float weight = gap > 0.0f ? p.smoothing : 1.0f - p.smoothing;
    return log1pf(expf(-fabsf(gap))) + (weight == 0.0f ? 0.0f : weight * fabsf(gap));
}
// d loss / d lp of a row of the pair's first sequence.
__device__ __forceinline__ float pair_slope(const PairArgsOnCard& p, float gap)
{
    return (p.smoothing / (1.0f + expf(-gap)) - (1.0f - p.smoothing) / (1.0f + expf(gap))) * (p.beta / (float)p.n_pairs);
}
// Both sums over the workgroup, in every thread.  Two barriers.
template <int NT>
__device__ __forceinline__ void reduce_pair(double (&sum)[2], double (&part)[2][NT / 64])
{
#pragma unroll
    for (int d = 32; d; d >>= 1) {
        sum[0] += __shfl_xor(sum[0], d);
        sum[1] += __shfl_xor(sum[1], d);
    }
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        part[0][threadIdx.x >> 6] = sum[0];
        part[1][threadIdx.x >> 6] = sum[1];
    }
    __syncthreads();
    sum[0] = part[0][0];
    sum[1] = part[1][0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) {
        sum[0] += part[0][w];
        sum[1] += part[1][w];
    }
}
// One workgroup per pair: the two rewards, the pair's loss, and d loss / d lp of every row of the pair.  Bound by its chain of reads
// (32 pairs of 90 rows 4.8 us).
__global__ void __launch_bounds__(kThreads) pair_kernel(PairArgsOnCard p, RowWork* work, double* each, int32_t blocks)
{
    __shared__ double s_part[2][kThreads / 64];
    for (int64_t k = blockIdx.x; k < p.n_pairs; k += blocks) {
        double sum[2] = {0.0, 0.0};
        add_pair(p, work, k, threadIdx.x, kThreads, sum);
        reduce_pair<kThreads>(sum, s_part);
        const double chosen = (double)p.beta * sum[0], rejected = (double)p.beta * sum[1];
        const float gap = (float)(chosen - rejected), slope = pair_slope(p, gap);
        if (threadIdx.x == 0) {
            p.rewards[2 * k] = (float)chosen;
            p.rewards[2 * k + 1] = (float)rejected;
            each[k] = (double)pair_loss(p, gap);
        }
        const int32_t b0 = p.begin[2 * k], b1 = p.begin[2 * k + 1], b2 = p.begin[2 * k + 2];
        for (int64_t i = (int64_t)max(b0, 0) + threadIdx.x; i < min(b1, p.rows); i += kThreads) work[i].down = slope;
        for (int64_t i = (int64_t)max(b1, 0) + threadIdx.x; i < min(b2, p.rows); i += kThreads) work[i].down = -slope;
    }
}

// All pairs by one workgroup, 16 lanes to a pair: the rewards and the loss.
template <int NT>
__device__ __forceinline__ void sum_pairs(const PairArgsOnCard& p, const RowWork* work, float* loss, double (&part)[NT / 64])
{
    double total = 0.0;
    const int lane = threadIdx.x & 15;
    for (int64_t k0 = 0; k0 < p.n_pairs; k0 += NT / 16) {
        const int64_t k = k0 + threadIdx.x / 16;
        double sum[2] = {0.0, 0.0};
        if (k < p.n_pairs) add_pair(p, work, k, lane, 16, sum);
#pragma unroll
        for (int d = 8; d; d >>= 1) {
            sum[0] += __shfl_xor(sum[0], d);
            sum[1] += __shfl_xor(sum[1], d);
        }
        if (lane == 0 && k < p.n_pairs) {
            const double chosen = (double)p.beta * sum[0], rejected = (double)p.beta * sum[1];
            p.rewards[2 * k] = (float)chosen;
            p.rewards[2 * k + 1] = (float)rejected;
            total += (double)pair_loss(p, (float)(chosen - rejected));
        }
    }
    total = reduce_sum<NT>(total, part);
    if (threadIdx.x == 0) *loss = (float)(total / (double)p.n_pairs);
}

// d loss / d lp of row i, by the whole workgroup: its sequence is looked for and the pair's rewards are summed again.  Of few rows and
// pairs this costs less than a launch that hands it on.
template <int NT>
__device__ __forceinline__ float slope_of_row(const PairArgsOnCard& p, const RowWork* work, int32_t i, int& found, double (&part)[2][NT / 64])
{
    if (threadIdx.x == 0) found = -1;
    __syncthreads();
    for (int k = threadIdx.x; k < 2 * p.n_pairs; k += NT)
        if (p.begin[k] <= i && i < p.begin[k + 1]) found = k;
    __syncthreads();
    const int k = __builtin_amdgcn_readfirstlane(found);
    if (k < 0) return 0.0f;
    double sum[2] = {0.0, 0.0};
    add_pair(p, work, k / 2, threadIdx.x, NT, sum);
    reduce_pair<NT>(sum, part);
    const float slope = pair_slope(p, (float)((double)p.beta * sum[0] - (double)p.beta * sum[1]));
    return k & 1 ? -slope : slope;
}

// The policy loss from the log-probabilities that a launch before has written: `span` rows to a workgroup, which leaves its sum in out, or
// the loss if it is the only one.  Up to 1,024 rows 2.0 us, a chain of two reads; 4,096 rows 4.1, 8,192 rows 6.6, 16,384 rows 12.1, bound by the
// exponentials of one compute unit (with the reads of four rows on their way together 3.3, 4.1, 6.3 and 10.5).
struct PolicySumArgs {
    const float* logprobs;
    const float* old_logprobs;
    const float* ref_logprobs;
    const float* advantages;
    const float* weights;
    const int32_t* tokens;
    float* loss;               // or NULL
    double* out;
    uint32_t rows, span;
    float clip_low, clip_high, kl_coef;
};
__global__ void __launch_bounds__(1024) policy_sum_kernel(PolicySumArgs a)
{
    __shared__ double s_part[16];
    const int64_t from = (int64_t)blockIdx.x * a.span, to = min(from + a.span, (int64_t)a.rows);
    double sum = 0.0;
    for (int64_t i = from + threadIdx.x; i < to; i += 1024) {
        const PolicyRow v = {a.old_logprobs[i], a.ref_logprobs ? a.ref_logprobs[i] : 0.0f, a.advantages[i], a.weights ? a.weights[i] : 1.0f};
        const float lp = a.logprobs[i];
        float e, d;
        policy_term(a.clip_low, a.clip_high, a.kl_coef, a.ref_logprobs, v, lp, &e, &d);
        if (a.tokens[i] != TDFA_NO_TOKEN && v.w != 0.0f && lp != -INFINITY) sum += (double)e;          // of rows that take part
    }
    sum = reduce_sum<1024>(sum, s_part);
    if (threadIdx.x == 0) {
        if (a.loss) *a.loss = (float)sum;
        else a.out[blockIdx.x] = sum;
    }
}

// What a gradient workgroup knows of its row: the token, the allowed bits, the statistics, d loss / d lp (0: the row takes no part).  Only
// what the caller gives is checked again.
struct GradRow {
    const uint32_t* bits;
    int32_t token;
    float2 stats;
    float down;
    float scale;               // exp(-ls), of fp32 rows
};
template <int NT>
__device__ __forceinline__ GradRow grad_row(const GivenGradArgs& a, uint32_t i)
{
    const float2 st = a.stats[i];
    const float down = a.down[i];
    const Row r = row_of(a, nullptr, i);
    return {r.bits, r.token, st, r.read && st.y != INFINITY ? down : 0.0f, expf(-fabsf(st.y))};
}
template <int NT>
__device__ __forceinline__ GradRow grad_row(const WorkGradArgs& a, uint32_t i)
{
    const float2 st = a.work[i].stats;
    const float down = a.work[i].down, scale = a.work[i].scale;
    const int32_t token = __builtin_amdgcn_readfirstlane(a.tokens[i]), q = a.allow ? __builtin_amdgcn_readfirstlane(a.states[i]) : 0;
    if (st.y == INFINITY) return {nullptr, token, st, 0.0f, 0.0f};
    return {a.allow ? bits_of(a.allow, q, a.n_tokens) : nullptr, token, st, down, scale};
}
template <int NT>
__device__ __forceinline__ GradRow grad_row(const FewPairsGradArgs& a, uint32_t i)
{
    __shared__ int s_found;
    __shared__ double s_sums[2][NT / 64];
    const float2 st = a.work[i].stats;
    const int32_t token = __builtin_amdgcn_readfirstlane(a.tokens[i]), q = a.allow ? __builtin_amdgcn_readfirstlane(a.states[i]) : 0;
    if (__builtin_amdgcn_readfirstlane(__float_as_int(st.y)) == 0x7F800000) return {nullptr, token, st, 0.0f, 0.0f};
    const float scale = a.work[i].scale, down = slope_of_row<NT>(a.pairs, a.work, (int32_t)i, s_found, s_sums);
    return {a.allow ? bits_of(a.allow, q, a.n_tokens) : nullptr, token, st, down, scale};
}
// What the first workgroup does beside the rows; false: nothing, it takes a row like the others.
template <int NT>
__device__ __forceinline__ bool first_block(const GivenGradArgs&) { return false; }
template <int NT>
__device__ __forceinline__ bool first_block(const WorkGradArgs& a)
{
    __shared__ double s_part[NT / 64];
    sum_losses<NT>(a.each, a.n, a.step, a.mean, a.loss, s_part);
    return true;
}
template <int NT>
__device__ __forceinline__ bool first_block(const FewPairsGradArgs& a)
{
    __shared__ double s_part[NT / 64];
    sum_pairs<NT>(a.pairs, a.work, a.loss, s_part);
    return true;
}
template <typename A> constexpr uint32_t kFirst = 1;          // workgroups before those of the rows
template <> constexpr uint32_t kFirst<GivenGradArgs> = 0;
template <int SPAN, typename A>
__device__ __forceinline__ int32_t parts_of(const A& a, int32_t) { return a.parts; }
template <int SPAN>
__device__ __forceinline__ int32_t parts_of(const FewPairsGradArgs&, int32_t n_groups) { return max(1, (n_groups + SPAN - 1) / SPAN); }

// grad[i][j] = down[i] c ([j = t] - p_j) over A, 0 elsewhere; 0 throughout in a row that takes no part.  A workgroup
// takes NT U groups of one row; the last of a row takes the elements behind the last whole group too.  Bound by the memory: 2,048 rows of
// 128,256 tokens in bf16 104 us (525 MB written and 255 MB of lines read, in part from the 256 MB cache that the sums have left full:
// 7.4 TB/s), 8 groups in flight per thread (4: 112, 2: 150).
template <typename A, int DTYPE, int NT, int U, bool BITS>
__global__ void __launch_bounds__(NT) token_grad_kernel(A a)
{
    constexpr int G = Elem<DTYPE>::kGroup;
    __shared__ uint2 s_masks[16];
    if (BITS && DTYPE == TDFA_BF16) {
        fill_masks(s_masks);
        __syncthreads();
    }
    if (blockIdx.x < kFirst<A>) {
        first_block<NT>(a);
        return;
    }
    const float c2 = a.inv_t * kLog2e;
    const int32_t n_groups = a.n_tokens / G, parts = parts_of<NT * U>(a, n_groups);
    const uint32_t w = blockIdx.x - kFirst<A>, i = w / (uint32_t)parts;
    const int32_t part = (int32_t)(w - i * (uint32_t)parts);
    const GradRow r = grad_row<NT>(a, i);
    const Slope q = shared_by_wave(slope_of<DTYPE>(r.down * a.inv_t, r.stats.x, fabsf(r.stats.y), r.scale, c2, signbit(r.stats.y)));
    const auto* row = row_at<DTYPE>(a.logits, i, a.stride16);
    auto* out = row_at<DTYPE>(a.grad, i, a.grad_stride16);
    const __amdgpu_buffer_rsrc_t to = buffer_of(out, (uint32_t)n_groups * 16u);
    const int32_t g0 = part * (NT * U), g = g0 + (int32_t)threadIdx.x;
    const int32_t behind = n_groups * G + (int32_t)threadIdx.x;
    if (q.d == 0.0f) {
#pragma unroll
        for (int k = 0; k < U; ++k) set_group(to, g + k * NT, make_uint4(0, 0, 0, 0));
        if (part == parts - 1 && behind < a.n_tokens) store_rounded(out + behind, 0.0f);
        return;
    }
    const float last = part == parts - 1 ? last_element<DTYPE>(a.n_tokens, row, r.bits, -1) : -INFINITY;
    uint4 x[U];
    uint32_t b[U];
    fetch<DTYPE, NT, U, BITS, true>(row_buffers<DTYPE>(row, r.bits, n_groups), g0, n_groups, x, b);
    const Writer<DTYPE> writer(q, c2);
    const Own own = own_of<DTYPE, NT, U>(r.token, g0);
    uint4 held = {};           // the groups with the token's own, which come last
    bool held_some = false;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const bool some = settle<DTYPE, BITS>(x[k], b[k], g + k * NT, n_groups, s_masks);
        if (k == own.k) {
            held = x[k];
            held_some = some;
        } else {
            writer.write(to, g + k * NT, x[k], some, false, own.mask, 0.0f);
        }
    }
    // lp from what the other elements are made of too: the statistics are the same whatever made them
    const auto lp_of = [&](float z) { return fmaf(z - q.ref, a.inv_t, -fabsf(r.stats.y)); };
    if (own.k >= 0) writer.write(to, g + own.k * NT, held, held_some, true, own.mask, q.d * rest_from(lp_of(element_of<DTYPE>(held, own.j))));
    if (part == parts - 1 && behind < a.n_tokens) store_rounded(out + behind, behind == r.token ? q.d * rest_from(lp_of(last)) : gradient_of<DTYPE>(last, q, c2));
}

constexpr int64_t kWholeGroups = 1024 * 16;
constexpr int kMaxParts = 64;
constexpr int64_t kPartRows = 384;

// One workgroup per row: the sum, the row's term, the gradient.  The row stays in registers between the sum and the gradient, R groups
// to a thread: 1,024 threads hold 256 KB, half of a compute unit's registers, and the row is read once.  Bound by the memory, on changing
// inputs: 1,024 rows of 128,256 tokens in bf16 without a constraint 95 us for 263 MB read and as much written (5.5 TB/s; an elementwise
// product of such matrices takes 87, a copy 100); 4,096 rows under one 280 us, 1.05 GB written and 0.51 GB of lines read (5.6 TB/s).  Vector
// instructions take two fifths of the time.  Two rows to a compute unit with half of each read twice: 316 us; workgroups that stay, and
// fetch the next row into the registers that the gradient leaves: 119 us for the 1,024.
template <int DTYPE, int NT, int R, bool BITS>
__global__ void __launch_bounds__(NT, 4) policy_row_kernel(PolicyRowArgs a)
{
    constexpr int G = Elem<DTYPE>::kGroup;
    __shared__ float s_part[NT / 64], s_running[2][NT / 64];
    __shared__ uint2 s_masks[16];
    __shared__ Slope s_slope;
    __shared__ float s_own;
    const uint32_t i = blockIdx.x;
    const Row r = row_of(a, a.weights, i);
    const PolicyRow v = policy_row(a, i);
    const float c2 = a.inv_t * kLog2e;
    const int32_t n_groups = a.n_tokens / G;
    if (BITS && DTYPE == TDFA_BF16) {
        fill_masks(s_masks);
        __syncthreads();
    }
    const auto* row = row_at<DTYPE>(a.logits, i, a.stride16);
    const RowBuffers buf = row_buffers<DTYPE>(row, r.bits, n_groups);
    Slope q = {0.0f, 0.0f, 0.0f, 0.0f};
    float last = -INFINITY, own_slope = 0.0f;
    uint4 x[R];
    uint32_t some = 0;
    uint32_t b[R];
    float z = -INFINITY;
    if (r.read) {                                          // the bits are on their way together with the token's logit
        fetch_bits<DTYPE, NT, R, BITS>(buf, 0, b);
        z = token_logit(r, row);
        last = last_element<DTYPE>(a.n_tokens, row, r.bits, r.token);
    }
    if (z > -INFINITY) {
        fetch_groups<DTYPE, NT, R, BITS, true>(buf, 0, n_groups, x, b);
        constexpr bool kMax = kRelativeToMax<DTYPE>;
        float m = kMax ? fmaxf(z, last) : z;
        const float nb = offset_of(m, c2);
        float sum[2] = {__builtin_amdgcn_exp2f(fmaf(last, c2, nb)), 0.0f}, own = 1.0f, s, ref = z;
        if constexpr (kMax) {
            add_groups_running<DTYPE, NT, R, BITS, false>(x, b, 0, n_groups, s_masks, r.token, c2, m, sum, some);
            s = sum_of_running<NT, false>(m, sum[0] + sum[1], c2, &ref, s_running);
        } else {
            add_groups<DTYPE, NT, R, BITS>(x, b, 0, n_groups, s_masks, r.token, c2, nb, sum, some);
            s = block_reduce<NT, false>(sum[0] + sum[1], s_part);
            own = own_term(z, c2, nb);
            s *= __builtin_amdgcn_rcpf(own);
        }
        const bool careful = !usable(own, s);
        if (careful) {
            ref = fmaxf(fmaxf(kLowest, z), last);
#pragma unroll
            for (int k = 0; k < R; ++k)
                if (some >> k & 1) ref = max_group<DTYPE>(x[k], ref);
            ref = block_reduce<NT, true>(ref, s_part);
            s = __builtin_amdgcn_exp2f((fmaxf(last, -INFINITY) - ref) * c2);
#pragma unroll
            for (int k = 0; k < R; ++k)
                if (some >> k & 1) add_group_careful<DTYPE>(x[k], c2, ref, s);
            s = block_reduce<NT, false>(s, s_part);
        }
        own = kMax || careful ? __builtin_amdgcn_exp2f((z - ref) * c2) : 1.0f;
        if (threadIdx.x < 64) {
            const Scored sc = score(z, ref, own, s, a.inv_t);
            const float lp = (float)sc.lp;
            float e = 0.0f, d = 0.0f;
            if (lp != -INFINITY) policy_term(a.clip_low, a.clip_high, a.kl_coef, a.ref_logprobs, v, lp, &e, &d);
            if (threadIdx.x == 0) {
                a.logprobs[i] = lp;
                s_slope = slope_of<DTYPE>(d * a.inv_t, sc.ref, sc.ls, sc.scale, c2, kMax || careful);
                s_own = d * a.inv_t * sc.rest;
            }
        }
        __syncthreads();
        q = shared_by_wave(s_slope);
        own_slope = s_own;
    } else {
        // A gradient may lie over the logits: no wavefront writes before all have read the token's logit (above, the sum's barriers see to it).
        if (r.read) __syncthreads();
        if (threadIdx.x == 0) a.logprobs[i] = r.lp;
    }
    if (!a.grad) return;
    auto* out = row_at<DTYPE>(a.grad, i, a.grad_stride16);
    const __amdgpu_buffer_rsrc_t to = buffer_of(out, (uint32_t)n_groups * 16u);
    const int32_t behind = n_groups * G + (int32_t)threadIdx.x;
    if (q.d == 0.0f) {
        for (int32_t g = threadIdx.x; g < n_groups; g += NT) set_group(to, g, make_uint4(0, 0, 0, 0));
        if (behind < a.n_tokens) store_rounded(out + behind, 0.0f);
        return;
    }
    some = __builtin_amdgcn_readfirstlane(some);
    const Writer<DTYPE> writer(shared_by_wave(q), c2);
    const Own own = own_of<DTYPE, NT, R>(r.token, 0);
#pragma unroll
    for (int k = 0; k < R; ++k) writer.write(to, (int32_t)threadIdx.x + k * NT, x[k], some >> k & 1, k == own.k, own.mask, own_slope);
    if (behind < a.n_tokens) store_rounded(out + behind, behind == r.token ? own_slope : gradient_of<DTYPE>(last, q, c2));
}

RowArgs row_args(const TokenRows& a, int64_t from)
{
    const int64_t esz = a.dtype == TDFA_F32 ? 4 : 2;
    return {a.allow, static_cast<const char*>(a.logits) + from * a.row_stride * esz, a.states ? a.states + from : nullptr, a.tokens + from,
            (uint32_t)(a.rows > 1 ? a.row_stride * esz / 16 : 0), (int32_t)std::min<int64_t>(a.n_states, INT32_MAX), a.n_tokens, a.inv_t};
}
uint32_t grad_stride16(const TokenRows& a, int64_t grad_stride) { return (uint32_t)(a.rows > 1 ? grad_stride * (a.dtype == TDFA_F32 ? 4 : 2) / 16 : 0); }
void* grad_from(const TokenRows& a, void* grad, int64_t grad_stride, int64_t from)
{
    return grad ? static_cast<char*>(grad) + from * grad_stride * (a.dtype == TDFA_F32 ? 4 : 2) : nullptr;
}

// What a call scores into.
struct Score {
    float* logprobs;
    float2* stats;             // for the caller, or NULL
    RowWork* work;             // for a loss, or NULL
    const PolicyArgs* policy;  // for the policy loss, or NULL
};
void fill(ScoreArgs& x, const TokenRows&, const Score& o, int64_t from)
{
    x.logprobs = o.logprobs + from;
    x.stats = o.stats ? o.stats + from : nullptr;
}
void fill(PairScoreArgs& x, const TokenRows&, const Score& o, int64_t from)
{
    x.logprobs = o.logprobs + from;
    x.work = o.work + from;
}
void fill_terms(PolicyTerms& x, const TokenRows& a, const PolicyArgs& p, float* logprobs, int64_t from)
{
    x.old_logprobs = p.old_logprobs + from;
    x.ref_logprobs = p.ref_logprobs ? p.ref_logprobs + from : nullptr;
    x.advantages = p.advantages + from;
    x.weights = a.weights ? a.weights + from : nullptr;
    x.logprobs = logprobs + from;
    x.clip_low = p.clip_low;
    x.clip_high = p.clip_high;
    x.kl_coef = p.kl_coef;
    x.grad_stride16 = 0;
}
void fill(PolicyScoreArgs& x, const TokenRows& a, const Score& o, int64_t from)
{
    fill_terms(x, a, *o.policy, o.logprobs, from);
    x.work = o.work + from;
}

template <typename A, int DTYPE, bool BITS>
int stats_launch(const TokenRows& a, const Score& o, hipStream_t stream)
{
    constexpr bool kLong = std::is_same_v<A, PolicyScoreArgs>;             // of a policy loss only what one_launch leaves
    const int32_t n_groups = a.n_tokens / Elem<DTYPE>::kGroup;
    for (int64_t from = 0; from < a.rows; from += kMaxBlocks) {
        const dim3 grid((unsigned)std::min(a.rows - from, kMaxBlocks));
        A x;
        static_cast<RowArgs&>(x) = row_args(a, from);
        fill(x, a, o, from);
        int rc = TDFA_OK;
        // Two rows or more to a compute unit, so that one is fetched while another is summed.  Rows too few to fill the card are shared by
        // more wavefronts each: 24 rows of 32,000 tokens in bf16 6.0 -> 5.1 us, 400 rows 8.2 -> 7.7; of 8,000 tokens 4.1 either way, 400
        // rows 4.5 -> 5.4.
        if (a.rows <= 512 && n_groups > 256 * 8 && n_groups <= 512 * 16) rc = launch(token_stats_kernel<A, DTYPE, 1024, 4, BITS>, grid, 1024, stream, x);
        else if (kLong || n_groups > 512 * 16) rc = launch(token_stats_kernel<A, DTYPE, 1024, 8, BITS>, grid, 1024, stream, x);
        else if constexpr (!kLong) {
            if (n_groups <= 64 * 4) rc = launch(token_stats_kernel<A, DTYPE, 64, 4, BITS>, grid, 64, stream, x);
            else if (n_groups <= 256 * 16) rc = launch(token_stats_kernel<A, DTYPE, 256, 8, BITS>, grid, 256, stream, x);
            else rc = launch(token_stats_kernel<A, DTYPE, 512, 8, BITS>, grid, 512, stream, x);
        }
        if (rc != TDFA_OK) return rc;
    }
    return TDFA_OK;
}

template <typename A, int DTYPE, bool BITS>
int parts_launch(const TokenRows& a, const Score& o, Part* out, hipStream_t stream)
{
    const int32_t n_groups = a.n_tokens / Elem<DTYPE>::kGroup, round = 256 * 8;
    const int32_t span = (n_groups + kMaxParts * round - 1) / (kMaxParts * round) * round, parts = (n_groups + span - 1) / span;
    A x;
    static_cast<RowArgs&>(x) = row_args(a, 0);
    fill(x, a, o, 0);
    const int rc = launch(part_stats_kernel<DTYPE, 256, 8, BITS>, dim3((unsigned)(a.rows * parts)), 256, stream, static_cast<RowArgs&>(x), a.weights, out, parts, span);
    if (rc != TDFA_OK) return rc;
    return launch(join_parts_kernel<A, DTYPE>, dim3((unsigned)((a.rows + kThreads / 64 - 1) / (kThreads / 64))), kThreads, stream, x,
                  static_cast<const Part*>(out), parts, (uint32_t)a.rows);
}

int64_t groups_of(const TokenRows& a) { return a.n_tokens / (a.dtype == TDFA_F32 ? Elem<TDFA_F32>::kGroup : Elem<TDFA_BF16>::kGroup); }

// Rows that are longer than a workgroup's registers, too few of them to fill the card, are shared out by parts, which a second launch joins:
// one row of 128,256 tokens in fp32 8.0 us by one workgroup, 5.6 so, 64 rows 12.9 and 10.0.  Up to 256 rows have a compute unit each, and the
// join costs more than the parts bring unless rows are very long (200 rows 14.1 and 15.8; of 256,000 tokens 28.0 and 24.8; in bf16 18.5 and
// 20.8, of 512,000 35.1 and 32.5); of 257 rows some compute units have two (300 rows 23.8 and 19.7; in bf16 of 256,000 29.9 and 27.1,
// of 140,000 18.6 and 19.3), and from some 400 on there is no difference (512 rows 31.0 and 30.9).
bool in_parts(const TokenRows& a)
{
    const int64_t n_groups = groups_of(a);
    return n_groups > kWholeGroups && (a.rows <= 64 || (a.rows > 256 && a.rows <= kPartRows) || (a.rows <= 256 && n_groups > 3 * kWholeGroups));
}

// parts: workspace for kMaxParts parts of each of the first kPartRows rows.
template <typename A>
int stats_of(const TokenRows& a, const Score& o, Part* parts, hipStream_t stream)
{
    if (in_parts(a)) {
        if (a.dtype == TDFA_F32) return a.allow ? parts_launch<A, TDFA_F32, true>(a, o, parts, stream) : parts_launch<A, TDFA_F32, false>(a, o, parts, stream);
        return a.allow ? parts_launch<A, TDFA_BF16, true>(a, o, parts, stream) : parts_launch<A, TDFA_BF16, false>(a, o, parts, stream);
    }
    if (a.dtype == TDFA_F32) return a.allow ? stats_launch<A, TDFA_F32, true>(a, o, stream) : stats_launch<A, TDFA_F32, false>(a, o, stream);
    return a.allow ? stats_launch<A, TDFA_BF16, true>(a, o, stream) : stats_launch<A, TDFA_BF16, false>(a, o, stream);
}

// set(x, from, parts) fills in what a launch for the rows from `from` on has beside the rows' arguments.
template <typename A, int DTYPE, bool BITS, typename F>
int grad_launch(const TokenRows& a, hipStream_t stream, F set)
{
    const int32_t n_groups = a.n_tokens / Elem<DTYPE>::kGroup;
    // Few rows in parts of half the size: gradients of 128 rows of 32,000 tokens in bf16 7 -> 6 us; 2,048 of 128,256 107 -> 112.
    constexpr bool kPairs = std::is_same_v<A, FewPairsGradArgs>;     // a row's slope is worked out by a whole workgroup
    const bool few = a.rows <= 128, tiny = !kPairs && n_groups <= 64 * 4;
    const int32_t span = tiny ? 64 * 4 : few ? 256 * 4 : 256 * 8, parts = std::max(1, (n_groups + span - 1) / span);
    const int64_t most = (4 * kMaxBlocks - 1) / parts;     // workgroups of 256 threads
    for (int64_t from = 0; from < a.rows; from += most) {
        const dim3 grid((unsigned)(std::min(a.rows - from, most) * parts + kFirst<A>));
        A x;
        set(x, from, parts);
        int rc = TDFA_OK;
        if (few && !tiny) rc = launch(token_grad_kernel<A, DTYPE, 256, 4, BITS>, grid, 256, stream, x);
        else if (!tiny) rc = launch(token_grad_kernel<A, DTYPE, 256, 8, BITS>, grid, 256, stream, x);
        else if constexpr (!kPairs) rc = launch(token_grad_kernel<A, DTYPE, 64, 4, BITS>, grid, 64, stream, x);
        if (rc != TDFA_OK) return rc;
    }
    return TDFA_OK;
}
template <typename A, typename F>
int grad_of(const TokenRows& a, hipStream_t stream, F set)
{
    if (a.dtype == TDFA_F32) return a.allow ? grad_launch<A, TDFA_F32, true>(a, stream, set) : grad_launch<A, TDFA_F32, false>(a, stream, set);
    return a.allow ? grad_launch<A, TDFA_BF16, true>(a, stream, set) : grad_launch<A, TDFA_BF16, false>(a, stream, set);
}

// The gradient from what the launches before have left, and the loss from n losses that lie `step` apart.
int grad_of_work(const TokenRows& a, const RowWork* work, const double* each, int64_t n, int32_t step, bool mean, float* loss, void* grad,
                 int64_t grad_stride, hipStream_t stream)
{
    return grad_of<WorkGradArgs>(a, stream, [&](WorkGradArgs& x, int64_t from, int32_t parts) {
        static_cast<RowArgs&>(x) = row_args(a, from);
        x.work = work + from;
        x.each = each;
        x.loss = loss;
        x.grad = grad_from(a, grad, grad_stride, from);
        x.grad_stride16 = grad_stride16(a, grad_stride);
        x.n = (uint32_t)n;
        x.parts = parts;
        x.step = step;
        x.mean = mean;
    });
}

template <int DTYPE, bool BITS>
int policy_launch(const TokenRows& a, const PolicyArgs& p, float* logprobs, void* grad, int64_t grad_stride, hipStream_t stream)
{
    const int32_t n_groups = a.n_tokens / Elem<DTYPE>::kGroup;
    for (int64_t from = 0; from < a.rows; from += kMaxBlocks) {
        const dim3 grid((unsigned)std::min(a.rows - from, kMaxBlocks));
        PolicyRowArgs x;
        static_cast<RowArgs&>(x) = row_args(a, from);
        fill_terms(x, a, p, logprobs, from);
        x.grad = grad_from(a, grad, grad_stride, from);
        x.grad_stride16 = grad_stride16(a, grad_stride);
        int rc;
        // The more wavefronts share a row, the sooner it is read: 1,500 rows of 32,000 tokens in bf16 34.4 us by 1,024 threads of 4 groups,
        // 38.5 by 256 of 16; 24 rows 9.1 and 10.4 (of 20,000 tokens, 1,500 rows 27.6 and 26.3).
        if (n_groups <= 64 * 8) rc = launch(policy_row_kernel<DTYPE, 64, 8, BITS>, grid, 64, stream, x);
        else if (n_groups <= 256 * 8) rc = launch(policy_row_kernel<DTYPE, 256, 8, BITS>, grid, 256, stream, x);
        else if (n_groups <= 1024 * 4) rc = launch(policy_row_kernel<DTYPE, 1024, 4, BITS>, grid, 1024, stream, x);
        else if (n_groups <= 1024 * 8) rc = launch(policy_row_kernel<DTYPE, 1024, 8, BITS>, grid, 1024, stream, x);
        else rc = launch(policy_row_kernel<DTYPE, 1024, 16, BITS>, grid, 1024, stream, x);
        if (rc != TDFA_OK) return rc;
    }
    return TDFA_OK;
}

// Whether a policy loss is scored and its gradient written by one launch, a workgroup per row that reads it once, or by two, which read
// it twice but share the second out by parts of rows.  Two are faster where few long rows leave compute units idle (24 rows of
// 128,256 tokens in bf16 14.8 us against 17.3, of 64,000 10.1 against 11.5; 40 rows 17.0 and 17.4, 11.5 and 11.8; 64 rows 19.1 and 18.0, 12.6
// and 12.0; 24, 40 and 64 rows of 60,000 in fp32 12.7, 14.2 and 16.5 against 13.9, 14.2 and 14.6) and where a row does not fit a
// workgroup's registers (300 rows of 256,000 in fp32 117 us, 167 with half of every row read twice by one launch).
bool one_launch(const TokenRows& a)
{
    const int64_t n_groups = groups_of(a);
    return n_groups <= kWholeGroups && (a.rows > 40 || n_groups <= 1024 * 4);
}

// Rows whose losses one workgroup sums, in 6.7 us; of more, each sums kSpanRows, in 4 us, and a further launch joins them in 2 to 5
// (16,384 rows by one workgroup 12.1).
constexpr int64_t kSumRows = 8192, kSpanRows = 2048;

// Workspace: Part [kMaxParts] of each of the first kPartRows rows, RowWork [rows], double [n_pairs] losses of the pairs.
int64_t parts_bytes(int64_t rows) { return (rows < kPartRows ? rows : kPartRows) * kMaxParts * (int64_t)sizeof(Part); }

}  // namespace

int64_t loss_workspace(int64_t rows, int64_t n_pairs) { return parts_bytes(rows) + (int64_t)sizeof(RowWork) * rows + 8 * n_pairs; }

bool token_logprobs_want_workspace(const TokenRows& a) { return in_parts(a); }

int launch_token_logprobs(const TokenRows& a, float* logprobs, float* stats, void* workspace, hipStream_t stream)
{
    if (a.rows == 0) return TDFA_OK;
    return stats_of<ScoreArgs>(a, Score{logprobs, reinterpret_cast<float2*>(stats), nullptr, nullptr}, static_cast<Part*>(workspace), stream);
}

int launch_token_grad(const TokenRows& a, const float* stats, const float* down, void* grad, int64_t grad_stride, hipStream_t stream)
{
    if (a.rows == 0) return TDFA_OK;
    return grad_of<GivenGradArgs>(a, stream, [&](GivenGradArgs& x, int64_t from, int32_t parts) {
        static_cast<RowArgs&>(x) = row_args(a, from);
        x.stats = reinterpret_cast<const float2*>(stats) + from;
        x.down = down + from;
        x.grad = grad_from(a, grad, grad_stride, from);
        x.grad_stride16 = grad_stride16(a, grad_stride);
        x.parts = parts;
    });
}

int launch_policy_loss(const TokenRows& a, const PolicyArgs& p, float* loss, float* logprobs, void* grad, int64_t grad_stride, void* workspace,
                       hipStream_t stream)
{
    if (a.rows && !(one_launch(a))) {
        RowWork* work = reinterpret_cast<RowWork*>(static_cast<char*>(workspace) + parts_bytes(a.rows));
        const int rc = stats_of<PolicyScoreArgs>(a, Score{logprobs, nullptr, work, &p}, static_cast<Part*>(workspace), stream);
        if (rc != TDFA_OK) return rc;
        constexpr int32_t step = sizeof(RowWork) / sizeof(double);
        if (grad) return grad_of_work(a, work, &work->value, a.rows, step, false, loss, grad, grad_stride, stream);
        return launch(loss_sum_kernel, dim3(1), 1024, stream, static_cast<const double*>(&work->value), (uint32_t)a.rows, step, 0, loss);
    }
    if (a.rows) {
        const int rc = a.dtype == TDFA_F32 ? (a.allow ? policy_launch<TDFA_F32, true>(a, p, logprobs, grad, grad_stride, stream)
                                                      : policy_launch<TDFA_F32, false>(a, p, logprobs, grad, grad_stride, stream))
                                           : (a.allow ? policy_launch<TDFA_BF16, true>(a, p, logprobs, grad, grad_stride, stream)
                                                      : policy_launch<TDFA_BF16, false>(a, p, logprobs, grad, grad_stride, stream));
        if (rc != TDFA_OK) return rc;
    }
    const bool alone = a.rows <= kSumRows;
    double* sums = static_cast<double*>(workspace);
    const unsigned blocks = alone ? 1u : (unsigned)((a.rows + kSpanRows - 1) / kSpanRows);
    const PolicySumArgs x = {logprobs, p.old_logprobs, p.ref_logprobs, p.advantages, a.weights, a.tokens, alone ? loss : nullptr, sums,
                             (uint32_t)a.rows, (uint32_t)(alone ? kSumRows : kSpanRows), p.clip_low, p.clip_high, p.kl_coef};
    const int rc = launch(policy_sum_kernel, dim3(blocks), 1024, stream, x);
    if (rc != TDFA_OK || alone) return rc;
    return launch(loss_sum_kernel, dim3(1), 1024, stream, static_cast<const double*>(sums), (uint32_t)blocks, 1, 0, loss);
}

int launch_preference_loss(const TokenRows& a, const PairArgs& p, float* loss, float* logprobs, void* grad, int64_t grad_stride, void* workspace,
                           hipStream_t stream)
{
    RowWork* work = reinterpret_cast<RowWork*>(static_cast<char*>(workspace) + parts_bytes(a.rows));
    double* each = reinterpret_cast<double*>(work + a.rows);
    if (a.rows) {
        const int rc = stats_of<PairScoreArgs>(a, Score{logprobs, nullptr, work, nullptr}, static_cast<Part*>(workspace), stream);
        if (rc != TDFA_OK) return rc;
    }
    const PairArgsOnCard pairs = {p.ref_logprobs, p.begin, p.rewards, p.n_pairs, (int32_t)a.rows, p.beta, p.smoothing};
    // Few rows and pairs without the launch between the other two, unless pairs are long, whose sums every workgroup of a gradient takes
    // again: 90 rows of 32,000 tokens in bf16 in 4 pairs 13.3 -> 11.7 us, 1,000 rows in 64 pairs 32.6 -> 30.4, in 4 pairs 32.9 -> 32.8, in
    // 2 pairs 33.8 -> 36.5 and in one 33.6 -> 39.2 (of 128,256 tokens 92.8 -> 91.1 in 4, 93.4 -> 92.3 in one, in fp32 163 -> 169; 300 rows of
    // few tokens in 128 pairs 10.7 -> 16.8), and 3 us less of the host.
    if (grad && a.rows && a.rows <= 1024 && a.rows <= 256 * (int64_t)p.n_pairs && p.n_pairs <= 64)
        return grad_of<FewPairsGradArgs>(a, stream, [&](FewPairsGradArgs& x, int64_t, int32_t) {
            const RowArgs r = row_args(a, 0);              // one launch: a row of 2^24 tokens has 4,096 parts at most, 2,048 where there are more than 128
            x = {r.allow, r.logits, r.states, r.tokens, work, grad, loss, pairs, r.stride16, grad_stride16(a, grad_stride), r.n_tokens, r.inv_t};
        });
    if (p.n_pairs) {
        const int32_t blocks = (int32_t)std::min<int64_t>(p.n_pairs, kMaxBlocks);
        const int rc = launch(pair_kernel, dim3((unsigned)blocks), kThreads, stream, pairs, work, each, blocks);
        if (rc != TDFA_OK) return rc;
    }
    if (grad && a.rows) return grad_of_work(a, work, each, p.n_pairs, 1, true, loss, grad, grad_stride, stream);
    return launch(loss_sum_kernel, dim3(1), 1024, stream, static_cast<const double*>(each), (uint32_t)p.n_pairs, 1, 1, loss);
}

}  // namespace tdfa
