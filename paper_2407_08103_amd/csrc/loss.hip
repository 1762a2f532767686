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
constexpr float kLowest = -3.402823466e38f;

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

// What is known about a row before its logits are read.
struct Row {
    const uint32_t* bits;      // its state's allowed bits, or NULL: every token is allowed
    int32_t token;
    bool live;                 // takes part
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

// (m, s) stands for the largest value m and the sum s of exp((z - m) c) of some logits; {kLowest, 0}: of none.  (A logit
// of -inf adds nothing to s whatever m is, and one of the type's lowest value is counted like any other.)
struct Sum {
    float m, s;
};
__device__ __forceinline__ Sum join(Sum a, Sum b, float c2)
{
    const float m = fmaxf(a.m, b.m);
    return {m, a.s * __builtin_amdgcn_exp2f((a.m - m) * c2) + b.s * __builtin_amdgcn_exp2f((b.m - m) * c2)};
}
__device__ __forceinline__ Sum wave_join(Sum a, float c2)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) a = join(a, Sum{__shfl_xor(a.m, d), __shfl_xor(a.s, d)}, c2);
    return a;
}

// One workgroup per row: its log-probability and its statistics {m, ln s}; {0, +inf} for a row that takes no part.
template <int DTYPE>
__global__ void __launch_bounds__(kThreads) token_stats_kernel(TokenRows a, float* logprobs, float2* stats)
{
    using E = typename Elem<DTYPE>::type;
    __shared__ Sum s_part[kThreads / 64];
    const float c2 = a.inv_t * kLog2e;
    for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
        const Row r = row_of<DTYPE>(a, i);
        if (!r.live) {
            if (threadIdx.x == 0) {
                if (logprobs) logprobs[i] = r.lp;
                if (stats) stats[i] = make_float2(0.0f, INFINITY);
            }
            continue;
        }
        const E* row = static_cast<const E*>(a.logits) + i * a.row_stride;
        Sum mine = {kLowest, 0.0f};
        for (int32_t t = threadIdx.x; t < a.n_tokens; t += kThreads) {
            if (!allowed(r.bits, t)) continue;
            const float z = to_f32(row[t]);
            if (z == z) {
                const float m = fmaxf(mine.m, z);
                mine = {m, mine.s * __builtin_amdgcn_exp2f((mine.m - m) * c2) + __builtin_amdgcn_exp2f((z - m) * c2)};
            }
        }
        mine = wave_join(mine, c2);
        __syncthreads();
        if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = mine;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < kThreads / 64; ++w) mine = join(mine, s_part[w], c2);
            const float ls = logf(mine.s), lp = (r.z - mine.m) * a.inv_t - ls;
            if (logprobs) logprobs[i] = lp;
            if (stats) stats[i] = lp == -INFINITY ? make_float2(0.0f, INFINITY) : make_float2(mine.m, ls);
        }
    }
}

// grad[i][j] = down[i] c ([j = t] - p_j) over A, 0 elsewhere; 0 throughout in a row that takes no part.
template <int DTYPE>
__global__ void __launch_bounds__(kThreads) token_grad_kernel(TokenRows a, const float2* stats, const float* down, void* grad, int64_t grad_stride)
{
    using E = typename Elem<DTYPE>::type;
    const float c2 = a.inv_t * kLog2e;
    for (int64_t i = blockIdx.x; i < a.rows; i += gridDim.x) {
        const Row r = row_of<DTYPE>(a, i);
        const E* row = static_cast<const E*>(a.logits) + i * a.row_stride;
        E* out = static_cast<E*>(grad) + i * grad_stride;
        const float2 st = stats[i];
        const bool live = r.live && st.y != INFINITY;
        const float d = live ? down[i] * a.inv_t : 0.0f;
        for (int32_t t = threadIdx.x; t < a.n_tokens; t += kThreads) {
            float g = 0.0f;
            if (d != 0.0f && allowed(r.bits, t)) {
                const float z = to_f32(row[t]);
                const float p = z == z ? __builtin_amdgcn_exp2f(((z - st.x) * a.inv_t - st.y) * kLog2e) : 0.0f;
                g = d * ((t == r.token ? 1.0f : 0.0f) - p);
            }
            store_rounded(out + t, g);
        }
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

__global__ void __launch_bounds__(kThreads)
policy_rows_kernel(PolicyArgs p, int64_t rows, const float* weights, const float* logprobs, const float2* stats, float* down, float* each)
{
    for (int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x; i < rows; i += (int64_t)gridDim.x * kThreads) {
        float e = 0.0f, d = 0.0f;
        if (stats[i].y != INFINITY) {
            policy_term(p, i, logprobs[i], &e, &d);
            const float w = weights ? weights[i] : 1.0f;
            e *= w;
            d *= w;
        }
        each[i] = e;
        down[i] = d;
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
pair_kernel(PairArgs p, int64_t rows, const float* logprobs, const float2* stats, float* down, double* each)
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
                if (stats[i].y != INFINITY) sum += (double)logprobs[i] - (double)p.ref_logprobs[i];
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

__global__ void __launch_bounds__(kThreads) zero_kernel(float* x, int64_t n)
{
    for (int64_t i = blockIdx.x * (int64_t)kThreads + threadIdx.x; i < n; i += (int64_t)gridDim.x * kThreads) x[i] = 0.0f;
}

unsigned blocks_for(int64_t n) { return (unsigned)(n < 1 << 16 ? n : 1 << 16); }

template <int DTYPE>
int stats_launch(const TokenRows& a, float* logprobs, float2* stats, hipStream_t stream)
{
    token_stats_kernel<DTYPE><<<blocks_for(a.rows), kThreads, 0, stream>>>(a, logprobs, stats);
    TDFA_HIP(hipGetLastError());
    return TDFA_OK;
}

int stats_of(const TokenRows& a, float* logprobs, float2* stats, hipStream_t stream)
{
    return a.dtype == TDFA_F32 ? stats_launch<TDFA_F32>(a, logprobs, stats, stream) : stats_launch<TDFA_BF16>(a, logprobs, stats, stream);
}

}  // namespace

int launch_token_logprobs(const TokenRows& a, float* logprobs, float* stats, void* workspace, hipStream_t stream)
{
    (void)workspace;
    if (a.rows == 0) return TDFA_OK;
    return stats_of(a, logprobs, reinterpret_cast<float2*>(stats), stream);
}

int launch_token_grad(const TokenRows& a, const float* stats, const float* down, void* grad, int64_t grad_stride, hipStream_t stream)
{
    if (a.rows == 0) return TDFA_OK;
    const float2* st = reinterpret_cast<const float2*>(stats);
    if (a.dtype == TDFA_F32) token_grad_kernel<TDFA_F32><<<blocks_for(a.rows), kThreads, 0, stream>>>(a, st, down, grad, grad_stride);
    else token_grad_kernel<TDFA_BF16><<<blocks_for(a.rows), kThreads, 0, stream>>>(a, st, down, grad, grad_stride);
    TDFA_HIP(hipGetLastError());
    return TDFA_OK;
}

// Workspace of the losses: double [n_pairs], float2 [rows] statistics, float [rows] d loss / d lp, float [rows] losses.
int64_t loss_workspace(int64_t rows, int64_t n_pairs) { return 8 * n_pairs + 16 * rows; }

int launch_policy_loss(const TokenRows& a, const PolicyArgs& p, float* loss, float* logprobs, void* grad, int64_t grad_stride, void* workspace,
                       hipStream_t stream)
{
    float2* stats = static_cast<float2*>(workspace);
    float* down = reinterpret_cast<float*>(stats + a.rows);
    float* each = down + a.rows;
    int rc = TDFA_OK;
    if (a.rows) {
        rc = stats_of(a, logprobs, stats, stream);
        if (rc != TDFA_OK) return rc;
        policy_rows_kernel<<<blocks_for((a.rows + kThreads - 1) / kThreads), kThreads, 0, stream>>>(p, a.rows, a.weights, logprobs, stats, down, each);
        TDFA_HIP(hipGetLastError());
    }
    loss_sum_kernel<float><<<1, 1024, 0, stream>>>(each, a.rows, 1.0, loss);
    TDFA_HIP(hipGetLastError());
    if (grad && a.rows) rc = launch_token_grad(a, reinterpret_cast<const float*>(stats), down, grad, grad_stride, stream);
    return rc;
}

int launch_preference_loss(const TokenRows& a, const PairArgs& p, float* loss, float* logprobs, void* grad, int64_t grad_stride, void* workspace,
                           hipStream_t stream)
{
    double* each = static_cast<double*>(workspace);
    float2* stats = reinterpret_cast<float2*>(each + p.n_pairs);
    float* down = reinterpret_cast<float*>(stats + a.rows);
    int rc = TDFA_OK;
    if (a.rows) {
        rc = stats_of(a, logprobs, stats, stream);
        if (rc != TDFA_OK) return rc;
        zero_kernel<<<blocks_for((a.rows + kThreads - 1) / kThreads), kThreads, 0, stream>>>(down, a.rows);     // rows of no sequence
        TDFA_HIP(hipGetLastError());
    }
    if (p.n_pairs) {
        pair_kernel<<<blocks_for(p.n_pairs), kThreads, 0, stream>>>(p, a.rows, logprobs, stats, down, each);
        TDFA_HIP(hipGetLastError());
    }
    loss_sum_kernel<double><<<1, 1024, 0, stream>>>(each, p.n_pairs, p.n_pairs ? 1.0 / (double)p.n_pairs : 0.0, loss);
    TDFA_HIP(hipGetLastError());
    if (grad && a.rows) rc = launch_token_grad(a, reinterpret_cast<const float*>(stats), down, grad, grad_stride, stream);
    return rc;
}

}  // namespace tdfa
