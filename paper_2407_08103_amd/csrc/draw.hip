// Draws from given random numbers and lists of the most likely tokens, under a constraint or none, for gfx950.
//
// A row has logits l (NaN counts as -inf), an allowed set A, m the largest l in A, and weights w_t = exp((l_t - m) / T).
// Tokens are ordered by their logit, the largest first, and by their id among equal ones.  With top_k, top_p and min_p
//     K = those whose logit reaches the k-th largest
//     P = those of K for which the tokens of K with a larger logit weigh less than top_p of what K weighs, and the largest
//     N = those of P with w_t >= min_p
// and the draw with number u is the first token of N, in that order, up to which the weights add up to more than u times what N
// weighs.  All three cuts leave a beginning of the order that ends between two different logits, so each is a threshold on the
// logit, and the draw is a threshold on the running sum: one search each.
//
// Which token it is hangs on where u falls between two sums, so weights are taken and added up in 64 bits.
#include "rows_device.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace tdfa {
namespace {

typedef unsigned long long u64;

// Order keys: the larger the logit the larger the key; NaN is -inf, -0 is +0.
__device__ __forceinline__ uint32_t key_of(float z)
{
    uint32_t u = __float_as_uint(fmaxf(z, -INFINITY) + 0.0f);
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7FFFFFFFu : ~key); }
constexpr uint32_t kKeyNegInf = 0x007FFFFFu, kKeyPosInf = 0xFF800000u;

constexpr int kList = 2048;            // tokens that are put in order in LDS

struct SelectArgs {
    const uint32_t* allow;     // or NULL: every token is allowed
    const void* logits;
    const int32_t* states;
    uint32_t stride16;
    int32_t n_states, n_tokens;
    float temperature;
};
struct DrawArgs : SelectArgs {
    const float* uniforms;
    const float4* params;      // or NULL: those below, and the temperature
    const int32_t* targets;    // of a dense table one for each state and token, of a packed one those of its edges; NULL: no table
    const int64_t* row_begin;  // of a packed table
    const uint32_t* dir;
    int32_t* tokens;
    int32_t* new_states;
    float* logprobs;
    int32_t top_k;
    float top_p, min_p;
};
struct TopArgs : SelectArgs {
    int32_t* ids;
    float* logprobs;
    int32_t k;
};

// What a row is drawn with.  Every value that the arrays of a call can hold means something.
struct Setting {
    double inv_t;              // 0: the most likely token
    double top_p, min_p, u;
    uint32_t top_k;            // 0: no cut
};
__device__ __forceinline__ Setting setting_of(const DrawArgs& a, uint32_t i)
{
    float4 v = {a.temperature, (float)a.top_k, a.top_p, a.min_p};
    Setting s;
    s.top_k = (uint32_t)a.top_k;
    if (a.params) {
        v = a.params[i];
        s.top_k = v.y >= 1.0f && v.y < 2147483648.0f ? (uint32_t)v.y : 0u;
    }
    const float u = a.uniforms[i];
    s.inv_t = v.x > 0.0f ? 1.0 / (double)v.x : 0.0;
    if (v.x == INFINITY) s.inv_t = 1e-300;                 // (all weights are 1)
    s.top_p = v.z >= 0.0f ? fminf(v.z, 1.0f) : v.z < 0.0f ? 0.0 : 1.0;
    s.min_p = fminf(fmaxf(v.w, 0.0f), 1.0f);
    s.u = fminf(fmaxf(u, 0.0f), 1.0f);
    return s;
}

// The weight of a logit beside the largest, m, which is above -inf.
__device__ __forceinline__ double weight_of(float z, float m, double inv_t)
{
    return z == m ? 1.0 : z > -INFINITY ? exp(((double)z - (double)m) * inv_t) : 0.0;
}

// A row and its allowed bits.
template <int DTYPE>
struct RowOf {
    const typename Elem<DTYPE>::type* row;
    const uint32_t* bits;
    int32_t n_tokens;
};

// f(token, logit) for every allowed token of a row, in no order.
template <int DTYPE, int NT, bool BITS, typename F>
__device__ __forceinline__ void for_each(const RowOf<DTYPE>& r, F&& f)
{
    constexpr int G = Elem<DTYPE>::kGroup, U = 4;
    const int32_t n_groups = r.n_tokens / G;
    const RowBuffers buf = row_buffers<DTYPE>(r.row, r.bits, n_groups);
    for (int32_t g0 = 0; g0 < n_groups; g0 += NT * U) {
        uint4 x[U];
        uint32_t b[U];
        fetch<DTYPE, NT, U, BITS>(buf, g0, n_groups, x, b);
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int32_t g = g0 + (int32_t)threadIdx.x + k * NT;
            const uint32_t on = BITS ? b[k] : g < n_groups ? (1u << G) - 1u : 0u;
            if (!__ballot(on != 0)) continue;
            float z[G];
            unpack<DTYPE>(x[k], z);
#pragma unroll
            for (int j = 0; j < G; ++j)
                if (on >> j & 1) f(g * G + j, z[j]);
        }
    }
    const int32_t t = n_groups * G + (int32_t)threadIdx.x;
    if (t < r.n_tokens && (!BITS || allowed(r.bits, t))) f(t, to_f32(r.row[t]));
}

// What the workgroup of a row shares.
template <int NT>
struct Shared {
    u64 list[kList];           // keys above, complements of ids below
    double cum[kList];
    u64 bin[256];
    double part[NT / 64];
    uint32_t word[NT / 64];
    uint32_t n;
    u64 found[2];
};

template <int NT>
__device__ __forceinline__ uint32_t block_sum(uint32_t v, uint32_t (&part)[NT / 64])
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < NT / 64; ++w) v += part[w];
    return v;
}
template <int NT>
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t (&part)[NT / 64])
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v = max(v, (uint32_t)__shfl_xor(v, d));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < NT / 64; ++w) v = max(v, part[w]);
    return v;
}

// Tokens that a row's bits allow.
template <int NT>
__device__ __forceinline__ uint32_t count_allowed(const uint32_t* bits, int32_t n_tokens, uint32_t (&part)[NT / 64])
{
    uint32_t c = 0;
    const int32_t words = (n_tokens + 31) >> 5;
    for (int32_t i = threadIdx.x; i < words; i += NT) {
        uint32_t w = bits[i];
        if (n_tokens - 32 * i < 32) w &= (1u << (n_tokens - 32 * i)) - 1u;
        c += __popc(w);
    }
    return block_sum<NT>(c, part);
}

// ---- a few tokens: put in order ----------------------------------------------------------------

// Puts list[0 .. n) in order, the largest first; list[n .. the next power of two) is overwritten.
template <int NT>
__device__ __forceinline__ void sort_list(u64 (&list)[kList], uint32_t n)
{
    uint32_t size = 64;
    while (size < n) size <<= 1;
    for (uint32_t i = n + threadIdx.x; i < size; i += NT) list[i] = 0;
    __syncthreads();
    for (uint32_t k = 2; k <= size; k <<= 1)
        for (uint32_t j = k >> 1; j; j >>= 1) {
            for (uint32_t i = threadIdx.x; i < size / 2; i += NT) {
                const uint32_t lo = (i / j) * 2 * j + (i & (j - 1)), hi = lo + j;
                const u64 x = list[lo], y = list[hi];
                if ((x < y) == ((lo & k) == 0)) {
                    list[lo] = y;
                    list[hi] = x;
                }
            }
            __syncthreads();
        }
}

// cum[i] = weights of list[0 .. i] added up, n of them.
template <int NT>
__device__ __forceinline__ void sum_list(Shared<NT>& s, uint32_t n, float m, double inv_t)
{
    const uint32_t per = (n + NT - 1) / NT, from = threadIdx.x * per;
    double mine = 0.0;
    for (uint32_t i = from; i < min(from + per, n); ++i) {
        mine += weight_of(logit_of((uint32_t)(s.list[i] >> 32)), m, inv_t);
        s.cum[i] = mine;
    }
    double upto = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const double other = __shfl_up(upto, d);
        if ((int)(threadIdx.x & 63) >= d) upto += other;
    }
    if ((threadIdx.x & 63) == 63) s.part[threadIdx.x >> 6] = upto;
    __syncthreads();
    double before = 0.0;
    for (uint32_t w = 0; w < threadIdx.x >> 6; ++w) before += s.part[w];
    const double below = __shfl_up(upto, 1);
    if (threadIdx.x & 63) before += below;
    for (uint32_t i = from; i < min(from + per, n); ++i) s.cum[i] += before;
    __syncthreads();
}

// The first i in 0 .. n for which holds(i), which holds from there on; n if it holds for none.  By one wavefront, 64 places at a time.
template <typename F>
__device__ __forceinline__ uint32_t first_where(uint32_t n, F&& holds)
{
    const uint32_t lane = threadIdx.x & 63;
    uint32_t from = 0, step = 1;
    while (step * 64 < n) step *= 64;
    for (;; step /= 64) {
        const uint32_t i = from + lane * step + (step - 1);                // the last of each stretch
        const u64 b = __ballot(i >= n || holds(i));
        from += (uint32_t)(b ? __builtin_ctzll(b) : 64) * step;
        if (step == 1 || from >= n) return min(from, n);
    }
}

struct Drawn {
    int32_t token;
    float lp;
};

// The draw from n >= 1 tokens in order with their running sums.  By one wavefront.
template <int NT>
__device__ __forceinline__ Drawn draw_of_list(const Shared<NT>& s, uint32_t n, float m, const Setting& q)
{
    const auto key = [&](uint32_t i) { return (uint32_t)(s.list[i] >> 32); };
    const auto id = [&](uint32_t i) { return (int32_t)~(uint32_t)s.list[i]; };
    const auto end_of = [&](uint32_t i) {                  // behind the tokens of the same logit
        const uint32_t k = key(i);
        return first_where(n, [&](uint32_t j) { return key(j) < k; });
    };
    if (m == -INFINITY || q.inv_t == 0.0) return {id(0), m == -INFINITY ? -INFINITY : 0.0f};
    uint32_t kept = n;
    if (q.top_k && q.top_k < n) kept = end_of(q.top_k - 1);
    if (q.top_p < 1.0) {
        const double enough = q.top_p * s.cum[kept - 1];
        kept = min(kept, end_of(min(kept - 1, first_where(n, [&](uint32_t i) { return s.cum[i] >= enough; }))));
    }
    if (q.min_p > 0.0) kept = min(kept, first_where(n, [&](uint32_t i) { return weight_of(logit_of(key(i)), m, q.inv_t) < q.min_p; }));
    const double total = s.cum[kept - 1], target = q.u * total;
    uint32_t at = first_where(n, [&](uint32_t i) { return s.cum[i] > target; });
    if (at >= kept) at = first_where(n, [&](uint32_t i) { return s.cum[i] >= total; });       // u is 1: the last that weighs anything
    return {id(at), (float)log(weight_of(logit_of(key(at)), m, q.inv_t) / total)};
}

// ---- any number of tokens: thresholds digit by digit -------------------------------------------

// Largest key first, values are added up until they reach `want` > 0: the key at which they do, and the sum before it.
// each(f) calls f(key, value) for the tokens; they add up to `want` at least.  Eight bits of the key by a pass.
template <int NT, typename E>
__device__ __forceinline__ uint32_t key_at(Shared<NT>& s, u64 want, u64* before, E&& each)
{
    uint32_t prefix = 0, fixed = 0;
    u64 above = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        __syncthreads();
        for (int i = threadIdx.x; i < 256; i += NT) s.bin[i] = 0;
        __syncthreads();
        each([&](uint32_t key, u64 value) {
            if ((key & fixed) == prefix && value) atomicAdd(&s.bin[key >> shift & 255u], value);
        });
        __syncthreads();
        if (threadIdx.x < 64) {
            const int lane = threadIdx.x;
            u64 v[4], mine = 0;                            // bins 255 - 4 lane .. 252 - 4 lane
#pragma unroll
            for (int j = 0; j < 4; ++j) mine += v[j] = s.bin[255 - 4 * lane - j];
            u64 upto = mine;
#pragma unroll
            for (int d = 1; d < 64; d <<= 1) {
                const u64 other = __shfl_up(upto, d);
                if (lane >= d) upto += other;
            }
            u64 sum = above + upto - mine;
            const bool here = sum < want && (want <= sum + mine || lane == 63);
            if (here) {
                int j = 0;
                for (; j < 3 && sum + v[j] < want; ++j) sum += v[j];
                s.found[0] = (u64)(255 - 4 * lane - j);
                s.found[1] = sum;
            }
        }
        __syncthreads();
        prefix |= (uint32_t)s.found[0] << shift;
        fixed |= 255u << shift;
        above = s.found[1];
    }
    *before = above;
    return prefix;
}

// The smallest whole number that is not below x y, for 0 <= x <= 1 with at most 24 significant bits.
__device__ __forceinline__ u64 share_of(double x, u64 y, bool up)
{
    if (!(x > 0.0)) return 0;
    int e;
    const u64 f = (u64)ldexp(frexp(x, &e), 24);            // x = f 2^(e - 24)
    const int shift = 24 - e;
    const unsigned __int128 p = (unsigned __int128)f * y;
    if (shift >= 100) return up && y ? 1 : 0;
    return (u64)((p + (up ? ((unsigned __int128)1 << shift) - 1 : 0)) >> shift);
}

// Weights as whole numbers, so that their sums do not depend on the order in which they are added: 2^bits times the weight, where
// n_tokens of them stay below 2^62.
struct Whole {
    float m;
    double inv_t, scale;
    __device__ __forceinline__ u64 of(float z) const { return (u64)(weight_of(z, m, inv_t) * scale + 0.5); }
};
__device__ __forceinline__ Whole whole_of(float m, double inv_t, int32_t n_tokens)
{
    return {m, inv_t, ldexp(1.0, 62 - (32 - __clz(max(n_tokens, 1))))};
}

template <int NT>
__device__ __forceinline__ u64 block_sum(u64 v, Shared<NT>& s)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s.bin[threadIdx.x >> 6] = v;
    __syncthreads();
    v = 0;
    for (int w = 0; w < NT / 64; ++w) v += s.bin[w];
    return v;
}

// The draw from a row of any kind, of which some token is allowed.
template <int DTYPE, int NT, bool BITS>
__device__ Drawn draw_by_digits(Shared<NT>& s, const RowOf<DTYPE>& r, const Setting& q)
{
    uint32_t top = 0;
    for_each<DTYPE, NT, BITS>(r, [&](int32_t, float z) { top = max(top, key_of(z)); });
    top = block_max<NT>(top, s.word);
    const float m = logit_of(top);
    uint32_t key = top;
    u64 nth = 1, before;
    float lp = m == -INFINITY ? -INFINITY : 0.0f;
    if (m != -INFINITY && q.inv_t != 0.0) {
        const Whole w = whole_of(m, q.inv_t, r.n_tokens);
        uint32_t cut = 0;                                  // the smallest key that is kept
        const auto weights = [&](auto&& f) { for_each<DTYPE, NT, BITS>(r, [&](int32_t, float z) { if (key_of(z) >= cut) f(key_of(z), w.of(z)); }); };
        const auto kept_weight = [&]() {
            u64 sum = 0;
            weights([&](uint32_t, u64 x) { sum += x; });
            return block_sum<NT>(sum, s);
        };
        if (q.top_k) {
            u64 n = 0;
            for_each<DTYPE, NT, BITS>(r, [&](int32_t, float) { ++n; });
            n = block_sum<NT>(n, s);
            if (q.top_k < n) cut = key_at<NT>(s, q.top_k, &before, [&](auto&& f) { for_each<DTYPE, NT, BITS>(r, [&](int32_t, float z) { f(key_of(z), (u64)1); }); });
        }
        if (q.top_p < 1.0) {
            const u64 enough = share_of(q.top_p, kept_weight(), true);
            cut = max(cut, enough ? key_at<NT>(s, enough, &before, weights) : top);
        }
        if (q.min_p > 0.0) {
            uint32_t least = top;
            for_each<DTYPE, NT, BITS>(r, [&](int32_t, float z) { if (weight_of(z, m, q.inv_t) >= q.min_p) least = min(least, key_of(z)); });
            cut = max(cut, ~block_max<NT>(~least, s.word));
        }
        const u64 total = kept_weight(), target = min(share_of(q.u, total, false), total - 1);
        key = key_at<NT>(s, target + 1, &before, weights);
        nth = (target - before) / w.of(logit_of(key)) + 1;
        lp = (float)log(weight_of(logit_of(key), m, q.inv_t) / ((double)total / w.scale));
    }
    // the nth token of that logit
    const uint32_t id = ~key_at<NT>(s, nth, &before, [&](auto&& f) { for_each<DTYPE, NT, BITS>(r, [&](int32_t t, float z) { f(~(uint32_t)t, (u64)(key_of(z) == key)); }); });
    return {(int32_t)id, lp};
}

// The allowed tokens of a row, in order, with their running sums; a row of at most kList of them.
template <int DTYPE, int NT, bool BITS>
__device__ __forceinline__ uint32_t list_row(Shared<NT>& s, const RowOf<DTYPE>& r, double inv_t, float* m)
{
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    for_each<DTYPE, NT, BITS>(r, [&](int32_t t, float z) { s.list[atomicAdd(&s.n, 1u)] = (u64)key_of(z) << 32 | ~(uint32_t)t; });
    __syncthreads();
    const uint32_t n = s.n;
    sort_list<NT>(s.list, n);
    *m = logit_of((uint32_t)(s.list[0] >> 32));
    if (*m != -INFINITY) sum_list<NT>(s, n, *m, inv_t);
    return n;
}

__device__ __forceinline__ int32_t target_of(const DrawArgs& a, int32_t q, int32_t token)
{
    if (!a.row_begin) return a.targets[(int64_t)q * a.n_tokens + token];
    const uint32_t* words = bits_of(a.allow, q, a.n_tokens) + (token >> 7 << 2);
    const int32_t at = token >> 5 & 3;
    uint32_t below = a.dir[(int64_t)q * (((int64_t)a.n_tokens + 127) / 128) + (token >> 7)];
    for (int32_t w = 0; w < at; ++w) below += __popc(words[w]);
    below += __popc(words[at] & ((1u << (token & 31)) - 1u));
    return a.targets[a.row_begin[q] + below];
}

// The state of row i, whether it is one of the table's (without a table: it always is), and its allowed bits.
struct StateOf {
    int32_t q;
    bool valid;
    const uint32_t* bits;
};
__device__ __forceinline__ StateOf state_of(const SelectArgs& a, uint32_t i)
{
    if (!a.allow) return {0, true, nullptr};
    const int32_t q = __builtin_amdgcn_readfirstlane(a.states[i]);
    const bool valid = q >= 0 && q < a.n_states;
    return {q, valid, valid ? bits_of(a.allow, q, a.n_tokens) : a.allow};
}

// One workgroup per sequence.
template <int DTYPE, int NT, bool BITS>
__global__ void __launch_bounds__(NT) draw_step_kernel(DrawArgs a)
{
    __shared__ Shared<NT> s;
    const uint32_t i = blockIdx.x;
    const StateOf st = state_of(a, i);
    const Setting q = setting_of(a, i);
    const RowOf<DTYPE> r = {row_at<DTYPE>(a.logits, i, a.stride16), st.bits, a.n_tokens};
    const uint32_t n = !st.valid ? 0u : BITS ? count_allowed<NT>(st.bits, a.n_tokens, s.word) : (uint32_t)a.n_tokens;
    Drawn d = {TDFA_NO_TOKEN, 0.0f};
    if (n > (uint32_t)kList) {
        d = draw_by_digits<DTYPE, NT, BITS>(s, r, q);
    } else if (n) {
        float m;
        list_row<DTYPE, NT, BITS>(s, r, q.inv_t, &m);
        if (threadIdx.x < 64) d = draw_of_list<NT>(s, n, m, q);
    }
    if (threadIdx.x == 0) {
        a.tokens[i] = d.token;
        if (a.targets) a.new_states[i] = !st.valid ? TDFA_DEAD : d.token == TDFA_NO_TOKEN ? st.q : target_of(a, st.q, d.token);
        if (a.logprobs) a.logprobs[i] = d.lp;
    }
}

// One workgroup per row: the k first tokens in order, and their log-probabilities.
template <int DTYPE, int NT, bool BITS>
__global__ void __launch_bounds__(NT) top_logprobs_kernel(TopArgs a)
{
    __shared__ Shared<NT> s;
    const uint32_t i = blockIdx.x, k = (uint32_t)a.k;
    const StateOf st = state_of(a, i);
    const RowOf<DTYPE> r = {row_at<DTYPE>(a.logits, i, a.stride16), st.bits, a.n_tokens};
    const double inv_t = 1.0 / (double)a.temperature;
    uint32_t n = !st.valid ? 0u : BITS ? count_allowed<NT>(st.bits, a.n_tokens, s.word) : (uint32_t)a.n_tokens;
    float m = -INFINITY;
    double total = 0.0;
    if (n > (uint32_t)kList) {
        uint32_t top = 0;
        for_each<DTYPE, NT, BITS>(r, [&](int32_t, float z) { top = max(top, key_of(z)); });
        m = logit_of(block_max<NT>(top, s.word));
        if (m != -INFINITY) {
            // the k-th largest key, and how many larger ones there are; of the tokens that have it those of the lowest ids
            u64 larger, unused;
            const uint32_t key = key_at<NT>(s, k, &larger, [&](auto&& f) { for_each<DTYPE, NT, BITS>(r, [&](int32_t, float z) { f(key_of(z), (u64)1); }); });
            const uint32_t last = ~key_at<NT>(s, k - larger, &unused, [&](auto&& f) {
                for_each<DTYPE, NT, BITS>(r, [&](int32_t t, float z) { f(~(uint32_t)t, (u64)(key_of(z) == key)); });
            });
            const Whole w = whole_of(m, inv_t, a.n_tokens);
            u64 sum = 0;
            if (threadIdx.x == 0) s.n = 0;
            __syncthreads();
            for_each<DTYPE, NT, BITS>(r, [&](int32_t t, float z) {
                sum += w.of(z);
                if (key_of(z) > key || (key_of(z) == key && (uint32_t)t <= last)) s.list[atomicAdd(&s.n, 1u)] = (u64)key_of(z) << 32 | ~(uint32_t)t;
            });
            total = (double)block_sum<NT>(sum, s) / w.scale;
            n = s.n;
            sort_list<NT>(s.list, n);
        }
    } else if (n) {
        list_row<DTYPE, NT, BITS>(s, r, inv_t, &m);
        total = s.cum[n - 1];
    }
    const double ln_total = m == -INFINITY ? 0.0 : m == INFINITY ? NAN : log(total);
    for (uint32_t j = threadIdx.x; j < k; j += NT) {
        int32_t id = TDFA_NO_TOKEN;
        float lp = -INFINITY;
        if (m != -INFINITY && j < n && (uint32_t)(s.list[j] >> 32) > kKeyNegInf) {
            id = (int32_t)~(uint32_t)s.list[j];
            lp = (float)(((double)logit_of((uint32_t)(s.list[j] >> 32)) - (double)m) * inv_t - ln_total);
        }
        a.ids[(uint64_t)i * k + j] = id;
        a.logprobs[(uint64_t)i * k + j] = lp;
    }
}

// fn(first row, number of rows) for the launches that the rows take.
template <typename F>
int by_launches(int64_t rows, F&& fn)
{
    for (int64_t from = 0; from < rows; from += kMaxBlocks) {
        const int rc = fn(from, (unsigned)std::min<int64_t>(kMaxBlocks, rows - from));
        if (rc != TDFA_OK) return rc;
    }
    return TDFA_OK;
}
void fill(SelectArgs& x, const LogitRows& a, int64_t from)
{
    const int64_t esz = a.dtype == TDFA_F32 ? 4 : 2;
    x.allow = a.allow;
    x.logits = static_cast<const char*>(a.logits) + from * a.row_stride * esz;
    x.states = a.states ? a.states + from : nullptr;
    x.stride16 = (uint32_t)(a.rows > 1 ? a.row_stride * esz / 16 : 0);
    x.n_states = (int32_t)std::min<int64_t>(a.n_states, INT32_MAX);
    x.n_tokens = a.n_tokens;
    x.temperature = a.temperature;
}

template <int DTYPE, int NT, bool BITS>
int draw_rows(const DrawArgs& x, unsigned rows, hipStream_t stream) { return launch(draw_step_kernel<DTYPE, NT, BITS>, dim3(rows), NT, stream, x); }
template <int DTYPE, int NT, bool BITS>
int top_rows(const TopArgs& x, unsigned rows, hipStream_t stream) { return launch(top_logprobs_kernel<DTYPE, NT, BITS>, dim3(rows), NT, stream, x); }

}  // namespace

int64_t select_workspace(int64_t, int64_t) { return 0; }

int launch_draw_step(const LogitRows& a, const DrawRows& d, void*, hipStream_t stream)
{
    return by_launches(a.rows, [&](int64_t from, unsigned rows) {
        DrawArgs x;
        fill(x, a, from);
        x.uniforms = d.uniforms + from;
        x.params = d.params ? reinterpret_cast<const float4*>(d.params) + from : nullptr;
        x.targets = d.delta ? d.delta : d.targets;
        x.row_begin = d.delta ? nullptr : d.row_begin;
        x.dir = d.dir;
        x.tokens = d.tokens + from;
        x.new_states = d.new_states ? d.new_states + from : nullptr;
        x.logprobs = d.logprobs ? d.logprobs + from : nullptr;
        x.top_k = d.top_k;
        x.top_p = d.top_p;
        x.min_p = d.min_p;
        if (a.dtype == TDFA_F32) return a.allow ? draw_rows<TDFA_F32, 1024, true>(x, rows, stream) : draw_rows<TDFA_F32, 1024, false>(x, rows, stream);
        return a.allow ? draw_rows<TDFA_BF16, 1024, true>(x, rows, stream) : draw_rows<TDFA_BF16, 1024, false>(x, rows, stream);
    });
}

int launch_top_logprobs(const LogitRows& a, int32_t k, int32_t* ids, float* logprobs, void*, hipStream_t stream)
{
    return by_launches(a.rows, [&](int64_t from, unsigned rows) {
        TopArgs x;
        fill(x, a, from);
        x.ids = ids + from * k;
        x.logprobs = logprobs + from * k;
        x.k = k;
        if (a.dtype == TDFA_F32) return a.allow ? top_rows<TDFA_F32, 1024, true>(x, rows, stream) : top_rows<TDFA_F32, 1024, false>(x, rows, stream);
        return a.allow ? top_rows<TDFA_BF16, 1024, true>(x, rows, stream) : top_rows<TDFA_BF16, 1024, false>(x, rows, stream);
    });
}

}  // namespace tdfa
