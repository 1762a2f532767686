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
// Which token it is hangs on where u falls between two sums, so weights are taken and added up in 64 bits.  (A list's order needs no sums: those of 32-bit
// logits take weights of 32 bits, and add them up in 64.)
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

// Tokens that are put in order in LDS.  16 bits: what is put in order are few tokens of a row; 32: the tokens of a step (below), which may be
// some hundreds.
template <int DTYPE> constexpr uint32_t kList = DTYPE == TDFA_F32 ? 1024 : 256;
constexpr uint32_t kFew = 256;         // tokens that are put in order without any other look at them

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

// What a row is drawn with, the same in all lanes.  Every value that the arrays of a call can hold means something.
struct Setting {
    float t, p, least, number;
    uint32_t top_k;            // 0: no cut
    __device__ __forceinline__ double inv_t() const { return t > 0.0f ? t == INFINITY ? 1e-300 : 1.0 / (double)t : 0.0; }       // 0: the first token; (next to 0: all weigh 1)
    __device__ __forceinline__ double top_p() const { return p >= 0.0f ? fminf(p, 1.0f) : p < 0.0f ? 0.0 : 1.0; }
    __device__ __forceinline__ double min_p() const { return fminf(fmaxf(least, 0.0f), 1.0f); }
    __device__ __forceinline__ double u() const { return fminf(fmaxf(number, 0.0f), 1.0f); }
};
__device__ __forceinline__ Setting setting_of(const DrawArgs& a, uint32_t i)
{
    Setting s = {a.temperature, a.top_p, a.min_p, 0.0f, (uint32_t)a.top_k};
    if (a.params) {
        const float4 v = a.params[i];
        const float k = shared_by_wave(v.y);
        s.t = shared_by_wave(v.x);
        s.p = shared_by_wave(v.z);
        s.least = shared_by_wave(v.w);
        s.top_k = k >= 1.0f && k < 2147483648.0f ? (uint32_t)k : 0u;
    }
    s.number = shared_by_wave(a.uniforms[i]);
    return s;
}

// A barrier for what lies in LDS, the only memory that threads hand one another anything in here: reads of a row stay on their way.
__device__ __forceinline__ void lds_barrier()
{
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// The same sums as borders of the lanes' intervals.  The sum of every lane is rounded in an order of its own, so that it may fall from one lane
// to the next, or rise where a lane adds nothing: a border is the largest sum up to it of a lane that adds something.
__device__ __forceinline__ double wave_borders(double v)
{
    const double sum = wave_upto(v);
    double top = v > 0.0 ? sum : 0.0;
    top = fmax(top, lanes_below<0x111, 0xF>(top));
    top = fmax(top, lanes_below<0x112, 0xF>(top));
    top = fmax(top, lanes_below<0x114, 0xF>(top));
    top = fmax(top, lanes_below<0x118, 0xF>(top));
    top = fmax(top, lanes_below<0x142, 0xA>(top));
    return fmax(top, lanes_below<0x143, 0xC>(top));
}
template <typename V>
__device__ __forceinline__ V wave_before(V upto) { return lanes_below<0x138, 0xF>(upto); }       // wave_shr 1

// A product that is rounded by itself.  A cut and the draw add up the same weights and have to find the same sums: as part of a fused product and sum, in one
// of them and not in the other, the draw with 1 went past the cut.
__device__ __forceinline__ double product(double x, double y)
{
#pragma clang fp contract(off)
    return x * y;
}

// The weight of a logit beside the largest, m, which is above -inf.
__device__ __forceinline__ double weight_of(float z, float m, double inv_t)
{
    return z == m ? 1.0 : z > -INFINITY ? exp(product((double)z - (double)m, inv_t)) : 0.0;
}

// A row and its allowed bits.
template <int DTYPE>
struct RowOf {
    const typename Elem<DTYPE>::type* row;
    const uint32_t* bits;
    int32_t n_tokens;
};

// f(token, logit) for every allowed token of a row, in no order.  (For rows that nothing faster takes: little code.)
template <int DTYPE, int NT, bool BITS, typename F>
__device__ __forceinline__ void for_each(const RowOf<DTYPE>& r, F&& f)
{
    constexpr int G = Elem<DTYPE>::kGroup;
    const int32_t n_groups = r.n_tokens / G;
    const RowBuffers buf = row_buffers<DTYPE>(r.row, r.bits, n_groups);
    for (int32_t g0 = 0; g0 < n_groups; g0 += NT) {
        uint4 x[1];
        uint32_t b[1];
        fetch<DTYPE, NT, 1, BITS>(buf, g0, n_groups, x, b);
        const int32_t g = g0 + (int32_t)threadIdx.x;
        for (uint32_t left = BITS ? b[0] : g < n_groups ? (1u << G) - 1u : 0u; left; left &= left - 1) {
            const int32_t j = __builtin_ctz(left);
            f(g * G + j, element_of<DTYPE>(x[0], j));
        }
    }
    const int32_t t = n_groups * G + (int32_t)threadIdx.x;
    if (t < r.n_tokens && (!BITS || allowed(r.bits, t))) f(t, to_f32(r.row[t]));
}

// The same row as the threads of a workgroup hold it: R > 0 groups each, in registers, or R = 0: read again by every look at it.
template <int DTYPE, int NT, int R, bool BITS>
struct Held {
    static constexpr int G = Elem<DTYPE>::kGroup, U = R ? R : 8, kAhead = U < 6 ? U : 6;
    static constexpr uint32_t kAll = (1u << G) - 1u;
    RowBuffers buf;
    int32_t n_groups;
    uint4 x[U];
    uint32_t b[(U + 3) / 4];   // allowed bits, of four groups each
    float last;                // the element behind the whole groups that belongs to this thread
    bool has_last;             // and whether it is allowed

    __device__ __forceinline__ void load(const RowOf<DTYPE>& r)
    {
        n_groups = r.n_tokens / G;
        buf = row_buffers<DTYPE>(r.row, r.bits, n_groups);
        // (before the groups: what is loaded after them arrives after them)
        const int32_t t = n_groups * G + (int32_t)threadIdx.x;
        has_last = t < r.n_tokens && (!BITS || allowed(r.bits, t));
        last = has_last ? to_f32(r.row[t]) : -INFINITY;
        if constexpr (R > 0) {
            load_bits(0);
            next_group();
#pragma unroll
            for (int k = 0; k < kAhead; ++k) load_group(k);
        }
    }
    __device__ __forceinline__ void load_bits(int32_t g0)
    {
        if constexpr (BITS) {
            uint32_t y[U];
            fetch_bits<DTYPE, NT, U, BITS>(buf, g0, y);
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int32_t g = g0 + (int32_t)threadIdx.x + k * NT;
                if (DTYPE == TDFA_F32) y[k] = g < n_groups ? y[k] >> ((g & 1) * 4) & 15u : 0u;
                b[k / 4] = k % 4 ? b[k / 4] | y[k] << (k % 4 * 8) : y[k];
            }
        }
    }
    // Groups are requested in the order in which they are looked at, kAhead of them before the first look, which requests the others: a
    // wavefront whose requests do not fit the queue waits with all that it has to do.
    __device__ __forceinline__ void load_group(int k, int32_t g0 = 0)
    {
        x[k] = group_at<false>(buf.x, BITS && bits_at(k) == 0 ? kNowhere : (uint32_t)(g0 + (int32_t)threadIdx.x + k * NT) * 16u);
        next_group();
    }
    __device__ __forceinline__ void load_rest()
    {
        if constexpr (R > 0)
#pragma unroll
            for (int k = kAhead; k < U; ++k) load_group(k);
    }
    __device__ __forceinline__ uint32_t bits_at(int k) const { return b[k / 4] >> (k % 4 * 8) & 0xFFu; }
    __device__ __forceinline__ uint32_t on_of(int k, int32_t g) const { return BITS ? bits_at(k) : g < n_groups ? kAll : 0u; }
    // f(group, its elements, which of them are allowed) for the groups of this thread; those of a wavefront lie side by side, and one
    // without an allowed token is passed over.
    template <bool ALL = false, bool FIRST = false, typename F>                 // ALL: none is passed over
    __device__ __forceinline__ void each(F&& f)
    {
        for (int32_t g0 = 0; g0 < (R ? 1 : n_groups); g0 += NT * U) {
            if constexpr (R == 0) {
                load_bits(g0);
#pragma unroll
                for (int k = 0; k < U; ++k) load_group(k, g0);
            }
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int32_t g = g0 + (int32_t)threadIdx.x + k * NT;
                const uint32_t on = on_of(k, g);
                if (FIRST && R > 0 && k + kAhead < U) load_group(k + kAhead);
                if (!ALL && !__ballot(on != 0)) continue;
                f(g, x[k], on);
                next_group();
            }
        }
    }
};

// What the workgroup of a row shares.
constexpr uint32_t kBins = 11273;       // see bin_of
constexpr uint32_t kSteps = 4096;      // see step_of
template <int DTYPE, int NT>
struct Shared {
    union {
        u64 bin[256];          // of one digit
        alignas(16) uint32_t count[DTYPE == TDFA_F32 ? 4 : kBins];
        uint32_t chunk[kBins];
        struct {
            u64 weight[DTYPE == TDFA_F32 ? kSteps : 1];
            uint32_t tokens[DTYPE == TDFA_F32 ? kSteps : 1];
        } step;
    };
    union {
        u64 list[kList<DTYPE>];    // keys above, complements of ids below
        double cum[kList<DTYPE>];  // of the sorted ones
    };
    u64 sorted[kList<DTYPE>];
    uint32_t rank[kList<DTYPE>];
    double part[NT / 64];
    uint32_t word[NT / 64], word2[NT / 64];
    uint32_t n;
    u64 found[2];
    double mass[3], end[3];
    u64 least;
    uint32_t at[4];
};

template <int NT>
__device__ __forceinline__ uint32_t block_sum(uint32_t v, uint32_t (&part)[NT / 64])
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    lds_barrier();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    lds_barrier();
    v = 0;
    for (int w = 0; w < NT / 64; ++w) v += part[w];
    return v;
}
template <int NT>
__device__ __forceinline__ uint32_t block_max(uint32_t v, uint32_t (&part)[NT / 64])
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v = max(v, (uint32_t)__shfl_xor(v, d));
    lds_barrier();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    lds_barrier();
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

// list[0 .. n) in order, the largest first, in sorted[]: every entry counts those above it.  n <= kList; three barriers.
template <int DTYPE, int NT>
__device__ __forceinline__ void sort_list(Shared<DTYPE, NT>& s, uint32_t n)
{
    for (uint32_t i = threadIdx.x; i < n; i += NT) s.rank[i] = 0;
    lds_barrier();
    uint32_t size = 64;
    while (size < n && size < NT) size <<= 1;              // threads side by side, and NT / size of them for one entry
    const uint32_t first = threadIdx.x / size, step = NT / size;
    for (uint32_t i = threadIdx.x & (size - 1); i < n; i += size) {
        const u64 mine = s.list[i];
        uint32_t above = 0;
        for (uint32_t j = first; j < n; j += step) above += s.list[j] > mine ? 1u : 0u;
        if (above) atomicAdd(&s.rank[i], above);
    }
    lds_barrier();
    for (uint32_t i = threadIdx.x; i < n; i += NT) s.sorted[s.rank[i]] = s.list[i];
    lds_barrier();
}

// cum[i] = weights of sorted[0 .. i] added up, n of them; it never falls, and does not rise at a token that weighs nothing.  By one wavefront.
template <int DTYPE, int NT>
__device__ __forceinline__ void sum_list(Shared<DTYPE, NT>& s, uint32_t n, float m, double inv_t)
{
    const uint32_t per = (n + 63) / 64, from = (threadIdx.x & 63) * per, to = min(from + per, n);
    double mine = 0.0;
    for (uint32_t i = from; i < to; ++i) {
        mine += weight_of(logit_of((uint32_t)(s.sorted[i] >> 32)), m, inv_t);
        s.cum[i] = mine;
    }
    const double end = wave_borders(mine), before = wave_before(end);
    for (uint32_t i = from; i < to; ++i) s.cum[i] = s.cum[i] == mine ? end : fmin(before + s.cum[i], end);
    wave_lds_sync();
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
template <int NT, int DTYPE>
__device__ __forceinline__ Drawn draw_of_list(const Shared<DTYPE, NT>& s, uint32_t n, float m, const Setting& q)
{
    const auto key = [&](uint32_t i) { return (uint32_t)(s.sorted[i] >> 32); };
    const auto id = [&](uint32_t i) { return (int32_t)~(uint32_t)s.sorted[i]; };
    const auto end_of = [&](uint32_t i) {                  // behind the tokens of the same logit
        const uint32_t k = key(i);
        return first_where(n, [&](uint32_t j) { return key(j) < k; });
    };
    if (m == -INFINITY || q.inv_t() == 0.0) return {id(0), m == -INFINITY ? -INFINITY : 0.0f};
    uint32_t kept = n;
    if (q.top_k && q.top_k < n) kept = end_of(q.top_k - 1);
    if (q.top_p() < 1.0) {
        const double enough = q.top_p() * s.cum[kept - 1];
        kept = min(kept, end_of(min(kept - 1, first_where(n, [&](uint32_t i) { return s.cum[i] >= enough; }))));
    }
    if (q.min_p() > 0.0) kept = min(kept, first_where(n, [&](uint32_t i) { return weight_of(logit_of(key(i)), m, q.inv_t()) < q.min_p(); }));
    const double total = s.cum[kept - 1], target = q.u() * total;
    uint32_t at = first_where(n, [&](uint32_t i) { return s.cum[i] > target; });
    if (at >= kept) at = first_where(n, [&](uint32_t i) { return s.cum[i] >= total; });       // u is 1: the last that weighs anything
    return {id(at), (float)log(weight_of(logit_of(key(at)), m, q.inv_t()) / total)};
}

// ---- any number of tokens: thresholds digit by digit -------------------------------------------

// Largest key first, values are added up until they reach `want` > 0: the key at which they do, and the sum before it.
// each(f) calls f(key, value) for the tokens; they add up to `want` at least.  Eight bits of the key by a pass.
template <int NT, int DTYPE, typename E>
__device__ __forceinline__ uint32_t key_at(Shared<DTYPE, NT>& s, u64 want, u64* before, E&& each)
{
    uint32_t prefix = 0, fixed = 0;
    u64 above = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
        lds_barrier();
        for (int i = threadIdx.x; i < 256; i += NT) s.bin[i] = 0;
        lds_barrier();
        each([&](uint32_t key, u64 value) {
            if ((key & fixed) == prefix && value) atomicAdd(&s.bin[key >> shift & 255u], value);
        });
        lds_barrier();
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
        lds_barrier();
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

// Weights as whole numbers, so that their sums do not depend on the order in which they are added: times the power of two with which
// those of the whole row, `sum` in all, stay below 2^62.  So n weights are off by n 2^-62 of the row's at most, however small each of them is.  (A cut leaves the larger
// ones: of n tokens with weights w in all it leaves k with k w / n at least, whose own are off by (k + n) 2^-62 of what it leaves.)
struct Whole {
    float m;
    double inv_t, scale;
    __device__ __forceinline__ u64 of(float z) const { return (u64)(weight_of(z, m, inv_t) * scale + 0.5); }
};
__device__ __forceinline__ Whole whole_of(float m, double inv_t, double sum) { return {m, inv_t, ldexp(1.0, 61 - ilogb(sum))}; }

// The sum over the workgroup, in every thread and in one order.
template <int NT>
__device__ __forceinline__ double block_sum(double v, double (&part)[NT / 64])
{
    v = lane_value(wave_upto(v), 63);
    lds_barrier();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    lds_barrier();
    v = 0.0;
    for (int w = 0; w < NT / 64; ++w) v += part[w];
    return v;
}
template <int NT, int DTYPE>
__device__ __forceinline__ u64 block_sum(u64 v, Shared<DTYPE, NT>& s)
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    lds_barrier();
    if ((threadIdx.x & 63) == 0) s.bin[threadIdx.x >> 6] = v;
    lds_barrier();
    v = 0;
    for (int w = 0; w < NT / 64; ++w) v += s.bin[w];
    return v;
}

// The draw from a row of any kind, of which some token is allowed.
template <int DTYPE, int NT, bool BITS>
__device__ __forceinline__ Drawn draw_by_digits(Shared<DTYPE, NT>& s, const RowOf<DTYPE>& r, const Setting& q)
{
    uint32_t top = 0;
    for_each<DTYPE, NT, BITS>(r, [&](int32_t, float z) { top = max(top, key_of(z)); });
    top = block_max<NT>(top, s.word);
    const float m = logit_of(top);
    uint32_t key = top;
    u64 nth = 1, before;
    float lp = m == -INFINITY ? -INFINITY : 0.0f;
    if (m != -INFINITY && q.inv_t() != 0.0) {
        double sum = 0.0;
        for_each<DTYPE, NT, BITS>(r, [&](int32_t, float z) { sum += weight_of(z, m, q.inv_t()); });
        const Whole w = whole_of(m, q.inv_t(), block_sum<NT>(sum, s.part));
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
        if (q.top_p() < 1.0) {
            const u64 enough = share_of(q.top_p(), kept_weight(), true);
            cut = max(cut, enough ? key_at<NT>(s, enough, &before, weights) : top);
        }
        if (q.min_p() > 0.0) {
            uint32_t least = top;
            for_each<DTYPE, NT, BITS>(r, [&](int32_t, float z) { if (weight_of(z, m, q.inv_t()) >= q.min_p()) least = min(least, key_of(z)); });
            cut = max(cut, ~block_max<NT>(~least, s.word));
        }
        const u64 total = kept_weight(), target = min(share_of(q.u(), total, false), total - 1);
        key = key_at<NT>(s, target + 1, &before, weights);
        nth = (target - before) / w.of(logit_of(key)) + 1;
        lp = (float)log(weight_of(logit_of(key), m, q.inv_t()) / ((double)total / w.scale));
    }
    // the nth token of that logit
    const uint32_t id = ~key_at<NT>(s, nth, &before, [&](auto&& f) { for_each<DTYPE, NT, BITS>(r, [&](int32_t t, float z) { f(~(uint32_t)t, (u64)(key_of(z) == key)); }); });
    return {(int32_t)id, lp};
}

// Takes hold of a row.  How many tokens are allowed; a barrier at least.
template <int DTYPE, int NT, int R, bool BITS>
__device__ __forceinline__ uint32_t load_row(Shared<DTYPE, NT>& s, Held<DTYPE, NT, R, BITS>& row, const RowOf<DTYPE>& r)
{
    row.load(r);
    if (!BITS) {
        lds_barrier();
        return (uint32_t)r.n_tokens;
    }
    if (R == 0) return count_allowed<NT>(r.bits, r.n_tokens, s.word);
    uint32_t n = row.has_last ? 1u : 0u;
#pragma unroll
    for (int k = 0; k < (row.U + 3) / 4; ++k) n += (uint32_t)__popc(row.b[k]);
    return block_sum<NT>(n, s.word);
}

// The tokens of a row for which wanted(token, logit) holds, in order, if there are at most kList.  maybe(a group's elements): whether it may
// for one of them.  How many there are; two to five barriers.
template <int DTYPE, int NT, int R, bool BITS, typename M, typename F>
__device__ __forceinline__ uint32_t list_of(Shared<DTYPE, NT>& s, Held<DTYPE, NT, R, BITS>& row, M&& maybe, F&& wanted)
{
    constexpr int G = Elem<DTYPE>::kGroup;
    if (threadIdx.x == 0) s.n = 0;
    lds_barrier();
    const auto add = [&](int32_t t, float z) {
        const uint32_t i = atomicAdd(&s.n, 1u);
        if (i < kList<DTYPE>) s.list[i] = (u64)key_of(z) << 32 | ~(uint32_t)t;
    };
    row.each([&](int32_t g, uint4 x, uint32_t on) {
        for (uint32_t left = maybe(x) ? on : 0u; left; left &= left - 1) {
            const int32_t j = __builtin_ctz(left);
            const float z = element_of<DTYPE>(x, j);
            if (wanted(g * G + j, z)) add(g * G + j, z);
        }
    });
    const int32_t behind = row.n_groups * G + (int32_t)threadIdx.x;
    if (row.has_last && wanted(behind, row.last)) add(behind, row.last);
    lds_barrier();
    const uint32_t n = (uint32_t)__builtin_amdgcn_readfirstlane((int)s.n);
    if (n <= kList<DTYPE>) sort_list(s, n);
    return n;
}
template <int DTYPE, int NT, int R, bool BITS>
__device__ __forceinline__ uint32_t list_all(Shared<DTYPE, NT>& s, Held<DTYPE, NT, R, BITS>& row)
{
    row.load_rest();
    return list_of<DTYPE, NT, R, BITS>(s, row, [](uint4) { return true; }, [](int32_t, float) { return true; });
}

// Tokens and weights of the threads before this one and with it, and the weights of all.  What one thread ends with is to the last bit what the
// next begins with, and a thread whose weights add nothing has an empty interval.  One barrier.
struct Sums {
    uint32_t n_before, n_upto;
    double before, upto, whole;
};
template <int NT, int DTYPE>
__device__ __forceinline__ Sums sums_of(Shared<DTYPE, NT>& s, uint32_t n, double w)
{
    const uint32_t n_sum = wave_upto(n), n_below = wave_before(n_sum);
    const double sum = wave_borders(w), below = wave_before(sum);
    if ((threadIdx.x & 63) == 63) {
        s.word2[threadIdx.x >> 6] = n_sum;
        s.part[threadIdx.x >> 6] = sum;
    }
    lds_barrier();
    // The same over the wavefronts; a lane's interval ends at its wavefront's end at most, and exactly there behind the last that adds anything.
    const uint32_t lane = threadIdx.x & 63, wave = (uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x) >> 6;
    const uint32_t n_waves = wave_upto(lane < NT / 64 ? s.word2[lane] : 0u);
    const double waves = wave_borders(lane < NT / 64 ? s.part[lane] : 0.0);
    const double base = wave ? lane_value(waves, (int)wave - 1) : 0.0, end = lane_value(waves, (int)wave), mine = lane_value(sum, 63);
    const uint32_t n_base = wave ? (uint32_t)__builtin_amdgcn_readlane((int)n_waves, (int)(wave - 1)) : 0u;
    return {n_base + n_below, n_base + n_sum, below == mine ? end : fmin(base + below, end), sum == mine ? end : fmin(base + sum, end),
            lane_value(waves, NT / 64 - 1)};
}

// ---- 16-bit logits: how many tokens have each logit ----------------------------------------------

// Logits of 16 bits take few values: with the number of tokens that have each, a row's weights need an exponential for a value, not for a
// token, and their sums do not depend on the order in which the tokens were counted.  Values of a magnitude from 2^-36 to 2^8 have a bin each, 128
// to a power of two, in the order of the values:
//     3: those up to -2^8, 4 .. 5635: negative ones, 5636: around zero, and NaN, 5637 .. 5639: just below 2^-36, 5640 .. 11271: positive ones,
//     11272: those from 2^8 on.
// Bins are read four at a time, hence the three before the positive ones and the place where it all begins.  (Of 10^5 logits spread like a few
// units around zero some lie below 2^-20: with bins from there on, one row of twenty was left to the digits.)
constexpr uint32_t kLowDown = 0x2D7Fu, kLowUp = kLowDown - 3, kHigh = 0x4380u, kHalf = kHigh - kLowDown - 1;     // in units of a bf16's last place
constexpr uint32_t kLowBin = 3, kZeroBin = kLowBin + kHalf + 1, kHighBin = kZeroBin + kHalf + 4;
static_assert(kHighBin + 1 == kBins && kHalf % 8 == 0 && kZeroBin % 4 == 0);
__device__ __forceinline__ uint32_t bin_of(float z)
{
    const float hi = __uint_as_float(kHigh << 16);
    const uint32_t up = __float_as_uint(__builtin_amdgcn_fmed3f(z, __uint_as_float(kLowUp << 16), hi));
    const uint32_t down = __float_as_uint(__builtin_amdgcn_fmed3f(-z, __uint_as_float(kLowDown << 16), hi));
    return (up + ((kZeroBin - kLowUp + kLowDown) << 16) - down) >> 16;
}
// The value of a bin that has one (the zero bin: 0).
__device__ __forceinline__ float value_of(uint32_t bin)
{
    return bin == kZeroBin ? 0.0f : __uint_as_float(bin > kZeroBin ? (kLowUp + bin - kZeroBin) << 16 : (kLowDown + kZeroBin - bin) << 16 | 0x80000000u);
}

// A thread's share of the bins that have a value: stretches of eight that lie together, the largest values first; the zero bin belongs to the
// stretch of the smallest positive values.
constexpr uint32_t kStretches = 2 * kHalf / 8;
template <int NT> constexpr uint32_t kShare = (kStretches + NT - 1) / NT;
__device__ __forceinline__ uint32_t top_of(uint32_t stretch) { return kHighBin - 1 - 8 * stretch - (stretch >= kHalf / 8 ? 4 : 0); }
__device__ __forceinline__ bool has_zero(uint32_t stretch) { return stretch == kHalf / 8 - 1; }
template <int NT>
__device__ __forceinline__ uint32_t counts_of(const Shared<TDFA_BF16, NT>& s, uint32_t stretch, uint32_t (&n)[8])       // the largest value's first; whether there are any
{
    const uint4 hi = *reinterpret_cast<const uint4*>(&s.count[top_of(stretch) - 3]), lo = *reinterpret_cast<const uint4*>(&s.count[top_of(stretch) - 7]);
    n[0] = hi.w; n[1] = hi.z; n[2] = hi.y; n[3] = hi.x; n[4] = lo.w; n[5] = lo.z; n[6] = lo.y; n[7] = lo.x;
    return (hi.x | hi.y | hi.z | hi.w) | (lo.x | lo.y | lo.z | lo.w);
}
// What a thread keeps of its share: of every stretch the weight of the first bin with tokens, and the factor from a weight to the next (the
// values of a stretch lie equally far from one another).
template <int NT>
struct Bins {
    double first[kShare<NT>], factor[kShare<NT>];
};
// f(bin, tokens, weight) in the order of the values, for bins with tokens.
template <int NT, typename F>
__device__ __forceinline__ void each_bin(const Shared<TDFA_BF16, NT>& s, const Bins<NT>& b, float m, double inv_t, F&& f)
{
#pragma unroll
    for (uint32_t p = 0; p < kShare<NT>; ++p) {
        const uint32_t o = threadIdx.x * kShare<NT> + p;
        if (o >= kStretches) return;
        uint32_t n[8];
        if (counts_of<NT>(s, o, n)) {
            double w = b.first[p];
            bool begun = false;
#pragma unroll
            for (uint32_t j = 0; j < 8; ++j) {
                if (begun) w *= b.factor[p];
                if (n[j]) {
                    f(top_of(o) - j, n[j], w);
                    begun = true;
                }
            }
        }
        if (has_zero(o) && s.count[kZeroBin]) f(kZeroBin, s.count[kZeroBin], weight_of(0.0f, m, inv_t));
    }
}

constexpr int32_t kCountedGroups = 64 * (int32_t)kBins;      // of longer rows find_nth has no room for the parts

// What the counts tell all threads of a workgroup, and this one of the bins before its own.
struct Counted : Sums {
    float m;                   // the largest logit
};

// Of the upper and the lower halves of four words the smallest each.
__device__ __forceinline__ uint32_t least_of(uint4 w)
{
    typedef unsigned short pair __attribute__((ext_vector_type(2)));
    const auto p = [](uint32_t x) { return __builtin_bit_cast(pair, x); };
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_min(__builtin_elementwise_min(p(w.x), p(w.y)), __builtin_elementwise_min(p(w.z), p(w.w))));
}

// Clears the counts, before a barrier.
template <int NT>
__device__ __forceinline__ void clear_counts(Shared<TDFA_BF16, NT>& s)
{
    for (uint32_t j = threadIdx.x; j < kBins / 4; j += NT) reinterpret_cast<uint4*>(s.count)[j] = make_uint4(0, 0, 0, 0);
    if (threadIdx.x < kBins % 4) s.count[kBins / 4 * 4 + threadIdx.x] = 0;
}

// Counts the tokens of a row by their logits, and weighs them.  One LDS atomic for each token of a group that has an allowed one: those of a
// wavefront meet in the same bins and banks (of the cycles in which LDS is at work 50 to 65 % are conflicts), which is most of the time until
// the counts are there.  Weights take two exponentials for a stretch that has tokens and a product from bin to bin, not one for each token.
// False: there are logits that the bins do not tell apart and that matter.
template <int NT, int R, bool BITS>
__device__ __forceinline__ bool count_row(Shared<TDFA_BF16, NT>& s, Held<TDFA_BF16, NT, R, BITS>& row, double inv_t, Bins<NT>& b, Counted& c)
{
    if (row.n_groups > kCountedGroups) return false;
    row.template each<false, true>([&](int32_t, uint4 x, uint32_t on) {
        float z[8];
        unpack<TDFA_BF16>(x, z);
        // (a token that is not allowed adds nothing, wherever; a group without any is not in the registers)
        if (on)
#pragma unroll
            for (int j = 0; j < 8; ++j) atomicAdd(&s.count[bin_of(z[j])], on >> j & 1u);
    });
    if (row.has_last) atomicAdd(&s.count[bin_of(row.last)], 1u);
    lds_barrier();
    if (s.count[kHighBin] | s.count[kZeroBin + 1] | s.count[kZeroBin + 2] | s.count[kZeroBin + 3]) return false;
    if (s.count[kZeroBin]) {                               // NaN counts as -inf, and other numbers than zero have no bin
        if (threadIdx.x < 2) s.at[threadIdx.x] = 0;
        lds_barrier();
        uint32_t odd = 0, nans = 0;
        const auto look = [&](float z) {
            nans += z != z ? 1u : 0u;
            odd += z != 0.0f && bin_of(z) == kZeroBin && z == z ? 1u : 0u;
        };
        row.each([&](int32_t, uint4 x, uint32_t on) {
            // magnitudes, those of NaN the largest: next to zero, or NaN?
            const uint4 w = make_uint4(x.x & 0x7FFF7FFFu, x.y & 0x7FFF7FFFu, x.z & 0x7FFF7FFFu, x.w & 0x7FFF7FFFu);
            const uint32_t least = least_of(w), most = ~least_of(make_uint4(~w.x, ~w.y, ~w.z, ~w.w));
            if ((least & 0xFFFFu) > kLowDown && least >> 16 > kLowDown && (most & 0xFFFFu) <= 0x7F80u && most >> 16 <= 0x7F80u) return;
            for (; on; on &= on - 1) look(element_of<TDFA_BF16>(x, __builtin_ctz(on)));
        });
        if (row.has_last) look(row.last);
        if (nans) atomicAdd(&s.at[0], nans);
        if (odd) atomicAdd(&s.at[1], odd);
        lds_barrier();
        if (s.at[1]) return false;
        if (threadIdx.x == 0) s.count[kZeroBin] -= s.at[0];
        lds_barrier();
    }
    // the largest logit, and the first bin with tokens of every stretch (8: none)
    uint32_t top = 0, begin[kShare<NT>];
#pragma unroll
    for (uint32_t p = 0; p < kShare<NT>; ++p) {
        const uint32_t o = threadIdx.x * kShare<NT> + p;
        begin[p] = 8;
        if (o >= kStretches) continue;
        uint32_t found = 0, n[8];
        if (counts_of<NT>(s, o, n)) {
#pragma unroll
            for (int j = 7; j >= 0; --j)
                if (n[j]) begin[p] = (uint32_t)j;
            found = top_of(o) - begin[p];
        }
        if (has_zero(o) && !found && s.count[kZeroBin]) found = kZeroBin;
        if (!top) top = found;
    }
    // lanes are in the order of the values
    const u64 some = __ballot(top != 0);
    top = some ? (uint32_t)__builtin_amdgcn_readlane((int)top, __builtin_ctzll(some)) : 0u;
    if ((threadIdx.x & 63) == 0) s.word[threadIdx.x >> 6] = top;
    lds_barrier();
    top = 0;
#pragma unroll
    for (int v = NT / 64 - 1; v >= 0; --v) top = s.word[v] ? s.word[v] : top;
    if (!top) return false;
    c.m = value_of(top);
    // what is not above -2^8 has to weigh next to nothing: less than 2^24 exp(-64) of the whole
    if (s.count[kLowBin] && !((-256.0 - (double)c.m) * inv_t < -64.0) && inv_t != 0.0) return false;
    uint32_t n = 0;
    double w = 0.0;
    if (inv_t != 0.0) {
#pragma unroll
        for (uint32_t p = 0; p < kShare<NT>; ++p) {
            b.first[p] = b.factor[p] = 0.0;
            if (begin[p] == 8) continue;
            const uint32_t at = top_of(threadIdx.x * kShare<NT> + p);
            b.first[p] = weight_of(value_of(at - begin[p]), c.m, inv_t);
            b.factor[p] = exp(((double)value_of(at - 7) - (double)value_of(at - 6)) * inv_t);
        }
        each_bin<NT>(s, b, c.m, inv_t, [&](uint32_t, uint32_t tokens, double weight) {
            n += tokens;
            w += product((double)tokens, weight);
        });
    }
    static_cast<Sums&>(c) = sums_of<NT>(s, n, w);
    return true;
}
// The nth (from 0) of the allowed tokens with logit v, by id, in the one thread that holds it; -1 in all others.
template <int DTYPE, int NT, int R, bool BITS>
__device__ __forceinline__ int32_t find_nth(Shared<DTYPE, NT>& s, Held<DTYPE, NT, R, BITS>& row, float v, uint32_t nth)
{
    constexpr int G = Elem<DTYPE>::kGroup;
    const auto matches = [&](uint4 x, uint32_t on) {
        float z[G];
        unpack<DTYPE>(x, z);
        uint32_t found = 0;
#pragma unroll
        for (int j = 0; j < G; ++j) found |= (z[j] == v ? 1u : 0u) << j;
        return found & on;
    };
    // Whether a group has any; 16 bits: two elements at a time, of zero without its sign.
    const uint32_t bits = (uint32_t)__builtin_amdgcn_readfirstlane((int)(DTYPE == TDFA_F32 ? __float_as_uint(v) : (__float_as_uint(v) >> 16) * 0x10001u));
    const bool zero = v == 0.0f;
    const auto maybe = [&](uint4 x) {
        if (zero) {
            constexpr uint32_t sign = DTYPE == TDFA_F32 ? 0x7FFFFFFFu : 0x7FFF7FFFu;
            x = make_uint4(x.x & sign, x.y & sign, x.z & sign, x.w & sign);
        }
        const uint4 w = make_uint4(x.x ^ bits, x.y ^ bits, x.z ^ bits, x.w ^ bits);
        if constexpr (DTYPE == TDFA_F32) return min(min(w.x, w.y), min(w.z, w.w)) == 0;
        const uint32_t m = least_of(w);
        return (m & 0xFFFFu) == 0 || m < 0x10000u;
    };
    // how many there are in every 64 groups, which a wavefront holds
    const uint32_t lane = threadIdx.x & 63, chunks = (uint32_t)(row.n_groups + 63) / 64;
    row.template each<true>([&](int32_t g, uint4 x, uint32_t on) {
        uint32_t n = 0;
        if (__ballot(maybe(x))) {
            const uint32_t found = matches(x, on);
#pragma unroll
            for (int j = 0; j < G; ++j) n += (uint32_t)__popcll(__ballot(found >> j & 1));
        }
        if (lane == 0 && (uint32_t)g < chunks * 64) s.chunk[g >> 6] = n;
    });
    lds_barrier();
    // every wavefront finds the chunk, and the one that holds it the token
    const uint32_t per = (chunks + 63) / 64;
    uint32_t mine = 0;
    for (uint32_t j = lane * per; j < min(lane * per + per, chunks); ++j) mine += s.chunk[j];
    const uint32_t upto = wave_upto(mine);
    const u64 here = __ballot(upto > nth);
    if (!here) {                                           // behind the whole groups: the tokens of the first threads
        const uint32_t left = nth - (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
        const bool match = row.has_last && row.last == v;
        const u64 behind = __ballot(match);
        return match && (uint32_t)__popcll(behind & ((1ull << lane) - 1)) == left ? row.n_groups * G + (int32_t)threadIdx.x : -1;
    }
    const int src = __builtin_ctzll(here);
    uint32_t chunk = lane * per, left = nth - (upto - mine);
    if ((int)lane == src)
        for (; left >= s.chunk[chunk]; ++chunk) left -= s.chunk[chunk];
    chunk = (uint32_t)__builtin_amdgcn_readlane((int)chunk, src);
    left = (uint32_t)__builtin_amdgcn_readlane((int)left, src);
    int32_t g = -1;
    uint32_t found = 0;
    if constexpr (R > 0) {
#pragma unroll
        for (int k = 0; k < R; ++k)
            if ((uint32_t)__builtin_amdgcn_readfirstlane((int)threadIdx.x + k * NT) >> 6 == chunk) {
                g = (int32_t)threadIdx.x + k * NT;
                found = matches(row.x[k], row.on_of(k, g));
            }
    } else if (threadIdx.x < 64) {
        g = (int32_t)(chunk * 64 + lane);
        uint32_t on = g < row.n_groups ? row.kAll : 0u;
        if constexpr (BITS) {
            const uint32_t byte = __builtin_amdgcn_raw_buffer_load_b8(row.buf.bits, DTYPE == TDFA_F32 ? g >> 1 : g, 0, 0);
            on &= DTYPE == TDFA_F32 ? byte >> ((g & 1) * 4) : byte;
        }
        found = matches(group_at<false>(row.buf.x, (uint32_t)g * 16u), on);
    }
    if (g < 0) return -1;
    const uint32_t n = (uint32_t)__popc(found), before = wave_upto(n) - n;
    if (left < before || left >= before + n) return -1;
    for (left -= before; left; --left) found &= found - 1;
    return g * G + __builtin_ctz(found);
}

// The draw from a row whose tokens have been counted, in the one thread that holds the token; the others have none.
template <int NT, int R, bool BITS>
__device__ __forceinline__ Drawn draw_of_counts(Shared<TDFA_BF16, NT>& s, Held<TDFA_BF16, NT, R, BITS>& row, const Bins<NT>& b, const Counted& c, const Setting& q)
{
    if (q.inv_t() == 0.0) return {find_nth<TDFA_BF16>(s, row, c.m, 0), 0.0f};
    double kept = c.whole;
    // Every cut leaves a beginning of the order: what it leaves of the weights, as far as it goes.
    if (q.top_k) {
        if (threadIdx.x == 0) s.mass[0] = kept;
        lds_barrier();
        if (c.n_before < q.top_k && q.top_k <= c.n_upto) {
            uint32_t n = c.n_before;
            double sum = c.before;
            each_bin<NT>(s, b, c.m, q.inv_t(), [&](uint32_t, uint32_t tokens, double w) {
                if (n < q.top_k) sum += product((double)tokens, w);
                n += tokens;
            });
            s.mass[0] = fmin(sum, c.upto);                 // (which is the next thread's beginning, however it has been rounded)
        }
        lds_barrier();
        kept = s.mass[0];
    }
    if (q.top_p() < 1.0 || q.min_p() > 0.0) {
        const double enough = fmax(q.top_p() * kept, 1e-300);
        if (threadIdx.x == 0) s.mass[1] = kept;
        if (threadIdx.x == 1) s.least = 0;
        lds_barrier();
        if (q.top_p() < 1.0 && c.before < enough && enough <= c.upto) {
            double sum = c.before;
            each_bin<NT>(s, b, c.m, q.inv_t(), [&](uint32_t, uint32_t tokens, double w) {
                if (sum < enough) sum += product((double)tokens, w);
            });
            s.mass[1] = fmin(sum, c.upto);
        }
        if (q.min_p() > 0.0) {
            double sum = c.before, least = 0.0;
            each_bin<NT>(s, b, c.m, q.inv_t(), [&](uint32_t, uint32_t tokens, double w) {
                sum += product((double)tokens, w);
                if (w >= q.min_p()) least = sum;
            });
            if (least > 0.0) atomicMax(&s.least, (u64)__double_as_longlong(fmin(least, c.upto)));
        }
        lds_barrier();
        kept = fmin(kept, s.mass[1]);
        if (q.min_p() > 0.0) kept = fmin(kept, __longlong_as_double((long long)s.least));
    }
    // the bin up to which the weights come to more than the target, which stays below what is kept
    const double target = fmin(q.u() * kept, __longlong_as_double(__double_as_longlong(kept) - 1));
    if (c.before <= target && target < c.upto) {
        double sum = c.before, before = sum, w_at = 1.0;
        uint32_t at = 0, tokens_at = 1;
        each_bin<NT>(s, b, c.m, q.inv_t(), [&](uint32_t bin, uint32_t tokens, double w) {
            if ((sum <= target && w > 0.0) || !at) {
                at = bin;
                tokens_at = tokens;
                before = sum;
                w_at = w;
            }
            sum += product((double)tokens, w);
        });
        s.at[0] = at;
        s.at[1] = (uint32_t)fmin(fmax((target - before) / w_at, 0.0), (double)(tokens_at - 1));
        s.mass[2] = w_at / kept;
    }
    lds_barrier();
    const float v = value_of(s.at[0]);
    const uint32_t nth = s.at[1];
    const double share = s.mass[2];
    const int32_t token = find_nth<TDFA_BF16>(s, row, v, nth);
    return {token, token >= 0 ? (float)log(share) : 0.0f};
}

// ---- 32-bit logits: tokens by the distance from the largest --------------------------------------

// Logits of 32 bits take too many values for a bin each.  Tokens are told apart by how far they lie below the largest logit, kPerUnit steps to
// a unit, which is a power of e of the weights; the tokens of the step that a search ends in are put in order.  Weights are added up as
// whole numbers, each as a part of the largest that its step can have: the sums do not depend on the order in which they are made, and keep their
// bits however small the weights are.  What lies kSteps or more below weighs less than 10^-22 of the largest and counts as nothing.
constexpr double kPerUnit = 80.0;

// exp(-x) for 0 <= x <= 1 / 80, by its series, off by 2^-47 of itself.
__device__ __forceinline__ double exp_near(double x)
{
    return fma(x, fma(x, fma(x, fma(x, fma(x, -1.0 / 120.0, 1.0 / 24.0), -1.0 / 6.0), 0.5), -1.0), 1.0);
}

// The largest logit of a row, by the first look at it.
template <int NT, int R, bool BITS>
__device__ __forceinline__ float largest_of(Shared<TDFA_F32, NT>& s, Held<TDFA_F32, NT, R, BITS>& row)
{
    float m = row.last;                                    // (NaN: passed over by all of these)
    m = fmaxf(m, -INFINITY);
    row.template each<false, true>([&](int32_t, uint4 x, uint32_t on) {
        x = make_uint4(on & 1 ? x.x : kNegInf<TDFA_F32>, on & 2 ? x.y : kNegInf<TDFA_F32>, on & 4 ? x.z : kNegInf<TDFA_F32>, on & 8 ? x.w : kNegInf<TDFA_F32>);
        m = max_group<TDFA_F32>(x, m);
    });
    m = wave_max(m);
    // (not in s.word: a wavefront without a token is here while others read there how many the row has)
    if ((threadIdx.x & 63) == 0) s.word2[threadIdx.x >> 6] = __float_as_uint(m);
    for (uint32_t j = threadIdx.x; j < kSteps; j += NT) {
        s.step.weight[j] = 0;
        s.step.tokens[j] = 0;
    }
    lds_barrier();
    for (int v = 0; v < NT / 64; ++v) m = fmaxf(m, __uint_as_float(s.word2[v]));
    return shared_by_wave(m);
}

// The step of a logit (NaN: the last), and how far it lies into it.
struct Steps {
    double m, scale;           // steps to a unit of the logits
    __device__ __forceinline__ uint32_t of(float z, double* into) const
    {
        const double y = fmin((m - (double)fmaxf(z, -INFINITY)) * scale, (double)(kSteps - 1));
        const uint32_t i = (uint32_t)y;
        *into = y - (double)i;
        return i;
    }
    __device__ __forceinline__ uint32_t of(float z) const
    {
        double unused;
        return of(z, &unused);
    }
    // The logits next to step i: so far around it that nothing of it is missed.  A distance from m and its step are rounded to 53 bits, and so is a
    // border: each is off by 2^-51 or less of the distance, however near to 0 the border itself lies, and by 2^-24 of the border in binary32.
    struct Band {
        float least, most;
        __device__ __forceinline__ bool any_of(uint4 x) const
        {
            float z[4];
            unpack<TDFA_F32>(x, z);
            bool any = false;
#pragma unroll
            for (int j = 0; j < 4; ++j) any |= z[j] >= least && z[j] <= most;
            return any;
        }
    };
    __device__ __forceinline__ Band band_of(uint32_t i) const
    {
        const double end = (double)(i + 1) / scale;
        const float lo = (float)(m - end), hi = (float)(m - (double)i / scale), around = (float)(end * 0x1p-45) + 1.0e-30f;
        return {shared_by_wave(lo - fabsf(lo) * 0x1p-21f - around), shared_by_wave(hi + fabsf(hi) * 0x1p-21f + around)};
    }
};

// (A thread has kSteps / NT steps that lie together.)
template <int NT>
__device__ __forceinline__ double step_weight(const Shared<TDFA_F32, NT>& s, uint32_t i, double unit) { return product((double)s.step.weight[i], unit); }

// Puts the tokens of a row in steps, and adds up.  An LDS atomic of 64 bits for each token, and one of 32 where a cut by number needs counts.
template <int NT, int R, bool BITS>
__device__ __forceinline__ Sums step_row(Shared<TDFA_F32, NT>& s, Held<TDFA_F32, NT, R, BITS>& row, const Steps& steps, int32_t n_tokens, bool counts)
{
    // 2^bits: n_tokens weights stay below 2^62, and one below 2^50
    const int bits = min(50, 62 - (32 - __clz(n_tokens)));
    const double one = ldexp(1.0, bits), shift = 0x1p52;
    const auto add = [&](float z) {
        double into;
        const uint32_t i = steps.of(z, &into);
        // (a sum with 2^52 has the whole number in its lower bits)
        const u64 w = (u64)__double_as_longlong(fma(exp_near(into * (1.0 / kPerUnit)), one, shift)) & ((1ull << 52) - 1);
        if (i < kSteps - 1) atomicAdd(&s.step.weight[i], w);
        if (counts) atomicAdd(&s.step.tokens[i], 1u);
    };
    row.each([&](int32_t, uint4 x, uint32_t on) {
        float z[4];
        unpack<TDFA_F32>(x, z);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (on >> j & 1) add(z[j]);
    });
    if (row.has_last) add(row.last);
    lds_barrier();
    constexpr uint32_t P = kSteps / NT;
    uint32_t n = 0;
    double w = 0.0, unit = exp(-(double)(threadIdx.x * P) * (1.0 / kPerUnit)) * ldexp(1.0, -bits);
#pragma unroll
    for (uint32_t j = 0; j < P; ++j) {
        if (counts) n += s.step.tokens[threadIdx.x * P + j];
        w += step_weight<NT>(s, threadIdx.x * P + j, unit);
        unit *= 0.98757780049388144;                       // exp(-1 / 80)
    }
    return sums_of<NT>(s, n, w);
}
// f(step, its tokens, its weight) for the steps of this thread in order.
template <int NT, typename F>
__device__ __forceinline__ void each_step(const Shared<TDFA_F32, NT>& s, int32_t n_tokens, F&& f)
{
    constexpr uint32_t P = kSteps / NT;
    const int bits = min(50, 62 - (32 - __clz(n_tokens)));
    double unit = exp(-(double)(threadIdx.x * P) * (1.0 / kPerUnit)) * ldexp(1.0, -bits);
    for (uint32_t j = 0; j < P; ++j) {
        f(threadIdx.x * P + j, s.step.tokens[threadIdx.x * P + j], step_weight<NT>(s, threadIdx.x * P + j, unit));
        unit *= 0.98757780049388144;
    }
}

// The draw from a row of 32-bit logits.  By the whole workgroup, the result is thread 0's; false: not to be had in this way.
template <int NT, int R, bool BITS>
__device__ __forceinline__ bool draw_of_steps(Shared<TDFA_F32, NT>& s, Held<TDFA_F32, NT, R, BITS>& row, int32_t n_tokens, const Setting& q, Drawn* d)
{
    const float m = largest_of<NT, R, BITS>(s, row);
    if (!(fabsf(m) < INFINITY)) return false;
    const double inv_t = q.inv_t();
    const auto key = [&](uint32_t i) { return (uint32_t)(s.sorted[i] >> 32); };
    if (inv_t == 0.0) {
        // (a group may hold larger logits too, of tokens that are not allowed)
        const uint32_t n = list_of<TDFA_F32, NT, R, BITS>(s, row, [&](uint4 x) { return max_group<TDFA_F32>(x, -INFINITY) >= m; }, [&](int32_t, float z) { return z == m; });
        if (n == 0 || n > kList<TDFA_F32>) return false;
        *d = {(int32_t)~(uint32_t)s.sorted[0], 0.0f};
        return true;
    }
    const Steps steps = {(double)m, inv_t * kPerUnit};
    const Sums c = step_row<NT, R, BITS>(s, row, steps, n_tokens, q.top_k != 0);
    if (threadIdx.x < 2) s.at[threadIdx.x] = kSteps;
    lds_barrier();
    double kept = c.whole;
    // Lists step i and adds up its weights from `base` on; false: too many.
    const auto look = [&](uint32_t i, double base) {
        const Steps::Band band = steps.band_of(i);
        const uint32_t n = list_of<TDFA_F32, NT, R, BITS>(s, row, [&](uint4 x) { return band.any_of(x); }, [&](int32_t, float z) { return steps.of(z) == i; });
        if (n == 0 || n > kList<TDFA_F32>) return 0u;
        if (threadIdx.x < 64) {
            sum_list(s, n, m, inv_t);
            for (uint32_t j = threadIdx.x; j < n; j += 64) s.cum[j] += base;
        }
        lds_barrier();
        return n;
    };
    const auto behind = [&](uint32_t n, uint32_t i) {      // the tokens that have the i-th one's logit
        const uint32_t k = key(i);
        return first_where(n, [&](uint32_t j) { return key(j) < k; });
    };
    // Weights up to the first `stay` of a step's tokens, no more than up to where the next step begins, however that has been rounded.
    const auto upto = [&](uint32_t stay, double end) { return fmin(s.cum[stay - 1], end); };
    if (q.top_k) {
        if (c.n_before < q.top_k && q.top_k <= c.n_upto) {
            uint32_t n = c.n_before;
            double sum = c.before;
            each_step<NT>(s, n_tokens, [&](uint32_t i, uint32_t tokens, double w) {
                if (n < q.top_k && q.top_k <= n + tokens) {
                    s.at[0] = i;
                    s.at[2] = q.top_k - n;
                    s.mass[0] = sum;
                    s.end[0] = fmin(sum + w, c.upto);
                }
                n += tokens;
                sum += w;
            });
        }
        lds_barrier();
        const uint32_t i = s.at[0], nth = s.at[2];
        const double base = s.mass[0];
        if (i < kSteps - 1) {                              // (a cut in the last step leaves all that weighs anything)
            const uint32_t n = look(i, base);
            if (!n) return false;
            kept = fmin(kept, upto(behind(n, min(nth, n) - 1), s.end[0]));
        }
    }
    double cut = kept;
    if (q.top_p() < 1.0) {
        const double enough = fmax(q.top_p() * kept, 1e-300);
        if (c.before < enough && enough <= c.upto) {
            double sum = c.before;
            each_step<NT>(s, n_tokens, [&](uint32_t i, uint32_t, double w) {
                if (w > 0.0 && (s.at[1] == kSteps || sum < enough)) {
                    s.at[1] = i;
                    s.mass[1] = sum;
                    s.end[1] = fmin(sum + w, c.upto);
                }
                sum += w;
            });
        }
        lds_barrier();
        const uint32_t i = s.at[1];
        const double base = s.mass[1];
        const uint32_t n = i < kSteps ? look(i, base) : 0u;
        if (!n) return false;
        cut = fmin(cut, upto(behind(n, min(n - 1, first_where(n, [&](uint32_t j) { return s.cum[j] >= enough; }))), s.end[1]));
    }
    // what weighs at least min_p ends in the step of its logarithm
    if (const uint32_t i = q.min_p() > 0.0 ? (uint32_t)fmin(fmax(-log(q.min_p()), 0.0) * kPerUnit, (double)(kSteps - 1)) : kSteps - 1; i < kSteps - 1) {
        if (threadIdx.x == i / (kSteps / NT)) {
            double sum = c.before;
            each_step<NT>(s, n_tokens, [&](uint32_t j, uint32_t, double w) {
                if (j == i) {
                    s.mass[2] = fmin(sum, c.upto);         // (as the next thread's steps begin)
                    s.end[2] = fmin(sum + w, c.upto);
                }
                sum += w;
            });
        }
        lds_barrier();
        const double base = s.mass[2];
        const Steps::Band band = steps.band_of(i);
        const uint32_t n = list_of<TDFA_F32, NT, R, BITS>(s, row, [&](uint4 x) { return band.any_of(x); }, [&](int32_t, float z) { return steps.of(z) == i; });
        if (n > kList<TDFA_F32>) return false;
        if (threadIdx.x < 64 && n) {
            sum_list(s, n, m, inv_t);
            for (uint32_t j = threadIdx.x; j < n; j += 64) s.cum[j] += base;
        }
        lds_barrier();
        const uint32_t stay = first_where(n, [&](uint32_t j) { return weight_of(logit_of(key(j)), m, inv_t) < q.min_p(); });
        cut = fmin(cut, stay ? upto(stay, s.end[2]) : base);
    }
    kept = fmin(kept, cut);
    const double target = fmin(q.u() * kept, __longlong_as_double(__double_as_longlong(kept) - 1));
    if (threadIdx.x == 0) s.at[3] = kSteps;
    lds_barrier();
    if (c.before <= target && target < c.upto) {
        double sum = c.before;
        each_step<NT>(s, n_tokens, [&](uint32_t i, uint32_t, double w) {
            if (w > 0.0 && (s.at[3] == kSteps || sum <= target)) {
                s.at[3] = i;
                s.mass[0] = sum;
            }
            sum += w;
        });
    }
    lds_barrier();
    const uint32_t i = s.at[3];
    const double base = s.mass[0];
    const uint32_t n = i < kSteps ? look(i, base) : 0u;
    if (!n) return false;
    // the last that weighs anything, where roundings leave the target behind all
    const double end = s.cum[n - 1];
    uint32_t at = first_where(n, [&](uint32_t j) { return s.cum[j] > target; });
    if (at >= n) at = first_where(n, [&](uint32_t j) { return s.cum[j] >= end; });
    *d = {(int32_t)~(uint32_t)s.sorted[at], (float)log(weight_of(logit_of(key(at)), m, inv_t) / kept)};
    return true;
}

// The first k tokens of a row of 32-bit logits, in order, in sorted[], and what the row weighs.  How many; 0: not to be had in this way.
template <int NT, int R, bool BITS>
__device__ __forceinline__ uint32_t top_of_steps(Shared<TDFA_F32, NT>& s, Held<TDFA_F32, NT, R, BITS>& row, uint32_t k, double inv_t, float* m, double* total)
{
    *m = largest_of<NT, R, BITS>(s, row);
    if (!(fabsf(*m) < INFINITY)) return 0;
    // Steps of the logits themselves, whatever the temperature, and in binary32: only the order has borders.  Weights are of binary32 too: the three roundings of an
    // exponent x and the exponential's last place leave them off by (1 + |x|) 2^-22 of themselves at most.  (Of 64 bits, by a polynomial: 500 rows of 32,000 36 -> 44 us.)
    // Their sum is of 64: next to the largest weight, which is 1, one of binary32 would lose what the logarithm of a nearly certain token is made of.
    const float top = *m, c2 = (float)(1.44269504088896340736 * inv_t);
    // (0 times infinity is no number, and a difference that overflows has to weigh nothing)
    if (!(c2 >= 0x1p-60f && c2 < INFINITY)) return 0;
    const auto step = [&](float z) { return (uint32_t)fminf((top - fmaxf(z, -INFINITY)) * (float)kPerUnit, (float)(kSteps - 1)); };
    double sum = 0.0;
    const auto add = [&](float z) {
        sum += (double)__builtin_amdgcn_exp2f((fmaxf(z, -INFINITY) - top) * c2);
        atomicAdd(&s.step.tokens[step(z)], 1u);
    };
    row.each([&](int32_t, uint4 x, uint32_t on) {
        float z[4];
        unpack<TDFA_F32>(x, z);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if (on >> j & 1) add(z[j]);
    });
    if (row.has_last) add(row.last);
    lds_barrier();
    constexpr uint32_t P = kSteps / NT;
    uint32_t n = 0;
#pragma unroll
    for (uint32_t j = 0; j < P; ++j) n += s.step.tokens[threadIdx.x * P + j];
    const Sums c = sums_of<NT>(s, n, sum);
    *total = c.whole;
    if (threadIdx.x == 0) s.at[0] = kSteps;
    lds_barrier();
    if (c.n_before < k && k <= c.n_upto) {
        n = c.n_before;
        for (uint32_t j = 0; j < P; ++j) {
            const uint32_t tokens = s.step.tokens[threadIdx.x * P + j];
            if (n < k && k <= n + tokens) s.at[0] = threadIdx.x * P + j;
            n += tokens;
        }
    }
    lds_barrier();
    const uint32_t last = s.at[0];
    if (last >= kSteps - 1) return 0;
    n = list_of<TDFA_F32, NT, R, BITS>(s, row, [&](uint4 x) { return step(fminf(max_group<TDFA_F32>(x, -INFINITY), top)) <= last; },     // (or above, if it is not allowed)
                                      [&](int32_t, float z) { return step(z) <= last; });
    return n > kList<TDFA_F32> ? 0u : n;
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

// One workgroup per sequence, that reads its row once (or, where it does not stay in registers, once for every look at it).  At most kFew allowed
// tokens are put in order; more are counted by their logits (16 bits) or weighed by steps (32), and every cut and the draw are searches in those
// sums.  What bounds it: one row, its chain of phases on one compute unit (bf16, 128,256 tokens, no constraint: 19 us, of which 9 to 12 until all
// tokens are counted, 4 for weights and their sums, 3 for the token among those of its logit); many rows, LDS atomics, one for each token, eight
// to a group of 16 bytes: 1,000 such rows 84 to 88 us, 2.9 to 3.1 TB/s.  fp32, 300 rows of 32,003 with three cuts: 53 to 55 us, 6 for the largest logit, 13 for
// the steps, 4 to 6 for each of up to four steps that are put in order.  (Thresholds digit by digit instead, ten looks at a row or more: 434, 1,900 and 373 us.)
template <int DTYPE, int NT, int R, bool BITS>
__global__ void __launch_bounds__(NT, NT > 256 ? 4 : DTYPE == TDFA_F32 ? 2 : 3) draw_step_kernel(DrawArgs a)
{
    __shared__ Shared<DTYPE, NT> s;
    const uint32_t i = blockIdx.x;
    const StateOf st = state_of(a, i);
    const Setting q = setting_of(a, i);
    const RowOf<DTYPE> r = {row_at<DTYPE>(a.logits, i, a.stride16), st.bits, a.n_tokens};
    Held<DTYPE, NT, R, BITS> row;
    if constexpr (DTYPE == TDFA_BF16) clear_counts<NT>(s);
    const uint32_t n = (uint32_t)__builtin_amdgcn_readfirstlane((int)(st.valid ? load_row<DTYPE, NT, R, BITS>(s, row, r) : 0u));
    Drawn d = {TDFA_NO_TOKEN, 0.0f};
    bool mine = threadIdx.x == 0;                          // this thread writes the result
    if (n > kFew) {
        bool done = false;
        if constexpr (DTYPE == TDFA_BF16) {
            Counted c;
            Bins<NT> b;
            done = count_row<NT, R, BITS>(s, row, q.inv_t(), b, c);
            if (done) {
                d = draw_of_counts<NT, R, BITS>(s, row, b, c, q);
                mine = d.token >= 0;
            }
        }
        if constexpr (DTYPE == TDFA_F32) done = draw_of_steps<NT, R, BITS>(s, row, a.n_tokens, q, &d);
        if (!done) d = draw_by_digits<DTYPE, NT, BITS>(s, r, q);
    } else if (n) {
        list_all<DTYPE, NT, R, BITS>(s, row);
        if (threadIdx.x < 64) {
            const float m = logit_of((uint32_t)(s.sorted[0] >> 32));
            if (m != -INFINITY) sum_list(s, n, m, q.inv_t());
            d = draw_of_list<NT>(s, n, m, q);
        }
    }
    if (mine) {
        a.tokens[i] = d.token;
        if (a.targets) a.new_states[i] = !st.valid ? TDFA_DEAD : d.token == TDFA_NO_TOKEN ? st.q : target_of(a, st.q, d.token);
        if (a.logprobs) a.logprobs[i] = d.lp;
    }
}

// The first k tokens of a row of any kind, in order, in sorted[], and what the row weighs.  How many there are, 0 if all are -inf.
template <int DTYPE, int NT, bool BITS>
__device__ __forceinline__ uint32_t top_by_digits(Shared<DTYPE, NT>& s, const RowOf<DTYPE>& r, uint32_t k, double inv_t, float* m, double* total)
{
    uint32_t top = 0;
    for_each<DTYPE, NT, BITS>(r, [&](int32_t, float z) { top = max(top, key_of(z)); });
    *m = logit_of(block_max<NT>(top, s.word));
    if (*m == -INFINITY) return 0;
    // the k-th largest key, and how many larger ones there are; of the tokens that have it those of the lowest ids
    u64 larger, unused;
    const uint32_t key = key_at<NT>(s, k, &larger, [&](auto&& f) { for_each<DTYPE, NT, BITS>(r, [&](int32_t, float z) { f(key_of(z), (u64)1); }); });
    const uint32_t last = ~key_at<NT>(s, k - larger, &unused, [&](auto&& f) {
        for_each<DTYPE, NT, BITS>(r, [&](int32_t t, float z) { f(~(uint32_t)t, (u64)(key_of(z) == key)); });
    });
    double sum = 0.0;
    if (threadIdx.x == 0) s.n = 0;
    lds_barrier();
    for_each<DTYPE, NT, BITS>(r, [&](int32_t t, float z) {
        sum += weight_of(z, *m, inv_t);
        if (key_of(z) > key || (key_of(z) == key && (uint32_t)t <= last)) s.list[atomicAdd(&s.n, 1u)] = (u64)key_of(z) << 32 | ~(uint32_t)t;
    });
    *total = block_sum<NT>(sum, s.part);
    const uint32_t n = s.n;
    sort_list(s, n);
    return n;
}

// The same from counts; 0: they do not tell.
template <int NT, int R, bool BITS>
__device__ __forceinline__ uint32_t top_of_counts(Shared<TDFA_BF16, NT>& s, Held<TDFA_BF16, NT, R, BITS>& row, uint32_t k, double inv_t, float* m, double* total)
{
    Counted c;
    Bins<NT> b;
    if (!count_row<NT, R, BITS>(s, row, inv_t, b, c)) return 0;
    *m = c.m;
    *total = c.whole;
    if (threadIdx.x == 0) s.at[0] = 0;
    lds_barrier();
    if (c.n_before < k && k <= c.n_upto) {
        uint32_t n = c.n_before;
        each_bin<NT>(s, b, c.m, inv_t, [&](uint32_t bin, uint32_t tokens, double) {
            if (n < k) {
                s.at[0] = bin;
                s.at[1] = n;
                s.at[2] = tokens;
            }
            n += tokens;
        });
    }
    lds_barrier();
    if (!s.at[0]) return 0;                                // fewer than k above -2^8
    const float v = value_of(s.at[0]);
    const uint32_t larger = s.at[1], equal = s.at[2];
    int32_t last = INT32_MAX;
    if (larger + equal > kList<TDFA_BF16>) {                // more than are wanted have that logit: those of the lowest ids
        const int32_t t = find_nth<TDFA_BF16>(s, row, v, k - larger - 1);
        if (t >= 0) s.at[3] = (uint32_t)t;
        lds_barrier();
        last = (int32_t)s.at[3];
    }
    return list_of<TDFA_BF16, NT, R, BITS>(s, row, [&](uint4 x) { return max_group<TDFA_BF16>(x, -INFINITY) >= v; },
                                           [&](int32_t t, float z) { return z > v || (z == v && t <= last); });
}

// One workgroup per row: the k first tokens in order, and their log-probabilities.  The same counts or steps give the logit that k tokens reach; those
// that do are put in order.  Bounds as for a draw: one row of 128,256 tokens in bf16 19 us, 2,048 rows under a constraint 130 to 136 (212 MB of groups with an
// allowed token, 292 MB read), 500 fp32 rows of 32,000 with 200 tokens listed 37.  (By digits: 195, 1,290 and 190 us.)
template <int DTYPE, int NT, int R, bool BITS>
__global__ void __launch_bounds__(NT, NT > 256 ? 4 : DTYPE == TDFA_F32 ? 2 : 3) top_logprobs_kernel(TopArgs a)
{
    __shared__ Shared<DTYPE, NT> s;
    const uint32_t i = blockIdx.x, k = (uint32_t)a.k;
    const StateOf st = state_of(a, i);
    const RowOf<DTYPE> r = {row_at<DTYPE>(a.logits, i, a.stride16), st.bits, a.n_tokens};
    const double inv_t = 1.0 / (double)a.temperature;
    Held<DTYPE, NT, R, BITS> row;
    if constexpr (DTYPE == TDFA_BF16) clear_counts<NT>(s);
    uint32_t n = (uint32_t)__builtin_amdgcn_readfirstlane((int)(st.valid ? load_row<DTYPE, NT, R, BITS>(s, row, r) : 0u));
    float m = -INFINITY;
    double total = 0.0;
    if (n > kFew) {
        n = 0;
        if constexpr (DTYPE == TDFA_BF16) n = top_of_counts<NT, R, BITS>(s, row, k, inv_t, &m, &total);
        else n = top_of_steps<NT, R, BITS>(s, row, k, inv_t, &m, &total);
        if (!n) n = top_by_digits<DTYPE, NT, BITS>(s, r, k, inv_t, &m, &total);
    } else if (n) {
        list_all<DTYPE, NT, R, BITS>(s, row);
        m = logit_of((uint32_t)(s.sorted[0] >> 32));
        if (m != -INFINITY) {
            if (threadIdx.x < 64) sum_list(s, n, m, inv_t);
            lds_barrier();
            total = s.cum[n - 1];
        }
    }
    const double ln_total = m == -INFINITY ? 0.0 : m == INFINITY ? NAN : log(total);
    for (uint32_t j = threadIdx.x; j < k; j += NT) {
        int32_t id = TDFA_NO_TOKEN;
        float lp = -INFINITY;
        if (m != -INFINITY && j < n && (uint32_t)(s.sorted[j] >> 32) > kKeyNegInf) {
            id = (int32_t)~(uint32_t)s.sorted[j];
            lp = (float)(((double)logit_of((uint32_t)(s.sorted[j] >> 32)) - (double)m) * inv_t - ln_total);
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

// launch_of(type, threads, groups to a thread, whether there is a constraint) for the shape that rows of n_groups take: in registers as
// long as they fit, few rows by more threads each.  Where there are several long rows to a compute unit, three of them at a time, each
// read two or three times, beat one that is held: 128,256 tokens in bf16, draws / lists of 2,048 rows under a constraint 156 -> 119 and
// 153 -> 118 us, 512 rows 48 -> 45 and 47 -> 44; without one 2,048 rows 174 -> 161 and 167 -> 158, 768 rows 73 -> 75 and 72 -> 68, 512 rows 51.5 ->
// 51.9 and 49.1 -> 49.9 (workgroups of 1,024 threads, of which one fits: 193 and 189).  Rows of 32,000 by 512 threads with 8 groups each against 256
// with 16: 300 rows 21 against 26, 1,500 rows 52 against 56.
template <int DTYPE, bool BITS, typename F>
int shaped(bool draws, int64_t rows, int32_t n_groups, F&& launch_of)
{
    using std::integral_constant;
    const integral_constant<int, DTYPE> type;
    const integral_constant<bool, BITS> bits;
    const auto go = [&](auto threads, auto groups) { return launch_of(type, threads, groups, bits); };
    if (n_groups <= 256 * 4) return go(integral_constant<int, 256>(), integral_constant<int, 4>());
    if (n_groups <= 1024 * 4 && rows <= 256) return go(integral_constant<int, 1024>(), integral_constant<int, 4>());
    if (n_groups <= 512 * 8) return go(integral_constant<int, 512>(), integral_constant<int, 8>());
    if constexpr (DTYPE == TDFA_F32) {
        // (With more in registers the compiler would keep some in memory.)  Draws, 1024 x 8 against 512 x 0: 32,003 tokens without a constraint 300 rows 66 ->
        // 59 us, 1,500 rows 196 -> 174; under one 300 rows 36 -> 53, 500 rows 58 -> 54, 1,500 rows 140 -> 121.  Lists: 500 rows of 32,000 27.8 -> 26.7,
        // but 1,500 rows of 60,000 96 -> 105, 1024 x 0 against it.
        if (rows > (BITS ? 448 : 256) && (draws || n_groups <= 1024 * 8)) return go(integral_constant<int, 512>(), integral_constant<int, 0>());
        if (n_groups <= 1024 * 8) return go(integral_constant<int, 1024>(), integral_constant<int, 8>());
    } else {
        if (n_groups <= 512 * 16) return go(integral_constant<int, 512>(), integral_constant<int, 16>());
        if (rows >= (BITS ? 512 : 768)) return go(integral_constant<int, 512>(), integral_constant<int, 0>());
        if (n_groups <= 1024 * 16) return go(integral_constant<int, 1024>(), integral_constant<int, 16>());
    }
    return go(integral_constant<int, 1024>(), integral_constant<int, 0>());
}
template <typename F>
int shaped(bool draws, const LogitRows& a, F&& launch_of)
{
    const int32_t n_groups = a.n_tokens / (a.dtype == TDFA_F32 ? 4 : 8);
    if (a.dtype == TDFA_F32) return a.allow ? shaped<TDFA_F32, true>(draws, a.rows, n_groups, launch_of) : shaped<TDFA_F32, false>(draws, a.rows, n_groups, launch_of);
    return a.allow ? shaped<TDFA_BF16, true>(draws, a.rows, n_groups, launch_of) : shaped<TDFA_BF16, false>(draws, a.rows, n_groups, launch_of);
}

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
        return shaped(true, a, [&](auto type, auto threads, auto groups, auto bits) {
            constexpr int DTYPE = decltype(type)::value, NT = decltype(threads)::value, R = decltype(groups)::value;
            return launch(draw_step_kernel<DTYPE, NT, R, decltype(bits)::value>, dim3(rows), NT, stream, x);
        });
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
        return shaped(false, a, [&](auto type, auto threads, auto groups, auto bits) {
            constexpr int DTYPE = decltype(type)::value, NT = decltype(threads)::value, R = decltype(groups)::value;
            return launch(top_logprobs_kernel<DTYPE, NT, R, decltype(bits)::value>, dim3(rows), NT, stream, x);
        });
    });
}

}  // namespace tdfa
