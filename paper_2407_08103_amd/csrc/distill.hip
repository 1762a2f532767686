// Distillation from a teacher's most likely tokens, under a constraint or none, with the gradient of the student's logits, for gfx950.
//
// A row has the student's logits z, an allowed set A, p = softmax of z c over A (c = 1 / temperature), and slots with a token and the
// teacher's value for it.  The slots that are live give the teacher's probabilities q; with a tail, what is missing from 1 is the probability r of all
// tokens of A that no live slot names, the tail, which the student gives p_tail.  The row's loss is the divergence
//     l = sum over slots of q (ln q - ln p) + r (ln r - ln p_tail)
// and with M = sum of q + r its gradient is
//     c (p_t M - the q of t's slots)  at the named tokens,      c (p_t M - r p_t / p_tail)  in the tail.
// The tail's terms are all exp((z_t - m) c) times one factor of the row, with m the largest logit of the tail: a sum over the tail
// relative to m is all that the first look at a row has to find out, however small the tail's part of it is.
#include "rows_device.h"

#include <algorithm>
#include <cmath>
#include <type_traits>

namespace tdfa {
namespace {

constexpr int kSlots = TDFA_TOP_MAX;
constexpr int kHash = 1024;            // places for the named tokens of a row
constexpr int kMarks = 16384;          // most groups that a workgroup takes: a byte for each says which of its tokens are named

struct DistillArgs {
    const uint32_t* allow;     // or NULL: every token is allowed
    const void* logits;
    const int32_t* states;
    const float* weights;      // or NULL
    const int32_t* ids;
    const float* values;
    float* losses;
    double* work;
    void* grad;                // or NULL
    uint32_t stride16, grad_stride16;
    int32_t n_states, n_tokens;
    int32_t k, tail;
    float temperature;
};
static_assert(sizeof(DistillArgs) <= 112, "the arguments of a launch that costs the host little");

// exp(x c) as 2 to the power of x hi + x lo: the two parts of log2(e) c, so that a sum of terms far below the largest keeps its bits.
// Both parts are above 0: an x of -inf gives 0, not the difference of two infinities.
struct Exponent {
    float hi, lo;
    __device__ __forceinline__ explicit Exponent(float temperature)
    {
        const double c2 = 1.44269504088896340736 / (double)temperature;
        hi = (float)c2;
        if ((double)hi >= c2) hi = __uint_as_float(__float_as_uint(hi) - 1u);
        lo = fmaxf((float)(c2 - (double)hi), 1.0e-45f);
    }
    __device__ __forceinline__ float of(float x) const { return __builtin_amdgcn_exp2f(fmaf(x, hi, x * lo)); }
};

constexpr uint32_t kNone = 0xFFFFFFFFu;

// The named tokens of a workgroup's part of a row.
struct Names {
    uint32_t marks[kMarks / 4];
    uint32_t key[kHash];       // tokens, kNone: free
    float value[kHash];        // gradient of the token
};
// What a workgroup shares that works out a row's numbers.
template <int NT>
struct Shared : Names {
    float running[2][NT / 64];
    // the slots: tokens (kNone: not live), places (the lowest bit: whether the slot owns it), the student's and the teacher's values
    uint32_t named[kSlots], place[kSlots];
    float logit[kSlots], given[kSlots];
    double far[kSlots], teacher[kSlots];       // exponentials relative to the largest of them, the teacher's probabilities
    struct { double part, mass, dot, low; } early;      // the sums of both, of q (ln q - ln of the exponential), and the lowest ln of one
    float top[kSlots / 64];    // the largest live logits
    double factor;
    int again, active;
    uint2 masks[16];
};

__device__ __forceinline__ uint32_t place_of(uint32_t id) { return id * 2654435761u >> 22; }
static_assert(kHash == 1 << 10);
// The place of token id, kNone if it is not named.
__device__ __forceinline__ uint32_t find(const Names& s, uint32_t id)
{
    for (uint32_t h = place_of(id);; h = (h + 1) & (kHash - 1)) {
        if (s.key[h] == id) return h;
        if (s.key[h] == kNone) return kNone;
    }
}
// Its place, made if it is new (*first).  kHash is four times the slots of a row: there is room.
__device__ __forceinline__ uint32_t enter(Names& s, uint32_t id, bool* first)
{
    for (uint32_t h = place_of(id);; h = (h + 1) & (kHash - 1)) {
        const uint32_t was = atomicCAS(&s.key[h], kNone, id);
        *first = was == kNone;
        if (*first || was == id) return h;
    }
}
// The marks are for `count` groups from g0 on; a token behind the row's whole groups has none.
template <int DTYPE>
__device__ __forceinline__ void mark(Names& s, int32_t id, int32_t g0, int32_t count)
{
    constexpr int G = Elem<DTYPE>::kGroup;
    const uint32_t g = (uint32_t)(id / G - g0);
    if (g < (uint32_t)count) atomicOr(&s.marks[g >> 2], 1u << ((g & 3) * 8 + id % G));
}
__device__ __forceinline__ uint32_t named_in(const Names& s, int32_t g) { return reinterpret_cast<const uint8_t*>(s.marks)[g]; }

template <int NT>
__device__ __forceinline__ void clear_names(Names& s, int32_t count)
{
    for (int j = threadIdx.x; j < kHash; j += NT) s.key[j] = kNone;
    for (int j = threadIdx.x; j < (count + 3) / 4; j += NT) s.marks[j] = 0;
}

// A value that is the same in all lanes, in scalar registers: next to a row's elements there are few others.
__device__ __forceinline__ double uniform(double v)
{
    const unsigned long long x = (unsigned long long)__double_as_longlong(v);
    return __longlong_as_double((long long)((unsigned long long)(uint32_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)x)));
}

// A group as it is loaded: its elements are taken out of it where they are used, not kept from one use to the next.
__device__ __forceinline__ void held(uint4& x) { asm volatile("" : "+v"(x.x), "+v"(x.y), "+v"(x.z), "+v"(x.w)); }

// -inf in place of what is not in the tail; `named` bits of a group of which b are allowed and that lies in the row.  False: there is
// nothing of the tail in the groups of the wavefront.
template <int DTYPE, bool BITS>
__device__ __forceinline__ bool keep_tail(uint4& x, uint32_t b, bool inside, uint32_t named, const uint2 (&masks)[16])
{
    constexpr uint32_t all = (1u << Elem<DTYPE>::kGroup) - 1u;
    const uint32_t on = (BITS ? b : inside ? all : 0u) & ~named;
    if (!__ballot(on != 0)) return false;
    if (__ballot(on != all)) x = keep_allowed<DTYPE>(x, on, masks);
    held(x);
    return true;
}

// Adds groups k0 .. k0 + B - 1, as far as the bits of `some` say, to a sum relative to a running maximum.  SAFE: NaN is passed over.
template <int DTYPE, int U, int B, bool SAFE>
__device__ __forceinline__ void add_running(uint4 (&x)[U], int k0, uint32_t some, const Exponent& c, float& m, float& sum)
{
    float top = m;
#pragma unroll
    for (int k = k0; k < k0 + B; ++k) {
        if (!(some >> k & 1)) continue;
        top = max_group<DTYPE>(x[k], top);
        next_group();
    }
    sum *= c.of(m - top);
    m = top;
#pragma unroll
    for (int k = k0; k < k0 + B; ++k) {
        if (!(some >> k & 1)) continue;
        float z[Elem<DTYPE>::kGroup];
        held(x[k]);
        unpack<DTYPE>(x[k], z);
#pragma unroll
        for (int j = 0; j < Elem<DTYPE>::kGroup; ++j) sum += c.of((SAFE ? fmaxf(z[j], -INFINITY) : z[j]) - m);
        next_group();
    }
}
// The same relative to a logit that is known before, by one rounded product and sum for an exponent: nb = -ref hi, rounded.
template <int DTYPE, int U>
__device__ __forceinline__ void add_relative(uint4 (&x)[U], int k, float hi, float nb, float (&sum)[2])
{
    float z[Elem<DTYPE>::kGroup];
    held(x[k]);
    unpack<DTYPE>(x[k], z);
#pragma unroll
    for (int j = 0; j < Elem<DTYPE>::kGroup; ++j) sum[j & 1] += __builtin_amdgcn_exp2f(fmaf(z[j], hi, nb));
    next_group();
}

// Running sums of all threads joined, relative to the largest maximum, in every thread.  Two barriers.
template <int NT>
__device__ __forceinline__ float join_running(float& m, float sum, const Exponent& c, float (&part)[2][NT / 64])
{
    const float top = wave_max(m);
    sum = wave_sum(sum * c.of(m - top));
    __syncthreads();
    if ((threadIdx.x & 63) == 0) {
        part[0][threadIdx.x >> 6] = top;
        part[1][threadIdx.x >> 6] = sum;
    }
    __syncthreads();
    m = part[0][0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) m = fmaxf(m, part[0][w]);
    sum = 0.0f;
#pragma unroll
    for (int w = 0; w < NT / 64; ++w) sum += part[1][w] * c.of(part[0][w] - m);
    return sum;
}

// What a row's gradients are made of: those of the tail are factor exp((z - ref) c).
struct Slope {
    float factor, log;         // log2 of |factor|, which may be beyond binary32
    float ref;
    bool careful;              // there is a NaN among the tail's logits, or something beyond the reach of binary32
};
// 16 bits: |factor| is in the exponent.  The largest of the tail may lie far above ref, and a factor that binary32 does not hold be that of gradients
// that it does.  Without the difference from ref as well it saves a product and a difference for each element and is off by 2^-14 or so of itself, beside a
// rounding by up to 2^-8.
struct Fold {
    float at;                  // NaN: not to be taken
    uint32_t sign;
};
__device__ __forceinline__ Fold fold_of(const Slope& q, const Exponent& c)
{
    const float nb = -(q.ref * c.hi);
    const bool folds = !q.careful && fabsf(nb) < 1024.0f;
    return {shared_by_wave(folds ? nb + q.log : __uint_as_float(0x7FC00000u)), __float_as_uint(q.factor) >> 31 ? 0x80008000u : 0u};
}
template <int DTYPE>
__device__ __forceinline__ float gradient_of(float z, const Slope& q, const Exponent& c)
{
    const float x = (q.careful ? fmaxf(z, -INFINITY) : z) - q.ref;
    if constexpr (DTYPE == TDFA_BF16) return copysignf(__builtin_amdgcn_exp2f(fmaf(x, c.hi, fmaf(x, c.lo, q.log))), q.factor);
    return q.factor * c.of(x);
}
// y in place of element j of a group.
template <int DTYPE>
__device__ __forceinline__ uint4 with_element(uint4 x, int32_t j, float y)
{
    const uint32_t v = DTYPE == TDFA_F32 ? __float_as_uint(y) : rounded_pair(y, y), m = DTYPE == TDFA_F32 ? 0xFFFFFFFFu : j & 1 ? 0xFFFF0000u : 0xFFFFu;
    const int32_t word = DTYPE == TDFA_F32 ? j : j >> 1;
    return where(make_uint4(word == 0 ? m : 0, word == 1 ? m : 0, word == 2 ? m : 0, word == 3 ? m : 0), v, x);
}
// Gradients of a group whose elements outside the tail are -inf.  some: there is any of the tail in the wavefront's groups.
template <int DTYPE>
__device__ __forceinline__ uint4 gradient_group(const Names& s, uint4 x, bool some, uint32_t named, int32_t g, const Slope& q, const Fold& f, const Exponent& c)
{
    constexpr int G = Elem<DTYPE>::kGroup;
    float z[G];
    if (!some) {
        x = make_uint4(0, 0, 0, 0);
    } else if (DTYPE == TDFA_BF16 && f.at == f.at) {
        held(x);
        unpack<DTYPE>(x, z);
#pragma unroll
        for (int j = 0; j < G; ++j) z[j] = __builtin_amdgcn_exp2f(fmaf(z[j], c.hi, f.at));
        x = pack<DTYPE>(z);
        x = make_uint4(x.x ^ f.sign, x.y ^ f.sign, x.z ^ f.sign, x.w ^ f.sign);
    } else {
        held(x);
        unpack<DTYPE>(x, z);
#pragma unroll
        for (int j = 0; j < G; ++j) z[j] = gradient_of<DTYPE>(z[j], q, c);
        x = pack<DTYPE>(z);
    }
    for (; named; named &= named - 1) {
        const int32_t j = __builtin_ctz(named);
        x = with_element<DTYPE>(x, j, s.value[find(s, (uint32_t)(g * G + j))]);
    }
    return x;
}

// What a workgroup knows of its row before it reads it, and the slot of this thread.
struct Head {
    int32_t id;
    float value, z;
    uint32_t word;             // the allowed bits with the token's
    bool named;                // the slot names a token and gives a value
    float weight;
    const uint32_t* bits;
    bool read;                 // the row's logits have to be read
};
template <int DTYPE, bool BITS>
__device__ __forceinline__ Head head_of(const DistillArgs& a, uint32_t i)
{
    Head h = {-1, 0.0f, -INFINITY, 0xFFFFFFFFu, false, 1.0f, a.allow, true};
    if ((int)threadIdx.x < a.k) {
        h.id = a.ids[(uint64_t)i * a.k + threadIdx.x];
        h.value = a.values[(uint64_t)i * a.k + threadIdx.x];
    }
    if (a.weights) h.weight = shared_by_wave(a.weights[i]);
    h.read = h.weight != 0.0f;
    if constexpr (BITS) {
        const int32_t q = __builtin_amdgcn_readfirstlane(a.states[i]);
        h.read = h.read && q >= 0 && q < a.n_states;
        if (h.read) h.bits = bits_of(a.allow, q, a.n_tokens);
    }
    h.named = h.read && h.id >= 0 && h.id < a.n_tokens && fabsf(h.value) < INFINITY;
    if (h.named) {                                         // (looked at in enter_slots, when the row is on its way too)
        if (BITS) h.word = h.bits[h.id >> 5];
        h.z = to_f32(row_at<DTYPE>(a.logits, i, a.stride16)[h.id]);
    }
    return h;
}
// Enters the slots; the marks are for the row's first `count` groups.  False: no slot is live.  Two barriers.
template <int DTYPE, int NT>
__device__ __forceinline__ bool enter_slots(Shared<NT>& s, const Head& h, int32_t count)
{
    clear_names<NT>(s, count);
    fill_masks(s.masks);
    if (threadIdx.x == 0) s.again = s.active = 0;
    __syncthreads();
    const bool live = h.named && (h.word >> (h.id & 31) & 1) && h.z > -INFINITY;
    if (threadIdx.x < kSlots) {
        const float top = wave_max(live ? h.z : -INFINITY);
        if ((threadIdx.x & 63) == 0) s.top[threadIdx.x >> 6] = top;
        s.named[threadIdx.x] = live ? (uint32_t)h.id : kNone;
    }
    if (live) {
        s.active = 1;
        bool owner;
        const uint32_t place = enter(s, (uint32_t)h.id, &owner);
        if (!owner) s.again = 1;
        mark<DTYPE>(s, h.id, 0, count);
        s.place[threadIdx.x] = place << 1 | (owner ? 1u : 0u);
        s.logit[threadIdx.x] = h.z;
        s.given[threadIdx.x] = h.value;
    }
    __syncthreads();
    return s.active;
}
// The largest logit of a live slot.
template <int NT>
__device__ __forceinline__ float top_slot(const Shared<NT>& s)
{
    float top = s.top[0];
#pragma unroll
    for (int w = 1; w < kSlots / 64; ++w) top = fmaxf(top, s.top[w]);
    return shared_by_wave(top);
}

// The sum over a wavefront, in binary64 and in one order.
__device__ __forceinline__ double wave_total(double v) { return lane_value(wave_upto(v), 63); }

// A row's numbers, in binary64: the loss, and what the gradients are made of, s.factor, and the value of every owner's place.  By the first
// wavefront, four slots to a lane: by a thread for each slot, with sums over the workgroup, it took 4 us of every row.
//
// What the slots give before the tail's sum is known, while the row is on its way: s.far the student's exponentials relative to the largest live
// logit, s.teacher the teacher's probabilities, as if every live slot counted.  (All of it behind the sum: 4,096 rows 362 -> 351 us, 1,024 rows with 128 slots
// 122 -> 115, 1,500 fp32 rows of 32,003 88 -> 79.)
template <int NT, typename F>
__device__ __forceinline__ void each_slot(const DistillArgs& a, const Shared<NT>& s, F&& f)       // f(slot) for the live slots of a lane (what it keeps of them lies in LDS)
{
    for (int j = (int)threadIdx.x; j < a.k; j += 64)
        if (s.named[j] != kNone) f(j);
}
template <int NT>
__device__ __forceinline__ void slot_numbers(const DistillArgs& a, Shared<NT>& s)
{
    if (threadIdx.x >= 64) return;
    if (s.again) {
        // Which of a token's slots came first is chance: the first of them owns it, so that sums over owners have one order.
        each_slot(a, s, [&](int j) {
            uint32_t owner = 1;
            for (int o = 0; o < j; ++o)
                if (s.named[o] == s.named[j]) owner = 0;
            s.place[j] = (s.place[j] & ~1u) | owner;
        });
    }
    const double inv_t = uniform(1.0 / (double)a.temperature), top = (double)top_slot(s);
    float best = -INFINITY;
    if (!a.tail) each_slot(a, s, [&](int j) { best = fmaxf(best, s.given[j]); });
    best = wave_max(best);
    double part = 0.0, mass = 0.0, dot = 0.0, low = 0.0;
    each_slot(a, s, [&](int j) {
        const double far = ((double)s.logit[j] - top) * inv_t, e = exp(far);
        const double ln_q = a.tail ? fmin((double)s.given[j], 0.0) : (double)s.given[j] - (double)best, q = exp(ln_q);
        s.far[j] = e;
        s.teacher[j] = q;
        if (s.place[j] & 1) part += e;
        mass += q;
        dot += q * (ln_q - far);
        low = fmin(low, far);
    });
    part = wave_total(part);
    mass = uniform(wave_total(mass));
    dot = wave_total(dot);
    low = -(double)wave_max(-(float)low);
    if (!a.tail) {
        const double share = uniform(1.0 / mass);          // (the best slot's is 1)
        each_slot(a, s, [&](int j) { s.teacher[j] *= share; });
        dot = dot * share - log(mass);
        mass = 1.0;
    }
    if (threadIdx.x == 0) s.early = {part, mass, dot, low};
    wave_lds_sync();
}
// All of it, with the tail's sum relative to ref.  A barrier behind it.
template <int NT>
__device__ __forceinline__ void row_numbers(const DistillArgs& a, uint32_t i, float weight, float ref, double sum, Shared<NT>& s)
{
    if (threadIdx.x < 64) {
        const double inv_t = uniform(1.0 / (double)a.temperature);
        sum = uniform(sum);
        const bool tail = sum != 0.0;                      // (NaN where an allowed logit is +inf, as everything below)
        const float top = top_slot(s), most = shared_by_wave(fmaxf(top, tail ? ref : -INFINITY));
        const double down = uniform(((double)ref - (double)most) * inv_t), slots_down = uniform(((double)top - (double)most) * inv_t);
        const double near = uniform(exp(slots_down)), total = uniform((tail ? exp(down) * sum : 0.0) + near * s.early.part), ln_total = uniform(log(total));
        double mass = uniform(s.early.mass), loss = s.early.dot + mass * (ln_total - slots_down);
        if ((float)(s.early.low + slots_down - ln_total) == -INFINITY) {
            // Some slot's log-probability may be beyond binary32: the teacher's probabilities without such slots.
            const auto ln_p = [&](int j) { return ((double)s.logit[j] - (double)most) * inv_t - ln_total; };
            const auto counts = [&](int j) { return (float)ln_p(j) != -INFINITY; };
            double part = 0.0;
            if (a.tail) {
                each_slot(a, s, [&](int j) { part += s.teacher[j] = counts(j) ? exp(fmin((double)s.given[j], 0.0)) : 0.0; });
                mass = uniform(wave_total(part));
            } else {
                float best = -INFINITY;
                each_slot(a, s, [&](int j) {
                    if (counts(j)) best = fmaxf(best, s.given[j]);
                });
                best = wave_max(best);
                each_slot(a, s, [&](int j) { part += s.teacher[j] = counts(j) ? exp((double)s.given[j] - (double)best) : 0.0; });
                mass = uniform(wave_total(part));
                const double share = mass > 0.0 ? 1.0 / mass : 0.0;
                each_slot(a, s, [&](int j) { s.teacher[j] *= share; });
                mass = mass > 0.0 ? 1.0 : 0.0;
            }
            part = 0.0;
            each_slot(a, s, [&](int j) {
                if (s.teacher[j] > 0.0) part += s.teacher[j] * (log(s.teacher[j]) - ln_p(j));
            });
            loss = wave_total(part);
        }
        double rest = 0.0;
        if (a.tail && tail) rest = uniform(fmax(1.0 - mass, 0.0));
        mass = uniform(mass + rest);
        if (rest > 0.0) loss += rest * (log(rest) - (down + log(sum) - ln_total));
        const double scale = uniform((double)weight * inv_t), each = uniform(mass * near / total);
        if (threadIdx.x == 0) {
            a.losses[i] = (float)loss;
            a.work[i] = (double)weight * loss;
            s.factor = tail ? scale * (mass * exp(down) / total - rest / sum) : 0.0;
        }
        wave_lds_sync();
        const bool again = s.again;
        each_slot(a, s, [&](int j) {
            if (!(s.place[j] & 1)) return;
            double teacher = s.teacher[j];
            if (again) {                                   // the slots of one token added up, in their order
                teacher = 0.0;
                for (int o = 0; o < a.k; ++o)
                    if (s.named[o] == s.named[j]) teacher += s.teacher[o];
            }
            s.value[s.place[j] >> 1] = (float)(scale * (s.far[j] * each - teacher));
        });
    }
    __syncthreads();
}
__device__ __forceinline__ void no_loss(const DistillArgs& a, uint32_t i)
{
    if (threadIdx.x == 0) {
        a.losses[i] = 0.0f;
        a.work[i] = 0.0;
    }
}

// One workgroup per row, of at most NT R groups, which stay in registers between the sum and the gradient.  16 bits: the sum is relative to the
// largest logit that is named, so that terms are added as they arrive; where that does not do, and in fp32, whose gradients would show what
// exponents lose far from the largest logit, relative to a running maximum.
// What bounds it: the memory where there are many rows, 4,096 rows of 128,256 tokens in bf16 350 us for 1.05 GB written and 0.4 GB
// of groups with an allowed token read (4.1 TB/s; a large copy runs at 4.7), 1,024 rows without a constraint 116 us (4.5); few rows, the chain of slots, row, sums, numbers (by one wavefront, in binary64) and
// gradients: 24 rows of 32,000 10 us, and 2 for the sum of their losses.  (A workgroup per row that reads it twice: 1,222, 323 and 28 us a call.)
template <int DTYPE, int NT, int R, bool BITS>
__global__ void __launch_bounds__(NT, 4) distill_row_kernel(DistillArgs a)
{
    constexpr int G = Elem<DTYPE>::kGroup, B = 4;          // B groups to a step of the running maximum
    static_assert(NT * R <= kMarks);
    __shared__ Shared<NT> s;
    const uint32_t i = blockIdx.x;
    const int tid = (int)threadIdx.x;
    const int32_t n_groups = a.n_tokens / G;
    const auto* row = row_at<DTYPE>(a.logits, i, a.stride16);
    auto* out = row_at<DTYPE>(a.grad, i, a.grad_stride16);
    const __amdgpu_buffer_rsrc_t to = buffer_of(out, (uint32_t)n_groups * 16u);
    const int32_t behind = n_groups * G + tid;
    const Head h = head_of<DTYPE, BITS>(a, i);
    uint4 x[R];
    uint32_t b[(R + 3) / 4];                               // allowed bits, of four groups each
    if (h.read) {
        const RowBuffers buf = row_buffers<DTYPE>(row, h.bits, n_groups);
        uint32_t y[R];
        fetch_bits<DTYPE, NT, R, BITS>(buf, 0, y);
        fetch_groups<DTYPE, NT, R, BITS, true>(buf, 0, n_groups, x, y);
#pragma unroll
        for (int k = 0; k < R; ++k) b[k / 4] = k % 4 ? b[k / 4] | y[k] << (k % 4 * 8) : y[k];
    }
    if (!h.read || !enter_slots<DTYPE, NT>(s, h, n_groups)) {
        no_loss(a, i);
        if (!a.grad) return;
        for (int32_t g = tid; g < n_groups; g += NT) set_group(to, g, make_uint4(0, 0, 0, 0));
        if (behind < a.n_tokens) store_rounded(out + behind, 0.0f);
        return;
    }
    slot_numbers(a, s);
    const Exponent c(a.temperature);
    const auto place_behind = [&]() { return behind < a.n_tokens ? find(s, (uint32_t)behind) : kNone; };
    const float last = last_element<DTYPE>(a.n_tokens, row, h.bits, place_behind() != kNone ? behind : -1);
    // The tail's sum, and the groups that have something of it (bits of `some`, for the wavefront) or a named token (bits of `names`).
    uint32_t some = 0, names = 0;
    float ref = -INFINITY, sum = NAN;
    double whole;
    const auto settle_group = [&](int k) {
        const int32_t g = tid + k * NT;
        const uint32_t named = g < n_groups ? named_in(s, g) : 0u;
        names |= (named ? 1u : 0u) << k;
        const bool any = keep_tail<DTYPE, BITS>(x[k], b[k / 4] >> (k % 4 * 8) & 0xFFu, g < n_groups, named, s.masks);
        some |= (any ? 1u : 0u) << k;
        return any;
    };
    if constexpr (DTYPE == TDFA_BF16) {
        ref = top_slot(s);
        const float nb = offset_of(ref, c.hi);
        float sums[2] = {__builtin_amdgcn_exp2f(fmaf(last, c.hi, nb)), 0.0f};
#pragma unroll
        for (int k = 0; k < R; ++k)
            if (settle_group(k)) add_relative<DTYPE>(x, k, c.hi, nb, sums);
        sum = block_reduce<NT, false>(sums[0] + sums[1], s.running[1]);
        // the rounding of ref hi is in all terms
        whole = (double)sum * (double)__builtin_amdgcn_exp2f(-fmaf(ref, c.hi, nb));
    }
    bool careful = false;
    if (DTYPE == TDFA_F32 || !(sum > 1.0e-30f && sum < 1.0e30f)) {
        const auto add_row = [&](auto safe) {
            constexpr bool SAFE = decltype(safe)::value;
            ref = fmaxf(last, kLowest);
            sum = c.of((SAFE ? fmaxf(last, -INFINITY) : last) - ref);
#pragma unroll
            for (int k = 0; k < R; k += B) {
                if (DTYPE == TDFA_F32 && !SAFE)
#pragma unroll
                    for (int j = 0; j < B; ++j) settle_group(k + j);
                add_running<DTYPE, R, B, SAFE>(x, k, some, c, ref, sum);
            }
            sum = join_running<NT>(ref, sum, c, s.running);
        };
        if (DTYPE == TDFA_F32) add_row(std::false_type());
        careful = DTYPE == TDFA_BF16 || !(sum < INFINITY);
        if (careful) add_row(std::true_type());
        whole = (double)sum;
    }
    row_numbers<NT>(a, i, h.weight, ref, whole, s);
    if (!a.grad) return;
    some = __builtin_amdgcn_readfirstlane(some);
    const double factor = s.factor;
    const Slope q = {shared_by_wave((float)factor), shared_by_wave(__builtin_amdgcn_logf((float)fabs(__builtin_amdgcn_frexp_mant(factor))) + (float)__builtin_amdgcn_frexp_exp(factor)),
                     shared_by_wave(ref), careful};
    const Fold f = fold_of(q, c);
#pragma unroll
    for (int k = 0; k < R; ++k) {
        const int32_t g = tid + k * NT;
        set_group(to, g, gradient_group<DTYPE>(s, x[k], some >> k & 1, names >> k & 1 ? named_in(s, g) : 0u, g, q, f, c));
        next_group();
    }
    if (behind < a.n_tokens) {
        // (read again, not kept in a register in between)
        const uint32_t place = place_behind();
        store_rounded(out + behind, place != kNone ? s.value[place] : gradient_of<DTYPE>(last_element<DTYPE>(a.n_tokens, row, h.bits, -1), q, c));
    }
}

// ---- rows that do not stay in registers: sums by parts, the numbers of the rows, gradients by parts ----------

struct PartArgs : DistillArgs {
    float2* parts;             // [rows][n_parts]: the largest logit of the tail in the part, and the sum relative to it, with its sign set if it was taken with care
    int32_t n_parts, span;     // groups to a part
};
struct NumbersArgs : DistillArgs {
    const float2* parts;
    uint2* named;              // [rows][k]: token and gradient of every slot (kNone: none)
    float4* slopes;            // [rows]: factor, ref, careful, whether the row takes part
    int32_t n_parts;
};
struct PartGradArgs {
    const uint32_t* allow;
    const void* logits;
    const int32_t* states;
    void* grad;
    const uint2* named;
    const float4* slopes;
    uint32_t stride16, grad_stride16;
    int32_t n_tokens, k, n_parts;
    float temperature;
};
static_assert(sizeof(PartGradArgs) <= 112);

// The sum of a part of a row's tail, and its last part's elements behind the whole groups.  Bound by the memory's lines that hold an allowed token, and
// in fp32 by the exponentials: 300 rows of 256,000 tokens 37 us.
template <int DTYPE, int NT, int U, bool BITS>
__global__ void __launch_bounds__(NT) distill_part_kernel(PartArgs a)
{
    constexpr int G = Elem<DTYPE>::kGroup, B = 4;
    __shared__ uint32_t s_marks[kMarks / 4];
    __shared__ uint2 s_masks[16];
    __shared__ float s_running[2][NT / 64];
    __shared__ uint32_t s_behind;
    const uint32_t i = blockIdx.x / (uint32_t)a.n_parts;
    const int32_t part = (int32_t)(blockIdx.x - i * (uint32_t)a.n_parts), n_groups = a.n_tokens / G, g0 = part * a.span, count = min(a.span, n_groups - g0);
    const int tid = (int)threadIdx.x;
    const auto* row = row_at<DTYPE>(a.logits, i, a.stride16);
    const bool ends = part == a.n_parts - 1;
    if (a.weights && a.weights[i] == 0.0f) return;
    const uint32_t* bits = a.allow;
    if constexpr (BITS) {
        const int32_t q = __builtin_amdgcn_readfirstlane(a.states[i]);
        if (q < 0 || q >= a.n_states) return;
        bits = bits_of(a.allow, q, a.n_tokens);
    }
    for (int j = tid; j < (count + 3) / 4; j += NT) s_marks[j] = 0;
    fill_masks(s_masks);
    if (tid == 0) s_behind = 0;
    __syncthreads();
    for (int j = tid; j < a.k; j += NT) {
        const int32_t id = a.ids[(uint64_t)i * a.k + j];
        // (of a token that is not allowed, or -inf, a mark changes nothing)
        if (id < 0 || id >= a.n_tokens || !(fabsf(a.values[(uint64_t)i * a.k + j]) < INFINITY)) continue;
        const int32_t g = id / G - g0;
        if (g >= 0 && g < count) atomicOr(&s_marks[g >> 2], 1u << ((g & 3) * 8 + id % G));
        else if (id >= n_groups * G) atomicOr(&s_behind, 1u << (id % G));
    }
    __syncthreads();
    const Exponent c(a.temperature);
    const RowBuffers buf = row_buffers<DTYPE>(row, bits, n_groups);
    const float last = ends && !(s_behind >> (tid & 31) & 1) ? last_element<DTYPE>(a.n_tokens, row, bits, -1) : -INFINITY;
    float m, sum;
    const auto add_part = [&](auto safe) {
        constexpr bool SAFE = decltype(safe)::value;
        m = fmaxf(last, kLowest);
        sum = c.of((SAFE ? fmaxf(last, -INFINITY) : last) - m);
        uint4 x[U];
        uint32_t b[U];
        for (int32_t at = 0; at < count; at += NT * U) {
            fetch<DTYPE, NT, U, BITS>(buf, g0 + at, g0 + count, x, b);
            uint32_t some = 0;
#pragma unroll
            for (int k = 0; k < U; k += B) {
#pragma unroll
                for (int j = k; j < k + B; ++j) {
                    const int32_t g = at + tid + j * NT;
                    const bool inside = g < count;
                    some |= (keep_tail<DTYPE, BITS>(x[j], inside ? b[j] : 0u, inside, inside ? reinterpret_cast<const uint8_t*>(s_marks)[g] : 0u, s_masks) ? 1u : 0u) << j;
                }
                add_running<DTYPE, U, B, SAFE>(x, k, some, c, m, sum);
            }
        }
        sum = join_running<NT>(m, sum, c, s_running);
    };
    add_part(std::false_type());
    const bool careful = !(sum < INFINITY);
    if (careful) add_part(std::true_type());
    if (tid == 0) a.parts[blockIdx.x] = make_float2(m, __uint_as_float(__float_as_uint(sum) | (careful ? 0x80000000u : 0u)));
}

// One workgroup per row: its numbers from its slots and the sums of its parts.
template <int DTYPE, bool BITS>
__global__ void __launch_bounds__(256) distill_numbers_kernel(NumbersArgs a)
{
    __shared__ Shared<256> s;
    const uint32_t i = blockIdx.x;
    const Head h = head_of<DTYPE, BITS>(a, i);
    const bool active = enter_slots<DTYPE, 256>(s, h, 0);
    float ref = kLowest;
    bool careful = false;
    double sum = 0.0;
    if (active) {
        const double inv_t = 1.0 / (double)a.temperature;
        for (int32_t p = 0; p < a.n_parts; ++p)
            if (a.parts[(uint64_t)i * a.n_parts + p].y != 0.0f) ref = fmaxf(ref, a.parts[(uint64_t)i * a.n_parts + p].x);
        for (int32_t p = 0; p < a.n_parts; ++p) {
            const float2 v = a.parts[(uint64_t)i * a.n_parts + p];
            careful = careful || __float_as_uint(v.y) >> 31;               // (also of a sum of 0, where the part has nothing but NaN)
            if (v.y != 0.0f) sum += fabs((double)v.y) * (v.x == ref ? 1.0 : exp(((double)v.x - (double)ref) * inv_t));
        }
        slot_numbers(a, s);
        row_numbers<256>(a, i, h.weight, ref, sum, s);
    } else {
        no_loss(a, i);
    }
    if ((int)threadIdx.x < a.k) {
        const uint32_t id = s.named[threadIdx.x];
        a.named[(uint64_t)i * a.k + threadIdx.x] = make_uint2(id, id != kNone ? __float_as_uint(s.value[s.place[threadIdx.x] >> 1]) : 0u);
    }
    if (threadIdx.x == 0) a.slopes[i] = make_float4(active ? (float)s.factor : 0.0f, ref, careful ? 1.0f : 0.0f, active ? 1.0f : 0.0f);
}

// Gradients of NT U groups of a row, the last part with the elements behind the whole groups.  Bound by the memory: the same rows 58 us, 307 MB
// written past the caches and the lines of the logits read again (numbers of the rows 8, sum of the losses 5).
template <int DTYPE, int NT, int U, bool BITS>
__global__ void __launch_bounds__(NT) distill_grad_kernel(PartGradArgs a)
{
    constexpr int G = Elem<DTYPE>::kGroup;
    __shared__ Names s;
    __shared__ uint2 s_masks[16];
    const uint32_t i = blockIdx.x / (uint32_t)a.n_parts;
    const int32_t part = (int32_t)(blockIdx.x - i * (uint32_t)a.n_parts), n_groups = a.n_tokens / G, g0 = part * NT * U, count = min(NT * U, n_groups - g0);
    const int tid = (int)threadIdx.x;
    const auto* row = row_at<DTYPE>(a.logits, i, a.stride16);
    auto* out = row_at<DTYPE>(a.grad, i, a.grad_stride16);
    const __amdgpu_buffer_rsrc_t to = buffer_of(out, (uint32_t)n_groups * 16u);
    const int32_t behind = part == a.n_parts - 1 ? n_groups * G + tid : a.n_tokens;
    const float4 v = a.slopes[i];
    if (shared_by_wave(v.w) == 0.0f) {
#pragma unroll
        for (int k = 0; k < U; ++k) set_group(to, g0 + tid + k * NT, make_uint4(0, 0, 0, 0));
        if (behind < a.n_tokens) store_rounded(out + behind, 0.0f);
        return;
    }
    const uint32_t* bits = BITS ? bits_of(a.allow, __builtin_amdgcn_readfirstlane(a.states[i]), a.n_tokens) : nullptr;
    uint2 mine = make_uint2(kNone, 0u);
    if (tid < a.k) mine = a.named[(uint64_t)i * a.k + tid];
    uint4 x[U];
    uint32_t b[U];
    fetch<DTYPE, NT, U, BITS, true>(row_buffers<DTYPE>(row, bits, n_groups), g0, n_groups, x, b);
    clear_names<NT>(s, count);
    fill_masks(s_masks);
    __syncthreads();
    static_assert(NT >= kSlots);
    if (mine.x != kNone && (int32_t)mine.x >= g0 * G && ((int32_t)mine.x < (g0 + count) * G || part == a.n_parts - 1)) {
        bool first;
        s.value[enter(s, mine.x, &first)] = __uint_as_float(mine.y);       // (slots of one token have the same)
        mark<DTYPE>(s, (int32_t)mine.x, g0, count);
    }
    __syncthreads();
    const Exponent c(a.temperature);
    const Slope q = {shared_by_wave(v.x), shared_by_wave(__builtin_amdgcn_logf(fabsf(v.x))), shared_by_wave(v.y), __builtin_amdgcn_readfirstlane(v.z != 0.0f) != 0};
    const Fold f = fold_of(q, c);
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const int32_t at = tid + k * NT, g = g0 + at;
        const uint32_t named = at < count ? named_in(s, at) : 0u;
        const bool some = keep_tail<DTYPE, BITS>(x[k], b[k], at < count, named, s_masks);
        set_group(to, g, gradient_group<DTYPE>(s, x[k], some, named, g, q, f, c));
        next_group();
    }
    if (behind < a.n_tokens) {
        const uint32_t place = find(s, (uint32_t)behind);
        const float last = last_element<DTYPE>(a.n_tokens, row, bits, -1);
        store_rounded(out + behind, place != kNone ? s.value[place] : gradient_of<DTYPE>(last, q, c));
    }
}

// Groups of the longest rows that stay in registers; with more of them the compiler would keep some in memory, in fp32 sooner.
constexpr int32_t held_groups(int dtype) { return dtype == TDFA_F32 ? 1024 * 8 : 1024 * 16; }

template <int DTYPE, bool BITS>
int rows_of(const DistillArgs& x, unsigned rows, hipStream_t stream)
{
    const int32_t n_groups = x.n_tokens / Elem<DTYPE>::kGroup;
    if (n_groups <= 256 * 4) return launch(distill_row_kernel<DTYPE, 256, 4, BITS>, dim3(rows), 256, stream, x);
    if (n_groups <= 512 * 8) return launch(distill_row_kernel<DTYPE, 512, 8, BITS>, dim3(rows), 512, stream, x);
    if constexpr (DTYPE == TDFA_F32) {
        return launch(distill_row_kernel<DTYPE, 1024, 8, BITS>, dim3(rows), 1024, stream, x);
    } else {
        if (n_groups <= 512 * 16) return launch(distill_row_kernel<DTYPE, 512, 16, BITS>, dim3(rows), 512, stream, x);
        return launch(distill_row_kernel<DTYPE, 1024, 16, BITS>, dim3(rows), 1024, stream, x);
    }
}

constexpr int kPartThreads = 256, kPartGroups = 8;        // groups in flight per thread of the launches over parts
constexpr int32_t kPiece = kPartThreads * kPartGroups;

int32_t groups_of(int dtype, int64_t n_tokens) { return (int32_t)(n_tokens / (dtype == TDFA_F32 ? 4 : 8)); }
// Few rows leave most compute units idle otherwise.
bool by_parts(int dtype, int64_t rows, int32_t n_groups) { return n_groups > held_groups(dtype) || (rows <= 40 && n_groups > 4096); }
// Groups to a part of the sums: about 1,024 workgroups, of whole pieces, none of more than kMarks groups.
int32_t span_of(int64_t rows, int32_t n_groups)
{
    const int64_t pieces = (n_groups + kPiece - 1) / kPiece, parts = std::max<int64_t>(1, std::min<int64_t>(pieces, 1024 / std::max<int64_t>(rows, 1)));
    return (int32_t)std::min<int64_t>(kMarks, (pieces + parts - 1) / parts * kPiece);
}
int64_t aligned(int64_t bytes) { return (bytes + 15) / 16 * 16; }

template <int DTYPE, bool BITS>
int parts_of(const DistillArgs& x, int64_t rows, int32_t span, float2* parts, uint2* named, float4* slopes, hipStream_t stream)
{
    const int32_t n_groups = x.n_tokens / Elem<DTYPE>::kGroup, n_parts = (n_groups + span - 1) / span;
    PartArgs p;
    static_cast<DistillArgs&>(p) = x;
    p.parts = parts;
    p.n_parts = n_parts;
    p.span = span;
    int rc = launch(distill_part_kernel<DTYPE, kPartThreads, kPartGroups, BITS>, dim3((unsigned)(rows * n_parts)), kPartThreads, stream, p);
    if (rc != TDFA_OK) return rc;
    NumbersArgs n;
    static_cast<DistillArgs&>(n) = x;
    n.parts = parts;
    n.named = named;
    n.slopes = slopes;
    n.n_parts = n_parts;
    rc = launch(distill_numbers_kernel<DTYPE, BITS>, dim3((unsigned)rows), 256, stream, n);
    if (rc != TDFA_OK || !x.grad) return rc;
    const int32_t grad_parts = (n_groups + kPiece - 1) / kPiece;
    const PartGradArgs g = {x.allow, x.logits, x.states, x.grad, named, slopes, x.stride16, x.grad_stride16, x.n_tokens, x.k, grad_parts, x.temperature};
    return launch(distill_grad_kernel<DTYPE, kPartThreads, kPartGroups, BITS>, dim3((unsigned)(rows * grad_parts)), kPartThreads, stream, g);
}

}  // namespace

// The rows' losses; where rows are taken by parts, of either type, the slots' and parts' numbers as well.
int64_t distill_workspace(int64_t rows, int64_t n_tokens, int64_t k)
{
    int64_t parts = 0;
    for (int dtype : {TDFA_F32, TDFA_BF16}) {
        const int32_t n = groups_of(dtype, n_tokens), span = span_of(rows, n);
        if (by_parts(dtype, rows, n)) parts = std::max<int64_t>(parts, (n + span - 1) / span);
    }
    return aligned(8 * rows) + (parts ? 16 * rows + aligned(8 * rows * k) + aligned(8 * rows * parts) : 0);
}

int launch_distill_loss(const LogitRows& a, const DistillRows& d, float* loss, void* grad, int64_t grad_stride, void* workspace, hipStream_t stream)
{
    const int64_t esz = a.dtype == TDFA_F32 ? 4 : 2;
    const int32_t n_groups = groups_of(a.dtype, a.n_tokens), span = span_of(a.rows, n_groups);
    const bool parted = by_parts(a.dtype, a.rows, n_groups);
    double* work = static_cast<double*>(workspace);
    float4* slopes = reinterpret_cast<float4*>(static_cast<char*>(workspace) + aligned(8 * a.rows));
    uint2* named = reinterpret_cast<uint2*>(slopes + a.rows);
    float2* parts = reinterpret_cast<float2*>(reinterpret_cast<char*>(named) + aligned(8 * a.rows * d.k));
    const int64_t n_parts = parted ? std::max((n_groups + span - 1) / span, (n_groups + kPiece - 1) / kPiece) : 1, step = std::max<int64_t>(1, kMaxBlocks / n_parts);
    for (int64_t from = 0; from < a.rows; from += step) {
        DistillArgs x;
        x.allow = a.allow;
        x.logits = static_cast<const char*>(a.logits) + from * a.row_stride * esz;
        x.states = a.states ? a.states + from : nullptr;
        x.weights = d.weights ? d.weights + from : nullptr;
        x.ids = d.ids + from * d.k;
        x.values = d.values + from * d.k;
        x.losses = d.losses + from;
        x.work = work + from;
        x.grad = grad ? static_cast<char*>(grad) + from * grad_stride * esz : nullptr;
        x.stride16 = (uint32_t)(a.rows > 1 ? a.row_stride * esz / 16 : 0);
        x.grad_stride16 = (uint32_t)(a.rows > 1 ? grad_stride * esz / 16 : 0);
        x.n_states = (int32_t)std::min<int64_t>(a.n_states, INT32_MAX);
        x.n_tokens = a.n_tokens;
        x.k = d.k;
        x.tail = d.tail;
        x.temperature = a.temperature;
        const int64_t rows = std::min<int64_t>(step, a.rows - from);
        const auto go = [&](auto dtype, auto bits) {
            constexpr int DTYPE = decltype(dtype)::value;
            constexpr bool BITS = decltype(bits)::value;
            return parted ? parts_of<DTYPE, BITS>(x, rows, span, parts, named, slopes, stream) : rows_of<DTYPE, BITS>(x, (unsigned)rows, stream);
        };
        using F32 = std::integral_constant<int, TDFA_F32>;
        using BF16 = std::integral_constant<int, TDFA_BF16>;
        const int rc = a.dtype == TDFA_F32 ? (a.allow ? go(F32(), std::true_type()) : go(F32(), std::false_type()))
                                           : (a.allow ? go(BF16(), std::true_type()) : go(BF16(), std::false_type()));
        if (rc != TDFA_OK) return rc;
    }
    return launch(loss_sum_kernel, dim3(1), 1024, stream, static_cast<const double*>(work), (uint32_t)a.rows, 1, 0, loss);
}

}  // namespace tdfa
