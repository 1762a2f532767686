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
constexpr int kMarks = 16384;          // bytes, one for a group of the row: the tokens of it that are named

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

template <int NT>
struct Shared {
    uint32_t marks[kMarks / 4];
    uint32_t key[kHash];       // named tokens, kNone: free
    float value[kHash];        // gradient of the token
    float running[2][NT / 64];
    double part[NT / 64];
    double teacher[kSlots];    // of rows that name a token twice
    uint32_t named[kSlots];
    float factor;              // of the tail's gradients
    int again, active;
    uint2 masks[16];
};
constexpr uint32_t kNone = 0xFFFFFFFFu;

__device__ __forceinline__ uint32_t place_of(uint32_t id) { return id * 2654435761u >> 22; }
static_assert(kHash == 1 << 10);
// The place of token id, kNone if it is not named.
template <int NT>
__device__ __forceinline__ uint32_t find(const Shared<NT>& s, uint32_t id)
{
    for (uint32_t h = place_of(id);; h = (h + 1) & (kHash - 1)) {
        if (s.key[h] == id) return h;
        if (s.key[h] == kNone) return kNone;
    }
}
// The named tokens of group g, as bits.  Groups kMarks apart share a byte, so of a longer row its bits are looked up.
template <int DTYPE, int NT>
__device__ __forceinline__ uint32_t named_in(const Shared<NT>& s, int32_t g, int32_t n_groups)
{
    constexpr int G = Elem<DTYPE>::kGroup;
    uint32_t b = reinterpret_cast<const uint8_t*>(s.marks)[g & (kMarks - 1)];
    if (n_groups > kMarks && b)
        for (int j = 0; j < G; ++j)
            if ((b >> j & 1) && find(s, (uint32_t)(g * G + j)) == kNone) b &= ~(1u << j);
    return b;
}

// Sum over the workgroup in binary64, in every thread and in one order.  Two barriers.
template <int NT>
__device__ __forceinline__ double block_total(double v, double (&part)[NT / 64])
{
#pragma unroll
    for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
    __syncthreads();
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
    __syncthreads();
    v = part[0];
#pragma unroll
    for (int w = 1; w < NT / 64; ++w) v += part[w];
    return v;
}

// -inf in place of what is not in the tail.
template <int DTYPE, bool BITS, int NT>
__device__ __forceinline__ void keep_tail(const Shared<NT>& s, uint4& x, uint32_t b, int32_t g, int32_t n_groups)
{
    constexpr uint32_t all = (1u << Elem<DTYPE>::kGroup) - 1u;
    uint32_t on = BITS ? b : g < n_groups ? all : 0u;
    if (on) on &= ~named_in<DTYPE>(s, g, n_groups);
    if (__ballot(on != all)) x = keep_allowed<DTYPE>(x, on, s.masks);
}

// Adds U groups to a sum relative to a running maximum.  SAFE: NaN is passed over.
template <int DTYPE, int U, bool SAFE>
__device__ __forceinline__ void add_running(const uint4 (&x)[U], const Exponent& c, float& m, float& sum)
{
    float top = m;
#pragma unroll
    for (int k = 0; k < U; ++k) top = max_group<DTYPE>(x[k], top);
    sum *= c.of(m - top);
    m = top;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        float z[Elem<DTYPE>::kGroup];
        unpack<DTYPE>(x[k], z);
#pragma unroll
        for (int j = 0; j < Elem<DTYPE>::kGroup; ++j) sum += c.of((SAFE ? fmaxf(z[j], -INFINITY) : z[j]) - m);
        next_group();
    }
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

// Gradients of one group whose elements outside the tail are -inf.
template <int DTYPE, int NT>
__device__ __forceinline__ uint4 gradient_group(const Shared<NT>& s, uint4 x, int32_t g, int32_t n_groups, const Exponent& c, float factor, float m, bool careful)
{
    constexpr int G = Elem<DTYPE>::kGroup;
    float z[G];
    unpack<DTYPE>(x, z);
#pragma unroll
    for (int j = 0; j < G; ++j) {
        const float d = (careful ? fmaxf(z[j], -INFINITY) : z[j]) - m;
        z[j] = factor * (DTYPE == TDFA_F32 ? c.of(d) : __builtin_amdgcn_exp2f(d * c.hi));
    }
    const uint32_t b = g < n_groups ? named_in<DTYPE>(s, g, n_groups) : 0u;
    if (b)
#pragma unroll
        for (int j = 0; j < G; ++j)
            if (b >> j & 1) z[j] = s.value[find(s, (uint32_t)(g * G + j))];
    return pack<DTYPE>(z);
}

// One workgroup per row.  R > 0: a row of at most NT R groups stays in registers between the sum and the gradient.  R = 0: a row of any
// length, read twice.
template <int DTYPE, int NT, int R, bool BITS>
__global__ void __launch_bounds__(NT, 4) distill_row_kernel(DistillArgs a)
{
    constexpr int G = Elem<DTYPE>::kGroup, U = R ? R : 8, B = 4;             // groups to a thread at a time, and in a step of the sum
    __shared__ Shared<NT> s;
    const uint32_t i = blockIdx.x;
    const int tid = (int)threadIdx.x;
    const int32_t n_groups = a.n_tokens / G;
    const auto* row = row_at<DTYPE>(a.logits, i, a.stride16);
    // the slot of this thread
    int32_t id = -1;
    float value = 0.0f;
    if (tid < a.k) {
        id = a.ids[(uint64_t)i * a.k + tid];
        value = a.values[(uint64_t)i * a.k + tid];
    }
    const float w = a.weights ? a.weights[i] : 1.0f;
    const int32_t q = BITS ? __builtin_amdgcn_readfirstlane(a.states[i]) : 0;
    const bool read = w != 0.0f && (!BITS || (q >= 0 && q < a.n_states));
    const uint32_t* bits = BITS && read ? bits_of(a.allow, q, a.n_tokens) : a.allow;
    const Exponent c(a.temperature);
    const double inv_t = 1.0 / (double)a.temperature;
    bool live = read && id >= 0 && id < a.n_tokens && fabsf(value) < INFINITY;
    float z = -INFINITY;
    if (live) {
        live = !BITS || allowed(bits, id);
        z = to_f32(row[id]);
        live = live && z > -INFINITY;
    }
    const RowBuffers buf = row_buffers<DTYPE>(row, bits, n_groups);
    uint4 x[U];
    uint32_t b[U];
    if (R && read) fetch<DTYPE, NT, U, BITS, true>(buf, 0, n_groups, x, b);
    for (int j = tid; j < kHash; j += NT) s.key[j] = kNone;
    for (int j = tid; j < min(kMarks, n_groups + 3) / 4; j += NT) s.marks[j] = 0;
    if (tid < kSlots) s.named[tid] = kNone;
    fill_masks(s.masks);
    if (tid == 0) s.again = s.active = 0;
    __syncthreads();
    // Every named token has a place; the slot that takes it first owns it.
    uint32_t place = kNone;
    bool owner = false;
    if (live) {
        s.active = 1;
        s.named[tid] = (uint32_t)id;
        for (place = place_of((uint32_t)id);; place = (place + 1) & (kHash - 1)) {
            const uint32_t was = atomicCAS(&s.key[place], kNone, (uint32_t)id);
            owner = was == kNone;
            if (owner || was == (uint32_t)id) break;
        }
        if (!owner) s.again = 1;
        if (id / G < n_groups) atomicOr(&s.marks[(id / G & (kMarks - 1)) >> 2], 1u << ((id / G & 3) * 8 + id % G));
    }
    __syncthreads();
    const int32_t behind = n_groups * G + tid;
    auto* out = row_at<DTYPE>(a.grad, i, a.grad_stride16);
    const __amdgpu_buffer_rsrc_t to = buffer_of(out, (uint32_t)n_groups * 16u);
    if (!s.active) {
        if (tid == 0) {
            a.losses[i] = 0.0f;
            a.work[i] = 0.0;
        }
        if (!a.grad) return;
        for (int32_t g = tid; g < n_groups; g += NT) set_group(to, g, make_uint4(0, 0, 0, 0));
        if (behind < a.n_tokens) store_rounded(out + behind, 0.0f);
        return;
    }
    // The tail: its largest logit m, and its sum relative to that.
    const uint32_t place_behind = behind < a.n_tokens ? find(s, (uint32_t)behind) : kNone;
    const float last = last_element<DTYPE>(a.n_tokens, row, bits, place_behind != kNone ? behind : -1);
    float m, sum;
    const auto add_row = [&](auto safe) {
        constexpr bool SAFE = decltype(safe)::value;
        m = fmaxf(last, kLowest);
        sum = c.of((SAFE ? fmaxf(last, -INFINITY) : last) - m);
        for (int32_t g0 = 0; g0 < (R ? 1 : n_groups); g0 += NT * U) {
            if (!R) fetch<DTYPE, NT, U, BITS>(buf, g0, n_groups, x, b);
#pragma unroll
            for (int k = 0; k < U; k += B) {
                uint4 y[B];
#pragma unroll
                for (int j = 0; j < B; ++j) {
                    if (!R || !SAFE) keep_tail<DTYPE, BITS>(s, x[k + j], b[k + j], g0 + tid + (k + j) * NT, n_groups);
                    y[j] = x[k + j];
                }
                add_running<DTYPE, B, SAFE>(y, c, m, sum);
            }
        }
        sum = join_running<NT>(m, sum, c, s.running);
    };
    add_row(std::false_type());
    const bool careful = !(sum < INFINITY);
    if (careful) add_row(std::true_type());
    const bool tail = sum != 0.0f;                         // (NaN where an allowed logit is +inf, as everything below)
    // The row's numbers, in binary64: the whole sum relative to the largest logit, the teacher's probabilities, the loss.
    const float most = block_reduce<NT, true>(fmaxf(live ? z : -INFINITY, tail ? m : -INFINITY), s.running[0]);
    const double down = ((double)m - (double)most) * inv_t, mine = live ? exp(((double)z - (double)most) * inv_t) : 0.0;
    const double total = (tail ? exp(down) * (double)sum : 0.0) + block_total<NT>(owner ? mine : 0.0, s.part);
    const double ln_total = log(total), lp = ((double)z - (double)most) * inv_t - ln_total;
    const bool counts = live && (float)lp != -INFINITY;
    double teacher, mass, rest = 0.0;
    if (a.tail) {
        teacher = counts ? exp(fmin((double)value, 0.0)) : 0.0;
        mass = block_total<NT>(teacher, s.part);
        if (tail) rest = fmax(1.0 - mass, 0.0);
        mass += rest;
    } else {
        const float best = block_reduce<NT, true>(counts ? value : -INFINITY, s.running[0]);
        teacher = counts ? exp((double)value - (double)best) : 0.0;
        mass = block_total<NT>(teacher, s.part);
        teacher = mass > 0.0 ? teacher / mass : 0.0;
        mass = mass > 0.0 ? 1.0 : 0.0;
    }
    double loss = block_total<NT>(teacher > 0.0 ? teacher * (log(teacher) - lp) : 0.0, s.part);
    if (rest > 0.0) loss += rest * (log(rest) - (down + log((double)sum) - ln_total));
    const double scale = (double)w * inv_t;
    if (tid == 0) {
        a.losses[i] = (float)loss;
        a.work[i] = (double)w * loss;
        s.factor = tail ? (float)(scale * (mass * exp(down) / total - rest / (double)sum)) : 0.0f;
    }
    if (!a.grad) return;
    if (s.again) {                                         // the slots of one token added up, in their order
        if (tid < kSlots) s.teacher[tid] = teacher;
        __syncthreads();
        if (owner) {
            teacher = 0.0;
            for (int j = 0; j < a.k; ++j)
                if (s.named[j] == (uint32_t)id) teacher += s.teacher[j];
        }
    }
    if (owner) s.value[place] = (float)(scale * (mine / total * mass - teacher));
    __syncthreads();
    const float factor = shared_by_wave(s.factor);
    for (int32_t g0 = 0; g0 < (R ? 1 : n_groups); g0 += NT * U) {
        if (!R) fetch<DTYPE, NT, U, BITS>(buf, g0, n_groups, x, b);
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int32_t g = g0 + tid + k * NT;
            if (!R) keep_tail<DTYPE, BITS>(s, x[k], b[k], g, n_groups);
            set_group(to, g, gradient_group<DTYPE>(s, x[k], g, n_groups, c, factor, m, careful));
            next_group();
        }
    }
    if (behind < a.n_tokens)
        store_rounded(out + behind, place_behind != kNone ? s.value[place_behind] : factor * c.of((careful ? fmaxf(last, -INFINITY) : last) - m));
}

template <int DTYPE, bool BITS>
int rows_of(const DistillArgs& x, unsigned rows, hipStream_t stream)
{
    const int32_t n_groups = x.n_tokens / Elem<DTYPE>::kGroup;
    if (n_groups <= 256 * 4) return launch(distill_row_kernel<DTYPE, 256, 4, BITS>, dim3(rows), 256, stream, x);
    if (n_groups <= 256 * 16) return launch(distill_row_kernel<DTYPE, 256, 16, BITS>, dim3(rows), 256, stream, x);
    if (n_groups <= 512 * 16) return launch(distill_row_kernel<DTYPE, 512, 16, BITS>, dim3(rows), 512, stream, x);
    if (n_groups <= 1024 * 16) return launch(distill_row_kernel<DTYPE, 1024, 16, BITS>, dim3(rows), 1024, stream, x);
    return launch(distill_row_kernel<DTYPE, 1024, 0, BITS>, dim3(rows), 1024, stream, x);
}

}  // namespace

int64_t distill_workspace(int64_t rows) { return 8 * rows; }

int launch_distill_loss(const LogitRows& a, const DistillRows& d, float* loss, void* grad, int64_t grad_stride, void* workspace, hipStream_t stream)
{
    const int64_t esz = a.dtype == TDFA_F32 ? 4 : 2;
    double* work = static_cast<double*>(workspace);
    for (int64_t from = 0; from < a.rows; from += kMaxBlocks) {
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
        const unsigned rows = (unsigned)std::min<int64_t>(kMaxBlocks, a.rows - from);
        const int rc = a.dtype == TDFA_F32 ? (a.allow ? rows_of<TDFA_F32, true>(x, rows, stream) : rows_of<TDFA_F32, false>(x, rows, stream))
                                           : (a.allow ? rows_of<TDFA_BF16, true>(x, rows, stream) : rows_of<TDFA_BF16, false>(x, rows, stream));
        if (rc != TDFA_OK) return rc;
    }
    return launch(loss_sum_kernel, dim3(1), 1024, stream, static_cast<const double*>(work), (uint32_t)a.rows, 1, 0, loss);
}

}  // namespace tdfa
