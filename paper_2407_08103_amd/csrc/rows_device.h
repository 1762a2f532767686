// Device code that the kernels over rows of logits share: a row's elements in groups of 16 bytes, its allowed bits, and what a
// workgroup makes of them.
#pragma once

#include <tuple>

#include "tdfa_internal.h"

namespace tdfa {
namespace {

constexpr float kLog2e = 1.44269504088896341f;
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

// Element j of a group.
template <int DTYPE>
__device__ __forceinline__ float element_of(uint4 x, int32_t j)
{
    if constexpr (DTYPE == TDFA_F32) {
        return __uint_as_float(j == 0 ? x.x : j == 1 ? x.y : j == 2 ? x.z : x.w);
    } else {
        const uint32_t w = j < 2 ? x.x : j < 4 ? x.y : j < 6 ? x.z : x.w;
        return __uint_as_float(j & 1 ? w & 0xFFFF0000u : w << 16);
    }
}
__device__ __forceinline__ uint4 where(uint4 mask, uint32_t y, uint4 x)         // y under the mask, x elsewhere
{
    return make_uint4((y & mask.x) | (x.x & ~mask.x), (y & mask.y) | (x.y & ~mask.y), (y & mask.z) | (x.z & ~mask.z), (y & mask.w) | (x.w & ~mask.w));
}

template <int DTYPE>
__device__ __forceinline__ const typename Elem<DTYPE>::type* row_at(const void* rows, uint32_t i, uint32_t stride16)
{
    return reinterpret_cast<const typename Elem<DTYPE>::type*>(static_cast<const char*>(rows) + (uint64_t)i * stride16 * 16u);
}
template <int DTYPE>
__device__ __forceinline__ typename Elem<DTYPE>::type* row_at(void* rows, uint32_t i, uint32_t stride16)
{
    return reinterpret_cast<typename Elem<DTYPE>::type*>(static_cast<char*>(rows) + (uint64_t)i * stride16 * 16u);
}
__device__ __forceinline__ const uint32_t* bits_of(const uint32_t* allow, int32_t q, int32_t n_tokens)
{
    return allow + (int64_t)q * ((((int64_t)n_tokens + 31) / 32 + 3) / 4 * 4);
}

__device__ __forceinline__ bool allowed(const uint32_t* bits, int32_t t)
{
    return !bits || (bits[t >> 5] >> (t & 31) & 1);
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

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// The whole groups of a row, and their allowed bits, as buffers: a read behind the end gives 0 and a write there is dropped, both
// without reaching the memory, so that no access needs a branch and the compiler knows how many are in flight.  (A row is at most
// 2^26 bytes long.)
struct RowBuffers {
    __amdgpu_buffer_rsrc_t x, bits;
};
__device__ __forceinline__ __amdgpu_buffer_rsrc_t buffer_of(const void* base, uint32_t bytes)
{
    return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, (int)bytes, 0x00027000);
}
template <int DTYPE>
__device__ __forceinline__ RowBuffers row_buffers(const void* row, const uint32_t* bits, int32_t n_groups)
{
    return {buffer_of(row, (uint32_t)n_groups * 16u), buffer_of(bits, DTYPE == TDFA_F32 ? (uint32_t)(n_groups + 1) / 2u : (uint32_t)n_groups)};
}
constexpr uint32_t kNowhere = 0x80000000u;
constexpr int kPastCaches = 2;             // the nt bit of an access
// ONCE: what is read is not read again, and leaves the caches to what is.
template <bool ONCE>
__device__ __forceinline__ uint4 group_at(__amdgpu_buffer_rsrc_t rows, uint32_t offset)
{
    const u32x4 x = __builtin_amdgcn_raw_buffer_load_b128(rows, (int)offset, 0, ONCE ? kPastCaches : 0);
    return make_uint4(x.x, x.y, x.z, x.w);
}
// Gradients are written past the caches: 1,024 rows of 128,256 tokens in bf16 113 us, 95 so.
__device__ __forceinline__ void set_group(__amdgpu_buffer_rsrc_t rows, int32_t g, uint4 x)
{
    const u32x4 y = {x.x, x.y, x.z, x.w};
    __builtin_amdgcn_raw_buffer_store_b128(y, rows, g * 16, 0, kPastCaches);
}
// What is made of one group is finished before the next is begun: the registers of eight elements at a time, not of all.
__device__ __forceinline__ void next_group() { __builtin_amdgcn_sched_barrier(0); }

// The allowed bits of groups g0 + threadIdx.x + k NT of a row, k < U, and the groups; those without an allowed token are not fetched.
template <int DTYPE, int NT, int U, bool BITS>
__device__ __forceinline__ void fetch_bits(const RowBuffers& row, int32_t g0, uint32_t (&b)[U])
{
    const int32_t g = g0 + (int32_t)threadIdx.x;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const int32_t at = g + k * NT;
        if constexpr (BITS) b[k] = __builtin_amdgcn_raw_buffer_load_b8(row.bits, DTYPE == TDFA_F32 ? at >> 1 : at, 0, 0);
        else b[k] = 0;
    }
}
template <int DTYPE, int NT, int U, bool BITS, bool ONCE = false>
__device__ __forceinline__ void fetch_groups(const RowBuffers& row, int32_t g0, int32_t n_groups, uint4 (&x)[U], uint32_t (&b)[U])
{
    const int32_t g = g0 + (int32_t)threadIdx.x;
#pragma unroll
    for (int k = 0; k < U; ++k) {
        const int32_t at = g + k * NT;
        if constexpr (BITS && DTYPE == TDFA_F32) b[k] = at < n_groups ? b[k] >> ((at & 1) * 4) & 15u : 0u;
        x[k] = group_at<ONCE>(row.x, BITS && b[k] == 0 ? kNowhere : (uint32_t)at * 16u);
    }
}
template <int DTYPE, int NT, int U, bool BITS, bool ONCE = false>
__device__ __forceinline__ void fetch(const RowBuffers& row, int32_t g0, int32_t n_groups, uint4 (&x)[U], uint32_t (&b)[U])
{
    fetch_bits<DTYPE, NT, U, BITS>(row, g0, b);
    fetch_groups<DTYPE, NT, U, BITS, ONCE>(row, g0, n_groups, x, b);
}

// Puts -inf where a token of group g is not allowed or the row is at its end.  False: so it is in the whole wavefront.
template <int DTYPE, bool BITS>
__device__ __forceinline__ bool settle(uint4& x, uint32_t b, int32_t g, int32_t n_groups, const uint2 (&masks)[16])
{
    if constexpr (BITS) {
        if (!__ballot(b != 0)) return false;
        x = keep_allowed<DTYPE>(x, b, masks);
        asm volatile("" : "+v"(x.x), "+v"(x.y), "+v"(x.z), "+v"(x.w));      // masked once, not again in every element
    } else {
        const int32_t g0 = __builtin_amdgcn_readfirstlane(g);             // (lanes are in the order of their groups)
        if (g0 >= n_groups) return false;
        if (g0 + 63 >= n_groups && g >= n_groups) {
            constexpr uint32_t none = kNegInf<DTYPE>;
            x = make_uint4(none, none, none, none);
        }
    }
    return true;
}

// -ref c2 as it is rounded by itself: the compiler, which does not see that it is a product, makes no product and sum one around it.
__device__ __forceinline__ float offset_of(float ref, float c2)
{
    float nb = -(ref * c2);
    asm("" : "+v"(nb));
    return nb;
}

template <int DTYPE>
__device__ __forceinline__ float max_group(uint4 x, float m)
{
    float z[Elem<DTYPE>::kGroup];
    unpack<DTYPE>(x, z);
#pragma unroll
    for (int j = 0; j < Elem<DTYPE>::kGroup; ++j) m = fmaxf(m, z[j]);
    return m;
}

// 2 to the power of (from - to) c2: what a sum relative to `from` is scaled by.  The roundings of from c2 and to c2 are in the terms (not
// if SAFE), so it is the difference of these.
template <bool SAFE>
__device__ __forceinline__ float rescale(float from, float to, float c2)
{
    return __builtin_amdgcn_exp2f(SAFE ? (from - to) * c2 : offset_of(to, c2) - offset_of(from, c2));
}

// The element behind the last whole group that belongs to this thread, -inf if there is none or it is token `without`.
template <int DTYPE>
__device__ __forceinline__ float last_element(int32_t n_tokens, const typename Elem<DTYPE>::type* row, const uint32_t* bits, int32_t without)
{
    const int32_t t = n_tokens / Elem<DTYPE>::kGroup * Elem<DTYPE>::kGroup + (int32_t)threadIdx.x;
    return t < n_tokens && t != without && allowed(bits, t) ? to_f32(row[t]) : -INFINITY;
}

// Over the 64 lanes of a wavefront, all of them active, by data-parallel primitives (no LDS); the result is uniform.
template <int CTRL>
__device__ __forceinline__ float lane_swap(float v)
{
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float lane_value(float v, int lane) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), lane)); }
__device__ __forceinline__ float wave_sum(float v)
{
    v += lane_swap<0xB1>(v);           // quad_perm [1,0,3,2]
    v += lane_swap<0x4E>(v);           // quad_perm [2,3,0,1]
    v += lane_swap<0x141>(v);          // row_half_mirror
    v += lane_swap<0x140>(v);          // row_mirror
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}
__device__ __forceinline__ float wave_max(float v)
{
    v = fmaxf(v, lane_swap<0xB1>(v));
    v = fmaxf(v, lane_swap<0x4E>(v));
    v = fmaxf(v, lane_swap<0x141>(v));
    v = fmaxf(v, lane_swap<0x140>(v));
    return fmaxf(fmaxf(lane_value(v, 0), lane_value(v, 16)), fmaxf(lane_value(v, 32), lane_value(v, 48)));
}
// What the lanes up to this one hold, added up, by data-parallel primitives; lanes that a step has nothing for add 0.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t lanes_below(uint32_t v) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, ROWS, 0xF, true); }
template <int CTRL, int ROWS>
__device__ __forceinline__ double lanes_below(double v)
{
    const unsigned long long x = (unsigned long long)__double_as_longlong(v);
    return __longlong_as_double((long long)((unsigned long long)lanes_below<CTRL, ROWS>((uint32_t)(x >> 32)) << 32 | lanes_below<CTRL, ROWS>((uint32_t)x)));
}
template <typename V>
__device__ __forceinline__ V wave_upto(V v)
{
    v += lanes_below<0x111, 0xF>(v);           // row_shr 1, 2, 4, 8
    v += lanes_below<0x112, 0xF>(v);
    v += lanes_below<0x114, 0xF>(v);
    v += lanes_below<0x118, 0xF>(v);
    v += lanes_below<0x142, 0xA>(v);           // row_bcast 15 into the second and fourth row
    v += lanes_below<0x143, 0xC>(v);           // row_bcast 31 into the upper two
    return v;
}
__device__ __forceinline__ double lane_value(double v, int lane)
{
    const unsigned long long x = (unsigned long long)__double_as_longlong(v);
    return __longlong_as_double((long long)((unsigned long long)(uint32_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)x, lane)));
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

// The sum of running ones over the workgroup, relative to its largest maximum, which goes to *ref, in every thread.  One barrier: the
// wavefronts leave a maximum and a sum each, and the lanes of every wavefront join those.
template <int NT, bool SAFE>
__device__ __forceinline__ float sum_of_running(float m, float s, float c2, float* ref, float (&part)[2][NT / 64])
{
    float top = wave_max(m);
    s = wave_sum(s * rescale<SAFE>(m, top, c2));
    if constexpr (NT > 64) {
        constexpr int W = NT / 64;
        static_assert(W == 4 || W == 8 || W == 16);
        if ((threadIdx.x & 63) == 0) {
            part[0][threadIdx.x >> 6] = top;
            part[1][threadIdx.x >> 6] = s;
        }
        __syncthreads();
        const float mine = part[0][threadIdx.x & (W - 1)];
        s = part[1][threadIdx.x & (W - 1)];
        top = fmaxf(mine, lane_swap<0xB1>(mine));
        top = fmaxf(top, lane_swap<0x4E>(top));
        if constexpr (W >= 8) top = fmaxf(top, lane_swap<0x141>(top));
        if constexpr (W >= 16) top = fmaxf(top, lane_swap<0x140>(top));
        s *= rescale<SAFE>(mine, top, c2);
        s += lane_swap<0xB1>(s);
        s += lane_swap<0x4E>(s);
        if constexpr (W >= 8) s += lane_swap<0x141>(s);
        if constexpr (W >= 16) s += lane_swap<0x140>(s);
        top = lane_value(top, 0);
        s = lane_value(s, 0);
    }
    *ref = top;
    return SAFE ? s : s * __builtin_amdgcn_exp2f(-fmaf(top, c2, offset_of(top, c2)));      // the rounding of top c2 is in all terms
}

__device__ __forceinline__ float shared_by_wave(float x) { return __int_as_float(__builtin_amdgcn_readfirstlane(__float_as_int(x))); }

// A sum over the workgroup, in thread 0.  One barrier.
template <int NT>
__device__ __forceinline__ double reduce_sum(double sum, double (&part)[NT / 64])
{
#pragma unroll
    for (int d = 32; d; d >>= 1) sum += __shfl_xor(sum, d);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    if (threadIdx.x == 0)
        for (int w = 1; w < NT / 64; ++w) sum += part[w];
    return sum;
}

// loss = the sum of n losses that lie `step` apart, or their mean, by one workgroup, in an order that depends on nothing but n and NT.
template <int NT>
__device__ __forceinline__ void sum_losses(const double* each, int64_t n, int32_t step, bool mean, float* loss, double (&part)[NT / 64])
{
    double sum = 0.0;
    for (int64_t i = threadIdx.x; i < n; i += NT) sum += each[i * step];
    sum = reduce_sum<NT>(sum, part);
    if (threadIdx.x == 0) *loss = (float)(mean && n ? sum / (double)n : sum);
}
[[maybe_unused]] __global__ void __launch_bounds__(1024) loss_sum_kernel(const double* each, uint32_t n, int32_t step, int32_t mean, float* loss)
{
    __shared__ double s_part[16];
    sum_losses<1024>(each, n, step, mean, loss, s_part);
}

// A launch that reports its own error (asking for the last one afterwards costs the host 0.4 us more).
template <typename... Params, typename... Args>
int launch(void (*kernel)(Params...), dim3 grid, unsigned threads, hipStream_t stream, Args... args)
{
    std::tuple<Params...> params(args...);
    return std::apply([&](Params&... p) -> int {
        void* at[] = {&p...};
        TDFA_HIP(hipLaunchKernel(reinterpret_cast<const void*>(kernel), grid, dim3(threads), at, 0, stream));
        return TDFA_OK;
    }, params);
}

// Workgroups of a launch, of 1,024 threads at most: a grid counts less than 2^32 threads, so that more rows go by several launches.
constexpr int64_t kMaxBlocks = 1 << 21;

}  // namespace
}  // namespace tdfa
