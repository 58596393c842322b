// Device parts that the attention kernels over a cache in E0M4 codes share.
//
// Softmax: p = 2^(t - ref + kShift) with t the score in powers of two.  Any reference gives the same quotient as long as nothing
// overflows, so it is only moved (and the sums rescaled) when a score exceeds it by more than kSlack: a lane compares its own
// scores, lanes only meet when one of them does.  P is rounded to fp16 for the product, at most 2^15 and with kShift + 24 = 32 powers
// of two below the reference.
#pragma once

#include "e0m4_kv4.h"

namespace e0m4 {

constexpr float kShift = 8.f, kSlack = 7.f;
constexpr float kLog2E = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();

// Kinds of instructions, for their order in a block; operands of products are read from LDS kAhead products before their own.
constexpr int kMfma = 0x8, kValu = 0x2, kTrans = 0x400, kDsRead = 0x100;
constexpr int kAhead = 4;

__device__ inline float bf16_low(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ inline float bf16_high(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }
__device__ inline uint32_t bf16_round(float f)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, f);
    if (f != f) return 0x7FC0u;
    return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

// What a row's weights take from its reference and sum (of 2^(t - ref + kShift)).
__device__ inline float2 row_norm(bool valid, float ref, float sum)
{
    return !valid || sum == 0.f ? float2{0.f, 0.f} : float2{ref, 256.f / sum};
}
static_assert(kShift == 8.f, "2^kShift over the sum");

// Four dims of a row's result from its sums; zeros for a row that sees nothing.
template <int DIM>
__device__ inline void finish(const Kv4Attention& a, int b, int h, int row, int d, bool valid, floatx4 acc, float ref, float sum)
{
    const float f = !valid || sum == 0.f ? 0.f : 1.f / sum;
    const int i = kv4_query_of(a, row), head = h * a.share + row - i * a.share;
    uint16_t* p = static_cast<uint16_t*>(a.out) + (((int64_t)b * a.n_new + i) * (a.kv_heads * a.share) + head) * DIM + d;
    uint32_t x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float y = f == 0.f ? 0.f : acc[j] * f;
        x[j] = a.bf16 ? bf16_round(y) : (uint32_t)__builtin_bit_cast(uint16_t, (half_t)y);
    }
    *reinterpret_cast<uint2*>(p) = uint2{x[0] | (x[1] << 16), x[2] | (x[3] << 16)};
    if (a.norm && d == 0) a.norm[((int64_t)b * a.kv_heads + h) * ((int64_t)a.n_new * a.share) + row] = row_norm(valid, ref, sum);
}

__device__ inline words4_t load16(__amdgpu_buffer_rsrc_t tile, int offset)
{
    return __builtin_bit_cast(words4_t, __builtin_amdgcn_raw_buffer_load_b128(tile, offset, 0, 0));
}

// The values of the cache are fp16, so queries are too; bfloat16 ones are scaled by the power of two that brings their row's largest into
// [1, 2), which the score's factor takes back: what is lost of them then is below 2^-25 of the largest.  A row is with the lanes
// ACROSS, 2 ACROSS, ... < LANES on, N pieces of 8 in each.
template <int N, int LANES, int ACROSS>
__device__ inline int bf16_row_exponent(const words4_t* raw)
{
    uint32_t top = 0;                   // largest magnitude, as bits
#pragma unroll
    for (int w = 0; w < N; ++w)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t l = raw[w][j] & 0x7FFFu, u = (raw[w][j] >> 16) & 0x7FFFu;
            top = l > top ? l : top;
            top = u > top ? u : top;
        }
#pragma unroll
    for (int d = ACROSS; d < LANES; d <<= 1) {
        const uint32_t o = __shfl_xor(top, d);
        top = o > top ? o : top;
    }
    const int e = (int)(top >> 7) - 127;
    return e == 128 || top == 0 ? 0 : e;                // (infinite, not a number, or all zeros)
}
__device__ inline half8_t bf16_scaled(words4_t raw, int e)
{
    half8_t q;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        q[2 * j] = (half_t)__builtin_ldexpf(bf16_low(raw[j]), -e);
        q[2 * j + 1] = (half_t)__builtin_ldexpf(bf16_high(raw[j]), -e);
    }
    return q;
}

// A row of queries as a lane has it, N pieces of 8 dims `step` dims apart from `first` on, in fp16; the row's other dims are with the lanes
// ACROSS (, 2 ACROSS) on.  Returns the factor of its scores, to powers of two.
template <int DIM, int N, int ACROSS>
__device__ inline float load_query_row(const Kv4Attention& a, int b, int h, int row, bool there, int first, int step, half8_t (&q)[N])
{
    float factor = kLog2E / __builtin_sqrtf((float)DIM);
    const int i = kv4_query_of(a, row), head = h * a.share + row - i * a.share;
    const uint16_t* p = static_cast<const uint16_t*>(a.q.data) + b * a.q.batch_ld + i * a.q.row_ld + head * a.q.head_ld + first;
    words4_t raw[N];
#pragma unroll
    for (int w = 0; w < N; ++w) raw[w] = there ? *reinterpret_cast<const words4_t*>(p + step * w) : words4_t{0, 0, 0, 0};
    if (!a.bf16) {
#pragma unroll
        for (int w = 0; w < N; ++w) q[w] = __builtin_bit_cast(half8_t, raw[w]);
        return factor;
    }
    const int e = bf16_row_exponent<N, 64, ACROSS>(raw);
#pragma unroll
    for (int w = 0; w < N; ++w) q[w] = bf16_scaled(raw[w], e);
    return __builtin_ldexpf(factor, e);
}

// The same row for the pass over the received weights; zeros where there is no query.
template <int N>
__device__ inline void keep_query_row(const Kv4Attention& a, int64_t row, int dim, bool there, int first, int step, const half8_t (&q)[N], float factor)
{
#pragma unroll
    for (int w = 0; w < N; ++w)
        *reinterpret_cast<half8_t*>(a.packed_q + row * dim + first + step * w) = there ? q[w] : half8_t{0, 0, 0, 0, 0, 0, 0, 0};
    if (first < 8) a.factors[row] = there ? factor : 0.f;
}

// Rows of the cache that a query at position `at` sees, by position: [from, to).
struct Kv4Seen {
    int from, to;
};
__device__ inline Kv4Seen kv4_seen(const Kv4Attention& a, int length, int at)
{
    return Kv4Seen{a.window && at - a.window + 1 > 0 ? at - a.window + 1 : 0, a.causal && at + 1 < length ? at + 1 : length};
}
__device__ inline const uint8_t* kv4_mask_row(const Kv4Attention& a, int b, int query)
{
    return a.mask ? a.mask + b * a.mask_batch_ld + query * a.mask_row_ld : nullptr;
}
// Truth values of a mask's row for GROUPS runs of 4 rows of the cache, the g-th one from first_row(g) on: bit 4 g + i.
template <int GROUPS, typename F>
__device__ inline uint32_t kv4_mask_bits(const Kv4Attention& a, int b, int query, F&& first_row)
{
    const uint8_t* mask = kv4_mask_row(a, b, query);
    uint32_t bits = 0;
    if (a.mask_words) {                                 // runs are aligned words, none of them across the mask's end
        uint32_t w[GROUPS];
#pragma unroll
        for (int g = 0; g < GROUPS; ++g) w[g] = *reinterpret_cast<const uint32_t*>(mask + (first_row(g) < a.mask_rows ? first_row(g) : 0));
#pragma unroll
        for (int g = 0; g < GROUPS; ++g)
#pragma unroll
            for (int i = 0; i < 4; ++i) bits |= first_row(g) < a.mask_rows && (w[g] >> (8 * i) & 0xFFu) ? 1u << (4 * g + i) : 0u;
    } else {
#pragma unroll 1
        for (int g = 0; g < GROUPS; ++g) {
            uint8_t m[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) m[i] = mask[first_row(g) + i < a.mask_rows ? first_row(g) + i : 0];
#pragma unroll
            for (int i = 0; i < 4; ++i) bits |= first_row(g) + i < a.mask_rows && m[i] ? 1u << (4 * g + i) : 0u;
        }
    }
    return bits;
}

}  // namespace e0m4
