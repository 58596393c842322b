// Rows into and out of a key/value cache in E0M4 codes: append (fit, encode and place), read (the values that the codes stand for)
// and eviction (selection by the attention that the rows received, then their codes moved to a smaller cache).  Layout:
// e0m4_kv4.h.  Compiled with -ffp-contract=off, as the quantiser is.
#include "e0m4_encode.h"
#include "e0m4_host.h"
#include "e0m4_kv4.h"

#include <type_traits>

namespace e0m4 {

namespace {

constexpr int kThreads = 256;
constexpr float kMost = 57344.0f;       // magnitude limit: scale stays under 65504, so that every value of a group is finite

typedef unsigned short ushort2_t __attribute__((ext_vector_type(2)));
typedef float float2_t __attribute__((ext_vector_type(2)));
typedef short short2_t __attribute__((ext_vector_type(2)));

__device__ inline float bf16_float(uint16_t b) { return __builtin_bit_cast(float, (uint32_t)b << 16); }

// Range of a group's values and 0, LANES neighbouring lanes with eight each: the largest value in the low half, the magnitude of the
// smallest in the high one, as 16-bit patterns of the rows' own type, which order like signed integers where they are positive.
// NaN counts as 0 and magnitudes are cut at kMost: patterns above its say whether there is anything to do.
__device__ inline uint32_t pack_max(uint32_t a, uint32_t b)
{
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(short2_t, a), __builtin_bit_cast(short2_t, b)));
}
template <int LANES, bool bf16>
__device__ inline void group_values(const uint4& raw, float (&x)[8], float& mn, float& mx)
{
    const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
    uint32_t up = 0, down = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        up = pack_max(up, w[j]);
        down = pack_max(down, w[j] ^ 0x80008000u);
    }
    // both halves' largest: (up, down) of either
    uint32_t range = pack_max(__builtin_amdgcn_perm(down, up, 0x05040100u), __builtin_amdgcn_perm(down, up, 0x07060302u));
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint16_t bits = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
        x[j] = bf16 ? bf16_float(bits) : (float)bits_half(bits);
    }
    const uint32_t most = bf16 ? 0x4760u : 0x7B00u;     // 57344 in either type
    if ((range & 0xFFFFu) > most || (range >> 16) > most) {
        float low = 0.f, high = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            x[j] = x[j] == x[j] ? x[j] : 0.f;
            x[j] = x[j] < -kMost ? -kMost : x[j];
            x[j] = x[j] > kMost ? kMost : x[j];
            low = fminf(low, x[j]);
            high = fmaxf(high, x[j]);
        }
        range = bf16 ? (__builtin_bit_cast(uint32_t, high) >> 16) | (__builtin_bit_cast(uint32_t, -low) & 0xFFFF0000u)
                     : (uint32_t)half_bits((half_t)high) | ((uint32_t)half_bits((half_t)-low) << 16);
        range &= 0x7FFF7FFFu;                           // (-0)
    }
    auto other = [](uint32_t v, auto ctrl) { return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, decltype(ctrl)::value, 0xF, 0xF, true); };
    range = pack_max(range, other(range, std::integral_constant<int, 0xB1>{}));             // (lanes as in group_range)
    range = pack_max(range, other(range, std::integral_constant<int, 0x4E>{}));
    if (LANES >= 8) range = pack_max(range, other(range, std::integral_constant<int, 0x141>{}));
    if (LANES == 16) range = pack_max(range, other(range, std::integral_constant<int, 0x140>{}));
    const uint16_t high = (uint16_t)range, low = (uint16_t)(range >> 16);
    mx = bf16 ? bf16_float(high) : (float)bits_half(high);
    mn = -(bf16 ? bf16_float(low) : (float)bits_half(low));
}
// The correctly rounded reciprocal of an fp16 number: from one within a unit in the last place, the remainder exact, one step (Markstein,
// as cited at Divisor; it fails for a divisor whose 24 bits are all ones only).
__device__ inline Divisor divisor_of_half(float d)
{
    const float r = __builtin_amdgcn_rcpf(d);
    return Divisor{d, __builtin_fmaf(__builtin_fmaf(-d, r, 1.0f), r, r)};
}

// encode_value of two finite values at once, in 16-bit halves: the image's bits plus half a code's step, at most the binade's last, have
// the code in fraction bits 9..6 (a step is 64 of them; the fifth fraction bit carries).
__device__ inline uint32_t encode_pair(float a, float b, const Divisor& sf, float bf)
{
    float t[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const float w = i ? b : a, q0 = w * sf.r;
        const float q = __builtin_fmaf(__builtin_fmaf(-q0, sf.d, w), sf.r, q0);
        t[i] = __builtin_amdgcn_fmed3f(q + bf, kLo, kHi);
    }
    const half2_t image = __builtin_convertvector((float2_t){t[0], t[1]}, half2_t);
    ushort2_t bits = __builtin_bit_cast(ushort2_t, image) + (ushort2_t){32, 32};
    bits = __builtin_elementwise_min(bits, (ushort2_t){0x43FF, 0x43FF});
    return __builtin_bit_cast(uint32_t, bits) & kFracMask2;
}
// A word from four pairs of codes in fraction bits 9..6 (the inverse of the packed layout's shifts).
__device__ inline uint32_t word_of_pairs(uint32_t p0, uint32_t p1, uint32_t p2, uint32_t p3)
{
    return p0 | (p1 >> 4) | (p2 << 4) | __builtin_amdgcn_alignbit(p3, p3, 24);
}

// One workgroup per tile of the cache that the new rows touch.  A row is DIM / 8 neighbouring threads with 8 values each; a group is
// G / 8 lanes, its range is found among them.  A thread's eight K codes are one word of the layout.  V codes go through LDS, 16 bits
// each, because a word of V holds eight rows; a word that also holds rows which stay is read and merged.  Two prompts of 2048 and 1536
// tokens, 40 heads: 27 us for 94 MB, which a copy moves in 18; about a hundred instructions for eight values take 12, and a workgroup
// does one after the other.  One token of a sequence 3.4 us.
template <int DIM, int G, bool BF16>
__global__ __launch_bounds__(kThreads) void kv4_append_kernel(uint8_t* __restrict__ cache, int64_t capacity, int64_t tiles, Kv4Rows keys,
                                                              Kv4Rows values, int64_t n_new, const int* __restrict__ starts,
                                                              const int* __restrict__ counts)
{
    using L = Kv4<DIM, G>;
    constexpr int kPerRow = DIM / 8, kRowsAtOnce = kThreads / kPerRow, kTimes = kKv4Rows / kRowsAtOnce;
    __shared__ __attribute__((aligned(16))) uint16_t vcode[kKv4Rows][DIM];   // (each in the fraction bits that it has in a pair)
    __shared__ __attribute__((aligned(16))) uint32_t pieces[DIM][4];
    const int b = blockIdx.z, h = blockIdx.y, t = threadIdx.x;
    const int64_t start = starts[b];
    const int64_t end = start + (counts ? clamp_count(counts[b], n_new) : n_new);
    const int64_t first = (start >= 0 ? start : start - (kKv4Rows - 1)) / kKv4Rows;        // tile of the first new row, rounded down
    const int64_t tile = first + blockIdx.x, row0 = tile * kKv4Rows;
    if (tile < 0 || tile >= tiles || row0 >= end) return;
    const int64_t lo64 = start > row0 ? start - row0 : 0, hi64 = (end < capacity ? end : capacity) - row0;
    const int lo = (int)lo64, hi = hi64 < kKv4Rows ? (int)hi64 : kKv4Rows;                  // new rows of this tile
    if (lo >= hi) return;
    uint8_t* out = cache + (((int64_t)b * gridDim.y + h) * tiles + tile) * L::kBytes;
    const int p = t % kPerRow, r0 = t / kPerRow;
    uint4 raw[2][kTimes];                               // (all rows are on their way before the first one's codes)
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
        for (int i = 0; i < kTimes; ++i) {
            const Kv4Rows& src = v ? values : keys;
            const int r = r0 + i * kRowsAtOnce;
            raw[v][i] = uint4{0, 0, 0, 0};
            if (r >= lo && r < hi)
                raw[v][i] = *reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(src.data) + b * src.batch_ld + h * src.head_ld + 8 * p +
                                                            (row0 + r - start) * src.row_ld);
        }
#pragma unroll
    for (int v = 0; v < 2; ++v)
#pragma unroll
        for (int i = 0; i < kTimes; ++i) {
            const int r = r0 + i * kRowsAtOnce;
            if (r < lo || r >= hi) continue;            // (all lanes of a row alike)
            float x[8];
            float mn, mx;
            group_values<G / 8, BF16>(raw[v][i], x, mn, mx);
            constexpr Divisor span = {kSpan, 1.0f / kSpan};                 // (what leaves quotient()'s range is below kMinScale)
            const half_t sh = (half_t)__builtin_amdgcn_fmed3f(quotient(mx - mn, span), kMinScale, kMaxScale);
            const Divisor sf = divisor_of_half((float)sh);
            const float z = __builtin_amdgcn_fmed3f(kLo - quotient(mn, sf), kLo, kHi);
            const half_t bh = bits_half(half_bits((half_t)z) & 0xFFC0u);
            const bool writes = p % (G / 8) == 0;       // one lane for the group's parameters
            const int g = 8 * p / G;
            uint32_t c[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) c[j] = encode_pair(x[2 * j], x[2 * j + 1], sf, (float)bh);
            if (v == 0) {
                *reinterpret_cast<uint32_t*>(out + L::k_word(r, 8 * p)) = word_of_pairs(c[0], c[1], c[2], c[3]);
                if (writes) *reinterpret_cast<uint32_t*>(out + L::k_param(r, g)) = (uint32_t)half_bits(sh) | ((uint32_t)half_bits(bh) << 16);
            } else {
                *reinterpret_cast<uint4*>(&vcode[r][8 * p]) = uint4{c[0], c[1], c[2], c[3]};
                if (writes) {
                    *reinterpret_cast<uint16_t*>(out + L::v_param(r, g)) = half_bits(sh);
                    *reinterpret_cast<uint16_t*>(out + L::v_param(r, g) + 64) = half_bits(bh);
                }
            }
        }
    __syncthreads();
    // V: four neighbouring dims of an octet per thread make a word each of four pieces
    if (t < DIM) {
        const int kq = t / (DIM / 4), d0 = t % (DIM / 4) * 4;
        uint32_t pair[4][4];                            // [dim][slots 2 i, 2 i + 1]
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint2 four[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int r = L::row_of(kq, 2 * i + j);
                four[j] = uint2{0, 0};
                if (r >= lo && r < hi) four[j] = *reinterpret_cast<const uint2*>(&vcode[r][d0]);
            }
            pair[0][i] = __builtin_amdgcn_perm(four[1].x, four[0].x, 0x05040100u);
            pair[1][i] = __builtin_amdgcn_perm(four[1].x, four[0].x, 0x07060302u);
            pair[2][i] = __builtin_amdgcn_perm(four[1].y, four[0].y, 0x05040100u);
            pair[3][i] = __builtin_amdgcn_perm(four[1].y, four[0].y, 0x07060302u);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i)
            pieces[d0 / 64 * 64 + kq * 16 + d0 % 16 + i][d0 % 64 / 16] = word_of_pairs(pair[i][0], pair[i][1], pair[i][2], pair[i][3]);
    }
    __syncthreads();
    if (t >= DIM) return;
    const int kq = (t >> 4) & 3;
    uint32_t stay = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int r = L::row_of(kq, j);
        if (r < lo || r >= hi) stay |= place_code(15u, j);
    }
    if (stay == ~0u) return;
    uint4* dst = reinterpret_cast<uint4*>(out + L::kVCodes) + t;
    uint4 word = *reinterpret_cast<const uint4*>(pieces[t]);
    if (stay) {
        const uint4 old = *dst;
        word = uint4{word.x | (old.x & stay), word.y | (old.y & stay), word.z | (old.z & stay), word.w | (old.w & stay)};
    }
    *dst = word;
}

// One workgroup per tile of the cache that the rows first ... first + rows - 1 touch: the codes' values go to LDS, whence rows are
// written out in whole.  Rows outside [0, min(length, capacity)) read as zeros.  Bound by memory: those two prompts in 17.5 us, 5.4 TB/s.
template <int DIM, int G>
__global__ __launch_bounds__(kThreads) void kv4_read_kernel(const uint8_t* __restrict__ cache, int64_t capacity, int64_t tiles,
                                                            const int* __restrict__ lengths, const int* __restrict__ firsts, int64_t rows,
                                                            half_t* __restrict__ keys, half_t* __restrict__ values)
{
    using L = Kv4<DIM, G>;
    constexpr int kStride = DIM + 8;                    // halves
    __shared__ __attribute__((aligned(16))) half_t kt[kKv4Rows * kStride], vt[kKv4Rows * kStride];
    const int b = blockIdx.z, h = blockIdx.y, t = threadIdx.x;
    const int64_t start = firsts ? firsts[b] : 0;
    const int64_t length = clamp_count(lengths[b], capacity);
    const int64_t first = (start >= 0 ? start : start - (kKv4Rows - 1)) / kKv4Rows;
    const int64_t tile = first + blockIdx.x, row0 = tile * kKv4Rows;
    if (row0 >= start + rows) return;
    const bool there = tile >= 0 && row0 < length;
    if (there) {
        const uint8_t* in = cache + (((int64_t)b * gridDim.y + h) * tiles + tile) * L::kBytes;
        const uint32_t hi = frac_mask_vgpr(), lo = frac_mask_low_vgpr();
        if (t < DIM) {
            const uint4 raw = reinterpret_cast<const uint4*>(in)[t];
            const uint32_t words[4] = {raw.x, raw.y, raw.z, raw.w};
            const int r = t & 15, kq = (t >> 4) & 3, piece = t >> 6;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int s = DIM == 64 ? w >> 1 : piece / (DIM >= 128 ? DIM / 128 : 1);
                const int lw = DIM == 64 ? w & 1 : piece % (DIM >= 128 ? DIM / 128 : 1) * 4 + w;
                const int row = 16 * s + r, d = kq * L::kLaneDims + 8 * lw;
                const uint32_t pw = *reinterpret_cast<const uint32_t*>(in + L::k_param(row, d / G));
                *reinterpret_cast<half8_t*>(&kt[row * kStride + d]) = kv4_values(words[w], pw, hi, lo);
            }
        }
        // two neighbouring dims of an octet per thread, so that a row gets them as one word
        if (t < DIM / 2) {
            const int n = 2 * (t & 7), kq = (t >> 3) & 3, tg = t >> 5;
            const uint4* piece = reinterpret_cast<const uint4*>(in + L::kVCodes) + tg * 64 + kq * 16 + n;
            const uint4 raw0 = piece[0], raw1 = piece[1];
            const uint32_t w0[4] = {raw0.x, raw0.y, raw0.z, raw0.w}, w1[4] = {raw1.x, raw1.y, raw1.z, raw1.w};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int d = 64 * tg + 16 * w + n;
                const words4_t* pp = reinterpret_cast<const words4_t*>(in + L::kVParams + d / G * 128 + kq * 16);
                const Kv4OctetParams o = kv4_octet_params(pp[0], pp[4]);
                const half8_t a = kv4_values_v(w0[w], o, hi, lo), c = kv4_values_v(w1[w], o, hi, lo);
#pragma unroll
                for (int j = 0; j < 8; ++j) *reinterpret_cast<half2_t*>(&vt[L::row_of(kq, j) * kStride + d]) = half2_t{a[j], c[j]};
            }
        }
    }
    __syncthreads();
    constexpr int kPerRow = DIM / 8;
    for (int i = t; i < kKv4Rows * kPerRow; i += kThreads) {
        const int r = i / kPerRow, d = i % kPerRow * 8;
        const int64_t row = row0 + r, at = row - start;
        if (at < 0 || at >= rows) continue;
        const bool in = there && row < length;
        half8_t k = {0, 0, 0, 0, 0, 0, 0, 0}, v = k;
        if (in) {
            k = *reinterpret_cast<const half8_t*>(&kt[r * kStride + d]);
            v = *reinterpret_cast<const half8_t*>(&vt[r * kStride + d]);
        }
        const int64_t dst = (((int64_t)b * rows + at) * gridDim.y + h) * DIM + d;
        *reinterpret_cast<half8_t*>(keys + dst) = k;
        *reinterpret_cast<half8_t*>(values + dst) = v;
    }
}

// Order of the received weights as an unsigned number: larger is more; -0 equals 0 and NaN counts as the most.
__device__ inline uint32_t rank_bits(float f)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, f + 0.0f);              // (-0 + 0 is 0)
    return f != f ? 0xFFFFFFFFu : u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ inline float weight_of_rank(uint32_t r) { return __builtin_bit_cast(float, r & 0x80000000u ? r ^ 0x80000000u : ~r); }

// Which rows stay.  One workgroup per (sequence, head): the need-th largest weight of the old rows by three passes of up to 2048 counters
// over its bits from the top, then one pass that counts and one that writes the rows above it, and the first ones that equal it, in
// order; a wavefront has a contiguous part of the rows in both, so that places come from ballots and sixteen sums.  A counter is
// four, one for every fourth lane: weights share their upper bits, and additions to one address follow each other.  After the
// first pass the ranks of the first kHeld rows are in LDS.  One compute unit has a head's rows (16000 of them in 18 to 22 us, 8000 in 13);
// what bounds it there are the additions in LDS, the barriers between the passes and the last one, which goes from 64 rows to the
// next.
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64, kBins = 2048, kCopies = 4, kHeld = 28672;
__global__ __launch_bounds__(kSelectThreads) void kv4_select_kernel(const float* __restrict__ received, int64_t capacity, int held_most,
                                                                    const int* __restrict__ lengths, int budget, int recent,
                                                                    int* __restrict__ kept, float* __restrict__ received_out)
{
    static_assert(kBins == 2 * kSelectThreads && kCopies == 4, "two counters of four copies per thread");
    extern __shared__ uint32_t held[];
    __shared__ __attribute__((aligned(16))) uint32_t count[kBins * kCopies];
    __shared__ uint32_t found[2];                       // prefix of the threshold, rows still needed under it
    __shared__ uint32_t above[kSelectWaves], equal[kSelectWaves];
    const int b = blockIdx.y, h = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t bh = (int64_t)b * gridDim.x + h;
    const float* w = received + bh * capacity;
    int* k = kept + bh * budget;
    float* ro = received_out + bh * budget;
    const int n = clamp_count(lengths[b], capacity);
    if (n <= budget) {
        for (int i = t; i < budget; i += kSelectThreads) {
            k[i] = i < n ? i : -1;
            ro[i] = i < n ? w[i] : 0.f;
        }
        return;
    }
    const int old = n - recent, need = budget - recent;     // need < old
    auto newest = [&]() {
        for (int i = t; i < recent; i += kSelectThreads) {
            k[need + i] = old + i;
            ro[need + i] = w[old + i];
        }
    };
    if (need == 0) {
        newest();
        return;
    }
    const int in_lds = old < held_most ? old : held_most;
    uint4* zero = reinterpret_cast<uint4*>(count) + 2 * t;
    zero[0] = zero[1] = uint4{0, 0, 0, 0};
    __syncthreads();
    constexpr int kAtOnce = 8;
    for (int i0 = t; i0 < old; i0 += kAtOnce * kSelectThreads) {
        float f[kAtOnce];
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) f[j] = i0 + j * kSelectThreads < old ? w[i0 + j * kSelectThreads] : 0.f;
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j) {
            const int i = i0 + j * kSelectThreads;
            if (i >= old) break;
            const uint32_t u = rank_bits(f[j]);
            if (i < in_lds) held[i] = u;
            atomicAdd(&count[(u >> 21) * kCopies + (lane & (kCopies - 1))], 1u);
        }
    }
    uint32_t prefix = 0, left = need;
    const int shifts[3] = {21, 10, 0}, masks[3] = {2047, 2047, 1023};
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
        __syncthreads();
        const uint4 lo = zero[0], hi = zero[1];         // counters 2 t and 2 t + 1
        const uint32_t c0 = (lo.x + lo.y) + (lo.z + lo.w), c1 = (hi.x + hi.y) + (hi.z + hi.w);
        uint32_t upto = c0 + c1;                        // rows in this lane's counters and those of the lanes above
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const uint32_t o = __shfl_down(upto, d);
            upto += lane + d < 64 ? o : 0u;
        }
        if (lane == 0) above[wave] = upto;
        zero[0] = zero[1] = uint4{0, 0, 0, 0};
        __syncthreads();
        uint32_t higher = upto - (c0 + c1);
        for (int i = wave + 1; i < kSelectWaves; ++i) higher += above[i];
        if (higher < left && left <= higher + c1) {
            found[0] = prefix | (uint32_t)(2 * t + 1) << shifts[pass];
            found[1] = left - higher;
        }
        higher += c1;
        if (higher < left && left <= higher + c0) {
            found[0] = prefix | (uint32_t)(2 * t) << shifts[pass];
            found[1] = left - higher;
        }
        __syncthreads();
        prefix = found[0];
        left = found[1];
        if (pass == 2) break;
        auto add = [&](uint32_t u) {
            if ((u ^ prefix) >> shifts[pass] == 0)
                atomicAdd(&count[((u >> shifts[pass + 1]) & masks[pass + 1]) * kCopies + (lane & (kCopies - 1))], 1u);
        };
#pragma unroll 4
        for (int i = t; i < in_lds; i += kSelectThreads) add(held[i]);
        for (int i = in_lds + t; i < old; i += kSelectThreads) add(rank_bits(w[i]));
    }
    const uint32_t threshold = prefix;                  // `left` rows that equal it stay
    const int part = ((old + kSelectWaves - 1) / kSelectWaves + 63) & ~63;
    const int begin = wave * part, end = begin + part < old ? begin + part : old;
    auto place = [&](auto rank) {
        uint32_t na = 0, ne = 0;
#pragma unroll 4
        for (int i = begin + lane; i < end; i += 64) {
            const uint32_t u = rank(i);
            na += u > threshold;
            ne += u == threshold;
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            na += __shfl_xor(na, d);
            ne += __shfl_xor(ne, d);
        }
        if (lane == 0) {
            above[wave] = na;
            equal[wave] = ne;
        }
        __syncthreads();
        uint32_t a0 = 0, e0 = 0;
        for (int i = 0; i < wave; ++i) {
            a0 += above[i];
            e0 += equal[i];
        }
        for (int i0 = begin; i0 < end; i0 += 64) {
            const int i = i0 + lane;
            const uint32_t u = i < end ? rank(i) : 0u;
            const uint64_t ma = __ballot(i < end && u > threshold), me = __ballot(i < end && u == threshold);
            uint32_t e = __builtin_amdgcn_mbcnt_hi((uint32_t)(me >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)me, e0));
            const uint32_t a = __builtin_amdgcn_mbcnt_hi((uint32_t)(ma >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)ma, a0));
            if (i < end && (u > threshold || (u == threshold && e < left))) {
                const uint32_t at = a + (e < left ? e : left);
                k[at] = i;
                ro[at] = weight_of_rank(u);
            }
            a0 += __popcll(ma);
            e0 += __popcll(me);
        }
    };
    // (a load from memory in the loop would wait for its stores: both are counted together)
    if (old <= in_lds) place([&](int i) { return held[i]; });
    else place([&](int i) { return rank_bits(w[i]); });
    newest();
}

// The rows that stay move to the smaller cache as they are, and the number of them becomes the sequence's length: here, because the
// selection's workgroups of all heads read the old one, which may stand in the same place.  One workgroup per tile of the smaller cache:
// words of K are copied, words of V put together from the eight rows' words, which takes nearly all of the old cache from memory: 46000
// rows of 40 heads to 16384 in 91 us, 265 MB read and 94 written, 3.9 TB/s.
template <int DIM, int G>
__global__ __launch_bounds__(DIM) void kv4_gather_kernel(const uint8_t* __restrict__ cache, int64_t tiles, const int* __restrict__ kept,
                                                              int budget, uint8_t* __restrict__ small, int64_t small_tiles, int64_t capacity,
                                                              const int* lengths, int* lengths_out)
{
    using L = Kv4<DIM, G>;
    __shared__ int rows[kKv4Rows];
    const int b = blockIdx.z, h = blockIdx.y, t = threadIdx.x;
    const int64_t bh = (int64_t)b * gridDim.y + h;
    if (blockIdx.x == 0 && h == 0 && t == 0) {
        const int n = clamp_count(lengths[b], capacity);
        lengths_out[b] = n < budget ? n : budget;
    }
    if (t < kKv4Rows) {
        const int64_t i = (int64_t)blockIdx.x * kKv4Rows + t;
        rows[t] = i < budget ? kept[bh * budget + i] : -1;
    }
    __syncthreads();
    if (rows[0] < 0) return;                            // rows that stay come first
    const uint8_t* in = cache + bh * tiles * L::kBytes;
    uint8_t* out = small + (bh * small_tiles + blockIdx.x) * L::kBytes;
    auto tile_of = [&](int row) { return in + (int64_t)(row / kKv4Rows) * L::kBytes; };
    const int kq = (t >> 4) & 3, block = t >> 6;        // a piece of K and one of V per thread
    {
        constexpr int kBlocks = DIM >= 128 ? DIM / 128 : 1;
        uint4 piece = {0, 0, 0, 0};
        if (DIM == 64) {
            const int r0 = rows[t & 15], r1 = rows[16 + (t & 15)];
            uint2 a = {0, 0}, c = {0, 0};
            if (r0 >= 0) a = *reinterpret_cast<const uint2*>(tile_of(r0) + L::k_word(r0 % kKv4Rows, kq * L::kLaneDims));
            if (r1 >= 0) c = *reinterpret_cast<const uint2*>(tile_of(r1) + L::k_word(r1 % kKv4Rows, kq * L::kLaneDims));
            piece = uint4{a.x, a.y, c.x, c.y};
        } else {
            const int row = rows[16 * (block / kBlocks) + (t & 15)];
            if (row >= 0) piece = *reinterpret_cast<const uint4*>(tile_of(row) + L::k_word(row % kKv4Rows, kq * L::kLaneDims + block % kBlocks * 32));
        }
        reinterpret_cast<uint4*>(out)[t] = piece;
    }
    uint4 from[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int row = rows[L::row_of(kq, j)];
        from[j] = uint4{0, 0, 0, 0};
        if (row >= 0) from[j] = reinterpret_cast<const uint4*>(tile_of(row) + L::kVCodes)[block * 64 + L::octet(row % kKv4Rows) * 16 + (t & 15)];
    }
    uint32_t word[4] = {0, 0, 0, 0};
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int slot = L::slot(rows[L::row_of(kq, j)] & (kKv4Rows - 1));
        const int shift = (0xE1 >> (slot >> 1 << 1) & 3) * 4 + 2 + (slot & 1) * 16;   // (nibble_shift: 6, 2, 10, 14 of a pair)
        const uint32_t src[4] = {from[j].x, from[j].y, from[j].z, from[j].w};
#pragma unroll
        for (int w = 0; w < 4; ++w) word[w] |= place_code(__builtin_amdgcn_alignbit(src[w], src[w], shift), j);
    }
    reinterpret_cast<uint4*>(out + L::kVCodes)[t] = uint4{word[0], word[1], word[2], word[3]};
    for (int i = t; i < kKv4Rows * L::kGroups; i += DIM) {
        const int r = i % kKv4Rows, g = i / kKv4Rows, row = rows[r];
        uint32_t kp = 0;
        uint16_t vs = 0, vb = 0;
        if (row >= 0) {
            const uint8_t* from = tile_of(row);
            kp = *reinterpret_cast<const uint32_t*>(from + L::k_param(row % kKv4Rows, g));
            vs = *reinterpret_cast<const uint16_t*>(from + L::v_param(row % kKv4Rows, g));
            vb = *reinterpret_cast<const uint16_t*>(from + L::v_param(row % kKv4Rows, g) + 64);
        }
        *reinterpret_cast<uint32_t*>(out + L::k_param(r, g)) = kp;
        *reinterpret_cast<uint16_t*>(out + L::v_param(r, g)) = vs;
        *reinterpret_cast<uint16_t*>(out + L::v_param(r, g) + 64) = vb;
    }
}

}  // namespace

int launch_kv4_append(void* cache, const e0m4_kv4_shape& s, const Kv4Rows& keys, const Kv4Rows& values, int dtype, int64_t n_new,
                      const int* starts, const int* counts, hipStream_t stream)
{
    const int64_t touched = (n_new + 2 * (kKv4Rows - 1)) / kKv4Rows, tiles = kv4_tiles(s.capacity);
    const dim3 grid((unsigned)touched, (unsigned)s.kv_heads, (unsigned)s.batch);
    return kv4_dispatch(s, [&](auto shape) -> int {
        constexpr int DIM = decltype(shape)::kDim, G = decltype(shape)::kGroup;
        auto launch = [&](auto kernel) -> int {
            hipLaunchKernelGGL(kernel, grid, dim3(kThreads), 0, stream, static_cast<uint8_t*>(cache), s.capacity, tiles, keys, values, n_new,
                               starts, counts);
            return check_launch();
        };
        return dtype == E0M4_KV4_BF16 ? launch(&kv4_append_kernel<DIM, G, true>) : launch(&kv4_append_kernel<DIM, G, false>);
    });
}

int launch_kv4_read(const void* cache, const e0m4_kv4_shape& s, const int* lengths, const int* first, int64_t rows, void* keys, void* values,
                    hipStream_t stream)
{
    const int64_t touched = (rows + (first ? 2 : 1) * (kKv4Rows - 1)) / kKv4Rows, tiles = kv4_tiles(s.capacity);
    const dim3 grid((unsigned)touched, (unsigned)s.kv_heads, (unsigned)s.batch);
    return kv4_dispatch(s, [&](auto shape) -> int {
        constexpr int DIM = decltype(shape)::kDim, G = decltype(shape)::kGroup;
        hipLaunchKernelGGL((kv4_read_kernel<DIM, G>), grid, dim3(kThreads), 0, stream, static_cast<const uint8_t*>(cache), s.capacity, tiles,
                           lengths, first, rows, static_cast<half_t*>(keys), static_cast<half_t*>(values));
        return check_launch();
    });
}

int launch_kv4_evict(const void* cache, const e0m4_kv4_shape& s, const float* received, const int* lengths, int budget, int recent,
                     void* small, const e0m4_kv4_shape& o, int* kept, int* lengths_out, float* received_out, hipStream_t stream)
{
    static std::atomic<uint64_t> allowed{0};
    int rc = allow_dynamic_lds(reinterpret_cast<const void*>(&kv4_select_kernel), kHeld * 4, allowed);
    if (rc != E0M4_OK) return rc;
    const int held = s.capacity < kHeld ? (int)s.capacity : kHeld;
    hipLaunchKernelGGL(kv4_select_kernel, dim3((unsigned)s.kv_heads, (unsigned)s.batch), dim3(kSelectThreads), held * 4, stream, received,
                       s.capacity, held, lengths, budget, recent, kept, received_out);
    rc = check_launch();
    if (rc != E0M4_OK) return rc;
    const dim3 grid((unsigned)kv4_tiles(budget), (unsigned)s.kv_heads, (unsigned)s.batch);
    return kv4_dispatch(s, [&](auto shape) -> int {
        constexpr int DIM = decltype(shape)::kDim, G = decltype(shape)::kGroup;
        hipLaunchKernelGGL((kv4_gather_kernel<DIM, G>), grid, dim3(DIM), 0, stream, static_cast<const uint8_t*>(cache),
                           kv4_tiles(s.capacity), kept, budget, static_cast<uint8_t*>(small), kv4_tiles(o.capacity), s.capacity, lengths, lengths_out);
        return check_launch();
    });
}

}  // namespace e0m4
