// Rows into and out of a key/value cache in E0M4 codes: append (fit, encode and place), read (the values that the codes stand for)
// and eviction (selection by the attention that the rows received, then their codes moved to a smaller cache).  Layout:
// e0m4_kv4.h.  Compiled with -ffp-contract=off, as the quantiser is.
#include "e0m4_encode.h"
#include "e0m4_host.h"
#include "e0m4_kv4.h"

namespace e0m4 {

namespace {

constexpr int kThreads = 256;
constexpr float kMost = 57344.0f;       // magnitude limit: scale stays under 65504, so that every value of a group is finite

__device__ inline float bf16_float(uint16_t b) { return __builtin_bit_cast(float, (uint32_t)b << 16); }

// One workgroup per tile of the cache that the new rows touch.  A row is DIM / 8 neighbouring threads with 8 values each; a group is
// G / 8 lanes, its range is found among them.  A thread's eight K codes are one word of the layout.  V codes go through LDS, a byte
// each, because a word of V holds eight rows; a word that also holds rows which stay is read and merged.
template <int DIM, int G>
__global__ __launch_bounds__(kThreads) void kv4_append_kernel(uint8_t* __restrict__ cache, int64_t capacity, int64_t tiles, Kv4Rows keys,
                                                              Kv4Rows values, int bf16, int64_t n_new, const int* __restrict__ starts,
                                                              const int* __restrict__ counts)
{
    using L = Kv4<DIM, G>;
    constexpr int kPerRow = DIM / 8, kRowsAtOnce = kThreads / kPerRow;
    __shared__ __attribute__((aligned(16))) uint8_t vcode[kKv4Rows][DIM];
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
#pragma unroll
    for (int v = 0; v < 2; ++v) {
        const Kv4Rows& src = v ? values : keys;
        const uint16_t* base = static_cast<const uint16_t*>(src.data) + b * src.batch_ld + h * src.head_ld + 8 * p;
        for (int r = r0; r < kKv4Rows; r += kRowsAtOnce) {
            if (r < lo || r >= hi) continue;            // (all lanes of a row alike)
            const uint4 raw = *reinterpret_cast<const uint4*>(base + (row0 + r - start) * src.row_ld);
            const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
            float x[8];
            float mn = 0.f, mx = 0.f;                   // the range always contains 0
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint16_t bits = (uint16_t)(w[j >> 1] >> (16 * (j & 1)));
                float f = bf16 ? bf16_float(bits) : (float)bits_half(bits);
                f = f == f ? f : 0.f;
                f = f < -kMost ? -kMost : f;
                f = f > kMost ? kMost : f;
                x[j] = f;
                mn = fminf(mn, f);
                mx = fmaxf(mx, f);
            }
            group_range<G / 8>(mn, mx);
            float s = (mx - mn) / kSpan;
            s = s < kMinScale ? kMinScale : s;
            s = s > kMaxScale ? kMaxScale : s;
            const half_t sh = (half_t)s;
            const Divisor sf = make_divisor((float)sh);
            float z = kLo - quotient(mn, sf);
            z = z < kLo ? kLo : z;
            z = z > kHi ? kHi : z;
            const half_t bh = bits_half(half_bits((half_t)z) & 0xFFC0u);
            uint32_t word = 0;
            uint64_t bytes = 0;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint32_t c = encode_value(x[j], sf, (float)bh);
                word |= place_code(c, j);
                bytes |= (uint64_t)c << (8 * j);
            }
            const bool writes = p % (G / 8) == 0;       // one lane for the group's parameters
            const int g = 8 * p / G;
            if (v == 0) {
                *reinterpret_cast<uint32_t*>(out + L::k_word(r, 8 * p)) = word;
                if (writes) *reinterpret_cast<uint32_t*>(out + L::k_param(r, g)) = (uint32_t)half_bits(sh) | ((uint32_t)half_bits(bh) << 16);
            } else {
                *reinterpret_cast<uint64_t*>(&vcode[r][8 * p]) = bytes;
                if (writes) {
                    *reinterpret_cast<uint16_t*>(out + L::v_param(r, g)) = half_bits(sh);
                    *reinterpret_cast<uint16_t*>(out + L::v_param(r, g) + 64) = half_bits(bh);
                }
            }
        }
    }
    __syncthreads();
    if (t >= DIM) return;                               // a piece of V per thread
    const int kq = (t >> 4) & 3, d0 = (t >> 6) * 64 + (t & 15);
    uint32_t stay = 0, word[4] = {0, 0, 0, 0};
    bool any = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int r = L::row_of(kq, j);
        if (r >= lo && r < hi) {
            any = true;
#pragma unroll
            for (int w = 0; w < 4; ++w) word[w] |= place_code(vcode[r][d0 + 16 * w], j);
        } else {
            stay |= place_code(15u, j);
        }
    }
    if (!any) return;
    uint4* dst = reinterpret_cast<uint4*>(out + L::kVCodes) + t;
    if (stay) {
        const uint4 old = *dst;
        word[0] |= old.x & stay;
        word[1] |= old.y & stay;
        word[2] |= old.z & stay;
        word[3] |= old.w & stay;
    }
    *dst = uint4{word[0], word[1], word[2], word[3]};
}

// One workgroup per tile of the cache that the rows first ... first + rows - 1 touch: the codes' values go to LDS, whence rows are
// written out in whole.  Rows outside [0, min(length, capacity)) read as zeros.
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
    const uint32_t u = __builtin_bit_cast(uint32_t, f + 0.0f);
    if (f != f) return 0xFFFFFFFFu;
    if (u == 0x80000000u) return 0x80000000u;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

// Which rows stay.  One workgroup per (sequence, head): the need-th largest weight of the old rows by four passes of 256 counters over
// its bytes from the top, then one pass that counts and one that writes the rows above it, and the first ones that equal it, in
// order; a wavefront has a contiguous part of the rows in both, so that places come from ballots and sixteen sums.
constexpr int kSelectThreads = 1024, kSelectWaves = kSelectThreads / 64;
__global__ __launch_bounds__(kSelectThreads) void kv4_select_kernel(const float* __restrict__ received, int64_t capacity,
                                                                    const int* __restrict__ lengths, int budget, int recent,
                                                                    int* __restrict__ kept, int* __restrict__ lengths_out,
                                                                    float* __restrict__ received_out)
{
    __shared__ uint32_t count[256];
    __shared__ uint32_t found[2];                       // prefix of the threshold, rows still needed under it
    __shared__ int above[kSelectWaves], equal[kSelectWaves];
    const int b = blockIdx.y, h = blockIdx.x, t = threadIdx.x, lane = t & 63, wave = t >> 6;
    const int64_t bh = (int64_t)b * gridDim.x + h;
    const float* w = received + bh * capacity;
    int* k = kept + bh * budget;
    float* ro = received_out + bh * budget;
    const int n = clamp_count(lengths[b], capacity);
    if (t == 0 && h == 0) lengths_out[b] = n < budget ? n : budget;
    if (n <= budget) {
        for (int i = t; i < budget; i += kSelectThreads) {
            k[i] = i < n ? i : -1;
            ro[i] = i < n ? w[i] : 0.f;
        }
        return;
    }
    const int old = n - recent, need = budget - recent;     // need < old
    for (int i = t; i < recent; i += kSelectThreads) {
        k[need + i] = old + i;
        ro[need + i] = w[old + i];
    }
    if (need == 0) return;
    uint32_t prefix = 0, left = need;
    for (int shift = 24; shift >= 0; shift -= 8) {
        for (int i = t; i < 256; i += kSelectThreads) count[i] = 0;
        __syncthreads();
        for (int i = t; i < old; i += kSelectThreads) {
            const uint32_t u = rank_bits(w[i]);
            if (shift == 24 || (u >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&count[(u >> shift) & 255u], 1u);
        }
        __syncthreads();
        if (wave == 0) {
            // lane l has the counters 4 l .. 4 l + 3; rows at or above its last one, from the top
            uint32_t c[4], sum = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) sum += c[j] = count[4 * lane + j];
            uint32_t upto = sum;
            for (int d = 1; d < 64; d <<= 1) {
                const uint32_t o = __shfl_down(upto, d);
                if (lane + d < 64) upto += o;
            }
            uint32_t higher = upto - sum;
            for (int j = 3; j >= 0; --j) {
                if (higher < left && left <= higher + c[j]) {
                    found[0] = prefix | ((uint32_t)(4 * lane + j) << shift);
                    found[1] = left - higher;
                }
                higher += c[j];
            }
        }
        __syncthreads();
        prefix = found[0];
        left = found[1];
    }
    const uint32_t threshold = prefix;                  // `left` rows that equal it stay
    const int part = ((old + kSelectWaves - 1) / kSelectWaves + 63) & ~63;
    const int begin = wave * part, end = begin + part < old ? begin + part : old;
    int na = 0, ne = 0;
    for (int i = begin + lane; i < end; i += 64) {
        const uint32_t u = rank_bits(w[i]);
        na += u > threshold;
        ne += u == threshold;
    }
    for (int d = 1; d < 64; d <<= 1) {
        na += __shfl_xor(na, d);
        ne += __shfl_xor(ne, d);
    }
    if (lane == 0) {
        above[wave] = na;
        equal[wave] = ne;
    }
    __syncthreads();
    int a0 = 0, e0 = 0;
    for (int i = 0; i < wave; ++i) {
        a0 += above[i];
        e0 += equal[i];
    }
    const uint64_t below = lane ? ~0ull >> (64 - lane) : 0ull;
    for (int i0 = begin; i0 < end; i0 += 64) {
        const int i = i0 + lane;
        const float f = i < end ? w[i] : 0.f;
        const uint32_t u = i < end ? rank_bits(f) : 0u;
        const uint64_t ma = __ballot(i < end && u > threshold), me = __ballot(i < end && u == threshold);
        const int ea = e0 + __popcll(me & below), aa = a0 + __popcll(ma & below);
        const bool is_above = (ma >> lane) & 1, is_equal = (me >> lane) & 1;
        if (is_above || (is_equal && ea < (int)left)) {
            const int at = aa + (ea < (int)left ? ea : (int)left);
            k[at] = i;
            ro[at] = f;
        }
        a0 += __popcll(ma);
        e0 += __popcll(me);
    }
}

// The rows that stay move to the smaller cache as they are.  One workgroup per tile of it: words of K are copied, words of V put
// together from the eight rows' words.
template <int DIM, int G>
__global__ __launch_bounds__(kThreads) void kv4_gather_kernel(const uint8_t* __restrict__ cache, int64_t tiles, const int* __restrict__ kept,
                                                              int budget, uint8_t* __restrict__ small, int64_t small_tiles)
{
    using L = Kv4<DIM, G>;
    __shared__ int rows[kKv4Rows];
    const int b = blockIdx.z, h = blockIdx.y, t = threadIdx.x;
    const int64_t bh = (int64_t)b * gridDim.y + h;
    if (t < kKv4Rows) {
        const int64_t i = (int64_t)blockIdx.x * kKv4Rows + t;
        rows[t] = i < budget ? kept[bh * budget + i] : -1;
    }
    __syncthreads();
    if (rows[0] < 0) return;                            // rows that stay come first
    const uint8_t* in = cache + bh * tiles * L::kBytes;
    uint8_t* out = small + (bh * small_tiles + blockIdx.x) * L::kBytes;
    auto tile_of = [&](int row) { return in + (int64_t)(row / kKv4Rows) * L::kBytes; };
    if (t < DIM) {
        {
            const int r = t & 15, kq = (t >> 4) & 3, piece = t >> 6;
            uint32_t word[4];
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int s = DIM == 64 ? w >> 1 : piece / (DIM >= 128 ? DIM / 128 : 1);
                const int lw = DIM == 64 ? w & 1 : piece % (DIM >= 128 ? DIM / 128 : 1) * 4 + w;
                const int row = rows[16 * s + r];
                word[w] = row < 0 ? 0u : *reinterpret_cast<const uint32_t*>(tile_of(row) + L::k_word(row % kKv4Rows, kq * L::kLaneDims + 8 * lw));
            }
            reinterpret_cast<uint4*>(out)[t] = uint4{word[0], word[1], word[2], word[3]};
        }
        const int kq = (t >> 4) & 3;
        uint32_t word[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = rows[L::row_of(kq, j)];
            if (row < 0) continue;
            const int rr = row % kKv4Rows, from = L::slot(rr);
            const uint4 raw = reinterpret_cast<const uint4*>(tile_of(row) + L::kVCodes)[(t & ~63) + L::octet(rr) * 16 + (t & 15)];
            const uint32_t src[4] = {raw.x, raw.y, raw.z, raw.w};
#pragma unroll
            for (int w = 0; w < 4; ++w) word[w] |= place_code(extract_code(src[w], from), j);
        }
        reinterpret_cast<uint4*>(out + L::kVCodes)[t] = uint4{word[0], word[1], word[2], word[3]};
    }
    for (int i = t; i < kKv4Rows * L::kGroups; i += kThreads) {
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
        hipLaunchKernelGGL((kv4_append_kernel<DIM, G>), grid, dim3(kThreads), 0, stream, static_cast<uint8_t*>(cache), s.capacity, tiles,
                           keys, values, dtype == E0M4_KV4_BF16, n_new, starts, counts);
        return check_launch();
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
    hipLaunchKernelGGL(kv4_select_kernel, dim3((unsigned)s.kv_heads, (unsigned)s.batch), dim3(kSelectThreads), 0, stream, received,
                       s.capacity, lengths, budget, recent, kept, lengths_out, received_out);
    const int rc = check_launch();
    if (rc != E0M4_OK) return rc;
    const dim3 grid((unsigned)kv4_tiles(budget), (unsigned)s.kv_heads, (unsigned)s.batch);
    return kv4_dispatch(s, [&](auto shape) -> int {
        constexpr int DIM = decltype(shape)::kDim, G = decltype(shape)::kGroup;
        hipLaunchKernelGGL((kv4_gather_kernel<DIM, G>), grid, dim3(kThreads), 0, stream, static_cast<const uint8_t*>(cache),
                           kv4_tiles(s.capacity), kept, budget, static_cast<uint8_t*>(small), kv4_tiles(o.capacity));
        return check_launch();
    });
}

}  // namespace e0m4
