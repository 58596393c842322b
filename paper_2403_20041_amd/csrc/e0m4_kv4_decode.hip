// Attention of few queries over a cache in E0M4 codes, and the sums of attention that its rows received.  Layout and what it gives
// the products: e0m4_kv4.h.
//
// A wavefront takes whole tiles of 32 rows by itself, 16 rows of queries at a time: it reads a tile's codes and parameters with wide
// loads straight into the operands' lanes, one tile ahead, dequantises them there, and keeps O^T and the softmax's state of its tiles in
// registers.  Nothing is shared between wavefronts until their results meet at the end: those of a workgroup in LDS, those of a
// chunk in the workspace, always in the same order.
//
// Softmax: p = 2^(t - ref + kShift) with t the score in powers of two.  Any reference gives the same quotient as long as nothing
// overflows, so it is only moved (and the sums rescaled) when a score exceeds it by more than kSlack: a lane compares its own
// scores, lanes only meet when one of them does.  P is rounded to fp16 for the product, at most 2^15 and with kShift + 24 = 32 powers
// of two below the reference; its sum is taken in fp32 before that rounding, whose errors are independent.
#include "e0m4_kv4.h"
#include "e0m4_host.h"

namespace e0m4 {

namespace {

constexpr int kCols = 16;               // rows of queries of a tile
constexpr float kShift = 8.f, kSlack = 7.f;
constexpr float kLog2E = 1.44269504088896340736f;
constexpr float kInf = __builtin_inff();

__device__ inline float bf16_low(uint32_t w) { return __builtin_bit_cast(float, w << 16); }
__device__ inline float bf16_high(uint32_t w) { return __builtin_bit_cast(float, w & 0xFFFF0000u); }
__device__ inline uint32_t bf16_round(float f)
{
    const uint32_t u = __builtin_bit_cast(uint32_t, f);
    if (f != f) return 0x7FC0u;
    return (u + 0x7FFFu + ((u >> 16) & 1u)) >> 16;
}

// Four dims of a row's result from its sums; zeros for a row that sees nothing.
template <int DIM>
__device__ inline void finish(const Kv4Attention& a, int b, int h, int row, int d, bool valid, floatx4 acc, float ref, float sum)
{
    const float f = !valid || sum == 0.f ? 0.f : 1.f / sum;
    const int i = row / a.share, head = h * a.share + row % a.share;
    uint16_t* p = static_cast<uint16_t*>(a.out) + (((int64_t)b * a.n_new + i) * (a.kv_heads * a.share) + head) * DIM + d;
    uint32_t x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float y = f == 0.f ? 0.f : acc[j] * f;
        x[j] = a.bf16 ? bf16_round(y) : (uint32_t)__builtin_bit_cast(uint16_t, (half_t)y);
    }
    *reinterpret_cast<uint2*>(p) = uint2{x[0] | (x[1] << 16), x[2] | (x[3] << 16)};
    if (a.lse && d == 0)
        a.lse[((int64_t)b * a.kv_heads + h) * ((int64_t)a.n_new * a.share) + row] = f == 0.f ? kInf : ref - kShift + __builtin_amdgcn_logf(sum);
}

// The lane's part of 16 rows of queries as the right operand of S^T = K Q^T: row row0 + lane % 16, dims kq * DIM/4 + 8 w.  The values
// of the cache are fp16, so queries are too; bfloat16 ones are scaled by the power of two that brings their row's largest into
// [1, 2), which `factor` takes back: what is lost of them then is below 2^-25 of the largest.
template <int DIM>
struct Queries {
    half8_t q[DIM / 32];
    float factor;                       // of a score, to powers of two
};
template <int DIM>
__device__ inline Queries<DIM> load_queries(const Kv4Attention& a, int b, int h, int row, bool there, int kq)
{
    Queries<DIM> out;
    out.factor = kLog2E / __builtin_sqrtf((float)DIM);
    const int i = row / a.share, head = h * a.share + row % a.share;
    const uint16_t* p = static_cast<const uint16_t*>(a.q.data) + b * a.q.batch_ld + i * a.q.row_ld + head * a.q.head_ld + kq * (DIM / 4);
    uint4 raw[DIM / 32];
#pragma unroll
    for (int w = 0; w < DIM / 32; ++w) raw[w] = there ? *reinterpret_cast<const uint4*>(p + 8 * w) : uint4{0, 0, 0, 0};
    if (!a.bf16) {
#pragma unroll
        for (int w = 0; w < DIM / 32; ++w) out.q[w] = __builtin_bit_cast(half8_t, raw[w]);
        return out;
    }
    uint32_t top = 0;                   // largest magnitude, as bits
#pragma unroll
    for (int w = 0; w < DIM / 32; ++w) {
        const uint32_t x[4] = {raw[w].x, raw[w].y, raw[w].z, raw[w].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t l = x[j] & 0x7FFFu, u = (x[j] >> 16) & 0x7FFFu;
            top = l > top ? l : top;
            top = u > top ? u : top;
        }
    }
    uint32_t o = __shfl_xor(top, 16);
    top = o > top ? o : top;
    o = __shfl_xor(top, 32);
    top = o > top ? o : top;
    int e = (int)(top >> 7) - 127;
    if (e == 128 || top == 0) e = 0;    // infinite, not a number, or all zeros
#pragma unroll
    for (int w = 0; w < DIM / 32; ++w) {
        const uint32_t x[4] = {raw[w].x, raw[w].y, raw[w].z, raw[w].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            out.q[w][2 * j] = (half_t)__builtin_ldexpf(bf16_low(x[j]), -e);
            out.q[w][2 * j + 1] = (half_t)__builtin_ldexpf(bf16_high(x[j]), -e);
        }
    }
    out.factor = __builtin_ldexpf(out.factor, e);
    return out;
}

// A tile's K as a wavefront's lanes have it from memory, and the same as operands.
template <int DIM, int G>
struct RawK {
    words4_t code[DIM / 64];
    uint32_t param[2][Kv4<DIM, G>::kLaneGroups];
};
__device__ inline words4_t load16(__amdgpu_buffer_rsrc_t tile, int offset)
{
    return __builtin_bit_cast(words4_t, __builtin_amdgcn_raw_buffer_load_b128(tile, offset, 0, 0));
}
template <int DIM, int G>
__device__ inline void load_k(__amdgpu_buffer_rsrc_t tile, int lane, RawK<DIM, G>& k)
{
    using L = Kv4<DIM, G>;
    const int kq = lane >> 4, r = lane & 15, g0 = kq * L::kLaneDims / G;
#pragma unroll
    for (int p = 0; p < L::kPieces; ++p) k.code[p] = load16(tile, (p * 64 + lane) * 16);
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int e = 0; e < L::kLaneGroups; ++e)
            k.param[s][e] = __builtin_amdgcn_raw_buffer_load_b32(tile, L::kKParams + ((g0 + e) * kKv4Rows + 16 * s + r) * 4, 0, 0);
}
// Operand of half s, step w (dims kq * DIM/4 + 8 w ...)
template <int DIM, int G>
__device__ inline half8_t operand_k(const RawK<DIM, G>& k, int s, int w, uint32_t hi, uint32_t lo)
{
    const uint32_t word = DIM == 64 ? k.code[0][2 * s + w] : k.code[s * (DIM / 128) + w / 4][w % 4];
    return kv4_values(word, k.param[s][Kv4<DIM, G>::kLaneGroups == 1 ? 0 : 8 * w / G], hi, lo);
}

template <int DIM, int G>
struct RawV {
    words4_t code[DIM / 64];
    words4_t scale[DIM / G], bias[DIM / G];
};
template <int DIM, int G>
__device__ inline void load_v(__amdgpu_buffer_rsrc_t tile, int lane, RawV<DIM, G>& v)
{
    using L = Kv4<DIM, G>;
    const int kq = lane >> 4;
#pragma unroll
    for (int p = 0; p < L::kPieces; ++p) v.code[p] = load16(tile, L::kVCodes + (p * 64 + lane) * 16);
#pragma unroll
    for (int g = 0; g < L::kGroups; ++g) {
        v.scale[g] = load16(tile, L::kVParams + g * 128 + kq * 16);
        v.bias[g] = load16(tile, L::kVParams + g * 128 + 64 + kq * 16);
    }
}
// Parameters of rows from `length` on become zeros: what memory holds there was perhaps never written, and 0 * NaN is NaN.
template <int DIM, int G>
__device__ inline void clear_v(RawV<DIM, G>& v, int row0, int kq, int length)
{
    using L = Kv4<DIM, G>;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        uint32_t m = 0;
        if (row0 + L::row_of(kq, 2 * j) < length) m |= 0xFFFFu;
        if (row0 + L::row_of(kq, 2 * j + 1) < length) m |= 0xFFFF0000u;
#pragma unroll
        for (int g = 0; g < L::kGroups; ++g) {
            v.scale[g][j] &= m;
            v.bias[g][j] &= m;
        }
    }
}

// Which of a tile's rows the lane's query sees: bit 4 s + i for row 16 s + 4 kq + i.  [from, to): by position.
__device__ inline uint32_t seen_rows(const Kv4Attention& a, int b, int row0, int kq, int query, int from, int to)
{
    uint32_t seen = 0;
    const uint8_t* m = a.mask ? a.mask + b * a.mask_batch_ld + query * a.mask_row_ld : nullptr;
#pragma unroll
    for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int row = row0 + 16 * s + 4 * kq + i;
            bool in = row >= from && row < to;
            if (m && in) in = row < a.mask_rows && m[row] != 0;
            seen |= in ? 1u << (4 * s + i) : 0u;
        }
    return seen;
}

template <int DIM, int G, int WAVES>
__global__ __launch_bounds__(WAVES * 64) void kv4_decode_kernel(Kv4Attention a)
{
    using L = Kv4<DIM, G>;
    constexpr int kSteps = DIM / 32, kDimTiles = DIM / 16, kStride = DIM + 4;
    extern __shared__ __attribute__((aligned(16))) float shared[];          // [wave][column][DIM + 4], then the statistics
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), col = lane & 15, kq = lane >> 4;
    const int b = blockIdx.z, h = blockIdx.y, chunk = blockIdx.x % a.chunks, row0 = blockIdx.x / a.chunks * kCols;
    const int rows = a.n_new * a.share, cols = rows - row0 < kCols ? rows - row0 : kCols;
    const Kv4Span span = kv4_span(a, b, row0, cols);
    const int tile0 = span.begin / kKv4Rows + chunk * a.chunk_tiles, tiles_end = (span.end + kKv4Rows - 1) / kKv4Rows;
    const int tile1 = tile0 + a.chunk_tiles < tiles_end ? tile0 + a.chunk_tiles : tiles_end;
    if (tile0 >= tile1 && a.chunks > 1) return;                             // (the sum knows)

    const int query = (row0 + col) / a.share, at = span.length - span.count + query;
    const bool valid = col < cols && query < span.count;
    const Queries<DIM> qs = load_queries<DIM>(a, b, h, valid ? row0 + col : 0, valid, kq);
    const int to = a.causal && at + 1 < span.length ? at + 1 : span.length;
    const int from = a.window && at - a.window + 1 > 0 ? at - a.window + 1 : 0;
    // rows that all of the tile's queries see by position
    const int first_query = row0 / a.share, last_query = (row0 + cols - 1) / a.share < span.count ? (row0 + cols - 1) / a.share : span.count - 1;
    const int all_from = a.window ? span.length - span.count + last_query - a.window + 1 : 0;
    const int all_to = a.causal ? span.length - span.count + first_query + 1 : span.length;

    const uint8_t* cache = a.cache + ((int64_t)b * a.kv_heads + h) * a.tiles * L::kBytes;
    const uint32_t hi = frac_mask_vgpr(), lo = frac_mask_low_vgpr();
    floatx4 o[kDimTiles];
#pragma unroll
    for (int d = 0; d < kDimTiles; ++d) o[d] = floatx4{0.f, 0.f, 0.f, 0.f};
    float ref = -kInf, sum = 0.f;

    RawK<DIM, G> k;
    RawV<DIM, G> v;
    int tile = tile0 + wave;
    {
        const __amdgpu_buffer_rsrc_t first = rsrc_if(cache + (int64_t)tile * L::kBytes, tile < tile1);
        load_k(first, lane, k);
        load_v(first, lane, v);
    }
    for (; tile < tile1; tile += WAVES) {
        // (behind the last one there is no access to memory)
        const __amdgpu_buffer_rsrc_t next = rsrc_if(cache + (int64_t)(tile + WAVES) * L::kBytes, tile + WAVES < tile1);
        floatx4 s[2] = {floatx4{0.f, 0.f, 0.f, 0.f}, floatx4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int w = 0; w < kSteps; ++w)
#pragma unroll
            for (int u = 0; u < 2; ++u)
                s[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(operand_k<DIM, G>(k, u, w, hi, lo), qs.q[w], s[u], 0, 0, 0);
        load_k(next, lane, k);
        const int r0 = tile * kKv4Rows;
        if (a.mask || r0 < all_from || r0 + kKv4Rows > all_to) {
            const uint32_t seen = seen_rows(a, b, r0, kq, valid ? query : 0, from, to);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[u][i] = (seen >> (4 * u + i)) & 1 ? s[u][i] : -kInf;
            if (r0 + kKv4Rows > span.length) clear_v<DIM, G>(v, r0, kq, span.length);
        }
        float top = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])), fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
        top *= qs.factor;
        if (__any(top > ref + kSlack)) {
            top = fmaxf(top, __shfl_xor(top, 16));
            top = fmaxf(top, __shfl_xor(top, 32));
            const float now = fmaxf(ref, top);
            const float down = now == -kInf ? 1.f : __builtin_amdgcn_exp2f(ref - now);
            ref = now;
            sum *= down;
#pragma unroll
            for (int d = 0; d < kDimTiles; ++d) o[d] *= down;
        }
        const float minus = ref == -kInf ? 0.f : kShift - ref;
        half8_t p;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], qs.factor, minus));
                sum += e;
                p[4 * u + i] = (half_t)e;
            }
#pragma unroll
        for (int pc = 0; pc < L::kPieces; ++pc) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int g = (64 * pc + 16 * w) / G;
                const Kv4OctetParams par = kv4_octet_params(v.scale[g], v.bias[g]);
                o[4 * pc + w] = __builtin_amdgcn_mfma_f32_16x16x32_f16(kv4_values_v(v.code[pc][w], par, hi, lo), p, o[4 * pc + w], 0, 0, 0);
            }
        }
        load_v(next, lane, v);
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);

    // the wavefronts' results, in their order
    float* stats = shared + WAVES * cols * kStride;                         // [wave][column] reference, then sum
    if (col < cols) {
        float* mine = shared + (wave * cols + col) * kStride + 4 * kq;
#pragma unroll
        for (int d = 0; d < kDimTiles; ++d) *reinterpret_cast<floatx4*>(mine + 16 * d) = o[d];
        if (kq == 0) {
            stats[wave * kCols + col] = ref;
            stats[(WAVES + wave) * kCols + col] = sum;
        }
    }
    __syncthreads();
    const int64_t bh = (int64_t)b * a.kv_heads + h;
    for (int i = t; i < cols * (DIM / 4); i += WAVES * 64) {
        const int c = i / (DIM / 4), d = i % (DIM / 4) * 4, row = row0 + c;
        float top = -kInf;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) top = fmaxf(top, stats[w * kCols + c]);
        floatx4 acc = {0.f, 0.f, 0.f, 0.f};
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) {
            const float f = top == -kInf ? 0.f : __builtin_amdgcn_exp2f(stats[w * kCols + c] - top);
            total += stats[(WAVES + w) * kCols + c] * f;
            acc += *reinterpret_cast<const floatx4*>(shared + (w * cols + c) * kStride + d) * f;
        }
        if (a.chunks > 1) {
            const int64_t at_row = (((int64_t)chunk * a.batch * a.kv_heads) + bh) * rows + row;
            *reinterpret_cast<floatx4*>(a.part_out + at_row * DIM + d) = acc;
            if (d == 0) a.part_stats[at_row] = float2{top, total};
        } else {
            finish<DIM>(a, b, h, row, d, row / a.share < span.count, acc, top, total);
        }
    }
}

// The sum over chunks, one workgroup per (sequence, head, row), a thread per four dims and quarter of the chunks.
template <int DIM>
__global__ __launch_bounds__(DIM) void kv4_combine_kernel(Kv4Attention a)
{
    constexpr int kParts = 4, kPer = DIM / 4;
    __shared__ floatx4 part[kParts][kPer];
    const int t = threadIdx.x, row = blockIdx.x, h = blockIdx.y, b = blockIdx.z, rows = a.n_new * a.share;
    const int row0 = row / a.tile_rows * a.tile_rows;
    const Kv4Span span = kv4_span(a, b, row0, rows - row0 < a.tile_rows ? rows - row0 : a.tile_rows);
    const int tiles = (span.end + kKv4Rows - 1) / kKv4Rows - span.begin / kKv4Rows;
    const int chunks = (tiles + a.chunk_tiles - 1) / a.chunk_tiles;
    const int64_t stride = (int64_t)a.batch * a.kv_heads * rows, at = ((int64_t)b * a.kv_heads + h) * rows + row;
    float top = -kInf, total = 0.f;
    for (int c = 0; c < chunks; ++c) top = fmaxf(top, a.part_stats[c * stride + at].x);
    const int d = t % kPer * 4, q = t / kPer;
    floatx4 acc = {0.f, 0.f, 0.f, 0.f};
    for (int c = 0; c < chunks; ++c) {
        const float2 st = a.part_stats[c * stride + at];
        const float f = top == -kInf ? 0.f : __builtin_amdgcn_exp2f(st.x - top);
        total += st.y * f;
        if (c % kParts == q) acc += *reinterpret_cast<const floatx4*>(a.part_out + (c * stride + at) * DIM + d) * f;
    }
    part[q][t % kPer] = acc;
    __syncthreads();
    if (q) return;
#pragma unroll
    for (int i = 1; i < kParts; ++i) acc += part[i][t];
    finish<DIM>(a, b, h, row, d, row / a.share < span.count, acc, top, total);
}

// What the rows of a tile of the cache received: one workgroup per tile, its wavefronts share the rows of queries.  K stays in
// registers as operands.
template <int DIM, int G>
__global__ __launch_bounds__(256) void kv4_received_kernel(Kv4Attention a, float* __restrict__ received)
{
    using L = Kv4<DIM, G>;
    constexpr int kSteps = DIM / 32, kWaves = 4;
    __shared__ float part[kWaves][kKv4Rows];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), col = lane & 15, kq = lane >> 4;
    const int tile = blockIdx.x, h = blockIdx.y, b = blockIdx.z, r0 = tile * kKv4Rows, rows = a.n_new * a.share;
    const int length = clamp_count(a.lengths[b], a.capacity), count = a.counts ? clamp_count(a.counts[b], a.n_new) : a.n_new;
    if (r0 >= length || count == 0) return;
    const int64_t bh = (int64_t)b * a.kv_heads + h;
    // queries that may see one of the tile's rows
    int i0 = 0, i1 = count;
    if (a.causal) {
        const int at = length - count, last = r0 + kKv4Rows < length ? r0 + kKv4Rows - 1 : length - 1;
        i0 = r0 - at > 0 ? r0 - at : 0;
        if (a.window && last + a.window - at < i1) i1 = last + a.window - at;
    }
    RawK<DIM, G> raw;
    load_k(make_rsrc(a.cache + (bh * a.tiles + tile) * L::kBytes), lane, raw);
    const uint32_t hi = frac_mask_vgpr(), lo = frac_mask_low_vgpr();
    half8_t k[2][kSteps];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int w = 0; w < kSteps; ++w) k[u][w] = operand_k<DIM, G>(raw, u, w, hi, lo);
    float got[2][4] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
    for (int row0 = (i0 * a.share) / kCols * kCols + wave * kCols; row0 < i1 * a.share; row0 += kWaves * kCols) {
        const int row = row0 + col, query = row / a.share, at = length - count + query;
        const bool valid = row < rows && query < count;
        const Queries<DIM> qs = load_queries<DIM>(a, b, h, valid ? row : 0, valid, kq);
        const float lse = valid ? a.lse[bh * rows + row] : kInf;
        floatx4 s[2] = {floatx4{0.f, 0.f, 0.f, 0.f}, floatx4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
        for (int w = 0; w < kSteps; ++w)
#pragma unroll
            for (int u = 0; u < 2; ++u) s[u] = __builtin_amdgcn_mfma_f32_16x16x32_f16(k[u][w], qs.q[w], s[u], 0, 0, 0);
        const int to = a.causal && at + 1 < length ? at + 1 : length;
        const int from = a.window && at - a.window + 1 > 0 ? at - a.window + 1 : 0;
        const uint32_t seen = valid ? seen_rows(a, b, r0, kq, query, from, to) : 0u;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                if ((seen >> (4 * u + i)) & 1) got[u][i] += __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], qs.factor, -lse));
    }
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float g = got[u][i];
#pragma unroll
            for (int d = 1; d < 16; d <<= 1) g += __shfl_xor(g, d);
            if (col == 0) part[wave][16 * u + 4 * kq + i] = g;
        }
    __syncthreads();
    if (t < kKv4Rows && r0 + t < length) {
        float g = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) g += part[w][t];
        received[bh * a.capacity + r0 + t] += g;
    }
}

}  // namespace

int launch_kv4_decode(const Kv4Attention& a, const e0m4_kv4_shape& s, hipStream_t stream)
{
    constexpr int kWaves = 4;
    const int64_t rows = (int64_t)a.n_new * a.share, row_tiles = (rows + kCols - 1) / kCols;
    const int cols = rows < kCols ? (int)rows : kCols;
    const int lds = (kWaves * cols * (s.dim + 4) + 2 * kWaves * kCols) * 4;
    const dim3 grid((unsigned)(row_tiles * a.chunks), (unsigned)a.kv_heads, (unsigned)a.batch);
    return kv4_dispatch(s, [&](auto shape) -> int {
        constexpr int DIM = decltype(shape)::kDim, G = decltype(shape)::kGroup;
        static std::atomic<uint64_t> allowed{0};
        const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(&kv4_decode_kernel<DIM, G, kWaves>), 160 * 1024, allowed);
        if (rc != E0M4_OK) return rc;
        hipLaunchKernelGGL((kv4_decode_kernel<DIM, G, kWaves>), grid, dim3(kWaves * 64), lds, stream, a);
        return check_launch();
    });
}

int launch_kv4_combine(const Kv4Attention& a, const e0m4_kv4_shape& s, hipStream_t stream)
{
    const dim3 grid((unsigned)(a.n_new * a.share), (unsigned)a.kv_heads, (unsigned)a.batch);
    switch (s.dim) {
        case 64: hipLaunchKernelGGL(kv4_combine_kernel<64>, grid, dim3(64), 0, stream, a); break;
        case 128: hipLaunchKernelGGL(kv4_combine_kernel<128>, grid, dim3(128), 0, stream, a); break;
        default: hipLaunchKernelGGL(kv4_combine_kernel<256>, grid, dim3(256), 0, stream, a); break;
    }
    return check_launch();
}

int launch_kv4_received(const Kv4Attention& a, const e0m4_kv4_shape& s, float* received, hipStream_t stream)
{
    const dim3 grid((unsigned)a.tiles, (unsigned)a.kv_heads, (unsigned)a.batch);
    return kv4_dispatch(s, [&](auto shape) -> int {
        constexpr int DIM = decltype(shape)::kDim, G = decltype(shape)::kGroup;
        hipLaunchKernelGGL((kv4_received_kernel<DIM, G>), grid, dim3(256), 0, stream, a, received);
        return check_launch();
    });
}

}  // namespace e0m4
