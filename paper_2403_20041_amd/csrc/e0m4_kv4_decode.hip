// Attention of few queries over a cache in E0M4 codes, and the sum of its chunks.  Layout and what it gives the products: e0m4_kv4.h;
// softmax: e0m4_kv4_attention.h.
//
// A wavefront takes whole tiles of 32 rows by itself, 16 rows of queries at a time: it reads a tile's codes and parameters with wide
// loads straight into the operands' lanes, one tile ahead, dequantises them there, and keeps O^T and the softmax's state of its tiles in
// registers.  Nothing is shared between wavefronts until their results meet at the end: those of a workgroup in LDS, those of a
// chunk in the workspace, always in the same order.
#include "e0m4_kv4_attention.h"
#include "e0m4_host.h"

#include <type_traits>

namespace e0m4 {

namespace {

constexpr int kCols = 16;               // rows of queries of a tile
// The lane's part of 16 rows of queries as the right operand of S^T = K Q^T: row row0 + lane % 16, dims kq * DIM/4 + 8 w.
template <int DIM>
struct Queries {
    half8_t q[DIM / 32];
    float factor;
};
template <int DIM>
__device__ inline Queries<DIM> load_queries(const Kv4Attention& a, int b, int h, int row, bool there, int kq)
{
    Queries<DIM> out;
    out.factor = load_query_row<DIM, DIM / 32, 16>(a, b, h, row, there, kq * (DIM / 4), 8, out.q);
    return out;
}

// A tile's K as a wavefront's lanes have it from memory, and the same as operands.
template <int DIM, int G>
struct RawK {
    words4_t code[DIM / 64];
    uint32_t param[2][Kv4<DIM, G>::kLaneGroups];
};
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

// Which of a tile's rows the lane's query sees: bit 4 s + i for row 16 s + 4 kq + i.
__device__ inline uint32_t seen_rows(const Kv4Attention& a, int b, int row0, int kq, int query, const Kv4Seen& by_place)
{
    auto row_of = [&](int i) { return row0 + 16 * (i >> 2) + 4 * kq + (i & 3); };
    uint32_t seen = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) seen |= row_of(i) >= by_place.from && row_of(i) < by_place.to ? 1u << i : 0u;
    if (a.mask) seen &= kv4_mask_bits<2>(a, b, query, [&](int g) { return row_of(4 * g); });
    return seen;
}

// What the rounding of P to fp16 leaves is multiplied too where the result is fp16, whose own rounding is no larger than that of the few
// weights that make a short row: by a second product (kRestSecond), or, where there are at most eight rows of queries, in the upper
// eight columns of the one that there is, which hold the same rows again (kRestColumns).  32 heads on 8, 32 sequences of up to 8192
// rows: 44.0 us in columns, 44.6 with a second product, 41.8 with neither; 64 sequences of 4000 rows of 64 dims 34.8, 35.7, 32.2; 16 of
// 8000 rows of 256 dims 85.6, 83.9, 81.7.
enum Rest { kRestNone, kRestSecond, kRestColumns };

// Bound: a tile of 32 rows is 4352 bytes (dim 128, group 128) and about 300 vector instructions, 208 of them dequantisation.  32 sequences
// of up to 8192 rows, 32 heads on 8: 182 MB in 48 us, of which a copy would take 35, the instructions 20 and the products 4: memory, and
// what of the rest does not fall behind its loads.  Four wavefronts a SIMD have a tile each on its way; two tiles ahead gained
// nothing (49 against 48 us).  4 of up to 16000 rows, 40 heads, with their scores kept: 272 MB in 67 us.  4.2 TB/s is the most that
// this kernel has drawn.
template <int DIM, int G, int WAVES, Rest REST>
__global__ __launch_bounds__(WAVES * 64, DIM == 256 ? 2 : DIM == 128 && G == 32 ? 3 : 4) void kv4_decode_kernel(Kv4Attention a)
{
    using L = Kv4<DIM, G>;
    constexpr int kSteps = DIM / 32, kDimTiles = DIM / 16, kStride = DIM + 4;
    extern __shared__ __attribute__((aligned(16))) float shared[];          // [wave][column][DIM + 4], then the statistics
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), kq = lane >> 4;
    const int col = REST == kRestColumns ? lane & 7 : lane & 15;
    const bool upper = REST == kRestColumns && (lane & 8);
    // (chunks are rotated from head to head: with a multiple of eight of them each would be one XCD's everywhere, and the last ones,
    // which short sequences do not have, leave theirs idle)
    const int b = blockIdx.z, h = blockIdx.y, chunk = (blockIdx.x + blockIdx.y + blockIdx.z * gridDim.y) % a.chunks, row0 = blockIdx.x / a.chunks * kCols;
    const int rows = a.n_new * a.share, cols = rows - row0 < kCols ? rows - row0 : kCols;
    const uint8_t* cache = a.cache + ((int64_t)b * a.kv_heads + h) * a.tiles * L::kBytes;
    RawK<DIM, G> k;
    RawV<DIM, G> v;
    // where a workgroup has all of a sequence's rows, its first tiles are on their way before their number is known
    const bool early = WAVES > 4 && a.window == 0;
    if (early) {
        const __amdgpu_buffer_rsrc_t first = rsrc_if(cache + (int64_t)wave * L::kBytes, wave < a.tiles);
        load_k(first, lane, k);
        load_v(first, lane, v);
    }
    const Kv4Span span = kv4_span(a, b, row0, cols);
    const int tile0 = span.begin / kKv4Rows + chunk * a.chunk_tiles, tiles_end = (span.end + kKv4Rows - 1) / kKv4Rows;
    const int tile1 = tile0 + a.chunk_tiles < tiles_end ? tile0 + a.chunk_tiles : tiles_end;
    const int query = kv4_query_of(a, row0 + col), at = span.length - span.count + query;
    const bool valid = col < cols && query < span.count;
    // (rows from the sequence's count on are read too, so that nobody waits for it; their results are not used)
    const Queries<DIM> qs = load_queries<DIM>(a, b, h, col < cols ? row0 + col : 0, col < cols, kq);
    if (a.packed_q && chunk == 0 && col < cols && !upper)
        keep_query_row<kSteps>(a, ((int64_t)b * a.kv_heads + h) * rows + row0 + col, DIM, valid, kq * (DIM / 4), 8, qs.q, qs.factor);
    if (tile0 >= tile1 && a.chunks > 1) return;                             // (the sum knows)
    const Kv4Seen by_place = kv4_seen(a, span.length, at);
    // rows that all of the tile's queries see by position
    const int first_query = kv4_query_of(a, row0), end_query = kv4_query_of(a, row0 + cols - 1), last_query = end_query < span.count ? end_query : span.count - 1;
    const int all_from = a.window ? span.length - span.count + last_query - a.window + 1 : 0;
    const int all_to = a.causal ? span.length - span.count + first_query + 1 : span.length;

    int tile = tile0 + wave;
    if (!early) {
        const __amdgpu_buffer_rsrc_t first = rsrc_if(cache + (int64_t)tile * L::kBytes, tile < tile1);
        load_k(first, lane, k);
        load_v(first, lane, v);
    }
    const uint32_t hi = frac_mask_vgpr(), lo = frac_mask_low_vgpr();
    floatx4 o[kDimTiles];
#pragma unroll
    for (int d = 0; d < kDimTiles; ++d) o[d] = floatx4{0.f, 0.f, 0.f, 0.f};
    float ref = -kInf, sum = 0.f;
    const float take_off = upper ? -1.f : 0.f;

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
            const uint32_t seen = seen_rows(a, b, r0, kq, valid ? query : 0, by_place);
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[u][i] = (seen >> (4 * u + i)) & 1 ? s[u][i] : -kInf;
            if (r0 + kKv4Rows > span.length) clear_v<DIM, G>(v, r0, kq, span.length);
        }
        if (a.scores && valid && !upper) {
            float* out = a.scores + (((int64_t)b * a.kv_heads + h) * rows + row0 + col) * (a.tiles * kKv4Rows) + r0 + 4 * kq;
            *reinterpret_cast<floatx4*>(out) = s[0] * qs.factor;
            *reinterpret_cast<floatx4*>(out + 16) = s[1] * qs.factor;
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
        half8_t p, rest;
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], qs.factor, minus));
                sum += e;
                const half_t near = (half_t)e;
                p[4 * u + i] = REST == kRestColumns ? (half_t)__builtin_fmaf((float)near, take_off, e) : near;
                if (REST == kRestSecond) rest[4 * u + i] = (half_t)(e - (float)near);
            }
#pragma unroll
        for (int pc = 0; pc < L::kPieces; ++pc) {
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                const int g = (64 * pc + 16 * w) / G;
                const Kv4OctetParams par = kv4_octet_params(v.scale[g], v.bias[g]);
                const half8_t values = kv4_values_v(v.code[pc][w], par, hi, lo);
                o[4 * pc + w] = __builtin_amdgcn_mfma_f32_16x16x32_f16(values, p, o[4 * pc + w], 0, 0, 0);
                if (REST == kRestSecond) o[4 * pc + w] = __builtin_amdgcn_mfma_f32_16x16x32_f16(values, rest, o[4 * pc + w], 0, 0, 0);
            }
        }
        load_v(next, lane, v);
    }
    sum += __shfl_xor(sum, 16);
    sum += __shfl_xor(sum, 32);
    if (REST == kRestColumns)
#pragma unroll
        for (int d = 0; d < kDimTiles; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[d][i] += other_lane<0x128>(o[d][i]);      // (eight lanes on in the row of 16)

    // the wavefronts' results, in their order
    float* stats = shared + WAVES * cols * kStride;                         // [wave][column] reference, then sum
    if (col < cols && !upper) {
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
            finish<DIM>(a, b, h, row, d, kv4_query_of(a, row) < span.count, acc, top, total);
        }
    }
}

// What chunks' results count for in a row's: 2^(reference - largest reference), by the lanes of a wavefront; returns the softmax's sum.
__device__ inline float chunk_factors(const float2* stats, int64_t stride, int chunks, int lane, float& top, float* factor)
{
    top = -kInf;
    for (int c = lane; c < chunks; c += 64) top = fmaxf(top, stats[c * stride].x);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    float total = 0.f;
    for (int c = lane; c < chunks; c += 64) {
        const float2 st = stats[c * stride];
        const float f = top == -kInf ? 0.f : __builtin_amdgcn_exp2f(st.x - top);
        if (factor) factor[c] = f;
        total += st.y * f;
    }
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) total += __shfl_xor(total, d);
    return total;
}
__device__ inline int chunks_of(const Kv4Attention& a, int b, int row, int rows, Kv4Span& span)
{
    const int row0 = row / a.tile_rows * a.tile_rows;
    span = kv4_span(a, b, row0, rows - row0 < a.tile_rows ? rows - row0 : a.tile_rows);
    const int tiles = (span.end + a.tile_keys - 1) / a.tile_keys - span.begin / a.tile_keys;
    return (tiles + a.chunk_tiles - 1) / a.chunk_tiles;
}

// The sum over chunks, a wavefront per row: it works out what they count for, then its lanes take four dims of one chunk after the other
// (of two or four chunks at a time where a row is shorter than 64 such pieces).  Workgroups beyond the rows' add what 2048 rows of
// the cache received, from the scores (tiles of 16 rows of queries, one of them at most).
constexpr int kCombineThreads = 256, kCombineRows = kCombineThreads / 64, kReceivedRows = 16, kReceivedKeys = 2048;
__host__ __device__ inline int combine_sums(const Kv4Attention& a) { return a.chunks > 1 ? (a.n_new * a.share + kCombineRows - 1) / kCombineRows : 0; }
template <int DIM>
__global__ __launch_bounds__(kCombineThreads) void kv4_combine_kernel(Kv4Attention a, float* __restrict__ received)
{
    constexpr int kPer = DIM / 4, kAtOnce = 64 / kPer;
    __shared__ float factors[kCombineRows][kKv4MaxChunks];
    __shared__ float2 norms[kReceivedRows];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), h = blockIdx.y, b = blockIdx.z, rows = a.n_new * a.share;
    const int64_t stride = (int64_t)a.batch * a.kv_heads * rows, bh = (int64_t)b * a.kv_heads + h;
    const int sums = combine_sums(a);
    Kv4Span span;
    if ((int)blockIdx.x < sums) {
        const int row = blockIdx.x * kCombineRows + wave;
        if (row >= rows) return;
        const int chunks = chunks_of(a, b, row, rows, span);
        const int64_t at = bh * rows + row;
        float* factor = factors[wave];
        float top;
        const float total = chunk_factors(a.part_stats + at, stride, chunks, lane, top, factor);
        // the other lanes' factors: a wavefront's LDS accesses stay in their order, if only the compiler keeps it
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
        const int d = lane % kPer * 4;
        const float* p = a.part_out + at * DIM + d;
        floatx4 acc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
        for (int c = lane / kPer; c < chunks; c += kAtOnce) acc += *reinterpret_cast<const floatx4*>(p + c * stride * DIM) * factor[c];
#pragma unroll
        for (int s = kPer; s < 64; s <<= 1)
#pragma unroll
            for (int i = 0; i < 4; ++i) acc[i] += __shfl_xor(acc[i], s);
        if (lane < kPer) finish<DIM>(a, b, h, row, d, kv4_query_of(a, row) < span.count, acc, top, total);
        return;
    }
    const int chunks = chunks_of(a, b, 0, rows, span), key0 = ((int)blockIdx.x - sums) * kReceivedKeys;
    if (key0 >= span.end || key0 + kReceivedKeys <= span.begin) return;
    if (a.chunks > 1) {
        for (int row = wave; row < rows; row += kCombineThreads / 64) {
            float top;
            const float total = chunk_factors(a.part_stats + bh * rows + row, stride, chunks, lane, top, nullptr);
            if (lane == 0) norms[row] = row_norm(kv4_query_of(a, row) < span.count, top, total);
        }
    } else if (t < rows) {
        norms[t] = a.norm[bh * rows + t];
    }
    __syncthreads();
    const int low = span.begin / kKv4Rows * kKv4Rows;
    const float* s = a.scores + bh * rows * (a.tiles * kKv4Rows);
    float* out = received + bh * a.capacity;
    int key[kReceivedKeys / kCombineThreads];
    float got[kReceivedKeys / kCombineThreads], old[kReceivedKeys / kCombineThreads];
#pragma unroll
    for (int j = 0; j < kReceivedKeys / kCombineThreads; ++j) {
        key[j] = key0 + t + j * kCombineThreads;
        key[j] = key[j] >= low && key[j] < span.end ? key[j] : -1;
        got[j] = 0.f;
        old[j] = key[j] >= 0 ? out[key[j]] : 0.f;
    }
    for (int row = 0; row < rows; ++row) {
        if (kv4_query_of(a, row) >= span.count) break;  // (their scores were not written)
#pragma unroll
        for (int j = 0; j < kReceivedKeys / kCombineThreads; ++j) {
            const float x = key[j] >= 0 ? s[row * (a.tiles * kKv4Rows) + key[j]] : -kInf;
            got[j] = x == -kInf ? got[j] : __builtin_fmaf(__builtin_amdgcn_exp2f(x - norms[row].x), norms[row].y, got[j]);
        }
    }
#pragma unroll
    for (int j = 0; j < kReceivedKeys / kCombineThreads; ++j)
        if (key[j] >= 0) out[key[j]] = old[j] + got[j];
}

template <int DIM, int G, int WAVES, Rest REST>
int launch_decode(const Kv4Attention& a, dim3 grid, int cols, hipStream_t stream)
{
    const int lds = (WAVES * cols * (DIM + 4) + 2 * WAVES * kCols) * 4;
    static std::atomic<uint64_t> allowed{0};
    const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(&kv4_decode_kernel<DIM, G, WAVES, REST>), 160 * 1024, allowed);
    if (rc != E0M4_OK) return rc;
    hipLaunchKernelGGL((kv4_decode_kernel<DIM, G, WAVES, REST>), grid, dim3(WAVES * 64), lds, stream, a);
    return check_launch();
}

}  // namespace

int launch_kv4_decode(const Kv4Attention& a, const e0m4_kv4_shape& s, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.n_new * a.share, row_tiles = (rows + kCols - 1) / kCols;
    const int cols = rows < kCols ? (int)rows : kCols;
    // 2^32 work items along a dimension are refused by the launch itself; only a forced kernel or chunk comes near: by choice these are at
    // most 12000 tiles of rows and chunks
    if (row_tiles * a.chunks * 512 > 0xffffffffLL) return E0M4_ERR_SHAPE;
    const dim3 grid((unsigned)(row_tiles * a.chunks), (unsigned)a.kv_heads, (unsigned)a.batch);
    return kv4_dispatch(s, [&](auto shape) -> int {
        constexpr int DIM = decltype(shape)::kDim, G = decltype(shape)::kGroup;
        const bool shared = a.chunks > 1 || a.chunk_tiles > kKv4ShortTiles;
        auto launch = [&](auto rest) -> int {
            constexpr Rest REST = decltype(rest)::value;
            return shared ? launch_decode<DIM, G, 4, REST>(a, grid, cols, stream) : launch_decode<DIM, G, 8, REST>(a, grid, cols, stream);
        };
        if (a.bf16) return launch(std::integral_constant<Rest, kRestNone>{});
        return cols <= 8 ? launch(std::integral_constant<Rest, kRestColumns>{}) : launch(std::integral_constant<Rest, kRestSecond>{});
    });
}

int launch_kv4_combine(const Kv4Attention& a, const e0m4_kv4_shape& s, float* received, hipStream_t stream)
{
    const int64_t blocks = received ? (s.capacity + kReceivedKeys - 1) / kReceivedKeys : 0;
    const dim3 grid((unsigned)(combine_sums(a) + blocks), (unsigned)a.kv_heads, (unsigned)a.batch);
    switch (s.dim) {
        case 64: hipLaunchKernelGGL(kv4_combine_kernel<64>, grid, dim3(kCombineThreads), 0, stream, a, received); break;
        case 128: hipLaunchKernelGGL(kv4_combine_kernel<128>, grid, dim3(kCombineThreads), 0, stream, a, received); break;
        default: hipLaunchKernelGGL(kv4_combine_kernel<256>, grid, dim3(kCombineThreads), 0, stream, a, received); break;
    }
    return check_launch();
}

}  // namespace e0m4
