// Layout of a key/value cache in E0M4 codes (e0m4_kv4_*), and what its kernels share.
//
// The cache of one (sequence, head of keys and values) is a run of tiles of 32 rows, each tile one contiguous stream:
//     K codes (16 dim bytes), V codes (16 dim bytes), K parameters, V parameters (128 dim / group bytes each).
// Both matrix products of attention contract what lies inside a lane's 32-bit words, without a transposition on the way:
//   K   S^T = K Q^T contracts the head dimension, so a word holds 8 consecutive dims of one row.  Lane kq * 16 + r of a 16-row half
//       s holds the dims kq * dim/4 ... of row 16 s + r (a quarter of the row: at most two groups' parameters per lane).
//   V   O^T = V^T P^T contracts rows, so a word holds 8 rows of one dim: the rows whose scores a lane has in its accumulators after
//       S^T, 4 kq + i and 16 + 4 kq + i (i = 0..3) of the tile for lane group kq; P goes from the accumulators into the product as
//       it is.  Such a set of 8 rows is an octet here; slot(row) is a row's place in it.
// In 16-byte pieces: K piece (s, c, kq, r) at (s * dim/128 + c) * 64 + kq * 16 + r holds the dims kq * dim/4 + 32 c ... + 31
// (dim 64: one piece per (kq, r), words 0, 1 of half 0 and 2, 3 of half 1); V piece (t, kq, n) at t * 64 + kq * 16 + n holds
// the dims 64 t + 16 w + n of octet kq in its words w.
// Parameters: K [group][row] words (scale low half, bias high half); V [group][scale or bias][octet][slot] fp16.
// A code's bits in its word are those of the packed weights (place_code).
#pragma once

#include "e0m4_device.h"
#include "e0m4_host.h"

namespace e0m4 {

typedef uint32_t words4_t __attribute__((ext_vector_type(4)));

constexpr int kKv4Rows = 32;                            // rows of a tile

__host__ __device__ constexpr int kv4_tile_bytes(int dim, int group) { return 32 * dim + 256 * (dim / group); }
__host__ __device__ inline int64_t kv4_tiles(int64_t capacity) { return (capacity + kKv4Rows - 1) / kKv4Rows; }

template <int DIM, int G>
struct Kv4 {
    static constexpr int kGroups = DIM / G;
    static constexpr int kPieces = DIM / 64;            // 16-byte pieces per lane and tile, of K as of V
    static constexpr int kVCodes = 16 * DIM;            // byte offsets in a tile
    static constexpr int kKParams = 32 * DIM;
    static constexpr int kVParams = 32 * DIM + 128 * kGroups;
    static constexpr int kBytes = kv4_tile_bytes(DIM, G);
    static constexpr int kLaneDims = DIM / 4;           // of K, contiguous
    static constexpr int kLaneGroups = G < kLaneDims ? kLaneDims / G : 1;
    // byte offset of the word with dims d .. d+7 (d a multiple of 8) of row
    __device__ static constexpr int k_word(int row, int d)
    {
        const int s = row >> 4, r = row & 15, kq = d / kLaneDims, w = d % kLaneDims / 8;
        const int piece = DIM == 64 ? 0 : s * (DIM / 128) + w / 4;
        const int word = DIM == 64 ? 2 * s + w : w % 4;
        return (piece * 64 + kq * 16 + r) * 16 + word * 4;
    }
    __device__ static constexpr int k_param(int row, int g) { return kKParams + (g * kKv4Rows + row) * 4; }
    __device__ static constexpr int octet(int row) { return (row & 15) >> 2; }
    __device__ static constexpr int slot(int row) { return (row >> 4) * 4 + (row & 3); }
    __device__ static constexpr int row_of(int octet, int slot) { return (slot >> 2) * 16 + octet * 4 + (slot & 3); }
    // byte offset of a row's scale (its bias is 64 bytes on)
    __device__ static constexpr int v_param(int row, int g) { return kVParams + g * 128 + (octet(row) * 8 + slot(row)) * 2; }
};

// A view of rows [batch, n, heads, dim] with the last dimension contiguous; strides in elements.
struct Kv4Rows {
    const void* data;
    int64_t batch_ld, row_ld, head_ld;
};

// ---- values of codes -----------------------------------------------------------------------------
// Two codes at a time to fp16((2 + c/8 - bias) * scale): c/8 - (bias - 2) is exact in fp16, the product is the one rounding.  Codes in
// fraction bits 5..2 (pairs 1 and 2 of a word, see the packed layout) read 32 + c/8 under the exponent of [32, 64), so that they
// only need another constant, bias + 30; eight codes take one rotate, four mask-ors, four additions and four products.
constexpr uint32_t kExp32Bits2 = 0x50005000u;           // sign 0, exponent of [32,64), both halves
__device__ inline half2_t splat(half_t h) { return half2_t{h, h}; }

__device__ inline void kv4_pairs(uint32_t word, uint32_t mask_hi, uint32_t mask_lo, half2_t (&p)[4])
{
    const uint32_t t = __builtin_amdgcn_alignbit(word, word, 8);
    p[0] = __builtin_bit_cast(half2_t, (word & mask_hi) | kExpBits2);
    p[1] = __builtin_bit_cast(half2_t, (word & mask_lo) | kExp32Bits2);
    p[2] = __builtin_bit_cast(half2_t, (t & mask_lo) | kExp32Bits2);
    p[3] = __builtin_bit_cast(half2_t, (t & mask_hi) | kExpBits2);
}
__device__ inline half8_t join(const half2_t (&p)[4])
{
    return half8_t{p[0][0], p[0][1], p[1][0], p[1][1], p[2][0], p[2][1], p[3][0], p[3][1]};
}
// Eight codes under one scale and bias (a word of K).
__device__ inline half8_t kv4_values(uint32_t word, uint32_t param, uint32_t mask_hi, uint32_t mask_lo)
{
    half2_t p[4];
    kv4_pairs(word, mask_hi, mask_lo, p);
    const half2_t s = splat(param_scale(param)), b = splat(param_bias(param)), b30 = b + splat((half_t)30.f);
    p[0] = (p[0] - b) * s;
    p[1] = (p[1] - b30) * s;
    p[2] = (p[2] - b30) * s;
    p[3] = (p[3] - b) * s;
    return join(p);
}
// Scales and biases of an octet in one group, as kv4_values_v takes them.
struct Kv4OctetParams {
    half2_t s[4], b[4];
};
__device__ inline Kv4OctetParams kv4_octet_params(words4_t scale, words4_t bias)
{
    Kv4OctetParams o;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t s = scale[i], b = bias[i];
        o.s[i] = __builtin_bit_cast(half2_t, s);
        o.b[i] = __builtin_bit_cast(half2_t, b);
        if (i == 1 || i == 2) o.b[i] += splat((half_t)30.f);
    }
    return o;
}
// Eight codes under eight scales and biases (a word of V).
__device__ inline half8_t kv4_values_v(uint32_t word, const Kv4OctetParams& o, uint32_t mask_hi, uint32_t mask_lo)
{
    half2_t p[4];
    kv4_pairs(word, mask_hi, mask_lo, p);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[i] = (p[i] - o.b[i]) * o.s[i];
    return join(p);
}

__device__ inline int clamp_count(int v, int64_t most) { return v < 0 ? 0 : (v < most ? v : (int)most); }

// ---- attention -----------------------------------------------------------------------------------
// One launch's view of e0m4_kv4_attention.  The rows of a head of keys and values are its queries' rows, row = i * share + h for the
// new token i and the h-th of its `share` query heads.
struct Kv4Attention {
    const uint8_t* cache;
    int64_t tiles;                                      // of a (sequence, head)
    Kv4Rows q;
    void* out;                                          // [batch, n_new, kv_heads * share, dim]
    const int* lengths;
    const int* counts;                                  // or null: n_new each
    const uint8_t* mask;                                // or null; [batch, n_new, mask_rows] by its strides
    int64_t mask_batch_ld, mask_row_ld;
    int mask_rows, mask_words;                          // (its runs of four rows can be read as words)
    int batch, kv_heads, share, n_new;
    uint32_t share_inverse;                             // 2^32 / share rounded up, 0 for 1: exact for the 2^22 rows that there may be
    int capacity, window;                               // window 0: none
    int causal, bf16;
    // Rows of the cache are dealt out in chunks of chunk_tiles tiles of tile_keys rows; with more than one chunk, partial results
    // meet in the workspace.
    int chunk_tiles, chunks;
    int tile_rows, tile_keys;                           // rows of queries that go through the cache together, rows of it at a time
    float* part_out;                                    // [chunk][batch][kv_heads][rows][dim]
    float2* part_stats;                                 // [chunk][batch][kv_heads][rows]: reference exponent, sum
    // for the received weights: [batch][kv_heads][rows] reference exponent and what 2^(score - reference) counts for (zero in rows that see
    // nothing).  A log2 of the sum would do in one number, but its rounding is that of a score's whole size.
    float2* norm;
    half_t* packed_q;                                   // [batch][kv_heads][rows][dim] queries as the products take them, and
    float* factors;                                     // [batch][kv_heads][rows] their scores' factors, or null
    float* scores;                                      // [batch][kv_heads][rows][tiles * 32] in powers of two, or null
};

// Grid of one workgroup for each sequence, head and one of `places`, place by place: x counts heads, y sequences and z places; places
// that z has no room for (65535) go to x in runs, the last of which may count beyond `places`.  A launch may have less than 2^32
// work items along a dimension: heads are at most 65535 and heads times places 2^36 (2^30 blocks of the cache; 2^25 blocks of queries
// in up to 2^11 chunks), so that x is at most 2^21 workgroups.
inline dim3 kv4_place_grid(const Kv4Attention& a, int64_t places)
{
    const int64_t run = (places + 65534) / 65535;
    return dim3((unsigned)(a.kv_heads * run), (unsigned)a.batch, (unsigned)((places + run - 1) / run));
}
__device__ inline int kv4_place(const Kv4Attention& a) { return blockIdx.z * (gridDim.x / a.kv_heads) + blockIdx.x / a.kv_heads; }

__device__ inline int kv4_query_of(const Kv4Attention& a, int row) { return a.share_inverse ? (int)__umulhi((uint32_t)row, a.share_inverse) : row; }

// What a tile of `n` rows of queries, the first one `row0`, looks at.
struct Kv4Span {
    int length, count;                                  // of the sequence
    int begin, end;                                     // rows of the cache that some query of the tile sees are among these
};
__device__ inline Kv4Span kv4_span(const Kv4Attention& a, int b, int row0, int n)
{
    Kv4Span s;
    s.length = clamp_count(a.lengths[b], a.capacity);
    s.count = a.counts ? clamp_count(a.counts[b], a.n_new) : a.n_new;
    const int i0 = kv4_query_of(a, row0);
    int i1 = kv4_query_of(a, row0 + n - 1);
    i1 = i1 < s.count ? i1 : s.count - 1;
    s.begin = 0;
    s.end = s.length;
    if (i0 >= s.count) s.end = 0;
    if (a.causal) {
        const int at = s.length - s.count;              // position of the first query
        s.end = s.end < at + i1 + 1 ? s.end : at + i1 + 1;
        if (a.window && at + i0 - a.window + 1 > 0) s.begin = at + i0 - a.window + 1;
    }
    if (s.end <= s.begin) s.begin = s.end = 0;
    return s;
}

template <int DIM, int G>
struct Kv4Tag {
    static constexpr int kDim = DIM, kGroup = G;
};
template <typename F>
int kv4_dispatch(const e0m4_kv4_shape& s, F&& f)
{
    switch (s.dim * 1000 + s.group) {
        case 64032: return f(Kv4Tag<64, 32>{});
        case 64064: return f(Kv4Tag<64, 64>{});
        case 128032: return f(Kv4Tag<128, 32>{});
        case 128064: return f(Kv4Tag<128, 64>{});
        case 128128: return f(Kv4Tag<128, 128>{});
        case 256032: return f(Kv4Tag<256, 32>{});
        case 256064: return f(Kv4Tag<256, 64>{});
        case 256128: return f(Kv4Tag<256, 128>{});
        default: return E0M4_ERR_SHAPE;
    }
}

int launch_kv4_append(void* cache, const e0m4_kv4_shape& s, const Kv4Rows& keys, const Kv4Rows& values, int dtype, int64_t n_new,
                      const int* starts, const int* counts, hipStream_t stream);
int launch_kv4_read(const void* cache, const e0m4_kv4_shape& s, const int* lengths, const int* first, int64_t rows, void* keys, void* values,
                    hipStream_t stream);
int launch_kv4_evict(const void* cache, const e0m4_kv4_shape& s, const float* received, const int* lengths, int budget, int recent,
                     void* small, const e0m4_kv4_shape& o, int* kept, int* lengths_out, float* received_out, hipStream_t stream);
// Attention: rows of queries in tiles of 16, a wavefront's tiles of the cache by itself; then, with several chunks, their sum.
constexpr int kKv4ShortTiles = 32;      // caches of so many tiles are one workgroup's
int launch_kv4_decode(const Kv4Attention& a, const e0m4_kv4_shape& s, hipStream_t stream);
// ... in workgroups of a.tile_rows rows (128; with dim 128 also 256), which share the dequantised rows of the cache.
constexpr int kKv4PrefillKeys = 64;
int launch_kv4_prefill(const Kv4Attention& a, const e0m4_kv4_shape& s, hipStream_t stream);
constexpr int kKv4MaxChunks = 2048;
// (received, unless null: the rows' weights from the scores, in the same launch)
int launch_kv4_combine(const Kv4Attention& a, const e0m4_kv4_shape& s, float* received, hipStream_t stream);
// received[j] += the weights of row j, from the rows' references and factors (norm)
int launch_kv4_received(const Kv4Attention& a, const e0m4_kv4_shape& s, float* received, hipStream_t stream);

}  // namespace e0m4
