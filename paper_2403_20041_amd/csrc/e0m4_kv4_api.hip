// C entries of the key/value cache in E0M4 codes: argument checks and the choice of kernels.  Every check happens on the host before
// anything is enqueued.
#include "e0m4_host.h"
#include "e0m4_kv4.h"

namespace e0m4 {

namespace {

constexpr int64_t kMaxCapacity = (int64_t)1 << 26, kMaxNew = (int64_t)1 << 20, kMaxGrid = 65535, kMaxShare = 1 << 10;
constexpr int64_t kMaxRows = (int64_t)1 << 38, kMaxSets = (int64_t)1 << 24;   // of all sequences and heads: their workgroups fit a grid

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

int check_kv4(const e0m4_kv4_shape* s)
{
    if (!s) return E0M4_ERR_NULL;
    if (s->batch < 0 || s->batch > kMaxGrid || s->kv_heads < 0 || s->kv_heads > kMaxGrid || s->capacity < 0 || s->capacity > kMaxCapacity)
        return E0M4_ERR_SHAPE;
    if (s->batch * s->kv_heads > kMaxSets || s->batch * s->kv_heads > kMaxRows / (s->capacity ? s->capacity : 1)) return E0M4_ERR_SHAPE;
    if (s->dim != 64 && s->dim != 128 && s->dim != 256) return E0M4_ERR_SHAPE;
    if ((s->group != 32 && s->group != 64 && s->group != 128) || s->group > s->dim) return E0M4_ERR_GROUP;
    return E0M4_OK;
}
bool empty(const e0m4_kv4_shape& s) { return s.batch == 0 || s.kv_heads == 0 || s.capacity == 0; }

// A view that the kernels read in 16-byte pieces.
int check_rows(const e0m4_kv4_rows* r)
{
    if (!r || !r->data) return E0M4_ERR_NULL;
    if (!aligned(r->data, 16)) return E0M4_ERR_ALIGN;
    if (((r->batch_ld | r->row_ld | r->head_ld) & 7) != 0) return E0M4_ERR_ALIGN;
    return E0M4_OK;
}
Kv4Rows view(const e0m4_kv4_rows& r) { return Kv4Rows{r.data, r.batch_ld, r.row_ld, r.head_ld}; }

size_t round16(size_t n) { return (n + 15) / 16 * 16; }

// How an attention call runs: the kernel, chunks of the cache, and what the workspace holds.
struct Plan {
    bool prefill, scores;
    int tile_rows, tile_keys, chunk_tiles, chunks;
    size_t out_bytes, stats_bytes, norm_bytes, scores_bytes, queries_bytes;
    size_t bytes() const { return out_bytes + stats_bytes + norm_bytes + scores_bytes + queries_bytes; }
};
// Chunks of the cache for many queries.  A workgroup of 128 rows takes 1.45 us for 64 rows of 128 dims alone on a compute unit and 2.1 beside
// another, one of 256 rows 2.1, the device 1.05 us for 128 rows when it is full.  Partial results go to memory and back and the launch
// that adds them takes 4 us at least.  32 heads on 2, us in 1, 2, 3, 4, 6 chunks (and by the estimate): 512 tokens behind 8000 rows
// 180, 113, 114, 102, 108 (193, 114, 117, 101, 111); 2048 tokens behind 14336 508, 561, 565, 586, 603.
int64_t prefill_chunks(const e0m4_kv4_shape& s, int64_t n_new, int64_t rows, int64_t sets, int tile_rows, int64_t units)
{
    const double unit = s.dim / 128.0, seen = n_new < s.capacity ? 1.0 - 0.5 * n_new / s.capacity : 0.5;
    const double full = sets * (tile_rows / 128) * units * seen * 1.05 * unit / 256;
    double best = 0;
    int64_t chunks = 1;
    for (int64_t c = 1; c <= 64 && c <= units; ++c) {
        const double chain = (double)((units + c - 1) / c) * (tile_rows == 256 || sets * c > 256 ? 2.1 : 1.45) * unit;
        const double time = (chain > full ? chain : full) + (c > 1 ? 4.0 + c * (double)rows * s.dim * 8 / 2.6e6 : 0.0);
        if (c == 1 || time < best) {
            best = time;
            chunks = c;
        }
    }
    return chunks;
}
// Everything here goes by the capacity, for the lengths are on the device: in caches much larger than their sequences, and under short
// windows, chunks are longer than the rows that there are would have them.  32 sequences of up to 8192 rows, 32 heads on 8, 47 us at
// that capacity, 62 and 95 at 4 and 16 times it; one of 701 rows 8.5, 11.8, 11.9; prompts 34, 33, 32.
Plan plan_attention(const e0m4_kv4_shape& s, int64_t heads, int64_t n_new, bool weights)
{
    Plan p;
    const int64_t rows = heads / s.kv_heads * n_new, all = s.batch * s.kv_heads * rows;
    const int force = knob(Knob::kv4_attention);
    // The kernel for few queries dequantises the cache again for every 16 rows of them, the other one shares it among 128, but has longer
    // chains and leaves a workgroup's missing rows idle.  8 sequences of 3000 rows and 8 heads, us of the two: 65 rows of queries 44
    // and 32, 97 rows 50 and 33; 8 of 500 rows and 8 heads, 129 rows of queries (9216 tiles taken) 16 and 18, 16 of them, 193 rows
    // (26624) 31 and 18; one of 16000 and 2 heads, 208 rows (13000) 26 and 23, of 3000 (2444) 13 and 15.  Up to 64 rows are the first
    // one's, which multiplies whole weights for fp16 results, though the other is the faster from about 33 on (31 and 26 us, 49 rows
    // 34 and 28).
    const int64_t taken = (s.capacity + kKv4Rows - 1) / kKv4Rows * s.batch * s.kv_heads * ((rows + 15) / 16);
    p.prefill = force ? force >= 2 : rows > 64 && taken > 12000;
    p.tile_keys = p.prefill ? kKv4PrefillKeys : kKv4Rows;
    const int64_t tiles = (s.capacity + p.tile_keys - 1) / p.tile_keys;
    auto sets = [&](int tile_rows) { return s.batch * s.kv_heads * ((rows + tile_rows - 1) / tile_rows); };
    int64_t chunk;
    if (p.prefill) {
        // 256 rows to a workgroup halve the dequantisation of 128, two workgroups of which a compute unit has at once: the larger ones where
        // they fill the device with like work (2048 tokens behind 14336, 508 us against 553), the smaller ones for prompts, whose rows
        // see from none to all of the others (1001 tokens of two sequences 33 against 37, 2048 tokens 55 against 62).
        p.tile_rows = s.dim == 128 && (force ? force == 3 : sets(256) >= 256 && 2 * n_new <= s.capacity) ? 256 : 128;
        const int64_t n = prefill_chunks(s, n_new, all, sets(p.tile_rows), p.tile_rows, tiles);
        chunk = (tiles + n - 1) / n;
    } else {
        // About three thousand workgroups, of eight tiles at least: shorter chunks spend their time on their beginnings, longer ones leave
        // compute units without work at the end (32 sequences of up to 256 tiles and 8 heads, 50 us in chunks of 8, 44 of 24, 50 of
        // 64; 16 of up to 126 tiles and a head of 256 dims 16.0 of 4, 15.2 of 8, 18.2 of 24).  Short caches are one workgroup's,
        // without a second launch for the sum: 22 tiles in 9.8 us, 14.3 in chunks.
        p.tile_rows = 16;
        chunk = tiles * sets(16) / 3072;
        if (chunk < 8) chunk = 8;
        if (tiles <= kKv4ShortTiles) chunk = tiles;
    }
    if (knob(Knob::kv4_chunk) > 0) chunk = knob(Knob::kv4_chunk);
    if (chunk < (tiles + kKv4MaxChunks - 1) / kKv4MaxChunks) chunk = (tiles + kKv4MaxChunks - 1) / kKv4MaxChunks;
    if (chunk > tiles) chunk = tiles;
    p.chunk_tiles = (int)chunk;
    p.chunks = (int)((tiles + chunk - 1) / chunk);
    p.scores = weights && !p.prefill && rows <= 16;
    p.out_bytes = p.chunks > 1 ? (size_t)p.chunks * all * s.dim * 4 : 0;
    p.stats_bytes = p.chunks > 1 ? round16((size_t)p.chunks * all * 8) : 0;
    p.norm_bytes = weights ? round16((size_t)all * 8) : 0;
    p.queries_bytes = weights && !p.scores ? (size_t)all * s.dim * 2 + round16((size_t)all * 4) : 0;
    p.scores_bytes = p.scores ? (size_t)all * kv4_tiles(s.capacity) * kKv4Rows * 4 : 0;
    return p;
}
int check_attention(const e0m4_kv4_shape* s, int64_t heads, int64_t n_new)
{
    const int rc = check_kv4(s);
    if (rc != E0M4_OK) return rc;
    if (heads < 0 || n_new < 0 || n_new > kMaxNew) return E0M4_ERR_SHAPE;
    if (s->kv_heads == 0 ? heads != 0 : heads % s->kv_heads != 0 || heads / s->kv_heads > kMaxShare || heads == 0) return E0M4_ERR_SHAPE;
    if (s->kv_heads && (heads / s->kv_heads * n_new > (int64_t)1 << 22 || s->batch * heads * n_new > (int64_t)1 << 32)) return E0M4_ERR_SHAPE;
    return E0M4_OK;
}

__global__ void kv4_zero_kernel(uint4* y, int64_t pieces)
{
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * blockDim.x) y[i] = uint4{0, 0, 0, 0};
}
int zero_fill(void* y, int64_t bytes, hipStream_t stream)
{
    const int64_t blocks = (bytes / 16 + 255) / 256;    // (a launch of 2^32 work items is refused)
    hipLaunchKernelGGL(kv4_zero_kernel, dim3((unsigned)(blocks < 65536 ? blocks : 65536)), dim3(256), 0, stream, static_cast<uint4*>(y), bytes / 16);
    return check_launch();
}

}  // namespace

}  // namespace e0m4

using namespace e0m4;

extern "C" {

size_t e0m4_kv4_bytes(const e0m4_kv4_shape* s)
{
    if (check_kv4(s) != E0M4_OK) return 0;
    return (size_t)s->batch * s->kv_heads * kv4_tiles(s->capacity) * kv4_tile_bytes(s->dim, s->group);
}

int e0m4_kv4_append(void* cache, const e0m4_kv4_shape* s, const e0m4_kv4_rows* keys, const e0m4_kv4_rows* values, int dtype, int64_t n_new,
                    const int32_t* starts, const int32_t* counts, void* stream)
{
    int rc = check_kv4(s);
    if (rc != E0M4_OK) return rc;
    if (n_new < 0 || n_new > kMaxCapacity || (dtype != E0M4_KV4_FP16 && dtype != E0M4_KV4_BF16)) return E0M4_ERR_SHAPE;
    if (empty(*s) || n_new == 0) return E0M4_OK;
    if (!cache || !starts) return E0M4_ERR_NULL;
    if ((rc = check_rows(keys)) != E0M4_OK || (rc = check_rows(values)) != E0M4_OK) return rc;
    if (!aligned(cache, 16) || !aligned(starts, 4) || !aligned(counts, 4)) return E0M4_ERR_ALIGN;
    return launch_kv4_append(cache, *s, view(*keys), view(*values), dtype, n_new, starts, counts, (hipStream_t)stream);
}

int e0m4_kv4_read(const void* cache, const e0m4_kv4_shape* s, const int32_t* lengths, const int32_t* first, int64_t rows, void* keys_f16,
                  void* values_f16, void* stream)
{
    const int rc = check_kv4(s);
    if (rc != E0M4_OK) return rc;
    if (rows < 0 || rows > kMaxCapacity) return E0M4_ERR_SHAPE;
    if (s->batch == 0 || s->kv_heads == 0 || rows == 0) return E0M4_OK;
    if ((!cache && s->capacity) || !lengths || !keys_f16 || !values_f16) return E0M4_ERR_NULL;
    if (!aligned(cache, 16) || !aligned(lengths, 4) || !aligned(first, 4) || !aligned(keys_f16, 16) || !aligned(values_f16, 16))
        return E0M4_ERR_ALIGN;
    return launch_kv4_read(cache, *s, lengths, first, rows, keys_f16, values_f16, (hipStream_t)stream);
}

size_t e0m4_kv4_attention_workspace_bytes(const e0m4_kv4_shape* s, int64_t heads, int64_t n_new, int with_weights)
{
    if (check_attention(s, heads, n_new) != E0M4_OK || empty(*s) || n_new == 0) return 0;
    return plan_attention(*s, heads, n_new, with_weights != 0).bytes();
}

int e0m4_kv4_attention(const e0m4_kv4_rows* queries, int dtype, int64_t heads, int64_t n_new, const void* cache, const e0m4_kv4_shape* s,
                       const int32_t* lengths, const int32_t* counts, int causal, int64_t window, const e0m4_kv4_mask* mask, float* weights,
                       void* out, void* workspace, size_t workspace_bytes, void* stream)
{
    int rc = check_attention(s, heads, n_new);
    if (rc != E0M4_OK) return rc;
    if (dtype != E0M4_KV4_FP16 && dtype != E0M4_KV4_BF16) return E0M4_ERR_SHAPE;
    if (window < 0 || (window > 0 && !causal)) return E0M4_ERR_SHAPE;
    if (mask && (mask->rows < 0 || mask->rows > kMaxCapacity)) return E0M4_ERR_SHAPE;
    if (s->batch == 0 || s->kv_heads == 0 || n_new == 0) return E0M4_OK;
    if (!out) return E0M4_ERR_NULL;
    if (!aligned(out, 16)) return E0M4_ERR_ALIGN;
    if (s->capacity == 0) return zero_fill(out, s->batch * n_new * heads * s->dim * 2, (hipStream_t)stream);
    if (!cache || !lengths || (mask && !mask->data && mask->rows)) return E0M4_ERR_NULL;
    if ((rc = check_rows(queries)) != E0M4_OK) return rc;
    if (!aligned(cache, 16) || !aligned(lengths, 4) || !aligned(counts, 4) || !aligned(weights, 4)) return E0M4_ERR_ALIGN;
    const Plan p = plan_attention(*s, heads, n_new, weights != nullptr);
    if (p.bytes() > 0) {
        if (!workspace) return E0M4_ERR_NULL;
        if (!aligned(workspace, 16)) return E0M4_ERR_ALIGN;
        if (workspace_bytes < p.bytes()) return E0M4_ERR_WORKSPACE;
    }
    Kv4Attention a = {};
    a.cache = static_cast<const uint8_t*>(cache);
    a.tiles = kv4_tiles(s->capacity);
    a.q = view(*queries);
    a.out = out;
    a.lengths = lengths;
    a.counts = counts;
    if (mask && mask->rows == 0) {                      // nothing is seen; any memory does for the address
        a.mask = static_cast<const uint8_t*>(cache);
    } else if (mask) {
        a.mask = static_cast<const uint8_t*>(mask->data);
        a.mask_batch_ld = mask->batch_ld;
        a.mask_row_ld = mask->row_ld;
        a.mask_rows = (int)mask->rows;
        a.mask_words = aligned(a.mask, 4) && ((mask->batch_ld | mask->row_ld | mask->rows) & 3) == 0;
    }
    a.batch = (int)s->batch;
    a.kv_heads = (int)s->kv_heads;
    a.share = (int)(heads / s->kv_heads);
    a.n_new = (int)n_new;
    a.share_inverse = a.share > 1 ? (uint32_t)((((uint64_t)1 << 32) + a.share - 1) / a.share) : 0;
    a.capacity = (int)s->capacity;
    a.window = window < s->capacity ? (int)window : 0;  // (one that is never left is none)
    a.causal = causal != 0;
    a.bf16 = dtype == E0M4_KV4_BF16;
    a.chunk_tiles = p.chunk_tiles;
    a.chunks = p.chunks;
    a.tile_rows = p.tile_rows;
    a.tile_keys = p.tile_keys;
    char* w = static_cast<char*>(workspace);
    a.part_out = reinterpret_cast<float*>(w);
    a.part_stats = reinterpret_cast<float2*>(w + p.out_bytes);
    a.norm = weights ? reinterpret_cast<float2*>(w + p.out_bytes + p.stats_bytes) : nullptr;
    if (p.queries_bytes) {
        a.packed_q = reinterpret_cast<half_t*>(w + p.out_bytes + p.stats_bytes + p.norm_bytes);
        a.factors = reinterpret_cast<float*>(a.packed_q + (size_t)a.batch * heads * n_new * s->dim);
    }
    a.scores = p.scores ? reinterpret_cast<float*>(w + p.out_bytes + p.stats_bytes + p.norm_bytes) : nullptr;
    rc = p.prefill ? launch_kv4_prefill(a, *s, (hipStream_t)stream) : launch_kv4_decode(a, *s, (hipStream_t)stream);
    if (rc == E0M4_OK && (a.chunks > 1 || p.scores)) rc = launch_kv4_combine(a, *s, p.scores ? weights : nullptr, (hipStream_t)stream);
    if (rc == E0M4_OK && weights && !p.scores) rc = launch_kv4_received(a, *s, weights, (hipStream_t)stream);
    return rc;
}

int e0m4_kv4_evict(const void* cache, const e0m4_kv4_shape* s, const float* received, const int32_t* lengths, int64_t budget, int64_t recent,
                   void* small, const e0m4_kv4_shape* o, int32_t* kept, int32_t* lengths_out, float* received_out, void* stream)
{
    int rc = check_kv4(s);
    if (rc != E0M4_OK || (rc = check_kv4(o)) != E0M4_OK) return rc;
    if (o->batch != s->batch || o->kv_heads != s->kv_heads || o->dim != s->dim || o->group != s->group) return E0M4_ERR_SHAPE;
    if (budget < 1 || budget > o->capacity || recent < 0 || recent > budget) return E0M4_ERR_SHAPE;
    if (s->batch == 0 || s->kv_heads == 0) return E0M4_OK;
    if (!small || !lengths || !kept || !lengths_out || !received_out || ((!cache || !received) && s->capacity)) return E0M4_ERR_NULL;
    if (!aligned(cache, 16) || !aligned(small, 16) || !aligned(received, 4) || !aligned(lengths, 4) || !aligned(kept, 4) ||
        !aligned(lengths_out, 4) || !aligned(received_out, 4))
        return E0M4_ERR_ALIGN;
    const uintptr_t c0 = reinterpret_cast<uintptr_t>(cache), c1 = reinterpret_cast<uintptr_t>(small);
    if (c0 < c1 + e0m4_kv4_bytes(o) && c1 < c0 + e0m4_kv4_bytes(s)) return E0M4_ERR_SHAPE;     // rows move while others are read
    return launch_kv4_evict(cache, *s, received, lengths, (int)budget, (int)recent, small, *o, kept, lengths_out, received_out,
                            (hipStream_t)stream);
}

}  // extern "C"
