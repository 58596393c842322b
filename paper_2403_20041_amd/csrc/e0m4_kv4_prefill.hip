// Attention of many queries over a cache in E0M4 codes.  Layout: e0m4_kv4.h; softmax: e0m4_kv4_attention.h.
//
// A workgroup takes 32 rows of queries per wavefront through the cache, 64 rows of it at a time: its threads dequantise them once for
// all, from registers that were loaded an iteration ahead, into the LDS buffer that the next iteration reads, and every wavefront
// multiplies what the present one holds.  S^T = K Q^T and O^T = V^T P^T in 32 x 32 x 16 products: a lane has one query (column) in
// both, so the softmax's state is its own, and P goes from the accumulators into the second product as it is.  For that K's rows are
// read in the order that gives a lane the rows of V's octets: accumulator 4 a + i of lane half kh is row 16 (a & 1) + 4 (2 (a >> 1) + kh)
// + i of a tile of 32, slot 4 (a & 1) + i of octet 2 (a >> 1) + kh.
//
// Bound: 32 products of 32 cycles and about 330 cycles of other instructions (four each, exponentials sixteen) per wavefront and 64
// rows share a SIMD between two wavefronts; 32 heads on 2, 2048 tokens behind 14336 rows take 513 us, 1004 TFLOP/s (a large library product:
// 1147), once some tens of passes have settled the clock, and 590 to 630 in the first ones.  Prompts are bound by the rows that see
// most: 64 rows of the cache follow each other every 1.4 to 2.1 us there.
//
// What the rounding of P to fp16 leaves is not multiplied here.  With a second product for it those 513 us are 720 and two prompts of
// 1001 tokens 46 instead of 37, for an error of fp16 results against 64 bits of 2.1e-4 (their own rounding) instead of 2.7e-4;
// bfloat16 results do not change (1.67e-3).
#include "e0m4_kv4_attention.h"

namespace e0m4 {

namespace {

constexpr int kKeys = kKv4PrefillKeys;  // rows of the cache per iteration

// One 16-byte piece of a tile's codes and its parameters, between memory and LDS.  A thread has pieces of K or of V: the wavefronts load
// what either needs, so that no branch stands between a load and its use an iteration later.
template <int DIM, int G>
struct Piece {
    static constexpr int kParts = G == 32 ? 2 : 1;      // groups of a piece of V
    static constexpr int kRows = DIM == 64 ? 2 : 1;     // rows of a piece of K
    words4_t code;
    words4_t scale[kParts], bias[kParts];               // of V
    uint32_t param[kRows];                              // of K
};

template <int DIM, int G, int WAVES>
__global__ __launch_bounds__(WAVES * 64, DIM == 256 ? 1 : 2) void kv4_prefill_kernel(Kv4Attention a)
{
    using L = Kv4<DIM, G>;
    constexpr int kThreads = WAVES * 64, kRows = WAVES * 32, kSteps = DIM / 16, kDimTiles = DIM / 32;
    constexpr int kKStride = DIM + 8, kVStride = kKeys + 8;                 // halves; the odd 16 bytes spread a column over the banks
    constexpr int kBuffer = kKeys * kKStride + DIM * kVStride;
    constexpr int kPieces = 4 * DIM / kThreads;                             // 64 rows of K, then of V, dealt to the threads
    static_assert(4 * DIM % kThreads == 0, "pieces per thread");
    constexpr int kBlocks = DIM >= 128 ? DIM / 128 : 1;
    constexpr bool kWhole = 2 * DIM % kThreads == 0;                        // a thread's first half are K's: known at compile time
    extern __shared__ __attribute__((aligned(16))) half_t buffer[];         // [2][K, V]
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), col = lane & 31, kh = lane >> 5;
    const int rows = a.n_new * a.share;
    // of all sequences and heads the rows that see most first
    const int h = blockIdx.x % a.kv_heads, b = blockIdx.y, place = kv4_place(a), chunk = place % a.chunks;
    const int block_row = ((rows + kRows - 1) / kRows - 1 - place / a.chunks) * kRows;
    if (block_row < 0) return;
    const int block_rows = rows - block_row < kRows ? rows - block_row : kRows;
    const Kv4Span span = kv4_span(a, b, block_row, block_rows);
    const int unit0 = span.begin / kKeys + chunk * a.chunk_tiles, units_end = (span.end + kKeys - 1) / kKeys;
    const int unit1 = unit0 + a.chunk_tiles < units_end ? unit0 + a.chunk_tiles : units_end;
    const int row = block_row + wave * 32 + col, query = kv4_query_of(a, row), at = span.length - span.count + query;
    const bool valid = row < rows && query < span.count;
    half8_t q[kSteps];
    const float factor = load_query_row<DIM, kSteps, 32>(a, b, h, valid ? row : 0, valid, 8 * kh, 16, q);
    if (a.packed_q && chunk == 0 && row < rows)
        keep_query_row<kSteps>(a, ((int64_t)b * a.kv_heads + h) * rows + row, DIM, valid, 8 * kh, 16, q, factor);
    if (unit0 >= unit1 && a.chunks > 1) return;
    const Kv4Seen by_place = kv4_seen(a, span.length, at);
    // this wavefront's rows: what some of them see, and what all of them see by position
    const int wave_row = block_row + wave * 32, wave_rows = rows - wave_row < 32 ? rows - wave_row : 32;
    Kv4Span own = {span.length, span.count, 0, 0};
    int all_from = 0, all_to = span.length;
    if (wave_rows > 0) {
        own = kv4_span(a, b, wave_row, wave_rows);
        const int i0 = kv4_query_of(a, wave_row), i1 = kv4_query_of(a, wave_row + wave_rows - 1), first = span.length - span.count;
        if (a.window) all_from = first + (i1 < span.count ? i1 : span.count - 1) - a.window + 1;
        if (a.causal) all_to = first + i0 + 1;
    }

    const uint8_t* cache = a.cache + ((int64_t)b * a.kv_heads + h) * a.tiles * L::kBytes;
    const uint32_t hi = frac_mask_vgpr(), lo = frac_mask_low_vgpr();
    Piece<DIM, G> piece[kPieces];
    // piece i of the thread: piece `id % DIM` of K (id < 2 DIM) or V of tile `id / DIM % 2` of the unit
    auto load = [&](int unit) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int id = (wave + i * WAVES) * 64, sub = id / DIM % 2, at_piece = id % DIM + lane;
            const bool is_v = kWhole ? i >= kPieces / 2 : id >= 2 * DIM;
            const int64_t tile = 2 * (int64_t)unit + sub;
            const __amdgpu_buffer_rsrc_t rs = rsrc_if(cache + tile * L::kBytes, unit < unit1 && tile < a.tiles);
            const int kq = (at_piece >> 4) & 3, block = at_piece >> 6;
            Piece<DIM, G>& p = piece[i];
            p.code = load16(rs, at_piece * 16 + (is_v ? L::kVCodes : 0));
            if (!kWhole || !is_v) {
                const int c = DIM == 64 ? 0 : block % kBlocks, s = DIM == 64 ? 0 : block / kBlocks;
                const int param = L::kKParams + (((kq * L::kLaneDims + 32 * c) / G) * kKv4Rows + 16 * s + (at_piece & 15)) * 4;
#pragma unroll
                for (int e = 0; e < Piece<DIM, G>::kRows; ++e) p.param[e] = __builtin_amdgcn_raw_buffer_load_b32(rs, param + 64 * e, 0, 0);
            }
            if (!kWhole || is_v) {
#pragma unroll
                for (int e = 0; e < Piece<DIM, G>::kParts; ++e) {
                    const int param = L::kVParams + ((block * 64 + 32 * e) / G) * 128 + kq * 16;
                    p.scale[e] = load16(rs, param);
                    p.bias[e] = load16(rs, param + 64);
                }
            }
        }
    };
    auto store = [&](int unit, half_t* into) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int id = (wave + i * WAVES) * 64, sub = id / DIM % 2, at_piece = id % DIM + lane;
            const bool is_v = kWhole ? i >= kPieces / 2 : id >= 2 * DIM;
            const int kq = (at_piece >> 4) & 3, block = at_piece >> 6;
            Piece<DIM, G>& p = piece[i];
            if (!is_v) {
                const int c = DIM == 64 ? 0 : block % kBlocks, s = DIM == 64 ? 0 : block / kBlocks;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int r = sub * 32 + 16 * (DIM == 64 ? w >> 1 : s) + (at_piece & 15);
                    const int d = kq * L::kLaneDims + (DIM == 64 ? 8 * (w & 1) : 32 * c + 8 * w);
                    *reinterpret_cast<half8_t*>(into + r * kKStride + d) = kv4_values(p.code[w], p.param[DIM == 64 ? w >> 1 : 0], hi, lo);
                }
            } else {
                const int r0 = unit * kKeys + sub * 32;
                if (r0 + 32 > span.length) {            // rows that were perhaps never written: 0 * NaN is NaN
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const uint32_t m = (r0 + L::row_of(kq, 2 * j) < span.length ? 0xFFFFu : 0u) |
                                           (r0 + L::row_of(kq, 2 * j + 1) < span.length ? 0xFFFF0000u : 0u);
#pragma unroll
                        for (int e = 0; e < Piece<DIM, G>::kParts; ++e) {
                            p.scale[e][j] &= m;
                            p.bias[e][j] &= m;
                        }
                    }
                }
                half_t* v = into + kKeys * kKStride + (block * 64 + (at_piece & 15)) * kVStride + (sub * 4 + kq) * 8;
#pragma unroll
                for (int w = 0; w < 4; ++w) {
                    const int e = Piece<DIM, G>::kParts == 2 ? w >> 1 : 0;
                    *reinterpret_cast<half8_t*>(v + 16 * w * kVStride) = kv4_values_v(p.code[w], kv4_octet_params(p.scale[e], p.bias[e]), hi, lo);
                }
            }
        }
    };

    floatx16 o[kDimTiles];
#pragma unroll
    for (int d = 0; d < kDimTiles; ++d)
#pragma unroll
        for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
    float ref = -kInf, sum = 0.f;
    const int key_row = (col & 7) | ((col >> 1) & 8) | ((col << 1) & 16);   // (bits 3 and 4 change places)

    load(unit0);
    store(unit0, buffer);
    load(unit0 + 1);
    for (int unit = unit0; unit < unit1; ++unit) {
        __syncthreads();
        const half_t* k = buffer + (unit - unit0) % 2 * kBuffer;
        if (unit + 1 < unit1) store(unit + 1, buffer + (unit + 1 - unit0) % 2 * kBuffer);
        load(unit + 2);
        const int r0 = unit * kKeys;
        if (r0 >= own.end || r0 + kKeys <= own.begin) continue;
        floatx16 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[u][i] = 0.f;
#pragma unroll
        for (int w = 0; w < kSteps; ++w)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                const half8_t kk = *reinterpret_cast<const half8_t*>(k + (32 * u + key_row) * kKStride + 16 * w + 8 * kh);
                s[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(kk, q[w], s[u], 0, 0, 0);
            }
        // operands are read kAhead products before their own
        __builtin_amdgcn_sched_group_barrier(kDsRead, kAhead, 0);
#pragma unroll
        for (int i = 0; i < 2 * kSteps - kAhead; ++i) {
            __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
            __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kMfma, kAhead, 0);
        auto row_of = [&](int u, int i) { return r0 + 32 * u + 16 * ((i >> 2) & 1) + 8 * (i >> 3) + 4 * kh + (i & 3); };
        if (a.mask) {
            const uint32_t seen = kv4_mask_bits<8>(a, b, valid ? query : 0, [&](int g) { return r0 + 32 * (g >> 2) + 16 * (g & 1) + 8 * ((g >> 1) & 1) + 4 * kh; });
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[u][i] = (seen >> (16 * u + i)) & 1 ? s[u][i] : -kInf;
        }
        if (r0 < all_from || r0 + kKeys > all_to) {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) s[u][i] = row_of(u, i) >= by_place.from && row_of(u, i) < by_place.to ? s[u][i] : -kInf;
        }
        float top = fmaxf(s[0][0], s[1][0]);
#pragma unroll
        for (int i = 1; i < 16; ++i) top = fmaxf(fmaxf(top, s[0][i]), s[1][i]);
        top *= factor;
        if (__any(top > ref + kSlack)) {
            top = fmaxf(top, __shfl_xor(top, 32));
            const float now = fmaxf(ref, top);
            const float down = now == -kInf ? 1.f : __builtin_amdgcn_exp2f(ref - now);
            ref = now;
            sum *= down;
#pragma unroll
            for (int d = 0; d < kDimTiles; ++d) o[d] *= down;
        }
        const float minus = ref == -kInf ? 0.f : kShift - ref;
        // P of 16 rows and the product before it side by side
        half8_t p, vv[2][kDimTiles];
        auto read_v = [&](int w) {
#pragma unroll
            for (int d = 0; d < kDimTiles; ++d)
                vv[w & 1][d] = *reinterpret_cast<const half8_t*>(k + kKeys * kKStride + (32 * d + col) * kVStride + (2 * w + kh) * 8);
        };
        auto weights = [&](int w) {
            half8_t r;
            float e[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                e[i] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[w >> 1][8 * (w & 1) + i], factor, minus));
                r[i] = (half_t)e[i];
            }
            sum += ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
            return r;
        };
        read_v(0);
        p = weights(0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            half8_t next;
            if (w < 3) {
                read_v(w + 1);
                next = weights(w + 1);
            }
#pragma unroll
            for (int d = 0; d < kDimTiles; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(vv[w & 1][d], p, o[d], 0, 0, 0);
            if (w < 3) {
                __builtin_amdgcn_sched_group_barrier(kDsRead, kDimTiles, 0);
#pragma unroll
                for (int d = 0; d < kDimTiles; ++d) {
                    __builtin_amdgcn_sched_group_barrier(kMfma, 1, 0);
                    __builtin_amdgcn_sched_group_barrier(kValu, 20 / kDimTiles, 0);
                    __builtin_amdgcn_sched_group_barrier(kTrans, 8 / kDimTiles, 0);
                }
                p = next;
            }
            __builtin_amdgcn_sched_barrier(0);
        }
    }
    sum += __shfl_xor(sum, 32);
    if (row >= rows) return;
    const int64_t bh = (int64_t)b * a.kv_heads + h, at_row = (((int64_t)chunk * a.batch * a.kv_heads) + bh) * rows + row;
    if (a.chunks > 1) {
#pragma unroll
        for (int d = 0; d < kDimTiles; ++d)
#pragma unroll
            for (int i = 0; i < 4; ++i)
                *reinterpret_cast<floatx4*>(a.part_out + at_row * DIM + 32 * d + 8 * i + 4 * kh) =
                    floatx4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
        if (kh == 0) a.part_stats[at_row] = float2{ref, sum};
        return;
    }
#pragma unroll
    for (int d = 0; d < kDimTiles; ++d)
#pragma unroll
        for (int i = 0; i < 4; ++i)
            finish<DIM>(a, b, h, row, 32 * d + 8 * i + 4 * kh, query < span.count,
                        floatx4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]}, ref, sum);
}

template <int DIM, int G, int WAVES>
int launch_prefill(const Kv4Attention& a, dim3 grid, hipStream_t stream)
{
    constexpr int kLds = 2 * (kKeys * (DIM + 8) + DIM * (kKeys + 8)) * 2;
    static std::atomic<uint64_t> allowed{0};
    const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(&kv4_prefill_kernel<DIM, G, WAVES>), kLds, allowed);
    if (rc != E0M4_OK) return rc;
    hipLaunchKernelGGL((kv4_prefill_kernel<DIM, G, WAVES>), grid, dim3(WAVES * 64), kLds, stream, a);
    return check_launch();
}

}  // namespace


int launch_kv4_prefill(const Kv4Attention& a, const e0m4_kv4_shape& s, hipStream_t stream)
{
    const int64_t rows = (int64_t)a.n_new * a.share, blocks = (rows + a.tile_rows - 1) / a.tile_rows;
    const dim3 grid = kv4_place_grid(a, blocks * a.chunks);
    return kv4_dispatch(s, [&](auto shape) -> int {
        constexpr int DIM = decltype(shape)::kDim, G = decltype(shape)::kGroup;
        if constexpr (DIM == 128)
            if (a.tile_rows == 256) return launch_prefill<DIM, G, 8>(a, grid, stream);
        return launch_prefill<DIM, G, 4>(a, grid, stream);
    });
}

}  // namespace e0m4
