// Low-rank adapters of rows (e0m4_lora): out[m] = base[m] + f[a] * B[a] (A[a] x[m]) with a the adapter that row m has chosen.
//
// Two launches over tiles of rows of one adapter (see e0m4_groups.h).  The first, H = X A^T: a workgroup's four wavefronts take 128-k chunks
// in turn, read rows of X and of A as the matrix cores take them and add their sums in LDS; few tiles are split along K over workgroups,
// each with a slab of its own.  The second, out = base + f H B^T: H is added up over the slabs in order and split into the sum of two 16-bit numbers (fp16
// after scaling its row by a power of two: 22 bits, bfloat16: 16), so that its rounding is far below that of the output; a wavefront has the rows of
// the tile and 64 columns at a time, of which a lane holds 16 neighbours of one row.
// What bounds it: memory, X once, base and out once, A and B of the adapters in use once (and from L2 for every further tile).
#include "e0m4_groups.h"

#include <algorithm>
#include <type_traits>

namespace e0m4 {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kWavesL = 4, kThreadsL = kWavesL * 64;
constexpr int kChunkK = 128;                    // k of a wavefront's turn
constexpr uint32_t kNowhere = 0x80000000u;      // beyond a buffer's end, whatever is added to it

struct LoraKernelArgs {
    const char* X;
    uint32_t x_ld;                              // bytes
    const GroupTile* tiles;
    const int* tile_count;
    const int* offsets;
    const int* order;
    int64_t rows;
    int adapters;
    const char* A;
    const char* B;
    int rank;
    const float* factors;
    int64_t N;
    uint32_t K;
    const char* base;
    int64_t base_ld;                            // bytes
    char* out;
    int64_t out_ld;                             // bytes
    float* H;                                   // [splits][rows][rank]
    int splits;
    uint32_t columns;                           // workgroups of a tile, second launch
    uint32_t tile_grid;                         // workgroups for tiles, second launch
};

template <bool BF>
__device__ inline floatx4 mfma16(const half8_t& a, const half8_t& b, const floatx4& v)
{
    if constexpr (BF) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), v, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, v, 0, 0, 0);
}

// H of a tile: MT times 16 rows, NT times 16 of the rank.  Lane (n = l%16, q = l/16) supplies A[16 j + n] and X[row 16 i + n] at k = 8 q ..
// + 7 of every step of 32, and holds H[row 16 i + n][16 j + 4 q ... + 3].
template <bool BF, int MT, int NT>
__global__ __launch_bounds__(kThreadsL, 2) void lora_shrink_kernel(LoraKernelArgs a)
{
    // steps of 32 k whose operands are requested together: as many as a hundred registers hold
    constexpr int U = (MT + NT) <= 6 ? 4 : (MT + NT) <= 12 ? 2 : 1;
    __shared__ __attribute__((aligned(16))) floatx4 red[kWavesL - 1][MT * NT][64];
    const uint32_t tile_no = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x / (uint32_t)a.splits)), split = blockIdx.x - tile_no * a.splits;
    if ((int)tile_no >= a.tile_count[0]) return;
    const GroupTile tile = a.tiles[tile_no];
    const int first = tile.begin + ((int)tile_no - tile.first_tile) * (16 * MT);
    const int M = min(16 * MT, tile.end - first);
    const int lane = threadIdx.x & 63, n_l = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const __amdgpu_buffer_rsrc_t x_rsrc = make_rsrc(a.X), a_rsrc = make_rsrc(a.A + (int64_t)tile.group * a.rank * a.K * 2);
    uint32_t x_off[MT], a_off[NT];
#pragma unroll
    for (int i = 0; i < MT; ++i) x_off[i] = 16 * i + n_l < M ? (uint32_t)a.order[first + 16 * i + n_l] * a.x_ld + (uint32_t)q * 16 : kNowhere;
#pragma unroll
    for (int j = 0; j < NT; ++j) a_off[j] = 16 * j + n_l < a.rank ? (uint32_t)(16 * j + n_l) * (a.K * 2) + (uint32_t)q * 16 : kNowhere;
    floatx4 acc[NT][MT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[j][i] = floatx4{0.f, 0.f, 0.f, 0.f};
    const int chunks = (int)((a.K + kChunkK - 1) / kChunkK);
    for (int ch = wave + kWavesL * (int)split; ch < chunks; ch += kWavesL * a.splits) {
#pragma unroll
        for (int s0 = 0; s0 < 4; s0 += U) {
            half8_t x[U][MT], w[U][NT];
#pragma unroll
            for (int s = 0; s < U; ++s) {
                const uint32_t k0 = (uint32_t)(ch * kChunkK + (s0 + s) * 32), out = k0 + q * 8 >= a.K ? kNowhere : 0u;
#pragma unroll
                for (int i = 0; i < MT; ++i) x[s][i] = __builtin_bit_cast(half8_t, __builtin_amdgcn_raw_buffer_load_b128(x_rsrc, (int)(x_off[i] | out), (int)(k0 * 2), 0));
#pragma unroll
                for (int j = 0; j < NT; ++j) w[s][j] = __builtin_bit_cast(half8_t, __builtin_amdgcn_raw_buffer_load_b128(a_rsrc, (int)(a_off[j] | out), (int)(k0 * 2), 0));
            }
#pragma unroll
            for (int s = 0; s < U; ++s)
#pragma unroll
                for (int j = 0; j < NT; ++j)
#pragma unroll
                    for (int i = 0; i < MT; ++i) acc[j][i] = mfma16<BF>(w[s][j], x[s][i], acc[j][i]);
        }
    }
    // the wavefronts' sums in order
    if (wave > 0) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < MT; ++i) red[wave - 1][j * MT + i][lane] = acc[j][i];
    }
    __syncthreads();
    if (wave > 0) return;
    float* h = a.H + ((int64_t)split * a.rows + first) * a.rank;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            floatx4 v = acc[j][i];
#pragma unroll
            for (int w = 0; w < kWavesL - 1; ++w) v += red[w][j * MT + i][lane];
            const int r = 16 * j + 4 * q, m = 16 * i + n_l;
            if (m < M && r < a.rank) *reinterpret_cast<floatx4*>(h + (int64_t)m * a.rank + r) = v;       // (the rank is a multiple of 8)
        }
    }
}

// base + f H B^T for a tile and 64 columns of a wavefront at a time; NT times 16 of the rank.  MFMA operands: the row of B in lane (n, q) of the j-th of four
// MFMAs is column 16 (n/4) + 4 j + n%4, so that a lane's results, 4 q .. + 3 of each, are the columns 16 q .. + 15 of row n; its 32 values of "k" are
// the 16 of the rank as the upper parts of H (q 0, 1), then the same as the lower parts (q 2, 3).
template <bool BF, int MT, int NT>
__global__ __launch_bounds__(kThreadsL, 2) void lora_expand_kernel(LoraKernelArgs a)
{
    typedef std::conditional_t<BF, __bf16, half_t> T;
    typedef T T8 __attribute__((ext_vector_type(8)));
    const int lane = threadIdx.x & 63, n_l = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (blockIdx.x >= a.tile_grid) {                    // rows without an adapter keep their base
        const int total = a.offsets[a.adapters];
        const int64_t pieces = a.N / 8;
        for (int64_t r = total + (int64_t)(blockIdx.x - a.tile_grid); r < a.rows; r += gridDim.x - a.tile_grid) {
            const int64_t row = a.order[r];
            for (int64_t p = threadIdx.x; p < pieces; p += kThreadsL) {
                u32x4 v = {0, 0, 0, 0};
                if (a.base) v = *reinterpret_cast<const u32x4*>(a.base + row * a.base_ld + p * 16);
                *reinterpret_cast<u32x4*>(a.out + row * a.out_ld + p * 16) = v;
            }
        }
        return;
    }
    const uint32_t tile_no = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x / a.columns)), part = blockIdx.x - tile_no * a.columns;
    if ((int)tile_no >= a.tile_count[0]) return;
    const GroupTile tile = a.tiles[tile_no];
    const int first = tile.begin + ((int)tile_no - tile.first_tile) * (16 * MT);
    const int M = min(16 * MT, tile.end - first);
    const float factor = a.factors ? a.factors[tile.group] : 1.f;
    int64_t row[MT];
    half8_t h[NT][MT];
    float scale[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) {
        const int m = 16 * i + n_l;
        row[i] = m < M ? a.order[first + m] : -1;
        float v[NT][8];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            const int r = 16 * j + 8 * (q & 1);
            floatx4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
            if (m < M && r < a.rank) {
                const float* src = a.H + (int64_t)(first + m) * a.rank + r;
                lo = *reinterpret_cast<const floatx4*>(src);
                hi = *reinterpret_cast<const floatx4*>(src + 4);
                for (int s = 1; s < a.splits; ++s) {
                    lo += *reinterpret_cast<const floatx4*>(src + (int64_t)s * a.rows * a.rank);
                    hi += *reinterpret_cast<const floatx4*>(src + (int64_t)s * a.rows * a.rank + 4);
                }
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[j][e] = lo[e];
                v[j][4 + e] = hi[e];
            }
        }
        // fp16: the row's largest magnitude is scaled into [1/2, 1) (powers of two: exact).  A row that holds an infinity or NaN is used as it is.
        scale[i] = factor;
        float down = 1.f;
        if constexpr (!BF) {
            float most = 0.f;
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(v[j][e]));
            most = fmaxf(most, __shfl_xor(most, 16));
            if (most > 0.f && most < INFINITY) {
                const int exponent = min(max(__builtin_amdgcn_frexp_expf(most), -126), 126);
                down = __builtin_amdgcn_ldexpf(1.f, -exponent);
                scale[i] = factor * __builtin_amdgcn_ldexpf(1.f, exponent);
            }
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            T8 part16;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float x = v[j][e] * down;
                const T upper = (T)x;
                const float rest = x - (float)upper;
                part16[e] = q < 2 ? upper : fabsf((float)upper) < INFINITY ? (T)rest : (T)0.f;
            }
            h[j][i] = __builtin_bit_cast(half8_t, part16);
        }
    }
    const char* adapter = a.B + (int64_t)tile.group * a.N * a.rank * 2;
    const int64_t step = (int64_t)a.columns * kWavesL * 64;
    for (int64_t c0 = ((int64_t)part * kWavesL + wave) * 64; c0 < a.N; c0 += step) {
        const int64_t col = c0 + 16 * q;                // this lane's results: columns col .. col + 15 of its rows
        u32x4 b[MT][2];
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                b[i][p] = u32x4{0, 0, 0, 0};
                if (a.base && row[i] >= 0 && col + 8 * p < a.N) b[i][p] = *reinterpret_cast<const u32x4*>(a.base + row[i] * a.base_ld + (col + 8 * p) * 2);
            }
        floatx4 acc[4][MT];
#pragma unroll
        for (int j4 = 0; j4 < 4; ++j4)
#pragma unroll
            for (int i = 0; i < MT; ++i) acc[j4][i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            half8_t w[4];
            const int r = 16 * j + 8 * (q & 1);
#pragma unroll
            for (int j4 = 0; j4 < 4; ++j4) {
                const int64_t n = c0 + 16 * (n_l >> 2) + 4 * j4 + (n_l & 3);
                w[j4] = half8_t{0, 0, 0, 0, 0, 0, 0, 0};
                if (n < a.N && r < a.rank) w[j4] = *reinterpret_cast<const half8_t*>(adapter + (n * a.rank + r) * 2);
            }
#pragma unroll
            for (int j4 = 0; j4 < 4; ++j4)
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[j4][i] = mfma16<BF>(w[j4], h[j][i], acc[j4][i]);
        }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const T8 from = __builtin_bit_cast(T8, b[i][p]);
                T8 o;
#pragma unroll
                for (int e = 0; e < 8; ++e) o[e] = (T)__builtin_fmaf(scale[i], acc[2 * p + e / 4][i][e % 4], (float)from[e]);
                if (row[i] >= 0 && col + 8 * p < a.N) *reinterpret_cast<u32x4*>(a.out + row[i] * a.out_ld + (col + 8 * p) * 2) = __builtin_bit_cast(u32x4, o);
            }
        }
    }
}

struct LoraPlan {
    int height_index;                           // tiles of 16 << this rows
    int splits;
    uint32_t columns;
    int64_t tiles;
};
LoraPlan plan_lora(int64_t rows, int64_t adapters, int rank, int64_t N, int64_t K)
{
    LoraPlan p;
    const int64_t each = rows / std::max<int64_t>(1, std::min(adapters, rows));        // rows of an adapter, if all are in use
    p.height_index = each <= 16 ? 0 : each <= 64 || rank > 64 ? 1 : 2;      // (64 rows of a rank of 128 do not fit the registers)
    p.tiles = most_tiles(rows, adapters, tile_height(p.height_index));
    const int64_t chunks = (K + kChunkK - 1) / kChunkK;
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({512 / std::max<int64_t>(p.tiles, 1), (chunks + kWavesL - 1) / kWavesL, 8}));
    const int64_t parts = (N + kWavesL * 64 - 1) / (kWavesL * 64);
    p.columns = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(parts, (1024 + p.tiles - 1) / std::max<int64_t>(p.tiles, 1)));
    return p;
}

template <bool BF, int MT, int NT>
int launch_lora_as(LoraKernelArgs a, const LoraPlan& p, bool copy, hipStream_t stream)
{
    const int64_t shrink = p.tiles * p.splits;
    a.tile_grid = (uint32_t)(p.tiles * p.columns);
    const int64_t expand = (int64_t)a.tile_grid + (copy ? std::min<int64_t>(a.rows, 256) : 0);
    if (shrink * kThreadsL > 0xffffffffLL || p.tiles * p.columns * kThreadsL > 0xf0000000LL) return E0M4_ERR_SHAPE;
    hipLaunchKernelGGL((lora_shrink_kernel<BF, MT, NT>), dim3((unsigned)shrink), dim3(kThreadsL), 0, stream, a);
    const int rc = check_launch();
    if (rc != E0M4_OK) return rc;
    hipLaunchKernelGGL((lora_expand_kernel<BF, MT, NT>), dim3((unsigned)expand), dim3(kThreadsL), 0, stream, a);
    return check_launch();
}

template <bool BF, int MT>
int launch_lora_rank(const LoraKernelArgs& a, const LoraPlan& p, bool copy, hipStream_t stream)
{
    if (a.rank <= 16) return launch_lora_as<BF, MT, 1>(a, p, copy, stream);
    if (a.rank <= 32) return launch_lora_as<BF, MT, 2>(a, p, copy, stream);
    if (a.rank <= 64) return launch_lora_as<BF, MT, 4>(a, p, copy, stream);
    if constexpr (MT <= 2) return launch_lora_as<BF, MT, 8>(a, p, copy, stream);
    else return E0M4_ERR_SHAPE;
}

template <bool BF>
int launch_lora_rows(const LoraKernelArgs& a, const LoraPlan& p, bool copy, hipStream_t stream)
{
    switch (p.height_index) {
        case 0: return launch_lora_rank<BF, 1>(a, p, copy, stream);
        case 1: return launch_lora_rank<BF, 2>(a, p, copy, stream);
        default: return launch_lora_rank<BF, 4>(a, p, copy, stream);
    }
}

}  // namespace

size_t lora_workspace_bytes(int64_t rows, int64_t adapters, int rank, int64_t N, int64_t K)
{
    return (size_t)plan_lora(rows, adapters, rank, N, K).splits * (size_t)rows * (size_t)rank * 4;
}

int launch_lora(const LoraArgs& l, void* workspace, hipStream_t stream)
{
    const LoraPlan p = plan_lora(l.rows, l.adapters, l.rank, l.N, l.K);
    const GroupPlan plan = plan_view(l.plan, l.rows, l.adapters);
    LoraKernelArgs a;
    a.X = static_cast<const char*>(l.X);
    a.x_ld = (uint32_t)(l.x_ld * 2);
    a.tiles = plan.tiles[p.height_index];
    a.tile_count = plan.class_ends[p.height_index] + kTileClasses - 1;
    a.offsets = plan.offsets;
    a.order = plan.order;
    a.rows = l.rows;
    a.adapters = (int)l.adapters;
    a.A = static_cast<const char*>(l.A);
    a.B = static_cast<const char*>(l.B);
    a.rank = l.rank;
    a.factors = l.factors;
    a.N = l.N;
    a.K = (uint32_t)l.K;
    a.base = static_cast<const char*>(l.base);
    a.base_ld = l.base_ld * 2;
    a.out = static_cast<char*>(l.out);
    a.out_ld = l.out_ld * 2;
    a.H = static_cast<float*>(workspace);
    a.splits = p.splits;
    a.columns = p.columns;
    a.tile_grid = 0;
    // (in place, with the same rows: nothing to copy)
    const bool copy = !(l.base == l.out && l.base_ld == l.out_ld);
    return l.dtype == E0M4_BF16 ? launch_lora_rows<true>(a, p, copy, stream) : launch_lora_rows<false>(a, p, copy, stream);
}

}  // namespace e0m4
