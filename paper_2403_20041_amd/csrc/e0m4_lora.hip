// Low-rank adapters of rows (e0m4_lora): out[m] = base[m] + f[a] * B[a] (A[a] x[m]) with a the adapter that row m has chosen.
//
// Two launches over tiles of rows of one adapter (see e0m4_groups.h).  The first, H = X A^T: a workgroup's four wavefronts take 128-k chunks
// in turn, read rows of X and of A as the matrix cores take them and add their sums in LDS; few tiles are split along K over workgroups,
// each with a slab of its own.  The second, out = base + f H B^T: H is added up over the slabs in order and split into the sum of three 16-bit numbers (fp16
// after scaling its row by a power of two), which hold all 24 bits of it: nothing is rounded between the two products.  A wavefront has the rows of
// the tile and 64 columns at a time, of which a lane holds two runs of 8 of one row.
// What bounds it: memory, X once, base and out once, A and B of the adapters in use once (and from L2 for every further tile).  3001 rows of five
// requests, rank 64, 4096 x 4096: 9 - 11 us and 16 - 19 of a floor of 16 together (A comes from L2 94 times, base and out pass through registers of few
// wavefronts, and each step of either launch waits for all that is under way, the second's stores too); 8192 rows of rank 16 42 of 41, of rank 64 71 of 42; 5253 rows of
// rank 16, 15832 x 7672 126 of 84; 4671 rows of 67 adapters of rank 128, 8008 x 2576 158 of 72; 64 rows with 40 adapters of rank 16 3.7 and 5.7 us, two launches' chains
// of loads, of rank 128 33 of 15.
#include "e0m4_groups.h"

#include <algorithm>
#include <type_traits>

namespace e0m4 {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));

constexpr int kWavesL = 4, kThreadsL = kWavesL * 64;
constexpr int kChunkK = 128;                    // k of a wavefront's turn
// For rows without an adapter.  64, 256 and 1024: 43, 15.8 and 11.1 us where none of 3001 rows of 4096 has one, 25.0, 21.5 and 21.7 where one in six has none; 64 rows
// 4.1 and 7.9 with any.
constexpr int64_t kCopyWorkgroups = 256;
constexpr uint32_t kNowhere = 0x80000000u;      // beyond a buffer's end, whatever is added to it

template <bool BF>
__device__ inline floatx4 mfma16(const half8_t& a, const half8_t& b, const floatx4& v)
{
    if constexpr (BF) return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), v, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, v, 0, 0, 0);
}

// Whole rows of 128 k are brought to LDS and turned around there: read as the matrix cores take them, 16 rows at a time and 64 bytes of each, rows come at 8 -
// 10 bytes per clock and compute unit (3001 rows by a rank of 64, 4096 k: 16 us).  Piece p (16 bytes) of row r lies at piece p ^ r%16 of its 256 bytes, by the
// choice of what a lane loads: the 16 rows of an operand read fall into 16 different bank groups.
constexpr int kChunkRowBytes = kChunkK * 2;

// H of a tile: MT times 16 rows, NT times 16 of the rank.  Lane (n = l%16, q = l/16) supplies A[16 j + n] and X[row 16 i + n] at k = 8 q ..
// + 7 of every step of 32, and holds H[row 16 i + n][16 j + 4 q ... + 3].  A wavefront has its operands of a chunk in registers when it
// requests the next one's into the same LDS.  (Arguments in registers from the start, as many as fit.)
template <bool BF, int MT, int NT>
__global__ __launch_bounds__(kThreadsL, 2) void lora_shrink_kernel(const void* plan, int rows, int adapters, const char* X, uint32_t x_ld, const char* A, uint32_t K,
                                                                    int rank, float* H, int splits)
{
    constexpr int HEIGHT = MT - 1;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const GroupPlan lay = plan_view(plan, rows, adapters);
    const uint32_t tile_no = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x / (uint32_t)splits)), split = blockIdx.x - tile_no * splits;
    const GroupTile tile = lay.tiles[HEIGHT][tile_no];  // (the list has room for a tile that is not there)
    if ((int)tile_no >= lay.class_ends[HEIGHT][kTileClasses - 1]) return;
    const int first = tile.begin + ((int)tile_no - tile.first_tile) * (16 * MT);
    const int M = min(16 * MT, tile.end - first);
    const int lane = threadIdx.x & 63, n_l = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    const __amdgpu_buffer_rsrc_t x_rsrc = make_rsrc(X), a_rsrc = make_rsrc(A + (int64_t)tile.group * rank * K * 2);
    unsigned char* mine = smem + wave * ((MT + NT) * 16 * kChunkRowBytes);
    // load e of 16 rows: rows 4 e + lane / 16
    uint32_t x_off[MT][4], a_off[NT][4], k_mine[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int r16 = 4 * e + q, piece = n_l ^ r16;
        k_mine[e] = (uint32_t)piece * 8;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int m = 16 * i + r16;
            x_off[i][e] = m < M ? (uint32_t)lay.order[first + m] * x_ld + (uint32_t)piece * 16 : kNowhere;
        }
#pragma unroll
        for (int j = 0; j < NT; ++j) a_off[j][e] = 16 * j + r16 < rank ? (uint32_t)(16 * j + r16) * (K * 2) + (uint32_t)piece * 16 : kNowhere;
    }
    uint32_t read_at[4];                                // of step s
#pragma unroll
    for (int s = 0; s < 4; ++s) read_at[s] = (uint32_t)(n_l * kChunkRowBytes + (((4 * s + q) ^ n_l) << 4));
    floatx4 acc[NT][MT];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[j][i] = floatx4{0.f, 0.f, 0.f, 0.f};
    const int chunks = (int)((K + kChunkK - 1) / kChunkK), apart = kWavesL * splits;
    auto load = [&](int ch) {
        const uint32_t k0 = (uint32_t)ch * kChunkK;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t out = k0 + k_mine[e] >= K ? kNowhere : 0u;
#pragma unroll
            for (int i = 0; i < MT; ++i) load_to_lds_b128(x_rsrc, mine + (i * 16 + 4 * e) * kChunkRowBytes, x_off[i][e] | out, k0 * 2);
#pragma unroll
            for (int j = 0; j < NT; ++j) load_to_lds_b128(a_rsrc, mine + ((MT + j) * 16 + 4 * e) * kChunkRowBytes, a_off[j][e] | out, k0 * 2);
        }
    };
    int ch = wave + kWavesL * (int)split;
    if (ch < chunks) load(ch);
    for (; ch < chunks; ch += apart) {
        wait_loads<0>();
        half8_t x[4][MT], w[4][NT];
#pragma unroll
        for (int s = 0; s < 4; ++s) {
#pragma unroll
            for (int i = 0; i < MT; ++i) x[s][i] = *reinterpret_cast<const half8_t*>(mine + i * 16 * kChunkRowBytes + read_at[s]);
#pragma unroll
            for (int j = 0; j < NT; ++j) w[s][j] = *reinterpret_cast<const half8_t*>(mine + (MT + j) * 16 * kChunkRowBytes + read_at[s]);
        }
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // read before it is written again
        __builtin_amdgcn_sched_barrier(0);
        if (ch + apart < chunks) load(ch + apart);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int s = 0; s < 4; ++s)
#pragma unroll
            for (int j = 0; j < NT; ++j)
#pragma unroll
                for (int i = 0; i < MT; ++i) acc[j][i] = mfma16<BF>(w[s][j], x[s][i], acc[j][i]);
    }
    // the wavefronts' sums in order
    floatx4* red = reinterpret_cast<floatx4*>(smem);    // [wavefronts - 1][NT * MT][64]
    __syncthreads();
    if (wave > 0) {
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int i = 0; i < MT; ++i) red[((wave - 1) * NT * MT + j * MT + i) * 64 + lane] = acc[j][i];
    }
    __syncthreads();
    if (wave > 0) return;
    float* h = H + ((int64_t)split * rows + first) * rank;
#pragma unroll
    for (int j = 0; j < NT; ++j) {
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            floatx4 v = acc[j][i];
#pragma unroll
            for (int w = 0; w < kWavesL - 1; ++w) v += red[(w * NT * MT + j * MT + i) * 64 + lane];
            const int r = 16 * j + 4 * q, m = 16 * i + n_l;
            if (m < M && r < rank) *reinterpret_cast<floatx4*>(h + (int64_t)m * rank + r) = v;       // (the rank is a multiple of 8)
        }
    }
}

// 16 rows of H as operands of the expanding product, NT times 16 of the rank, and what their product is to be multiplied with.  H is the sum of three 16-bit
// parts: each is what the ones before it left, rounded, and what it leaves is exact in fp32.  An operand's 32 values of "k" are 16 of the rank for two parts, the
// first (q 0, 1) and the second (q 2, 3), or the third and zeros.  (Two parts leave 16 of bfloat16's 24 bits: 415 rows of rank 128 have 2.3e-3 of the results rounded
// the other way than the exact sums, 1.9e-4 with three; fp32 operands have 3.6e-4.  The third one costs 30.0 -> 31.5 us with 3001 rows of rank 64, 4096 x 4096, 148 -> 158
// with 4671 of rank 128, 8008 x 2576, 42.3 -> 42.5 with 8192 of rank 16.)
constexpr int kPartPairs = 2;
template <bool BF, int NT>
__device__ inline void split_rows(const float* H, bool in, int rank, int splits, int64_t slab, float factor, int q, half8_t (&h)[kPartPairs][NT], float& scale)
{
    typedef std::conditional_t<BF, __bf16, half_t> T;
    typedef T T8 __attribute__((ext_vector_type(8)));
    float v[NT][8];
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int r = 16 * j + 8 * (q & 1);
        floatx4 lo = {0.f, 0.f, 0.f, 0.f}, hi = lo;
        if (in && r < rank) {
            for (int s = 0; s < splits; ++s) {
                lo += *reinterpret_cast<const floatx4*>(H + r + s * slab);
                hi += *reinterpret_cast<const floatx4*>(H + r + s * slab + 4);
            }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[j][e] = lo[e];
            v[j][4 + e] = hi[e];
        }
    }
    // fp16: the row's largest magnitude is scaled into [2^14, 2^15) (powers of two: exact), so that what is 2^-15 of it still has all its bits above the least
    // number of the type, 2^-24, and what is 2^-28 of it eleven.  A row that holds an infinity is used as it is; NaN (which the maximum passes over) stays NaN.
    scale = factor;
    float up = 1.f;
    if constexpr (!BF) {
        float most = 0.f;
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
            for (int e = 0; e < 8; ++e) most = fmaxf(most, fabsf(v[j][e]));
        most = fmaxf(most, __shfl_xor(most, 16));
        if (most > 0.f && most < INFINITY) {
            const int exponent = min(max(__builtin_amdgcn_frexp_expf(most) - 15, -126), 126);
            up = __builtin_amdgcn_ldexpf(1.f, -exponent);
            scale = factor * __builtin_amdgcn_ldexpf(1.f, exponent);
        }
    }
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        T8 pair[kPartPairs];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const float x = v[j][e] * up;
            const T first = (T)x;
            const float rest = fabsf((float)first) < INFINITY ? x - (float)first : 0.f;     // (NaN, too, is in the first part alone)
            const T second = (T)rest;
            pair[0][e] = q < 2 ? first : second;
            pair[1][e] = q < 2 ? (T)(rest - (float)second) : (T)0.f;
        }
#pragma unroll
        for (int p = 0; p < kPartPairs; ++p) h[p][j] = __builtin_bit_cast(half8_t, pair[p]);
    }
}

// base + f H B^T for a tile and 64 columns of a wavefront at a time; NT times 16 of the rank.  The row of B in lane (n, q) of the j-th of four
// MFMAs is column 8 (n/4) + 4 (j%2) + 32 (j/2) + n%4, so that a lane's results, 4 q .. + 3 of each, are the columns 8 q .. + 7 and 32 + 8 q .. + 7 of row n and
// four lanes read and write 64 bytes of it side by side.  The 64 rows of B are one piece
// of memory that comes to LDS as it is, but for the order of 16-byte pieces in a row (see order_of): up to a rank of 48 one set of columns ahead; beyond, into the same LDS
// once its operands are in registers, which leaves room for more workgroups of a compute unit (64 rows of 40 adapters of rank 128: 41 us with two sets, 33 with one; 3001
// rows of rank 64, 4096 x 4096, 38.5 and 31.6, 8192 93 and 71).
// With more than 16 rows the wavefronts make the operands of 16 rows each and share them through LDS.
__host__ __device__ constexpr int expand_sets(int NT) { return NT >= 4 ? 1 : 2; }
__host__ __device__ constexpr int operand_lds(int MT, int NT) { return MT > 1 ? kPartPairs * NT * MT * 1024 + MT * 64 : 0; }
__host__ __device__ constexpr int expand_lds(int MT, int NT) { return operand_lds(MT, NT) + kWavesL * expand_sets(NT) * 64 * NT * 32; }
template <bool BF, int MT, int NT>
__global__ __launch_bounds__(kThreadsL, 2) void lora_expand_kernel(const void* plan, int rows, int adapters, uint32_t columns, uint32_t tile_grid, const float* H, int rank,
                                                                    int splits, const char* B, const float* factors, int N, const char* base, char* out,
                                                                    int64_t base_ld, int64_t out_ld)
{
    typedef std::conditional_t<BF, __bf16, half_t> T;
    typedef T T8 __attribute__((ext_vector_type(8)));
    constexpr int HEIGHT = MT - 1;
    constexpr bool kShared = MT > 1;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    half8_t* operands = reinterpret_cast<half8_t*>(smem);                               // [pairs of parts][NT][MT][64]
    float* scales = reinterpret_cast<float*>(smem + kPartPairs * NT * MT * 1024);       // [MT * 16]
    const GroupPlan lay = plan_view(plan, rows, adapters);
    const int lane = threadIdx.x & 63, n_l = lane & 15, q = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (blockIdx.x >= tile_grid) {                      // rows without an adapter keep their base
        const int total = lay.offsets[adapters];
        const int64_t pieces = N / 8;
        for (int64_t r = total + (int64_t)(blockIdx.x - tile_grid); r < rows; r += gridDim.x - tile_grid) {
            const int64_t row = lay.order[r];
            for (int64_t p = threadIdx.x; p < pieces; p += kThreadsL) {
                u32x4 v = {0, 0, 0, 0};
                if (base) v = *reinterpret_cast<const u32x4*>(base + row * base_ld + p * 16);
                *reinterpret_cast<u32x4*>(out + row * out_ld + p * 16) = v;
            }
        }
        return;
    }
    const uint32_t tile_no = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x / columns)), part = blockIdx.x - tile_no * columns;
    const GroupTile tile = lay.tiles[HEIGHT][tile_no];  // (the list has room for a tile that is not there)
    if ((int)tile_no >= lay.class_ends[HEIGHT][kTileClasses - 1]) return;
    const int first = tile.begin + ((int)tile_no - tile.first_tile) * (16 * MT);
    const int M = min(16 * MT, tile.end - first);
    const float factor = factors ? factors[tile.group] : 1.f;
    const int64_t slab = (int64_t)rows * rank;

    // ---- rows of B: load e brings pieces 64 e .. + 63 of the 64 rows' pieces
    const int ppr = rank / 8;                           // pieces of a row
    const uint32_t reciprocal = small_reciprocal(ppr), adapter_pieces = (uint32_t)N * (uint32_t)ppr;
    // Where piece p of row 8 a + b (+ 4, + 32) lies among the row's, a power of two of them: the 16 rows of an operand read (all a and b of a j) fall into different
    // bank groups, for two pieces a row into half as many.
    auto order_of = [&](int p, int a, int b) -> int {
        switch (ppr) {
            case 16: return p ^ (4 * a + b);
            case 8: return p ^ (2 * a + (b >> 1));
            case 4: return p ^ a;
            case 2: return p ^ (a >> 1);
            default: return p;
        }
    };
    uint32_t piece_at[2 * NT];                          // (in the adapter, for its first columns)
#pragma unroll
    for (int e = 0; e < 2 * NT; ++e) {
        const uint32_t f = (uint32_t)(e * 64 + lane), r = small_quotient(f, reciprocal), p = f - r * ppr;
        piece_at[e] = r * ppr + (uint32_t)order_of((int)p, (int)(r >> 3) & 3, (int)r & 3);
    }
    const __amdgpu_buffer_rsrc_t b_rsrc = make_rsrc(B + (int64_t)tile.group * N * rank * 2);
    constexpr int kSets = expand_sets(NT);
    unsigned char* w_lds = smem + operand_lds(MT, NT) + wave * (kSets * 64 * NT * 32);
    uint32_t w_at[NT];                                  // of step j, MFMA 0; the rank's end: any piece, its operand is zeroed
#pragma unroll
    for (int j = 0; j < NT; ++j) {
        const int p = 2 * j + (q & 1);
        w_at[j] = (uint32_t)((8 * (n_l >> 2) + (n_l & 3)) * rank * 2 + order_of(p < ppr ? p : 0, n_l >> 2, n_l & 3) * 16);
    }
    auto load_w = [&](int at, int set) {
#pragma unroll
        for (int e = 0; e < 2 * NT; ++e) {
            if (e < ppr) {
                const uint32_t piece = (uint32_t)at * (uint32_t)ppr + piece_at[e];
                load_to_lds_b128(b_rsrc, w_lds + set * (64 * NT * 32) + e * 1024, piece < adapter_pieces ? piece * 16 : kNowhere, 0);
            }
        }
    };
    const int step = (int)columns * kWavesL * 64;
    int c0 = ((int)part * kWavesL + wave) * 64;
    if (c0 < N) load_w(c0, 0);

    int64_t row[MT];
#pragma unroll
    for (int i = 0; i < MT; ++i) row[i] = 16 * i + n_l < M ? lay.order[first + 16 * i + n_l] : -1;
    u32x4 b[MT][2];
    auto load_base = [&](int at) {
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int col = at + 8 * q + 32 * p;
                b[i][p] = u32x4{0, 0, 0, 0};
                if (base && row[i] >= 0 && col < N) b[i][p] = *reinterpret_cast<const u32x4*>(base + row[i] * base_ld + (int64_t)col * 2);
            }
    };
    load_base(c0);
    half8_t mine[kPartPairs][NT];
    float scale[MT];
    if constexpr (kShared) {
        if (wave < MT) {
            const int m = 16 * wave + n_l;
            split_rows<BF, NT>(H + (int64_t)(first + m) * rank, m < M, rank, splits, slab, factor, q, mine, scale[0]);
#pragma unroll
            for (int p = 0; p < kPartPairs; ++p)
#pragma unroll
                for (int j = 0; j < NT; ++j) operands[((p * NT + j) * MT + wave) * 64 + lane] = mine[p][j];
            if (q == 0) scales[m] = scale[0];
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < MT; ++i) scale[i] = scales[16 * i + n_l];
    } else {
        split_rows<BF, NT>(H + (int64_t)(first + n_l) * rank, n_l < M, rank, splits, slab, factor, q, mine, scale[0]);
    }
    int set = 0;
    for (; c0 < N; c0 += step) {
        wait_loads<0>();                                // these columns' rows of B
        __builtin_amdgcn_sched_barrier(0);
        if (kSets == 2 && c0 + step < N) load_w(c0 + step, set ^ 1);
        __builtin_amdgcn_sched_barrier(0);
        const int col = c0 + 8 * q;                     // this lane's results: columns col .. + 7 and col + 32 .. + 7 of its rows
        floatx4 acc[4][MT];
#pragma unroll
        for (int j4 = 0; j4 < 4; ++j4)
#pragma unroll
            for (int i = 0; i < MT; ++i) acc[j4][i] = floatx4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int j = 0; j < NT; ++j) {
            half8_t w[4];
#pragma unroll
            for (int j4 = 0; j4 < 4; ++j4) {
                w[j4] = *reinterpret_cast<const half8_t*>(w_lds + set * (64 * NT * 32) + w_at[j] + (4 * (j4 & 1) + 32 * (j4 >> 1)) * rank * 2);
                if (2 * j + (q & 1) >= ppr) w[j4] = half8_t{0, 0, 0, 0, 0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < MT; ++i) {
#pragma unroll
                for (int p = 0; p < kPartPairs; ++p) {
                    const half8_t h = kShared ? operands[((p * NT + j) * MT + i) * 64 + lane] : mine[p][j];
#pragma unroll
                    for (int j4 = 0; j4 < 4; ++j4) acc[j4][i] = mfma16<BF>(w[j4], h, acc[j4][i]);
                }
            }
        }
        if (kSets == 1) {
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // read before it is written again
            __builtin_amdgcn_sched_barrier(0);
            if (c0 + step < N) load_w(c0 + step, 0);
            __builtin_amdgcn_sched_barrier(0);
        }
        u32x4 o[MT][2];
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const T8 from = __builtin_bit_cast(T8, b[i][p]);
                T8 v;
#pragma unroll
                for (int e = 0; e < 8; ++e) v[e] = (T)__builtin_fmaf(scale[i], acc[2 * p + e / 4][i][e % 4], (float)from[e]);
                o[i][p] = __builtin_bit_cast(u32x4, v);
            }
        }
        load_base(c0 + step);
#pragma unroll
        for (int i = 0; i < MT; ++i) {
#pragma unroll
            for (int p = 0; p < 2; ++p)
                if (row[i] >= 0 && col + 32 * p < N) *reinterpret_cast<u32x4*>(out + row[i] * out_ld + (int64_t)(col + 32 * p) * 2) = o[i][p];
        }
        set ^= kSets - 1;
    }
}

struct LoraPlan {
    int shrink_height, expand_height;           // tiles of 16 or 32 rows (0 or 1)
    int splits;
    int64_t shrink_tiles, expand_tiles;
    uint32_t columns;
};
// Tiles of 16 rows for H, of 32 where adapters have many rows of a rank that would be read too often; of 32 for the second launch, of 16 where adapters have
// no more rows.  3001 rows of five requests, rank 64, 4096 x 4096, both launches, in us (rows of a tile in the first / second launch, splits, workgroups per tile in the
// second): 16/16 1 4 31.0, 16/32 1 4 31.4, 32/32 1 4 33.9, 2 4 31.3, 32/16 2 4 31.9, 16/32 1 16 33.7, 32/32 2 16 35.2; 512 rows of two, rank 32: 16/16 2 12.1,
// 16/32 2 11.4, 4 11.5, 8 13.5, 32/32 2 12.5; 64 rows of 40 adapters, rank 16: 1, 2, 4 and 8 splits 9.7, 8.6, 8.5, 9.3; 8192 rows of four, rank 16: 16/32 1 with 2, 4 and 8
// workgroups per tile 45.5, 43.3, 42.0, 32/32 1 8 45.9.  Adapters are counted as if all of them were in use.
// Workgroups of the second launch: a rank of 32 or less has little to bring before its first column, and 1024 against 2048 take 43.3 and 42.0 (8192 rows of four, rank
// 16) and 134 and 127 (5253 of one, rank 16, 15832 x 7672).  Beyond that 448, 896 and 2048 take 31.6, 34.6 and 35.5 (3001 rows, rank 64), 32.4, 40.4 and 40.4 (64 rows of
// 40 adapters, rank 128), 158, 175 and 187 (4671 of 67, rank 128, 8008 x 2576), 84, 96 and 134 (5000 of one, rank 128, 4096 x 4096), and 70.6, 69.1 and 71.9 (8192, rank 64).
LoraPlan plan_lora(int64_t rows, int64_t adapters, int rank, int64_t N, int64_t K)
{
    LoraPlan p;
    const int64_t each = rows / std::max<int64_t>(1, std::min(adapters, rows));        // rows of an adapter, if all are in use
    p.shrink_height = each > 64 && rank > 32 && rank <= 64 ? 1 : 0;         // (32 rows of a rank of 128 do not fit the LDS)
    p.expand_height = each > 16 ? 1 : 0;
    p.shrink_tiles = most_tiles(rows, adapters, tile_height(p.shrink_height));
    p.expand_tiles = most_tiles(rows, adapters, tile_height(p.expand_height));
    const int64_t chunks = (K + kChunkK - 1) / kChunkK;
    p.splits = (int)std::max<int64_t>(1, std::min<int64_t>({256 / p.shrink_tiles, (chunks + kWavesL - 1) / kWavesL, 4}));
    const int64_t parts = (N + kWavesL * 64 - 1) / (kWavesL * 64), workgroups = rank > 32 ? 448 : 2048;
    p.columns = (uint32_t)std::max<int64_t>(1, std::min<int64_t>(parts, (workgroups + p.expand_tiles - 1) / p.expand_tiles));
    return p;
}

template <bool BF, int MT, int NT>
int launch_shrink(const LoraArgs& a, const LoraPlan& p, float* H, hipStream_t stream)
{
    const int64_t grid = p.shrink_tiles * p.splits;
    constexpr int lds = kWavesL * (MT + NT) * 16 * kChunkRowBytes;
    static_assert(lds >= (kWavesL - 1) * NT * MT * 1024 && lds <= 160 * 1024, "sums fit, and all fits the LDS of a compute unit");
    static std::atomic<uint64_t> lds_allowed{0};
    const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(&lora_shrink_kernel<BF, MT, NT>), lds, lds_allowed);
    if (rc != E0M4_OK) return rc;
    hipLaunchKernelGGL((lora_shrink_kernel<BF, MT, NT>), dim3((unsigned)grid), dim3(kThreadsL), lds, stream, a.plan, (int)a.rows, (int)a.adapters,
                       static_cast<const char*>(a.X), (uint32_t)(a.x_ld * 2), static_cast<const char*>(a.A), (uint32_t)a.K, a.rank, H, p.splits);
    return check_launch();
}
template <bool BF, int MT, int NT>
int launch_expand(const LoraArgs& a, const LoraPlan& p, const float* H, hipStream_t stream)
{
    const int64_t tiles = p.expand_tiles * p.columns;
    // (in place, with the same rows: nothing to copy)
    const int64_t grid = tiles + (a.base == a.out ? 0 : std::min<int64_t>(a.rows, kCopyWorkgroups));
    constexpr int lds = expand_lds(MT, NT);
    static_assert(lds <= 160 * 1024, "the LDS of a compute unit");
    static std::atomic<uint64_t> lds_allowed{0};
    const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(&lora_expand_kernel<BF, MT, NT>), lds, lds_allowed);
    if (rc != E0M4_OK) return rc;
    hipLaunchKernelGGL((lora_expand_kernel<BF, MT, NT>), dim3((unsigned)grid), dim3(kThreadsL), lds, stream, a.plan, (int)a.rows, (int)a.adapters, p.columns,
                       (uint32_t)tiles, H, a.rank, p.splits, static_cast<const char*>(a.B), a.factors, (int)a.N, static_cast<const char*>(a.base),
                       static_cast<char*>(a.out), a.base_ld * 2, a.out_ld * 2);
    return check_launch();
}

// f(bool, rows / 16, rank / 16 rounded up to a power of two) as constants
template <typename F>
int with_sizes(bool bf16, int height, int rank, F&& f)
{
    auto by_rank = [&](auto bf, auto mt) -> int {
        if (rank <= 16) return f(bf, mt, std::integral_constant<int, 1>{});
        if (rank <= 32) return f(bf, mt, std::integral_constant<int, 2>{});
        if (rank <= 64) return f(bf, mt, std::integral_constant<int, 4>{});
        return f(bf, mt, std::integral_constant<int, 8>{});
    };
    auto by_rows = [&](auto bf) -> int {
        return height == 0 ? by_rank(bf, std::integral_constant<int, 1>{}) : by_rank(bf, std::integral_constant<int, 2>{});
    };
    return bf16 ? by_rows(std::true_type{}) : by_rows(std::false_type{});
}

}  // namespace

size_t lora_workspace_bytes(int64_t rows, int64_t adapters, int rank, int64_t N, int64_t K)
{
    return (size_t)plan_lora(rows, adapters, rank, N, K).splits * (size_t)rows * (size_t)rank * 4;
}

int launch_lora(const LoraArgs& a, void* workspace, hipStream_t stream)
{
    const LoraPlan p = plan_lora(a.rows, a.adapters, a.rank, a.N, a.K);
    // (both launches fit their grids, or neither goes out)
    if (p.shrink_tiles * p.splits * kThreadsL > 0xffffffffLL || (p.expand_tiles * p.columns + kCopyWorkgroups) * kThreadsL > 0xffffffffLL) return E0M4_ERR_SHAPE;
    float* H = static_cast<float*>(workspace);
    const int rc = with_sizes(a.dtype == E0M4_BF16, p.shrink_height, a.rank, [&](auto bf, auto mt, auto nt) -> int {
        if constexpr (decltype(mt)::value > 1 && decltype(nt)::value != 4) return E0M4_ERR_SHAPE;     // (plan_lora takes them for ranks of 33 to 64 alone)
        else return launch_shrink<decltype(bf)::value, decltype(mt)::value, decltype(nt)::value>(a, p, H, stream);
    });
    if (rc != E0M4_OK) return rc;
    return with_sizes(a.dtype == E0M4_BF16, p.expand_height, a.rank, [&](auto bf, auto mt, auto nt) -> int {
        return launch_expand<decltype(bf)::value, decltype(mt)::value, decltype(nt)::value>(a, p, H, stream);
    });
}

}  // namespace e0m4
