// Products of a layout's rows with the quantised weights of their groups, many rows to a group (e0m4_matmul_grouped and its like): tiles of up to
// 128 rows of one group and 256 weight rows (gated: 128 of the gate and the same of the up projection).
//     Y[p, n] = sum_k X[row(p), k] * dequant(codes of p's group)[n, k], and with the gated product silu(gate) * up of the two halves of n.
//
// Four wavefronts side by side, 64 weight rows each, two workgroups to a compute unit.  Per K slice of 64 (four MFMA sub-steps of 16):
//   - rows of X come from where the layout's entries say straight to an LDS ring of four stages, two and a half slices ahead, and are read as 16-byte
//     fragments one sub-step ahead of their use; 128-byte rows whose eight pieces are XOR-swizzled with (row / 2) % 8;
//   - codes never touch LDS: lane (n = l%32, h = l/32) reads the chunk of row n with k = 32h .. 32h + 31 of the slice ahead of time (8-bit codes: two
//     chunks), and word s of it is dequantised in registers one sub-step ahead of MFMA s, whose k are {8s..8s+7} and {32+8s..32+8s+7};
//   - one barrier per slice, after sub-step 1.
// A tile whose group has fewer rows left is computed in as many 32-row blocks as it has, by a loop of its own: with 128 groups of 256 rows on
// average a third of the tiles are not whole.  Classes of tiles by that number come one after the other (prompt of 1001 tokens with 6 of 64 experts, bfloat16
// 2816 x 2048: 98 us in the groups' order, 89 by classes; 4096 with 8 of 128, 1536 x 2048, 211 and 207).
// What bounds it: with whole tiles the clock that the chip holds under matrix instructions (4096 tokens with 2 of 8, 4096 x 13696: 767 - 824 us, 1115 - 1200
// TFLOP/s, a library's product of 8192^3 on the same card 1078); with short ones the dequantisation, 31 vector instructions a sub-step whatever
// the rows, which is as long as 96 rows' products take.  Few tiles leave compute units without a workgroup or with a wavefront to a SIMD, which does not fill
// it: parts of K side by side then (256 tokens with 2 of 8, 4096 x 4096: 44 us, in two parts 30).
#include "e0m4_groups.h"

#include <algorithm>
#include <type_traits>

namespace e0m4 {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

constexpr int BK = 64;
constexpr int kRowBytes = BK * 2, kStages = 4;
constexpr int TN = 2;                           // operand blocks of 32 weight rows per wavefront

struct ManyArgs {
    const void* X;
    const void* codes;
    void* Y;
    const void* plan;
    int rows, groups;
    uint32_t N, K;
    uint32_t n_tiles;
    uint32_t share, share_reciprocal;           // share 0: rows of X lie in the layout's order
};

// A tile is 32 TM rows and 64 WN columns; KS groups of WN wavefronts take a part of K each, and their sums are added in LDS.  (Arguments one by one, in registers
// from the start)
template <int FMT, int G, bool GATED, int TM, int WN, int KS>
__global__ __launch_bounds__(64 * WN * KS, 2) void grouped_many_kernel(const char* X, const char* codes, void* Y, const void* plan, int rows, int groups,
                                                                               uint32_t N32, uint32_t K32, uint32_t n_tiles, uint32_t share,
                                                                               uint32_t share_reciprocal)
{
    const GroupPlan lists = plan_view(plan, rows, groups);
    constexpr int HEIGHT = TM == 4 ? 3 : 2;
    static_assert(tile_height(HEIGHT) == 32 * TM, "a list of tiles");
    constexpr int BM = 32 * TM, BN = 64 * WN;
    constexpr int kThreads = 64 * WN;                   // of a part of K
    constexpr int kStageBytes = BM * kRowBytes;
    constexpr bool E8 = FMT == kGroupedE8, BF = FMT == kGroupedBf16;
    constexpr int PD = E8 ? 2 : 4, S = kStages, L = S - 1;      // slices of codes in registers, stages of X, how far ahead X is requested
    constexpr int RP = kThreads / 8;                    // rows of X per loader pass
    constexpr int PA = BM / RP;                         // passes
    constexpr int NCH = E8 ? 2 : 1;
    static_assert(32 % RP == 0, "a 32-row block is whole loader passes");
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];

    // Work items: class after class, in each the tiles of a group, its row tiles first, column after column, so that neighbours share their weights.
    // Each XCD takes a contiguous run of every class and shares rows of X and weights in its L2.
    const uint32_t xcd = blockIdx.x % kNumXcd;
    uint32_t turn = blockIdx.x / kNumXcd, from = 0, item = 0;
    bool found = false;
#pragma unroll
    for (int c = 0; c < kTileClasses; ++c) {
        const uint32_t to = (uint32_t)lists.class_ends[HEIGHT][c] * n_tiles, each = (to - from + kNumXcd - 1) / kNumXcd;
        if (!found && turn < each) {
            item = from + xcd * each + turn;
            found = true;
            if (item >= to) return;
        }
        turn -= found ? 0 : each;
        from = to;
    }
    if (!found) return;
    const GroupTile tile = lists.tiles[HEIGHT][(uint32_t)__builtin_amdgcn_readfirstlane((int)(item / n_tiles))];
    const int group_rows = tile.end - tile.begin;       // (those of its tiles of this class)
    const uint32_t in_group = item - (uint32_t)tile.first_tile * n_tiles, m_tiles = (uint32_t)(group_rows + BM - 1) / BM;
    const uint32_t tile_n = (uint32_t)__builtin_amdgcn_readfirstlane((int)(in_group / m_tiles)), tile_m = in_group - tile_n * m_tiles;
    const int first = __builtin_amdgcn_readfirstlane(tile.begin + (int)tile_m * BM);
    const int M = __builtin_amdgcn_readfirstlane(min(BM, tile.end - first));        // rows of this tile
    const int64_t N = N32, K = K32;
    const int64_t n_out = GATED ? N / 2 : N;
    const int64_t n0 = (int64_t)tile_n * (GATED ? BN / 2 : BN);
    const int part = KS > 1 ? __builtin_amdgcn_readfirstlane((int)threadIdx.x / kThreads) : 0;
    const int t = KS > 1 ? (int)threadIdx.x % kThreads : (int)threadIdx.x;
    const int lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const uint32_t fmask = frac_mask_vgpr();
    const PackedLayout<G> lay(E8 ? 2 * K : K);
    // (4-bit codes fill whole k blocks of two slices; 8-bit codes have a block per slice, and their last pair may lack one)
    const int slices = E8 ? (int)((K + BK - 1) / BK) : 2 * (int)k_blocks(K);
    const int pairs = (slices + 1) / 2;
    const int kt_begin = KS > 1 ? __builtin_amdgcn_readfirstlane(2 * (pairs * part / KS)) : 0;
    const int kt_end = KS > 1 ? __builtin_amdgcn_readfirstlane(2 * (pairs * (part + 1) / KS)) : 2 * pairs;
    const int kt_last = KS > 1 ? min(kt_end, slices) : slices;

    // ---- rows of X: 8 lanes cover one 128-byte row slice; pass p handles row RP * p + t / 8.  Rows that the tile lacks, and k beyond K, are requested
    // beyond the buffer's end.
    constexpr uint32_t kNowhere = 0x80000000u;
    const int a_row = t >> 3, a_piece = (t & 7) ^ ((a_row >> 1) & 7);
    const char* x_base = share ? X : X + (int64_t)first * K * 2;
    uint32_t a_off[PA];
#pragma unroll
    for (int p = 0; p < PA; ++p) {
        const int row = a_row + RP * p;
        uint32_t at = (uint32_t)row;
        if (share && row < M) at = small_quotient((uint32_t)lists.order[first + row], share_reciprocal);
        a_off[p] = row < M ? at * (K32 * 2) + (uint32_t)a_piece * 16 : kNowhere;
    }
    const uint32_t a_lds_off = (uint32_t)(wave * 8 * kRowBytes);

    // ---- codes: operand block j of this wavefront covers 32 weight rows; gated, block 0 the gate's and block 1 the same of the up projection
    const int b_h = lane >> 5, b_r = lane & 15;
    const int64_t nrb = row_blocks(N), rb_tile = n0 / kBlockRows;
    const uint4* group_codes = reinterpret_cast<const uint4*>(codes + (int64_t)tile.group * (nrb * lay.nkb * block_bytes(G)));
    const uint4* b_codes = group_codes + lay.code_index(rb_tile, 0);
    const uint32_t* b_params = reinterpret_cast<const uint32_t*>(group_codes) + lay.param_index(rb_tile, 0);
    const uint32_t rb_stride = (uint32_t)lay.nkb * block_bytes(G);
    uint32_t b_code_off[TN], b_param_off[TN];           // (row blocks beyond the last: that one again, never stored)
#pragma unroll
    for (int j = 0; j < TN; ++j) {
        int64_t rb;
        if (GATED) rb = min(rb_tile + wave * 2 + ((lane >> 4) & 1), nrb / 2 - 1) - rb_tile + j * (nrb / 2);
        else rb = min(rb_tile + wave * 4 + 2 * j + ((lane >> 4) & 1), nrb - 1) - rb_tile;
        b_code_off[j] = (uint32_t)rb * rb_stride + (uint32_t)((E8 ? 2 * b_h : b_h) * kBlockRows + b_r) * 16;
        b_param_off[j] = (uint32_t)rb * rb_stride + (uint32_t)b_r * 4 + (G == 32 ? b_h * 64 : 0);
    }

    // ---- fragment read position: row 32 i + l%32, piece 4 h + s
    uint32_t frag_off[4];
#pragma unroll
    for (int s = 0; s < 4; ++s) frag_off[s] = (uint32_t)((lane & 31) * kRowBytes + (((4 * b_h + s) ^ ((lane >> 1) & 7)) << 4));

    u32x4 bset[PD][TN][NCH];
    uint32_t pwset[PD][TN];
    half8_t fa[2][TM];
    uint32_t fb[2][TN][4];
    floatx16 acc[TM][TN];
    constexpr int NB = (1 + NCH) * TN;                  // loads of a slice's codes and parameters

    // (slices beyond the last are requested through a resource of no bytes: the number of requests stays, memory is not read)
    // piece p of a slice's rows, piece i of its codes and parameters
    auto load_a = [&](int kt, uint32_t stage_off, int p) {
        const __amdgpu_buffer_rsrc_t rsrc = rsrc_if(x_base, kt < kt_last);
        const uint32_t k0 = (uint32_t)kt * BK;
        const uint32_t out = (int64_t)k0 + a_piece * 8 >= K ? kNowhere : 0u;
        load_to_lds_b128(rsrc, smem + stage_off + a_lds_off + p * RP * kRowBytes, a_off[p] | out, k0 * 2);
    };
    auto load_b = [&](int kt, int set, int i) {
        const uint32_t k0 = (uint32_t)kt * BK;
        const int j = i / (1 + NCH), c = i % (1 + NCH);
        if (c < NCH) {
            const int soff = E8 ? (int)((k0 / BK) * kBlockCodeBytes) : (int)((k0 / kCodesPerChunk) * (kBlockRows * 16));
            bset[set][j][c] = __builtin_amdgcn_raw_buffer_load_b128(rsrc_if(b_codes, kt < kt_last), (int)b_code_off[j] + c * kBlockRows * 16, soff, 0);
        } else {
            const int soff = E8 ? (int)((k0 / BK) * (kBlockRows * 4)) : (int)((k0 / G) * (kBlockRows * 4));
            pwset[set][j] = __builtin_amdgcn_raw_buffer_load_b32(rsrc_if(b_params, kt < kt_last), (int)b_param_off[j], soff, 0);
        }
    };
    auto read_frag = [&](uint32_t stage_off, int s, int i) -> half8_t {
        return *reinterpret_cast<const half8_t*>(smem + stage_off + frag_off[s] + i * 32 * kRowBytes);
    };
    // The dequantisation of a sub-step's operands, in eight units of two weights (pair u % 4 of operand u / 4) and three stages: the codes' values, their
    // difference from the bias (exact; bfloat16: one fp32 fused multiply-add per weight, exact too), the product with the scale, rounded once.
    struct Unit {
        uint32_t w1;
        half2_t diff;
        floatx2 wide;
    };
    auto unit_codes = [&](int set, int s, int u) -> uint32_t {
        const int j = u >> 2, p = u & 3;
        if (E8) {
            const uint32_t m8 = fmask | (fmask >> 4), w8 = bset[set][j][(s >> 1) * (NCH - 1)][2 * (s & 1) + (p >> 1)];   // eight fraction bits of both halves
            return ((p & 1 ? __builtin_amdgcn_alignbit(w8, w8, 8) : w8) & m8) | kExpBits2;
        }
        const uint32_t word = bset[set][j][0][s];
        return p == 0 ? w1_pair_bits<0>(word, fmask) : p == 1 ? w1_pair_bits<1>(word, fmask) : p == 2 ? w1_pair_bits<2>(word, fmask) : w1_pair_bits<3>(word, fmask);
    };
    auto unit_middle = [&](int set, int u, Unit& v) {
        const uint32_t pw = pwset[set][u >> 2];
        const half2_t q = __builtin_bit_cast(half2_t, v.w1);
        if (BF) {
            const float sf = __builtin_bit_cast(float, pw << 16), nb = -__builtin_bit_cast(float, pw & 0xFFFF0000u) * sf;
            v.wide = floatx2{__builtin_fmaf((float)q[0], sf, nb), __builtin_fmaf((float)q[1], sf, nb)};
        } else {
            const half_t bi = param_bias(pw);
            v.diff = q - half2_t{bi, bi};
        }
    };
    auto unit_last = [&](int set, int u, const Unit& v) -> uint32_t {
        if (BF) return __builtin_bit_cast(uint32_t, __builtin_convertvector(v.wide, bf16x2_t));
        const half_t sc = param_scale(pwset[set][u >> 2]);
        return __builtin_bit_cast(uint32_t, v.diff * half2_t{sc, sc});
    };
    // One sub-step: the products of fa[now], fb[now], and behind each of them some of the instructions that prepare the next one's operands (`step` of slice
    // in `set`, rows from stage `from`) and some requests, so that one wavefront keeps the matrix pipe busy.  The stages of a unit stand apart: a product behind the
    // difference that it takes leaves an issue slot empty.  2 % less time than with the compiler's order between products (4096 tokens with 2 of 8 experts, 4096 x
    // 13696: 808 -> 796 us; holding each stage to its place is no faster).
    auto sub_step = [&](auto tm_c, int now, uint32_t from, int set, int s, auto request) {
        constexpr int TMX = decltype(tm_c)::value, SLOTS = TMX * TN;
        auto first_unit = [](int slot) -> int { return slot <= 0 ? 0 : slot >= SLOTS ? 8 : 8 * slot / SLOTS; };
        Unit v[8];
        auto stage = [&](int which, int slot) {
#pragma unroll
            for (int u = 0; u < 8; ++u) {
                if (u < first_unit(slot) || u >= first_unit(slot + 1) || slot < 0 || slot >= SLOTS) continue;
                if (which == 0) v[u].w1 = unit_codes(set, s, u);
                if (which == 1) unit_middle(set, u, v[u]);
                if (which == 2) fb[now ^ 1][u >> 2][u & 3] = unit_last(set, u, v[u]);
            }
        };
#pragma unroll
        for (int m = 0; m < SLOTS; ++m) {
            const int i = m / TN, j = m % TN;
            const half8_t w = __builtin_bit_cast(half8_t, u32x4{fb[now][j][0], fb[now][j][1], fb[now][j][2], fb[now][j][3]});
            acc[i][j] = BF ? __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8_t, fa[now][i]), __builtin_bit_cast(bf16x8_t, w), acc[i][j], 0, 0, 0)
                           : __builtin_amdgcn_mfma_f32_32x32x16_f16(fa[now][i], w, acc[i][j], 0, 0, 0);
            if (m < TMX) fa[now ^ 1][m] = read_frag(from, s, m);
            request(m, SLOTS);
            stage(2, m - 2);
            stage(1, m - 1);
            stage(0, m);
            __builtin_amdgcn_sched_barrier(0);
        }
        stage(2, SLOTS - 2);
        stage(1, SLOTS - 1);
        __builtin_amdgcn_sched_barrier(0);
        stage(2, SLOTS - 1);
        __builtin_amdgcn_sched_barrier(0);
    };

    auto write_rows = [&](auto tm_c) {
        using out_t = std::conditional_t<BF, __bf16, half_t>;
        typedef out_t out8_t __attribute__((ext_vector_type(8)));
        constexpr int TMX = decltype(tm_c)::value;
        constexpr int COLS = GATED ? 32 : 64, ROWS = 1024 / COLS, kChunks = TMX * 32 / ROWS;
        constexpr int PPR = COLS / 8, RPP = 64 / PPR;   // 16-byte pieces per row, rows per pass (two passes per chunk)
        constexpr int kStride = COLS + 4, NJ = COLS / 32, NR = 16 / NJ;
        auto value = [&](int i, int r, int j) -> float {
            if constexpr (GATED) return silu_f32(acc[i][0][r]) * acc[i][1][r];
            else return acc[i][j][r];
        };
        out_t* y = static_cast<out_t*>(Y) + (int64_t)first * n_out + n0;
        const int wcol = wave * COLS, cols = (int)min((int64_t)(GATED ? BN / 2 : BN), n_out - n0);
        const uint32_t ld = (uint32_t)n_out;
        if ((n_out & 7) != 0) {                         // rows that are not whole 16-byte pieces: element by element (never gated)
            const int col0 = wcol + (lane & 31), row0 = 4 * (lane >> 5);
#pragma unroll
            for (int j = 0; j < NJ; ++j) {
                if (col0 + 32 * j < cols) {
#pragma unroll
                    for (int i = 0; i < TMX; ++i)
#pragma unroll
                        for (int r = 0; r < 16; ++r) {
                            const int row = row0 + 32 * i + 8 * (r >> 2) + (r & 3);
                            if (row < M) y[(uint32_t)row * ld + (uint32_t)(col0 + 32 * j)] = (out_t)value(i, r, j);
                        }
                }
            }
            return;
        }
        // A wavefront turns 4 KiB of sums at a time around in a piece of LDS of its own (the ring is free by then) and writes whole 16-byte pieces.
        constexpr uint32_t kTurnBytes = 32 * (32 + 4) * 4;
        static_assert(kTurnBytes >= 16 * (64 + 4) * 4 && kTurnBytes * WN <= (uint32_t)KS * kStages * kStageBytes, "fits the stages");
        float* turn_lds = reinterpret_cast<float*>(smem + wave * kTurnBytes);
        const int prow = lane / PPR, pcol = (lane % PPR) * 8;
        const int my_rows = wcol + pcol < cols ? M - prow : 0;
        const uint32_t o0 = (uint32_t)prow * ld + (uint32_t)(wcol + pcol);
        __syncthreads();                                // every wavefront has left the K loop's stages (or the other parts' sums)
#pragma unroll
        for (int ch = 0; ch < kChunks; ++ch) {
#pragma unroll
            for (int j = 0; j < NJ; ++j)
#pragma unroll
                for (int rr = 0; rr < NR; ++rr)
                    turn_lds[(8 * (rr >> 2) + 4 * (lane >> 5) + (rr & 3)) * kStride + 32 * j + (lane & 31)] =
                        value(ch * ROWS / 32, (ch * ROWS % 32) / 2 + rr, j);
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int p = 0; p < 2; ++p) {
                const int dr = ch * ROWS + p * RPP;
                const float* src = turn_lds + (p * RPP + prow) * kStride + pcol;
                const floatx4 lo = *reinterpret_cast<const floatx4*>(src), hi = *reinterpret_cast<const floatx4*>(src + 4);
                out8_t o;
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    o[e] = (out_t)lo[e];
                    o[4 + e] = (out_t)hi[e];
                }
                if (dr < my_rows) *reinterpret_cast<out8_t*>(y + (o0 + (uint32_t)dr * ld)) = o;
            }
            __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
            __builtin_amdgcn_wave_barrier();            // the piece of LDS is read before it is written again
        }
    };

    // The tile on TMX 32-row blocks
    auto run = [&](auto tm_c) {
        constexpr int TMX = decltype(tm_c)::value, PAX = TMX * 32 / RP;
        const uint32_t ring = (uint32_t)part * S * kStageBytes;
#pragma unroll
        for (int i = 0; i < TMX; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int r = 0; r < 16; ++r) acc[i][j][r] = 0.f;
        // One K slice.  On entry: stage `cur` holds slice kt; fa[0], fb[0] hold its sub-step 0 operands; bset[set] holds its codes; the next PD - 1
        // slices' codes and the next L - 1 slices' rows are in flight.  (REST: one of the last two slices, which request nothing)
        auto step = [&](auto rest_c, int kt, int set, uint32_t cur, uint32_t nxt, uint32_t last) {
            constexpr bool REST = decltype(rest_c)::value;
            auto nothing = [](int, int) {};
            sub_step(tm_c, 0, cur, set, 1, nothing);
            sub_step(tm_c, 1, cur, set, 2, nothing);
            wait_loads<REST ? 0 : (L - 1) * NB + (L - 2) * PAX>();
            __builtin_amdgcn_s_barrier();   // slice kt+1 is complete in stage `nxt`, and nobody reads slice kt-1 any more
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            sub_step(tm_c, 0, cur, set, 3, [&](int m, int slots) {
#pragma unroll
                for (int p = 0; p < PAX; ++p)
                    if (!REST && p >= PAX * m / slots && p < PAX * (m + 1) / slots) load_a(kt + L, last, p);
            });
            sub_step(tm_c, 1, nxt, (set + 1) % PD, 0, [&](int m, int slots) {
#pragma unroll
                for (int i = 0; i < NB; ++i)
                    if (!REST && i >= NB * m / slots && i < NB * (m + 1) / slots) load_b(kt + PD, set, i);
            });
        };
        // (in the order that the loop keeps up: slice kt requests rows L slices on, then codes PD slices on)
#pragma unroll
        for (int d = -(PD > L ? PD : L); d < 0; ++d) {
            if (d + L >= 0) {
#pragma unroll
                for (int p = 0; p < PAX; ++p) load_a(kt_begin + d + L, ring + (uint32_t)(d + L) * kStageBytes, p);
            }
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
            if (d + PD >= 0) {
#pragma unroll
                for (int i = 0; i < NB; ++i) load_b(kt_begin + d + PD, d + PD, i);
            }
            asm volatile("" ::: "memory");
            __builtin_amdgcn_sched_barrier(0);
        }
        wait_loads<(L - 1) * PAX + (PD < L ? PD : L) * NB>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
#pragma unroll
        for (int i = 0; i < TMX; ++i) fa[0][i] = read_frag(ring, 0, i);
#pragma unroll
        for (int u = 0; u < 8; ++u) {
            Unit v;
            v.w1 = unit_codes(0, 0, u);
            unit_middle(0, u, v);
            fb[0][u >> 2][u & 3] = unit_last(0, u, v);
        }
        uint32_t so[S];                                 // stages of slices kt, kt + 1, ..., kt - 1
#pragma unroll
        for (int i = 0; i < S; ++i) so[i] = ring + (uint32_t)i * kStageBytes;
        auto advance_ring = [&]() {                     // by two slices
            uint32_t tmp[S];
#pragma unroll
            for (int i = 0; i < S; ++i) tmp[i] = so[(i + 2) % S];
#pragma unroll
            for (int i = 0; i < S; ++i) so[i] = tmp[i];
        };
        int kt = kt_begin;
        for (; kt + PD <= kt_end; kt += PD) {
#pragma unroll
            for (int d = 0; d < PD; d += 2) {
                step(std::false_type{}, kt + d, d, so[0], so[1], so[S - 1]);
                step(std::false_type{}, kt + d + 1, d + 1, so[1], so[2], so[0]);
                advance_ring();
            }
        }
        if (PD == 4 && kt < kt_end) {
            step(std::true_type{}, kt, 0, so[0], so[1], so[S - 1]);
            step(std::true_type{}, kt + 1, 1, so[1], so[2], so[0]);
        }
        wait_loads<0>();                                // (what was requested beyond the range has arrived before the stages are used otherwise)
        if constexpr (KS > 1) {
            // The parts' sums are added to the first's, in the order of K, through LDS.  Parts of one pair of slices fewer wait at the barriers of
            // two steps more.
            if (kt_end - kt_begin < 2 * ((pairs + KS - 1) / KS)) {
                __syncthreads();
                __syncthreads();
            }
            __syncthreads();                            // every wavefront has left the K loop's stages
            floatx4* sums = reinterpret_cast<floatx4*>(smem);
            constexpr int kPart = TMX * TN * 4 * kThreads;
            static_assert((KS - 1) * TM * TN * 4 * kThreads * 16 <= KS * kStages * kStageBytes, "fits the stages");
            if (part > 0) {
#pragma unroll
                for (int i = 0; i < TMX; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int q = 0; q < 4; ++q)
                            sums[(part - 1) * kPart + ((i * TN + j) * 4 + q) * kThreads + t] =
                                floatx4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
            }
            __syncthreads();
            if (part > 0) return;
#pragma unroll
            for (int s = 0; s < KS - 1; ++s)
#pragma unroll
                for (int i = 0; i < TMX; ++i)
#pragma unroll
                    for (int j = 0; j < TN; ++j)
#pragma unroll
                        for (int q = 0; q < 4; ++q) {
                            const floatx4 v = sums[s * kPart + ((i * TN + j) * 4 + q) * kThreads + t];
#pragma unroll
                            for (int e = 0; e < 4; ++e) acc[i][j][4 * q + e] += v[e];
                        }
        }
        write_rows(tm_c);
    };
    if constexpr (TM >= 4) {
        if (M > 96) return run(std::integral_constant<int, 4>{});
        if (M > 64) return run(std::integral_constant<int, 3>{});
    }
    if (M > 32) run(std::integral_constant<int, 2>{});
    else run(std::integral_constant<int, 1>{});
}

template <int FMT, int G, bool GATED, int TM, int WN, int KS>
int launch_many(const ManyArgs& f, int64_t rows, int64_t groups, hipStream_t stream)
{
    constexpr int lds = KS * kStages * 32 * TM * kRowBytes, threads = 64 * WN * KS;
    ManyArgs a = f;
    const int64_t columns = GATED ? 32 * WN : 64 * WN, n_out = GATED ? a.N / 2 : a.N;
    a.n_tiles = (uint32_t)((n_out + columns - 1) / columns);
    const int64_t grid = grouped_workgroups(rows, groups, 32 * TM, a.n_tiles);
    if (grid * threads > kMaxWorkItems) return E0M4_ERR_SHAPE;
    static std::atomic<uint64_t> lds_allowed{0};
    const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(&grouped_many_kernel<FMT, G, GATED, TM, WN, KS>), lds, lds_allowed);
    if (rc != E0M4_OK) return rc;
    hipLaunchKernelGGL((grouped_many_kernel<FMT, G, GATED, TM, WN, KS>), dim3((unsigned)grid), dim3(threads), lds, stream, static_cast<const char*>(a.X),
                       static_cast<const char*>(a.codes), a.Y, a.plan, a.rows, a.groups, a.N, a.K, a.n_tiles, a.share, a.share_reciprocal);
    return check_launch();
}

template <int FMT, int G, bool GATED>
int launch_many_shape(const ManyArgs& a, int64_t rows, int64_t groups, int height, int columns, hipStream_t stream)
{
    if (height == 128 && columns == 256) return launch_many<FMT, G, GATED, 4, 4, 1>(a, rows, groups, stream);
    if (height == 128 && columns == 128) return launch_many<FMT, G, GATED, 4, 2, 2>(a, rows, groups, stream);
    if (height == 64 && columns == 128) return launch_many<FMT, G, GATED, 2, 2, 4>(a, rows, groups, stream);
    return E0M4_ERR_SHAPE;
}

}  // namespace

int launch_grouped_many(const GroupedArgs& g, int format, int height, int columns, hipStream_t stream)
{
    ManyArgs a;
    a.X = g.X;
    a.codes = g.codes;
    a.Y = g.Y;
    a.plan = g.plan;
    a.rows = (int)g.rows;
    a.groups = (int)g.groups;
    a.N = (uint32_t)g.N;
    a.K = (uint32_t)g.K;
    a.n_tiles = 0;
    a.share = (uint32_t)g.share;
    a.share_reciprocal = small_reciprocal(g.share);
    auto go = [&](auto fmt_c, auto g_c) -> int {
        constexpr int FMT = decltype(fmt_c)::value, G = decltype(g_c)::value;
        return g.swiglu ? launch_many_shape<FMT, G, true>(a, g.rows, g.groups, height, columns, stream)
                        : launch_many_shape<FMT, G, false>(a, g.rows, g.groups, height, columns, stream);
    };
    using G32 = std::integral_constant<int, 32>;
    using G64 = std::integral_constant<int, 64>;
    using G128 = std::integral_constant<int, 128>;
    if (format == kGroupedE8) return go(std::integral_constant<int, kGroupedE8>{}, G128{});
    auto go_g = [&](auto fmt_c) -> int { return g.group == 32 ? go(fmt_c, G32{}) : g.group == 64 ? go(fmt_c, G64{}) : go(fmt_c, G128{}); };
    return format == kGroupedBf16 ? go_g(std::integral_constant<int, kGroupedBf16>{}) : go_g(std::integral_constant<int, kGroupedFp16>{});
}

}  // namespace e0m4
