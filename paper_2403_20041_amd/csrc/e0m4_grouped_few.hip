// Products of a layout's rows with the quantised weights of their groups, few rows to a group (e0m4_matmul_grouped and its like): tiles of 16 or 32
// rows of one group, the weight operand of the matrix cores made in registers from the packed codes.
//     Y[p, n] = sum_k X[row(p), k] * dequant(codes of p's group)[n, k], and with the gated product silu(gate) * up of the two halves of n.
//
// A workgroup has one tile and R consecutive row blocks (16 weight rows; R / 2 blocks of the gate and the same of the up projection); its four
// wavefronts take every fourth k block, each with its own part of X, and add their sums in LDS at the end, in order.  The rows of X come
// from where the layout's entries say, straight to LDS, whole rows of a k block, and are turned around there into the matrix cores' operands; rows that
// a tile lacks are requested beyond the buffer's end, which gives zeros without an access to memory.
// What bounds it: the stream of the used groups' weights, which come once for every tile; X comes from L2 for every R row blocks.  32 tokens with 8 of
// 128 experts, 2048 x 768 in groups of 64: 19 us, 5 TB/s; 13 with 2 of 8, gated 27392 x 4096 in 8 bits: 121 us where six of the experts are read, 694 MB, 156 where all are, 926.  One token with 8 of 128, gated
// 1536 x 2048: 6.0 us of which 2.7 are its bytes' (the tile, its rows, their data and the sums are one chain).  More rows to a tile than 32, and more row
// blocks than four, were slower throughout (64 rows 66 - 82 us where 16 take 35).
#include "e0m4_groups.h"

#include <algorithm>
#include <type_traits>

namespace e0m4 {

namespace {

typedef unsigned int u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float floatx2 __attribute__((ext_vector_type(2)));

constexpr int kFewWaves = 4;
constexpr int kFewThreads = kFewWaves * 64;
// K blocks of weights that a wavefront has under way (R 2 or 4).  One less, these and one more: 64 tokens with 8 of 128 experts, gated 1536 x 2048, 36.0, 36.0 and 38.4 us with
// 16 rows and R 4, 36.2, 35.6 and 38.0 with R 2, 39.2, 42.4 and 43.1 with 32 rows; 8 with 2 of 8, 14336 x 4096, 38.4, 38.3 and 39.9, 35.5, 35.8 and 38.1, 40.9, 43.3 and 44.2.
constexpr int few_weights_ahead(int R) { return R == 4 ? 2 : 3; }

struct FewArgs {
    const void* X;
    const void* codes;
    void* Y;
    const void* plan;
    int rows, groups;
    uint32_t N, K;
    uint32_t chunks;                            // workgroups of a tile
    uint32_t kind;                              // log2 of the codes' group, and 16 times the entries per row of X (0: rows lie in the layout's order)
    uint32_t share_reciprocal;
};

template <int N, int I = 0, typename F>
__device__ inline void for_each_of(F&& f)
{
    if constexpr (I < N) {
        f(std::integral_constant<int, I>{});
        for_each_of<N, I + 1>(f);
    }
}

// MT: tiles of 16 rows; R: row blocks.  Every weight is rounded to 16 bits before the product, as the dequant entry points do: a row's result
// depends on the tile that it falls into only by the order of sums.  (The codes' exact values, with scale and bias applied to a group's sums in
// fp32, would take 28 instead of 60 vector instructions per weight operand and 4 - 6 % less time, bfloat16 6 - 12 %, and be off by half a step of
// each weight: 35.0 and 33.1 us for 64 tokens with 8 of 128 experts, gated 1536 x 2048.)
// (Arguments one by one, in registers from the start.)
template <int FMT, int MT, int R, bool GATED>
__global__ __launch_bounds__(kFewThreads, 2) void grouped_few_kernel(const char* X, const char* codes, void* Y, const void* plan, int rows, int groups, uint32_t N,
                                                                       uint32_t K, uint32_t chunks, uint32_t kind, uint32_t share_reciprocal)
{
    constexpr int NP = FMT == kGroupedE8 ? 2 : 4;       // MFMAs per k block
    constexpr int BLK = NP * 32;                        // weights of a row per k block
    constexpr int DW = few_weights_ahead(R);
    constexpr int PPR = NP * 4, RPI = 64 / PPR, RB = PPR * 16, XE = NP;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const GroupPlan lay = plan_view(plan, rows, groups);
    constexpr int HEIGHT = MT - 1;
    static_assert(tile_height(HEIGHT) == 16 * MT, "a list of tiles");
    const uint32_t share = kind >> 4;
    const int group_shift = (int)(kind & 15);
    const uint32_t tile_no = (uint32_t)__builtin_amdgcn_readfirstlane((int)(blockIdx.x / chunks)), chunk = blockIdx.x - tile_no * chunks;
    // (the list has room for a tile that is not there)
    const GroupTile tile = lay.tiles[HEIGHT][tile_no];
    if ((int)tile_no >= lay.class_ends[HEIGHT][kTileClasses - 1]) return;
    const int first = tile.begin + ((int)tile_no - tile.first_tile) * (16 * MT);
    const int M = min(16 * MT, tile.end - first);       // rows of this tile
    const int nkb = (int)((K + BLK - 1) / BLK);
    const int pw = kBlockRows << (7 - group_shift);   // parameter words per k block (8-bit codes: 16)
    const uint32_t rb_stride = (uint32_t)nkb * (uint32_t)(kBlockCodeBytes + 4 * pw);

    const int t = threadIdx.x;
    const int lane = t & 63;
    const int wave = __builtin_amdgcn_readfirstlane(t >> 6);
    const int n_l = lane & 15, g_l = lane >> 4;
    const uint32_t fmask = frac_mask_vgpr();
    const uint32_t half_blocks = N / 2 / kBlockRows;
    const uint32_t blocks = GATED ? half_blocks : (N + kBlockRows - 1) / kBlockRows;      // of a half
    constexpr int RH = GATED ? R / 2 : R;               // row blocks of a half
    const uint32_t rb0 = chunk * RH;
    const char* wg_base = codes + (int64_t)tile.group * ((int64_t)((N + kBlockRows - 1) / kBlockRows) * rb_stride) + (uint64_t)rb0 * rb_stride;
    uint32_t rb_off[R];                                 // (beyond the last: that one again, its sums are not used); gated: gate, up, gate, up
#pragma unroll
    for (int r = 0; r < R; ++r) {
        const uint32_t s = min((uint32_t)(GATED ? r / 2 : r), blocks - 1 - rb0) + (GATED && (r & 1) ? half_blocks : 0u);
        rb_off[r] = (uint32_t)__builtin_amdgcn_readfirstlane((int)(s * rb_stride));
    }
    const uint32_t code_voff = lane * 16;
    const uint32_t param_voff = (uint32_t)nkb * kBlockCodeBytes + 4 * (((g_l * kCodesPerChunk) >> group_shift) * kBlockRows + n_l);
    const uint32_t pb = 4 * pw;
    u32x4 c[DW][R];
    uint32_t pwd[DW][R];
    auto load_w = [&](int kb, int d) {
        const __amdgpu_buffer_rsrc_t rsrc = rsrc_if(wg_base, kb < nkb);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            c[d][r] = __builtin_amdgcn_raw_buffer_load_b128(rsrc, (int)code_voff, (int)(rb_off[r] + (uint32_t)kb * kBlockCodeBytes), 0);
            pwd[d][r] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, (int)param_voff, (int)(rb_off[r] + (uint32_t)kb * pb), 0);
        }
    };
    // Rows of X.  (row, 16-byte piece) of a k block lies at row * RB + 16 * (piece ^ swizzle(row)), by the choice of the piece that a lane
    // loads: the 16 rows of an operand read fall into 16 different bank groups.
    unsigned char* xl = smem + wave * (MT * 16 * RB);
    auto swizzle = [](int row) -> int { return FMT == kGroupedE8 ? (row >> 1) & 7 : row & 15; };
    const char* x_base = share ? X : X + (int64_t)first * K * 2;
    constexpr uint32_t kNowhere = 0x80000000u;          // beyond the resource, whatever is added to it
    uint32_t x_voff[MT][XE], x_rd[NP];
    const int last_piece = (int)(K - (uint32_t)(nkb - 1) * BLK) / 8;    // pieces of a row in the last k block
    bool x_tail[XE];
#pragma unroll
    for (int e = 0; e < XE; ++e) {
        const int j = (lane % PPR) ^ swizzle(e * RPI + lane / PPR);
        x_tail[e] = j >= last_piece;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
            const int row = 16 * i + e * RPI + lane / PPR;
            uint32_t at = (uint32_t)row;
            if (share && row < M) at = small_quotient((uint32_t)lay.order[first + row], share_reciprocal);
            x_voff[i][e] = row < M ? at * (K * 2) + (uint32_t)j * 16 : kNowhere;
        }
    }
#pragma unroll
    for (int e = 0; e < NP; ++e) x_rd[e] = (uint32_t)(n_l * RB + (((g_l * NP + e) ^ swizzle(n_l)) << 4));
    auto load_x = [&](int kb) {
        const __amdgpu_buffer_rsrc_t rsrc = rsrc_if(x_base, kb < nkb);
#pragma unroll
        for (int i = 0; i < MT; ++i)
#pragma unroll
            for (int e = 0; e < XE; ++e) {
                const uint32_t voff = kb == nkb - 1 && x_tail[e] ? kNowhere : x_voff[i][e];
                load_to_lds_b128(rsrc, xl + (i * 16 + e * RPI) * RB, voff, (uint32_t)kb * RB);
            }
    };
#pragma unroll
    for (int d = 0; d < DW; ++d) {
        if (d == 0) load_x(wave);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        load_w(wave + d * kFewWaves, d);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    }

    auto pair = [](half2_t w1, half2_t bias2, half2_t scale2) -> half2_t { return (w1 - bias2) * scale2; };  // difference exact, product rounded once
    // the weight operand of MFMA p: word p of the chunk (8-bit codes: words 2p and 2p + 1), to the bits of the dequant entry points
    auto dequant = [&](const u32x4& cc, uint32_t pw1, int p) -> half8_t {
        if (FMT == kGroupedBf16) {
            // one fp32 fused multiply-add per weight (products and difference are exact), then one rounding
            const float sf = __builtin_bit_cast(float, pw1 << 16);
            const float nb = -__builtin_bit_cast(float, pw1 & 0xFFFF0000u) * sf;
            const half2_t q[4] = {w1_pair<0>(cc[p], fmask), w1_pair<1>(cc[p], fmask), w1_pair<2>(cc[p], fmask), w1_pair<3>(cc[p], fmask)};
            bf16x2_t o[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const floatx2 f = {__builtin_fmaf((float)q[e][0], sf, nb), __builtin_fmaf((float)q[e][1], sf, nb)};
                o[e] = __builtin_convertvector(f, bf16x2_t);
            }
            return *reinterpret_cast<const half8_t*>(o);
        }
        const half_t sc = param_scale(pw1), bi = param_bias(pw1);
        const half2_t s2 = {sc, sc}, b2 = {bi, bi};
        half2_t o[4];
        if (FMT == kGroupedE8) {
            const uint32_t m8 = fmask | (fmask >> 4);   // eight fraction bits of both halves
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t w8 = cc[2 * (p & 1) + h];
                o[2 * h] = pair(__builtin_bit_cast(half2_t, (w8 & m8) | kExpBits2), b2, s2);
                o[2 * h + 1] = pair(__builtin_bit_cast(half2_t, (__builtin_amdgcn_alignbit(w8, w8, 8) & m8) | kExpBits2), b2, s2);
            }
        } else {
            o[0] = pair(w1_pair<0>(cc[p], fmask), b2, s2);
            o[1] = pair(w1_pair<1>(cc[p], fmask), b2, s2);
            o[2] = pair(w1_pair<2>(cc[p], fmask), b2, s2);
            o[3] = pair(w1_pair<3>(cc[p], fmask), b2, s2);
        }
        return *reinterpret_cast<const half8_t*>(o);
    };
    auto mfma = [](const half8_t& x, const half8_t& w, const floatx4& v) -> floatx4 {
        if constexpr (FMT == kGroupedBf16)
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, x), __builtin_bit_cast(bf16x8_t, w), v, 0, 0, 0);
        else return __builtin_amdgcn_mfma_f32_16x16x32_f16(x, w, v, 0, 0, 0);
    };
    floatx4 acc[R][MT];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < MT; ++i) acc[r][i] = floatx4{0.f, 0.f, 0.f, 0.f};

    // One k block: its X from LDS to registers, whereupon the next one's is requested into the same place; its weights' registers are
    // requested again for DW of this wavefront's blocks on.
    auto block = [&](auto rest_c, int kb, auto u_c) {
        constexpr int u = decltype(u_c)::value;
        // (behind this block's X, requested in the block before, come only that block's weights; behind the first block's all of the
        // prologue's)
        if (u == 0 && kb < kFewWaves) wait_loads<DW * 2 * R>();
        else wait_loads<(decltype(rest_c)::value && u > 0) ? 0 : 2 * R>();
        half8_t xa[NP][MT];
#pragma unroll
        for (int p = 0; p < NP; ++p)
#pragma unroll
            for (int i = 0; i < MT; ++i) xa[p][i] = *reinterpret_cast<const half8_t*>(xl + i * (16 * RB) + x_rd[p]);
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");          // read before it is written again
        __builtin_amdgcn_sched_barrier(0);
        if (!decltype(rest_c)::value || kb + kFewWaves < nkb) load_x(kb + kFewWaves);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int p = 0; p < NP; ++p) {
#pragma unroll
                for (int r = 0; r < R; ++r) {
                    const half8_t w = dequant(c[u % DW][r], pwd[u % DW][r], p);
#pragma unroll
                    for (int i = 0; i < MT; ++i) acc[r][i] = mfma(xa[p][i], w, acc[r][i]);
                }
            }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        load_w(kb + DW * kFewWaves, u % DW);
        asm volatile("" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
    };
    int kb = wave;
    for (; kb + (DW - 1) * kFewWaves < nkb; kb += DW * kFewWaves) {
        for_each_of<DW>([&](auto u_c) { block(std::false_type{}, kb + decltype(u_c)::value * kFewWaves, u_c); });
    }
    for_each_of<DW - 1>([&](auto u_c) {
        if (kb + decltype(u_c)::value * kFewWaves < nkb) block(std::true_type{}, kb + decltype(u_c)::value * kFewWaves, u_c);
    });

    // The wavefronts' sums, added in order: lane l holds rows 4 (l/16) .. + 3 of every 16, weight row l%16.
    floatx4* red = reinterpret_cast<floatx4*>(smem);    // [wavefronts][R][MT][64]
    wait_loads<0>();                                    // (what was requested beyond the last block has arrived)
    __syncthreads();
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < MT; ++i) red[((wave * R + r) * MT + i) * 64 + lane] = acc[r][i];
    __syncthreads();
    const int64_t n_out = GATED ? N / 2 : N;
    for (int idx = t; idx < RH * MT * 64; idx += kFewThreads) {
        const int s = idx / (MT * 64), i = (idx / 64) % MT, l = idx % 64;
        auto total = [&](int r) -> floatx4 {
            const floatx4* src = red + (r * MT + i) * 64 + l;
            floatx4 v = src[0];
#pragma unroll
            for (int w = 1; w < kFewWaves; ++w) v += src[w * R * MT * 64];
            return v;
        };
        floatx4 v = total(GATED ? 2 * s : s);
        if constexpr (GATED) {
            const floatx4 up = total(2 * s + 1);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = silu_f32(v[e]) * up[e];
        }
        const int64_t col = (int64_t)(rb0 + s) * kBlockRows + (l & 15);
        if (col >= n_out) continue;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const int m = 16 * i + 4 * (l >> 4) + e;
            if (m >= M) continue;
            const int64_t at = (int64_t)(first + m) * n_out + col;
            if (FMT == kGroupedBf16) static_cast<__bf16*>(Y)[at] = (__bf16)v[e];
            else static_cast<half_t*>(Y)[at] = (half_t)v[e];
        }
    }
}

template <int FMT, int MT, int R, bool GATED>
int launch_few(const FewArgs& f, hipStream_t stream)
{
    constexpr int lds = std::max(kFewWaves * R * MT * 64 * 16, kFewWaves * MT * 16 * (FMT == kGroupedE8 ? 128 : 256));
    FewArgs a = f;
    const uint32_t blocks = GATED ? a.N / 2 / kBlockRows : (uint32_t)row_blocks(a.N);
    constexpr uint32_t RH = GATED ? R / 2 : R;
    a.chunks = (blocks + RH - 1) / RH;
    const int64_t grid = grouped_workgroups(a.rows, a.groups, 16 * MT, a.chunks);
    if (grid * kFewThreads > kMaxWorkItems) return E0M4_ERR_SHAPE;
    static std::atomic<uint64_t> lds_allowed{0};
    const int rc = allow_dynamic_lds(reinterpret_cast<const void*>(&grouped_few_kernel<FMT, MT, R, GATED>), lds, lds_allowed);
    if (rc != E0M4_OK) return rc;
    hipLaunchKernelGGL((grouped_few_kernel<FMT, MT, R, GATED>), dim3((unsigned)grid), dim3(kFewThreads), lds, stream, static_cast<const char*>(a.X),
                       static_cast<const char*>(a.codes), a.Y, a.plan, a.rows, a.groups, a.N, a.K, a.chunks, a.kind, a.share_reciprocal);
    return check_launch();
}

template <int FMT, bool GATED>
int launch_few_as(const FewArgs& f, int height, int row_blocks, hipStream_t stream)
{
    if (height == 32 && row_blocks == 4) return launch_few<FMT, 2, 4, GATED>(f, stream);
    if (height == 16 && row_blocks == 4) return launch_few<FMT, 1, 4, GATED>(f, stream);
    if (height == 16 && row_blocks == 2) return launch_few<FMT, 1, 2, GATED>(f, stream);
    return E0M4_ERR_SHAPE;
}

}  // namespace

int launch_grouped_few(const GroupedArgs& a, int format, int height, int row_blocks, hipStream_t stream)
{
    FewArgs f;
    f.X = a.X;
    f.codes = a.codes;
    f.Y = a.Y;
    f.plan = a.plan;
    f.rows = (int)a.rows;
    f.groups = (int)a.groups;
    f.N = (uint32_t)a.N;
    f.K = (uint32_t)a.K;
    f.chunks = 0;
    f.kind = (uint32_t)a.share << 4 | (format == kGroupedE8 || a.group == 128 ? 7 : a.group == 64 ? 6 : 5);
    f.share_reciprocal = small_reciprocal(a.share);
    auto go = [&](auto fmt_c) -> int {
        constexpr int FMT = decltype(fmt_c)::value;
        return a.swiglu ? launch_few_as<FMT, true>(f, height, row_blocks, stream) : launch_few_as<FMT, false>(f, height, row_blocks, stream);
    };
    switch (format) {
        case kGroupedFp16: return go(std::integral_constant<int, kGroupedFp16>{});
        case kGroupedE8: return go(std::integral_constant<int, kGroupedE8>{});
        default: return go(std::integral_constant<int, kGroupedBf16>{});
    }
}

}  // namespace e0m4
