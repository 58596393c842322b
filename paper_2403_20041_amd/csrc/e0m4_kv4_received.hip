// What the rows of a cache in E0M4 codes received: received[j] += sum over rows of queries of 2^(score - reference) times what the
// attention left for the row (e0m4_kv4.h, norm).  Scores are formed a second time: kept from the first, they would take four bytes each, 8 / dim of the
// operations' time at the card's rates, twice.
//
// A workgroup owns 256 rows of the cache, so no two add to one number.  Four pairs of wavefronts hold 64 rows of K each as operands in
// registers, dequantised once; all rows of queries pass by through LDS, 64 at a time, half of them for either wavefront of a pair.
// A lane sums what its own query gives to its rows of K; lanes and pairs meet at the end.
//
// Bound: arithmetic of the exponentials beside the products, and the first rows of a causal prompt, which all queries see: 2048 tokens,
// 40 heads in 49 to 53 us.
#include "e0m4_kv4_attention.h"

namespace e0m4 {

namespace {

constexpr int kThreads = 512, kKeys = 256, kQueries = 64;

template <int DIM, int G>
__global__ __launch_bounds__(kThreads) void kv4_received_kernel(Kv4Attention a, float* __restrict__ received)
{
    using L = Kv4<DIM, G>;
    constexpr int kSteps = DIM / 16, kStride = DIM + 8, kPerRow = DIM / 8, kPieces = kQueries * kPerRow / kThreads;
    __shared__ __attribute__((aligned(16))) half_t staged[2][kQueries * kStride];
    __shared__ float part[2][kKeys];
    const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), col = lane & 31, kh = lane >> 5;
    const int set = wave & 3, half = wave >> 2, rows = a.n_new * a.share;
    // rows of the cache that most queries see first
    const int h = blockIdx.x % a.kv_heads, b = blockIdx.y, key0 = kv4_place(a) * kKeys;
    const int length = clamp_count(a.lengths[b], a.capacity), count = a.counts ? clamp_count(a.counts[b], a.n_new) : a.n_new;
    if (key0 >= length || count == 0) return;
    const int64_t bh = (int64_t)b * a.kv_heads + h;
    // queries that may see one of the workgroup's rows
    const int first = length - count;
    int i0 = 0, i1 = count;
    if (a.causal) {
        const int last = key0 + kKeys < length ? key0 + kKeys - 1 : length - 1;
        i0 = key0 - first > 0 ? key0 - first : 0;
        if (a.window && last + a.window - first < i1) i1 = last + a.window - first;
    }
    const int begin = i0 * a.share / kQueries * kQueries, end = i1 * a.share;
    if (begin >= end) return;

    // K: row 32 u + col of the wavefront's 64, dims 16 w + 8 kh
    const int own = key0 + 64 * set;
    const uint32_t hi = frac_mask_vgpr(), lo = frac_mask_low_vgpr();
    half8_t k[2][kSteps];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
        const int64_t tile = own / kKv4Rows + u;
        const __amdgpu_buffer_rsrc_t rs = rsrc_if(a.cache + (bh * a.tiles + tile) * L::kBytes, tile < a.tiles);
#pragma unroll
        for (int w = 0; w < kSteps; ++w) {
            const int d = 16 * w + 8 * kh;
            const uint32_t word = __builtin_amdgcn_raw_buffer_load_b32(rs, L::k_word(col, d), 0, 0);
            const uint32_t param = __builtin_amdgcn_raw_buffer_load_b32(rs, L::k_param(col, d / G), 0, 0);
            k[u][w] = kv4_values(word, param, hi, lo);
        }
    }

    // queries, an iteration ahead in registers; a lane's own factor and sum
    words4_t raw[kPieces];
    float factor, next_factor;
    float2 norm, next_norm;
    const half_t* packed = a.packed_q + bh * rows * DIM;
    auto load = [&](int row0) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const int r = row0 + (t + i * kThreads) / kPerRow;
            raw[i] = words4_t{0, 0, 0, 0};
            if (r < rows) raw[i] = *reinterpret_cast<const words4_t*>(packed + (int64_t)r * DIM + t % kPerRow * 8);
        }
        const int r = row0 + 32 * half + col;
        next_factor = 0.f;
        next_norm = float2{0.f, 0.f};
        if (r < rows) {
            next_factor = a.factors[bh * rows + r];
            next_norm = a.norm[bh * rows + r];
        }
    };
    auto store = [&](int into) {
#pragma unroll
        for (int i = 0; i < kPieces; ++i)
            *reinterpret_cast<words4_t*>(&staged[into][(t + i * kThreads) / kPerRow * kStride + t % kPerRow * 8]) = raw[i];
    };

    float got[2][16];
#pragma unroll
    for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 16; ++i) got[u][i] = 0.f;
    load(begin);
    store(0);
    factor = next_factor;
    norm = next_norm;
    load(begin + kQueries);
    int at = 0;
    for (int row0 = begin; row0 < end; row0 += kQueries, at ^= 1) {
        __syncthreads();
        const float by = factor, ref = norm.x, weight = norm.y;
        factor = next_factor;
        norm = next_norm;
        store(at ^ 1);
        load(row0 + 2 * kQueries);
        const int mine = row0 + 32 * half;              // this wavefront's rows of queries
        const int q0 = kv4_query_of(a, mine), q1 = kv4_query_of(a, mine + 31);
        if (a.causal && first + q1 < own) continue;     // (they see none of its rows)
        const half_t* q = &staged[at][(32 * half + col) * kStride + 8 * kh];
        floatx16 s[2];
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) s[u][i] = 0.f;
#pragma unroll
        for (int w = 0; w < kSteps; ++w) {
            const half8_t qq = *reinterpret_cast<const half8_t*>(q + 16 * w);
#pragma unroll
            for (int u = 0; u < 2; ++u) s[u] = __builtin_amdgcn_mfma_f32_32x32x16_f16(k[u][w], qq, s[u], 0, 0, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kDsRead, kAhead, 0);
#pragma unroll
        for (int i = 0; i < kSteps - kAhead; ++i) {
            __builtin_amdgcn_sched_group_barrier(kMfma, 2, 0);
            __builtin_amdgcn_sched_group_barrier(kDsRead, 1, 0);
        }
        __builtin_amdgcn_sched_group_barrier(kMfma, 2 * kAhead, 0);
        auto row_of = [&](int u, int i) { return own + 32 * u + 8 * (i >> 2) + 4 * kh + (i & 3); };
        uint32_t seen = ~0u;
        if (a.mask) {
            const int query = kv4_query_of(a, mine + col);
            seen = kv4_mask_bits<8>(a, b, query < count ? query : 0, [&](int g) { return own + 8 * g + 4 * kh; });
        }
        const bool some = a.mask || (a.causal && first + q0 + 1 < own + 64) || (a.window && first + q1 - a.window + 1 > own);
        if (some) {
            const Kv4Seen by_place = kv4_seen(a, length, first + kv4_query_of(a, mine + col));
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) {
                    const bool in = row_of(u, i) >= by_place.from && row_of(u, i) < by_place.to && (seen >> (16 * u + i)) & 1;
                    const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], by, -ref));
                    got[u][i] = in ? __builtin_fmaf(e, weight, got[u][i]) : got[u][i];
                }
        } else {
#pragma unroll
            for (int u = 0; u < 2; ++u)
#pragma unroll
                for (int i = 0; i < 16; ++i) got[u][i] = __builtin_fmaf(__builtin_amdgcn_exp2f(__builtin_fmaf(s[u][i], by, -ref)), weight, got[u][i]);
        }
    }
    // 32 sums over 32 lanes: at each step a lane gives away half of its sums and adds the other half of another's, until lane `col` has
    // the sum of number 16 u + i = col
    float v[32];
#pragma unroll
    for (int i = 0; i < 32; ++i) v[i] = got[i >> 4][i & 15];
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1)
#pragma unroll
        for (int i = 0; i < d; ++i) {
            float low = v[i], high = v[i + d];
            asm volatile("" : "+v"(low), "+v"(high));   // (or the choice becomes one of an index that no register has)
            v[i] = (col & d ? high : low) + __shfl_xor(col & d ? low : high, d);
        }
    part[half][64 * set + 32 * (col >> 4) + 8 * ((col >> 2) & 3) + 4 * kh + (col & 3)] = v[0];
    __syncthreads();
    if (t < kKeys && key0 + t < length) received[bh * a.capacity + key0 + t] += part[0][t] + part[1][t];
}

}  // namespace

int launch_kv4_received(const Kv4Attention& a, const e0m4_kv4_shape& s, float* received, hipStream_t stream)
{
    const dim3 grid = kv4_place_grid(a, (s.capacity + kKeys - 1) / kKeys);
    return kv4_dispatch(s, [&](auto shape) -> int {
        constexpr int DIM = decltype(shape)::kDim, G = decltype(shape)::kGroup;
        hipLaunchKernelGGL((kv4_received_kernel<DIM, G>), grid, dim3(kThreads), 0, stream, a, received);
        return check_launch();
    });
}

}  // namespace e0m4
