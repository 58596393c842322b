// Rows laid out by the weights that they choose: the router's choice of experts, the layout of the entries by expert, and the weighted
// sum of a token's rows.
//
// Choice: a token is LANES lanes, each with every LANES-th logit in registers.  k times the largest is found (a maximum in each lane, then over
// the lanes by DPP), and the lowest index among those that equal it; what was chosen becomes -infinity, which no logit is (they are
// clamped to finite numbers).  softmax over the chosen ones: exp(l - largest) / sum, sigmoid: through
// log sigmoid(l) = min(l, 0) - log1p(exp(-|l|)), so that the weights of very unlikely experts still add up to one.
//
// Layout: a stable counting sort.  The entries of a group keep their order, so results depend on nothing but the choice: counts are
// integers, an entry's rank among its like within a wavefront comes from ballots over the bits of its group, and wavefronts and workgroups
// count in order.  Up to 1024 entries are one workgroup's work (choice, counts, places and tiles in one launch), of 64 tokens at most, as many as it
// chooses for at once; otherwise a first launch chooses and counts per workgroup, and every workgroup of a second one adds up the counts before its own.
// What bounds it: launches, and the chains of a few hundred dependent instructions in each.  One token of 64 experts 4.7 us, 32 of 128 with 8 chosen 8.7, 128
// 10.9, 4096 13.3 in a graph (traced, the choice 6.3 and the places 7.7).
#include "e0m4_groups.h"

#include <float.h>

namespace e0m4 {

namespace {

constexpr int kWg = 1024;                       // threads of a workgroup that lays entries out
// ... of few tokens by few experts: its barriers are cheaper.  In 256 and 1024 threads one token of 64 experts takes 4.7 and 6.2 us, 16 of 128 with 8 chosen 6.3 and 8.6, as
// many as it chooses for at once; 60 of 16 with 2 chosen 5.7 and 4.5, 64 of 64 with 4 chosen 9.0 and 5.9.
constexpr int kSmallWg = 256;
constexpr int kSmallTokens = 16;
// More tokens to choose for, or entries than threads: two launches.  64 of 64 experts with 4 chosen 5.9 us in one and 9.6 in two, of 128 with 8 chosen 8.9 and 10.3; 128 of
// them 13.8 and 10.9, 256 of 64 with 4 chosen 12.2 and 10.4 (128 of those 8.0 and 10.0).
constexpr int kOneWorkgroupTokens = 64;
constexpr int kCountThreads = 512;
// Entries of a workgroup of the first of two launches, at least.  128, 256 and 512: 4096 tokens of 128 experts with 8 chosen 14.8, 13.3 and 16.2 us, 128 of them 11.0, 10.9
// and 14.2; 256 of 64 with 4 chosen 9.0, 10.4 and 14.0.
constexpr int kCountEntries = 256;

template <int LANES>
__device__ inline float lanes_max(float v)
{
    v = fmaxf(v, other_lane<0xB1>(v));
    v = fmaxf(v, other_lane<0x4E>(v));
    v = fmaxf(v, other_lane<0x141>(v));
    v = fmaxf(v, other_lane<0x140>(v));
    if (LANES == 64) {
        v = fmaxf(v, __shfl_xor(v, 16));
        v = fmaxf(v, __shfl_xor(v, 32));
    }
    return v;
}
template <int CTRL>
__device__ inline uint32_t other_lane_u32(uint32_t v)
{
    return (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, CTRL, 0xF, 0xF, true);
}
template <int LANES>
__device__ inline uint32_t lanes_min(uint32_t v)
{
    v = min(v, other_lane_u32<0xB1>(v));
    v = min(v, other_lane_u32<0x4E>(v));
    v = min(v, other_lane_u32<0x141>(v));
    v = min(v, other_lane_u32<0x140>(v));
    if (LANES == 64) {
        v = min(v, (uint32_t)__shfl_xor((int)v, 16));
        v = min(v, (uint32_t)__shfl_xor((int)v, 32));
    }
    return v;
}
// (the order of the additions is the same in all lanes: both sides of an exchange add the same two numbers)
template <int LANES>
__device__ inline float lanes_sum(float v)
{
    v += other_lane<0xB1>(v);
    v += other_lane<0x4E>(v);
    v += other_lane<0x141>(v);
    v += other_lane<0x140>(v);
    if (LANES == 64) {
        v += __shfl_xor(v, 16);
        v += __shfl_xor(v, 32);
    }
    return v;
}

// (as kernel arguments one by one, in registers from the start)
struct Route {
    const void* logits;
    int* experts;
    float* weights;
    const int* count;
    int64_t logits_ld;
    int tokens, groups;
    float factor;
    int dtype, k, sigmoid, renormalise;
};
#define ROUTE_PARAMETERS const void *logits, int *experts, float *weights, void *plan, const int *count, int64_t logits_ld, int tokens, int groups, float factor, uint32_t kind
#define ROUTE_ARGUMENTS a.logits, a.experts, a.weights, plan, a.count, a.logits_ld, (int)a.tokens, a.groups, a.factor, \
                        (uint32_t)(a.dtype | a.sigmoid << 2 | a.renormalise << 3 | a.k << 4)
#define ROUTE Route{logits, experts, weights, count, logits_ld, tokens, groups, factor, (int)(kind & 3), (int)(kind >> 4), (int)(kind >> 2 & 1), (int)(kind >> 3 & 1)}

__device__ inline float logit_at(const Route& a, int64_t at)
{
    float v;
    if (a.dtype == E0M4_FP32) v = static_cast<const float*>(a.logits)[at];
    else if (a.dtype == E0M4_BF16) v = __builtin_bit_cast(float, (uint32_t)static_cast<const uint16_t*>(a.logits)[at] << 16);
    else v = (float)static_cast<const half_t*>(a.logits)[at];
    // finite numbers, NaN the lowest
    return v == v ? fminf(fmaxf(v, -FLT_MAX), FLT_MAX) : -FLT_MAX;
}

// The k experts of one token (LANES lanes, PER logits each) and their weights; lane j < k gets the j-th.
template <int LANES, int PER>
__device__ inline void choose(const Route& a, int64_t token, int lane, int& expert, float& weight)
{
    float v[PER];
    const int64_t row = token * a.logits_ld;
#pragma unroll
    for (int i = 0; i < PER; ++i) {
        const int e = i * LANES + lane;
        v[i] = e < a.groups ? logit_at(a, row + e) : -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < PER; ++i) top = fmaxf(top, v[i]);
    top = lanes_max<LANES>(top);
    float all = 0.f;
    if (!a.sigmoid && !a.renormalise) {
#pragma unroll
        for (int i = 0; i < PER; ++i) all += expf(v[i] - top);
        all = lanes_sum<LANES>(all);
    }
    float mine = -INFINITY, best = top;
    expert = -1;
    for (int j = 0; j < a.k; ++j) {
        if (j > 0) {
            best = v[0];
#pragma unroll
            for (int i = 1; i < PER; ++i) best = fmaxf(best, v[i]);
            best = lanes_max<LANES>(best);
        }
        uint32_t at = 0xFFFFFFFFu;
#pragma unroll
        for (int i = PER - 1; i >= 0; --i) at = v[i] == best ? (uint32_t)(i * LANES + lane) : at;
        at = lanes_min<LANES>(at);
        if (lane == j) {
            mine = best;
            expert = (int)at;
        }
#pragma unroll
        for (int i = 0; i < PER; ++i) v[i] = at == (uint32_t)(i * LANES + lane) ? -INFINITY : v[i];
    }
    const bool one = lane < a.k;
    if (a.sigmoid && !a.renormalise) {
        weight = one ? 1.f / (1.f + expf(-mine)) : 0.f;
    } else {
        float s = mine;
        if (a.sigmoid) s = fminf(mine, 0.f) - log1pf(expf(-fabsf(mine)));
        // (the first chosen one has the largest score of either kind)
        const float largest = a.sigmoid ? lanes_max<LANES>(one ? s : -INFINITY) : top;
        const float p = one ? expf(s - largest) : 0.f;
        const float total = lanes_sum<LANES>(p);
        weight = p / (a.renormalise ? total : all);
    }
    weight *= a.factor;
}

// Experts and weights of tokens first ... last - 1 by a workgroup of THREADS; `kept` gets the experts too.
template <int THREADS, int LANES, int PER>
__device__ inline void choose_tokens(const Route& a, int64_t first, int64_t last, int* kept)
{
    const int lane = threadIdx.x % LANES;
    const int64_t there = a.count ? (int64_t)min(max(a.count[0], 0), 0x7fffffff) : a.tokens;
    // (all lanes of a wavefront stay, for the exchanges among them)
    for (int64_t base = first; base < last; base += THREADS / LANES) {
        const int64_t token = base + threadIdx.x / LANES;
        int expert;
        float weight;
        choose<LANES, PER>(a, token < last ? token : last - 1, lane, expert, weight);
        if (token < last && lane < a.k) {
            const int chosen = token < there ? expert : -1;
            a.experts[token * a.k + lane] = chosen;
            a.weights[token * a.k + lane] = token < there ? weight : 0.f;
            kept[(token - first) * a.k + lane] = chosen;
        }
    }
}

__device__ inline int group_of(int index, int groups) { return (unsigned)index < (unsigned)groups ? index : groups; }

// Numbers of a group that are summed up over the groups before it: rows, tiles of 16, 32 and 64 rows, tiles of 128 rows by class.
constexpr int kSums = 1 + (kTileHeights - 1) + kTileClasses;
struct Sums {
    int v[kSums];
};
template <int CTRL, int ROWS>
__device__ inline int shifted(int v)                    // another lane's v, 0 where there is none
{
    return __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xF, false);
}
// Sums over the threads before this one, and over the first `threads`.
template <int WAVES>
__device__ inline void scan(const Sums& mine, Sums& before, Sums& all, Sums (&waves)[WAVES], int threads)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Sums s = mine;
#pragma unroll
    for (int i = 0; i < kSums; ++i) {                   // within rows of 16 lanes, then over the rows
        int v = s.v[i];
        v += shifted<0x111, 0xF>(v);
        v += shifted<0x112, 0xF>(v);
        v += shifted<0x114, 0xF>(v);
        v += shifted<0x118, 0xF>(v);
        v += shifted<0x142, 0xA>(v);
        v += shifted<0x143, 0xC>(v);
        s.v[i] = v;
    }
    if (lane == 63) waves[wave] = s;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kSums; ++i) {
        before.v[i] = s.v[i] - mine.v[i];
        all.v[i] = 0;
    }
    for (int w = 0; w * 64 < threads; ++w) {
#pragma unroll
        for (int i = 0; i < kSums; ++i) {
            const int n = waves[w].v[i];
            if (w < wave) before.v[i] += n;
            all.v[i] += n;
        }
    }
}

struct Layout {
    GroupPlan plan;
    int64_t rows;
    const int* index;
    int groups;
    int bits;                                   // of a group's number, that of `groups` itself included
};
__device__ inline Layout make_layout(const void* plan, const int* index, int rows, int groups)
{
    return Layout{plan_view(plan, rows, groups), rows, index, groups, 32 - __builtin_clz((unsigned)groups)};
}

// Offsets and tile lists, part `part` of `parts`; thread g has group g (`total` rows), the one behind the last those of none.  Where its entries begin.
template <int WAVES>
__device__ inline int lay_out_groups(const Layout& a, int total, int part, int parts, Sums (&waves)[WAVES])
{
    const int g = threadIdx.x;
    Sums mine = {}, before, all;
    const int last = total % tile_height(kTileHeights - 1), whole = total / tile_height(kTileHeights - 1);
    const int last_class = last == 0 ? -1 : last > 96 ? 0 : last > 64 ? 1 : last > 32 ? 2 : 3;
    if (g <= a.groups) mine.v[0] = total;
    if (g < a.groups) {
#pragma unroll
        for (int i = 0; i < kTileHeights - 1; ++i) mine.v[1 + i] = (total + tile_height(i) - 1) / tile_height(i);
        mine.v[kTileHeights] = whole + (last_class == 0 ? 1 : 0);
#pragma unroll
        for (int c = 1; c < kTileClasses; ++c) mine.v[kTileHeights + c] = last_class == c ? 1 : 0;
    }
    scan(mine, before, all, waves, a.groups + 1);
    const int begin = before.v[0], end = begin + total;
    if (g <= a.groups && part == 0) {
        a.plan.offsets[g] = begin;
        if (g == a.groups) {
            int sum = 0;
#pragma unroll
            for (int i = 0; i < kTileHeights - 1; ++i) {
#pragma unroll
                for (int c = 0; c < kTileClasses; ++c) a.plan.class_ends[i][c] = all.v[1 + i];
            }
#pragma unroll
            for (int c = 0; c < kTileClasses; ++c) {
                sum += all.v[kTileHeights + c];
                a.plan.class_ends[kTileHeights - 1][c] = sum;
            }
        }
    }
    if (g < a.groups) {
#pragma unroll
        for (int i = 0; i < kTileHeights - 1; ++i) {
            for (int t = part; t < mine.v[1 + i]; t += parts) a.plan.tiles[i][before.v[1 + i] + t] = GroupTile{g, before.v[1 + i], begin, end};
        }
        GroupTile* tiles = a.plan.tiles[kTileHeights - 1];
        const int whole_end = last_class == 0 ? end : begin + whole * tile_height(kTileHeights - 1);
        for (int t = part; t < mine.v[kTileHeights]; t += parts)
            tiles[before.v[kTileHeights] + t] = GroupTile{g, before.v[kTileHeights], begin, whole_end};
        int of_class = all.v[kTileHeights];             // where the class begins
#pragma unroll
        for (int c = 1; c < kTileClasses; ++c) {
            if (last_class == c && part == 0) tiles[of_class + before.v[kTileHeights + c]] = GroupTile{g, of_class + before.v[kTileHeights + c], whole_end, end};
            of_class += all.v[kTileHeights + c];
        }
    }
    return begin;
}

// Rank of an entry among those of its group in its wavefront, and how many there are.
__device__ inline int rank_among_like(int g, bool in, int bits, int& like_in_wave)
{
    uint64_t like = __ballot(in);
    for (int b = 0; b < bits; ++b) {
        const uint64_t set = __ballot((g >> b) & 1);
        like &= ((g >> b) & 1) ? set : ~set;
    }
    like_in_wave = __popcll(like);
    return __popcll(like & (((uint64_t)1 << (threadIdx.x & 63)) - 1));
}

template <int THREADS>
struct LayoutLds {
    int next[THREADS];                          // where the next entry of a group goes
    uint16_t chunk[THREADS / 64][THREADS];      // entries of a group in a wavefront's 64, then in those of the wavefronts before
    Sums waves[THREADS / 64];
};
template <int THREADS>
__device__ inline void clear_chunks(LayoutLds<THREADS>& lds, int groups)
{
    if ((int)threadIdx.x <= groups) {
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) lds.chunk[w][threadIdx.x] = 0;
    }
}
// Thread g: chunk[w][g] becomes the sum over the wavefronts before w; the sum over all.
template <int THREADS>
__device__ inline int sum_chunks(LayoutLds<THREADS>& lds, int groups)
{
    int sum = 0;
    if ((int)threadIdx.x <= groups) {
        int n[THREADS / 64];
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) n[w] = lds.chunk[w][threadIdx.x];
#pragma unroll
        for (int w = 0; w < THREADS / 64; ++w) {
            lds.chunk[w][threadIdx.x] = (uint16_t)sum;
            sum += n[w];
        }
    }
    return sum;
}

// Few entries, one to a thread at most, and groups, one to a thread with the one behind the last: everything in one workgroup.
template <int THREADS, int LANES, int PER, bool CHOOSE>
__global__ __launch_bounds__(THREADS) void route_small_kernel(ROUTE_PARAMETERS)
{
    const Route r = ROUTE;
    const Layout a = make_layout(plan, experts, tokens * r.k, groups);
    __shared__ LayoutLds<THREADS> lds;
    __shared__ int kept[THREADS];
    clear_chunks(lds, a.groups);
    const int t = threadIdx.x;
    const bool in = t < (int)a.rows;
    if constexpr (CHOOSE) choose_tokens<THREADS, LANES, PER>(r, 0, r.tokens, kept);
    __syncthreads();
    const int g = in ? group_of(CHOOSE ? kept[t] : a.index[t], a.groups) : 0;
    int like;
    const int rank = rank_among_like(g, in, a.bits, like);
    if (in && rank == 0) lds.chunk[t >> 6][g] = (uint16_t)like;
    __syncthreads();
    const int total = sum_chunks(lds, a.groups);
    lds.next[t] = lay_out_groups(a, total, 0, 1, lds.waves);
    __syncthreads();
    if (in) {
        const int to = lds.next[g] + lds.chunk[t >> 6][g] + rank;
        a.plan.order[to] = t;
        a.plan.place[t] = g < a.groups ? to : -1;
    }
}

// Many entries, first launch: the choice, and counts of the workgroup's entries.
template <int LANES, int PER, bool CHOOSE>
__global__ __launch_bounds__(kCountThreads) void route_count_kernel(ROUTE_PARAMETERS, int tokens_each)
{
    const Route r = ROUTE;
    const Layout a = make_layout(plan, experts, tokens * r.k, groups);
    __shared__ int counted[kMaxGroups + 1];
    __shared__ int kept[kCountThreads / LANES * kMaxChoices];
    for (int i = threadIdx.x; i <= a.groups; i += kCountThreads) counted[i] = 0;
    const int64_t first = (int64_t)blockIdx.x * tokens_each, last = min(first + tokens_each, (int64_t)r.tokens);
    __syncthreads();
    if constexpr (CHOOSE) {
        // (as many tokens at a time as the workgroup has lanes for)
        for (int64_t at = first; at < last; at += kCountThreads / LANES) {
            const int64_t to = min(at + kCountThreads / LANES, last);
            choose_tokens<kCountThreads, LANES, PER>(r, at, to, kept);
            if (plan == nullptr) continue;    // (no layout is wanted)
            __syncthreads();
            for (int i = threadIdx.x; i < (int)(to - at) * r.k; i += kCountThreads) atomicAdd(&counted[group_of(kept[i], a.groups)], 1);
            __syncthreads();
        }
    } else {
        for (int64_t i = first + threadIdx.x; i < last; i += kCountThreads) atomicAdd(&counted[group_of(a.index[i], a.groups)], 1);
        __syncthreads();
    }
    if (plan == nullptr) return;
    for (int i = threadIdx.x; i <= a.groups; i += kCountThreads) a.plan.counts[(int64_t)blockIdx.x * (a.groups + 1) + i] = counted[i];
}

// ... second launch: workgroup p places the entries that workgroups p * each ... of the first counted.
__global__ __launch_bounds__(kWg) void route_place_kernel(const int* index, void* plan, int rows, int groups, int blocks, int each, int64_t entries_each)
{
    const Layout a = make_layout(plan, index, rows, groups);
    __shared__ LayoutLds<kWg> lds;
    __shared__ int total[kWg], before[kWg];
    const int n = a.groups + 1, t = threadIdx.x;
    if (t < n) total[t] = before[t] = 0;
    __syncthreads();
    // Thread (part, g) adds up every parts-th workgroup's count of g.
    const int parts = kWg / n, g_mine = t % n, part = t / n, mine = blockIdx.x * each;
    if (part < parts) {
        int sum = 0, early = 0;
        const int* counts = a.plan.counts + g_mine;
        for (int b = part; b < blocks; b += parts * 8) {
            int c[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) c[i] = b + i * parts < blocks ? counts[(b + i * parts) * n] : 0;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                sum += c[i];
                early += b + i * parts < mine ? c[i] : 0;
            }
        }
        atomicAdd(&total[g_mine], sum);
        atomicAdd(&before[g_mine], early);
    }
    __syncthreads();
    const int begin = lay_out_groups(a, t < n ? total[t] : 0, blockIdx.x, gridDim.x, lds.waves);
    lds.next[t] = begin + (t < n ? before[t] : 0);
    // 1024 entries at a time
    const int64_t first = mine * entries_each, last = min((int64_t)(mine + each) * entries_each, a.rows);
    for (int64_t base = first; base < last; base += kWg) {
        clear_chunks(lds, a.groups);
        __syncthreads();
        const int64_t entry = base + t;
        const bool in = entry < last;
        const int g = in ? group_of(a.index[entry], a.groups) : 0;
        int like;
        const int rank = rank_among_like(g, in, a.bits, like);
        if (in && rank == 0) lds.chunk[t >> 6][g] = (uint16_t)like;
        __syncthreads();
        const int sum = sum_chunks(lds, a.groups);
        __syncthreads();
        if (in) {
            const int to = lds.next[g] + lds.chunk[t >> 6][g] + rank;
            a.plan.order[to] = (int)entry;
            a.plan.place[entry] = g < a.groups ? to : -1;
        }
        __syncthreads();
        if (t <= a.groups) lds.next[t] += sum;
    }
}

template <int LANES, int PER, bool CHOOSE>
int launch_route_as(const RouteArgs& a, void* plan, hipStream_t stream)
{
    const int64_t rows = a.tokens * a.k;
    if (plan && rows <= kSmallWg && a.tokens <= (CHOOSE ? kSmallTokens : kSmallWg) && a.groups < kSmallWg) {
        hipLaunchKernelGGL((route_small_kernel<kSmallWg, LANES, PER, CHOOSE>), dim3(1), dim3(kSmallWg), 0, stream, ROUTE_ARGUMENTS);
        return check_launch();
    }
    if (plan && rows <= kWg && (!CHOOSE || a.tokens <= kOneWorkgroupTokens)) {
        hipLaunchKernelGGL((route_small_kernel<kWg, LANES, PER, CHOOSE>), dim3(1), dim3(kWg), 0, stream, ROUTE_ARGUMENTS);
        return check_launch();
    }
    int64_t each = (kCountEntries + a.k - 1) / a.k;
    if (each * kMaxCountBlocks < a.tokens) each = (a.tokens + kMaxCountBlocks - 1) / kMaxCountBlocks;
    const int blocks = (int)((a.tokens + each - 1) / each);
    const int together = each * a.k < kWg ? (int)(kWg / (each * a.k)) : 1;
    if (blocks == 0) return E0M4_OK;
    hipLaunchKernelGGL((route_count_kernel<LANES, PER, CHOOSE>), dim3((unsigned)blocks), dim3(kCountThreads), 0, stream, ROUTE_ARGUMENTS, (int)each);
    const int rc = check_launch();
    if (rc != E0M4_OK || !plan) return rc;
    hipLaunchKernelGGL(route_place_kernel, dim3((unsigned)((blocks + together - 1) / together)), dim3(kWg), 0, stream, a.experts, plan, (int)rows, a.groups,
                       blocks, together, each * a.k);
    return check_launch();
}

}  // namespace

int launch_route(const RouteArgs& a, void* plan, hipStream_t stream)
{
    if (!a.logits) return launch_route_as<16, 1, false>(a, plan, stream);
    if (a.groups <= 16) return launch_route_as<16, 1, true>(a, plan, stream);
    if (a.groups <= 64) return launch_route_as<16, 4, true>(a, plan, stream);
    if (a.groups <= 128) return launch_route_as<16, 8, true>(a, plan, stream);
    if (a.groups <= 256) return launch_route_as<16, 16, true>(a, plan, stream);
    return launch_route_as<64, 16, true>(a, plan, stream);
}

// ---- weighted sum of a token's rows ----------------------------------------------------------------------------------

namespace {

constexpr int kCombineThreads = 256;

// Bound by memory: 4096 tokens with 8 rows of 2048, bfloat16, 168 MB in 30 us.  A wavefront: 64 pieces of V columns of one token.  All of a token's rows are requested before the first is used; sums in fp32, in the order
// of the token's choices, one rounding.
template <typename T, int V>
__global__ __launch_bounds__(kCombineThreads) void combine_kernel(const T* __restrict__ Y, const float* __restrict__ weights, const int* __restrict__ place,
                                                                  const T* base, T* out, int64_t items, uint32_t chunks, int64_t N, int k)
{
    typedef T vec __attribute__((ext_vector_type(V)));
    const int64_t item = (int64_t)blockIdx.x * (kCombineThreads / 64) + __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
    if (item >= items) return;
    const uint32_t token = (uint32_t)__builtin_amdgcn_readfirstlane((int)((uint32_t)item / chunks));
    const int64_t col = ((int64_t)((uint32_t)item - token * chunks) * 64 + (threadIdx.x & 63)) * V;
    if (col >= N) return;
    float sum[V];
    const int64_t o = (int64_t)token * N + col;
    if (base) {
        const vec b = *reinterpret_cast<const vec*>(base + o);
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] = (float)b[e];
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] = 0.f;
    }
    constexpr int AT = 8;
    for (int j0 = 0; j0 < k; j0 += AT) {
        vec y[AT];
#pragma unroll
        for (int j = 0; j < AT; ++j) {
            if (j0 + j < k) {
                const int at = place[(int64_t)token * k + j0 + j];
                if (at >= 0) y[j] = *reinterpret_cast<const vec*>(Y + (int64_t)at * N + col);
            }
        }
#pragma unroll
        for (int j = 0; j < AT; ++j) {
            if (j0 + j < k && place[(int64_t)token * k + j0 + j] >= 0) {
                const float w = weights[(int64_t)token * k + j0 + j];
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] = __builtin_fmaf(w, (float)y[j][e], sum[e]);
            }
        }
    }
    vec r;
#pragma unroll
    for (int e = 0; e < V; ++e) r[e] = (T)sum[e];
    *reinterpret_cast<vec*>(out + o) = r;
}

template <typename T, int V>
int launch_combine_as(const void* Y, int64_t N, const float* weights, const int* place, int64_t tokens, int k, const void* base, void* out, hipStream_t stream)
{
    const int64_t chunks = (N + 64 * V - 1) / (64 * V), items = tokens * chunks, blocks = (items + kCombineThreads / 64 - 1) / (kCombineThreads / 64);
    if (items > 0x7fffffffLL || blocks * kCombineThreads > 0xffffffffLL) return E0M4_ERR_SHAPE;
    hipLaunchKernelGGL((combine_kernel<T, V>), dim3((unsigned)blocks), dim3(kCombineThreads), 0, stream, static_cast<const T*>(Y), weights, place,
                       static_cast<const T*>(base), static_cast<T*>(out), items, (uint32_t)chunks, N, k);
    return check_launch();
}

template <typename T>
int launch_combine_t(const void* Y, int64_t N, const float* weights, const int* place, int64_t tokens, int k, const void* base, void* out, hipStream_t stream)
{
    if (N % 8 == 0) return launch_combine_as<T, 8>(Y, N, weights, place, tokens, k, base, out, stream);
    if (N % 2 == 0) return launch_combine_as<T, 2>(Y, N, weights, place, tokens, k, base, out, stream);
    return launch_combine_as<T, 1>(Y, N, weights, place, tokens, k, base, out, stream);
}

}  // namespace

int launch_combine(const void* Y, int64_t N, const float* weights, const void* plan, int64_t tokens, int k, int64_t groups, const void* base, void* out, int dtype,
                   hipStream_t stream)
{
    const int* place = plan_view(plan, tokens * k, groups).place;
    return dtype == E0M4_BF16 ? launch_combine_t<__bf16>(Y, N, weights, place, tokens, k, base, out, stream)
                              : launch_combine_t<half_t>(Y, N, weights, place, tokens, k, base, out, stream);
}

}  // namespace e0m4
