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
// count in order.  Few entries are one workgroup's work (choice, counts, places and tiles in one launch); otherwise a first launch
// chooses and counts per workgroup, and every workgroup of a second one adds up the counts before its own.
// What bounds it: launches, and the chains of a few hundred dependent instructions in each.
#include "e0m4_groups.h"

#include <float.h>

namespace e0m4 {

namespace {

constexpr int kWg = 1024;
constexpr int kWaves = kWg / 64;
// Entries of a call that one workgroup takes
constexpr int64_t kOneWorkgroup = 2048;
constexpr int kCountEntries = 256;              // entries of a workgroup of the first of two launches, at least
constexpr int kCountThreads = 256;

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

struct Route {
    const void* logits;
    int64_t tokens, logits_ld;
    int dtype, groups, k, sigmoid, renormalise;
    float factor;
    const int* count;
    int* experts;
    float* weights;
};

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

// Experts and weights of tokens first ... last - 1 by a workgroup of THREADS.
template <int THREADS, int LANES, int PER>
__device__ inline void choose_tokens(const Route& a, int64_t first, int64_t last)
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
            a.experts[token * a.k + lane] = token < there ? expert : -1;
            a.weights[token * a.k + lane] = token < there ? weight : 0.f;
        }
    }
}

__device__ inline int group_of(int index, int groups) { return (unsigned)index < (unsigned)groups ? index : groups; }

// Running sums over the workgroup's threads of five numbers each; before[i] is the sum over the threads before this one, total[i] over all.
struct Five {
    int v[1 + kTileHeights];
};
__device__ inline Five scan_five(const Five& mine, Five (&waves)[kWaves])
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    Five s = mine;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
#pragma unroll
        for (int i = 0; i < 1 + kTileHeights; ++i) {
            const int o = __shfl_up(s.v[i], d);
            if (lane >= d) s.v[i] += o;
        }
    }
    if (lane == 63) waves[wave] = s;
    __syncthreads();
    Five before = s;
#pragma unroll
    for (int i = 0; i < 1 + kTileHeights; ++i) before.v[i] -= mine.v[i];
    for (int w = 0; w < wave; ++w) {
#pragma unroll
        for (int i = 0; i < 1 + kTileHeights; ++i) before.v[i] += waves[w].v[i];
    }
    return before;
}

struct Layout {
    GroupPlan plan;
    int64_t rows;
    const int* index;
    int groups;
    int bits;                                   // of a group's number, that of `groups` itself included
};

// LDS of the layout's workgroups
struct LayoutLds {
    int next[kMaxGroups + 1];                   // where the next entry of a group goes
    int first[1 + kTileHeights][kMaxGroups + 1];// where groups (and their tiles of each height) begin
    uint16_t chunk[kWaves][kMaxGroups + 1];     // entries of a group in a wavefront's 64
    Five waves[kWaves];
};

// Offsets and tile lists, part `part` of `parts` (rows of a group: `total` of thread g), and next[g] = begin of g + before.
__device__ inline void lay_out_groups(const Layout& a, LayoutLds& lds, int total, int before, int part, int parts)
{
    const int g = threadIdx.x;
    Five mine = {};
    if (g <= a.groups) {
        mine.v[0] = total;
#pragma unroll
        for (int i = 0; i < kTileHeights; ++i) mine.v[1 + i] = g < a.groups ? (total + tile_height(i) - 1) / tile_height(i) : 0;
    }
    const Five begin = scan_five(mine, lds.waves);
    if (g <= a.groups) {
        lds.next[g] = begin.v[0] + before;
#pragma unroll
        for (int i = 0; i < 1 + kTileHeights; ++i) lds.first[i][g] = begin.v[i];
        if (part == 0) {
            a.plan.offsets[g] = begin.v[0];
            if (g == a.groups) {
#pragma unroll
                for (int i = 0; i < kTileHeights; ++i) a.plan.tile_counts[i] = begin.v[1 + i];
            }
        }
    }
    __syncthreads();
#pragma unroll 1
    for (int i = 0; i < kTileHeights; ++i) {
        const int* first = lds.first[1 + i];
        const int tiles = first[a.groups];
        for (int t = part * kWg + threadIdx.x; t < tiles; t += parts * kWg) {
            int lo = 0, hi = a.groups;          // the last group that begins at or before t
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if (first[mid] <= t) lo = mid;
                else hi = mid;
            }
            // (of groups that begin at the same tile all but the last are empty)
            a.plan.tiles[i][t] = GroupTile{lo, first[lo], lds.first[0][lo], lds.first[0][lo + 1]};
        }
    }
}

// Entries first ... last - 1 to their places, 1024 at a time.
__device__ inline void place_entries(const Layout& a, LayoutLds& lds, int64_t first, int64_t last)
{
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    for (int64_t base = first; base < last; base += kWg) {
        if ((int)threadIdx.x <= a.groups) {
#pragma unroll
            for (int w = 0; w < kWaves; ++w) lds.chunk[w][threadIdx.x] = 0;
        }
        __syncthreads();
        const int64_t entry = base + threadIdx.x;
        const bool in = entry < last;
        const int g = in ? group_of(a.index[entry], a.groups) : 0;
        uint64_t like = __ballot(in);
        for (int b = 0; b < a.bits; ++b) {
            const uint64_t set = __ballot((g >> b) & 1);
            like &= ((g >> b) & 1) ? set : ~set;
        }
        const int rank = __popcll(like & (((uint64_t)1 << lane) - 1));
        if (in && rank == 0) lds.chunk[wave][g] = (uint16_t)__popcll(like);
        __syncthreads();
        if ((int)threadIdx.x <= a.groups) {     // counts of the wavefronts before
            int sum = 0;
#pragma unroll
            for (int w = 0; w < kWaves; ++w) {
                const int n = lds.chunk[w][threadIdx.x];
                lds.chunk[w][threadIdx.x] = (uint16_t)sum;
                sum += n;
            }
            lds.first[0][threadIdx.x] = sum;    // (the groups' begins are not needed any more)
        }
        __syncthreads();
        if (in) {
            const int to = lds.next[g] + lds.chunk[wave][g] + rank;
            a.plan.order[to] = (int)entry;
            a.plan.place[entry] = g < a.groups ? to : -1;
        }
        __syncthreads();
        if ((int)threadIdx.x <= a.groups) lds.next[threadIdx.x] += lds.first[0][threadIdx.x];
    }
}

// Few entries: everything in one workgroup.
template <int LANES, int PER, bool CHOOSE>
__global__ __launch_bounds__(kWg) void route_small_kernel(Route r, Layout a)
{
    __shared__ LayoutLds lds;
    int* count = lds.first[1];                  // (read by the thread of its group before begins come there)
    if ((int)threadIdx.x <= a.groups) count[threadIdx.x] = 0;
    if constexpr (CHOOSE) choose_tokens<kWg, LANES, PER>(r, 0, r.tokens);
    __syncthreads();                            // (the choice is read back by other threads of the workgroup: the barrier waits for the stores)
    for (int64_t i = threadIdx.x; i < a.rows; i += kWg) atomicAdd(&count[group_of(a.index[i], a.groups)], 1);
    __syncthreads();
    lay_out_groups(a, lds, (int)threadIdx.x <= a.groups ? count[threadIdx.x] : 0, 0, 0, 1);
    __syncthreads();
    place_entries(a, lds, 0, a.rows);
}

// Many entries, first launch: the choice, and counts of the workgroup's entries.
template <int LANES, int PER, bool CHOOSE>
__global__ __launch_bounds__(kCountThreads) void route_count_kernel(Route r, Layout a, int64_t tokens_each)
{
    __shared__ int count[kMaxGroups + 1];
    for (int i = threadIdx.x; i <= a.groups; i += kCountThreads) count[i] = 0;
    const int64_t first = (int64_t)blockIdx.x * tokens_each, last = min(first + tokens_each, r.tokens);
    if constexpr (CHOOSE) choose_tokens<kCountThreads, LANES, PER>(r, first, last);
    if (a.plan.offsets == nullptr) return;      // (no layout is wanted)
    __syncthreads();
    for (int64_t i = first * r.k + threadIdx.x; i < last * r.k; i += kCountThreads) atomicAdd(&count[group_of(a.index[i], a.groups)], 1);
    __syncthreads();
    for (int i = threadIdx.x; i <= a.groups; i += kCountThreads) a.plan.counts[(int64_t)blockIdx.x * (a.groups + 1) + i] = count[i];
}

// ... second launch: workgroup p places the entries that workgroups p * each ... of the first counted.
__global__ __launch_bounds__(kWg) void route_place_kernel(Layout a, int blocks, int each, int64_t entries_each)
{
    __shared__ LayoutLds lds;
    int *total = lds.first[1], *before = lds.first[2];     // (read by the thread of their group before begins come there)
    const int n = a.groups + 1;
    if ((int)threadIdx.x < n) total[threadIdx.x] = before[threadIdx.x] = 0;
    __syncthreads();
    // Thread (part, g) adds up every parts-th workgroup's count of g.
    const int parts = kWg / n, g = threadIdx.x % n, part = threadIdx.x / n, mine = blockIdx.x * each;
    if (part < parts) {
        int sum = 0, early = 0;
        for (int b = part; b < blocks; b += parts) {
            const int c = a.plan.counts[(int64_t)b * n + g];
            sum += c;
            early += b < mine ? c : 0;
        }
        atomicAdd(&total[g], sum);
        atomicAdd(&before[g], early);
    }
    __syncthreads();
    const bool in = (int)threadIdx.x < n;
    lay_out_groups(a, lds, in ? total[threadIdx.x] : 0, in ? before[threadIdx.x] : 0, blockIdx.x, gridDim.x);
    __syncthreads();
    place_entries(a, lds, mine * entries_each, min((int64_t)(mine + each) * entries_each, a.rows));
}

template <int LANES, int PER, bool CHOOSE>
int launch_route_as(const Route& r, const Layout& a, hipStream_t stream)
{
    if (a.plan.offsets && a.rows <= kOneWorkgroup) {
        hipLaunchKernelGGL((route_small_kernel<LANES, PER, CHOOSE>), dim3(1), dim3(kWg), 0, stream, r, a);
        return check_launch();
    }
    int64_t each = (kCountEntries + r.k - 1) / r.k;
    if (each * kMaxCountBlocks < r.tokens) each = (r.tokens + kMaxCountBlocks - 1) / kMaxCountBlocks;
    const int blocks = (int)((r.tokens + each - 1) / each);
    hipLaunchKernelGGL((route_count_kernel<LANES, PER, CHOOSE>), dim3((unsigned)blocks), dim3(kCountThreads), 0, stream, r, a, each);
    const int rc = check_launch();
    if (rc != E0M4_OK || !a.plan.offsets) return rc;
    const int together = each * r.k < kWg ? (int)(kWg / (each * r.k)) : 1;
    hipLaunchKernelGGL(route_place_kernel, dim3((unsigned)((blocks + together - 1) / together)), dim3(kWg), 0, stream, a, blocks, together, each * r.k);
    return check_launch();
}

}  // namespace

int launch_route(const RouteArgs& args, void* plan, hipStream_t stream)
{
    const Route r{args.logits, args.tokens, args.logits_ld, args.dtype, args.groups, args.k, args.sigmoid, args.renormalise, args.factor, args.count, args.experts,
                  args.weights};
    Layout a = {};
    a.rows = args.tokens * args.k;
    if (plan) a.plan = plan_view(plan, a.rows, args.groups);
    a.index = args.experts;
    a.groups = args.groups;
    while ((1 << a.bits) <= args.groups) ++a.bits;
    if (!args.logits) return launch_route_as<16, 1, false>(r, a, stream);
    if (args.groups <= 16) return launch_route_as<16, 1, true>(r, a, stream);
    if (args.groups <= 64) return launch_route_as<16, 4, true>(r, a, stream);
    if (args.groups <= 128) return launch_route_as<16, 8, true>(r, a, stream);
    if (args.groups <= 256) return launch_route_as<16, 16, true>(r, a, stream);
    return launch_route_as<64, 16, true>(r, a, stream);
}

// ---- weighted sum of a token's rows ----------------------------------------------------------------------------------

namespace {

constexpr int kCombineThreads = 256;

// A wavefront: 64 pieces of V columns of one token.  All of a token's rows are requested before the first is used; sums in fp32, in the order
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
