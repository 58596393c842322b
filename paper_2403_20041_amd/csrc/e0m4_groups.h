// Rows laid out by the weights that they choose (e0m4_groups, e0m4_route): the memory of such a layout, and what the kernels that read it need
// of it.
#pragma once

#include "e0m4_device.h"
#include "e0m4_host.h"

namespace e0m4 {

constexpr int64_t kMaxGroupRows = (int64_t)1 << 24;
constexpr int kMaxGroups = 1023;                // with the group of rows that choose none, one thread of a workgroup each
constexpr int kMaxChoices = 16;                 // experts of a token
constexpr int kMaxShare = 255;                  // entries per row of X

// Tiles: rows of one group, so many at most.  A kernel has a workgroup (or several) for every tile of the height that it was built for;
// how many there are only the device knows, so it is launched for as many as there can be.  Tiles of 128 rows are listed by classes, those of
// more than 96, 64, 32 rows and the others, each by groups: long work comes first, and every XCD gets its share of each.
constexpr int kTileHeights = 4;
constexpr int kTileClasses = 4;
__host__ __device__ constexpr int tile_height(int i) { return 16 << i; }    // 16, 32, 64, 128
__host__ __device__ inline int64_t most_tiles(int64_t rows, int64_t groups, int height) { return rows / height + (groups < rows ? groups : rows); }

struct GroupTile {
    int group;
    int first_tile;                             // of the group, in this list (and class)
    int begin, end;                             // the rows of these tiles: positions in the layout
};

// Layout in memory, in 32-bit words: offsets [groups + 1], order [rows] and place [rows], each padded to a multiple of four words, then
// where the classes of each height end in its list (heights below 128: one class), the lists of tiles, and the counts of the first
// launch's workgroups.  Kernels are given its beginning and find the rest themselves: arguments that fit the registers that a launch fills (14 to 16 of
// them) are there at once, others cost a load from memory each time that they are first used, 6 us of a kernel of 15.
__host__ __device__ constexpr int64_t round4(int64_t n) { return (n + 3) & ~(int64_t)3; }
constexpr int64_t kMaxCountBlocks = 256;
struct GroupPlan {
    int* offsets;
    int* order;
    int* place;
    int* class_ends[kTileHeights];              // [kTileClasses]
    GroupTile* tiles[kTileHeights];
    int* counts;                                // [workgroups][groups + 1]
};
inline int64_t plan_words(int64_t rows, int64_t groups)
{
    int64_t n = round4(groups + 1) + 2 * round4(rows) + kTileHeights * kTileClasses;
    for (int i = 0; i < kTileHeights; ++i) n += 4 * most_tiles(rows, groups, tile_height(i));
    return n + kMaxCountBlocks * round4(groups + 1);
}
__host__ __device__ inline GroupPlan plan_view(const void* plan, int64_t rows, int64_t groups)
{
    int* w = static_cast<int*>(const_cast<void*>(plan));
    GroupPlan p;
    p.offsets = w;
    p.order = p.offsets + round4(groups + 1);
    p.place = p.order + round4(rows);
    int* at = p.place + round4(rows);
    for (int i = 0; i < kTileHeights; ++i, at += kTileClasses) p.class_ends[i] = at;
    for (int i = 0; i < kTileHeights; ++i) {
        p.tiles[i] = reinterpret_cast<GroupTile*>(at);
        at += 4 * most_tiles(rows, groups, tile_height(i));
    }
    p.counts = at;
    return p;
}

// x / d for x < 2^24, 1 <= d <= 255: the product with the rounded-up reciprocal is off by less than x / 2^32 < 1 / d.
__host__ __device__ inline uint32_t small_reciprocal(int64_t d) { return d > 1 ? (uint32_t)((((uint64_t)1 << 32) + d - 1) / d) : 0; }
__device__ inline uint32_t small_quotient(uint32_t x, uint32_t reciprocal) { return reciprocal ? __umulhi(x, reciprocal) : x; }

// The expert choice of a router, and the layout (see e0m4.h).  logits null: `experts` is read, one entry per token, and laid out.
struct RouteArgs {
    const void* logits;
    int dtype;
    int64_t tokens, logits_ld;
    int groups, k, sigmoid, renormalise;
    float factor;
    const int* count;
    int* experts;
    float* weights;
};
int launch_route(const RouteArgs& a, void* plan, hipStream_t stream);
int launch_combine(const void* Y, int64_t N, const float* weights, const void* plan, int64_t tokens, int k, int64_t groups, const void* base, void* out,
                   int dtype, hipStream_t stream);

// Products of the rows of a layout with their groups' weights (see e0m4.h).
struct GroupedArgs {
    const void* X;
    int64_t share;                              // entries per row of X; 0: rows lie in the layout's order
    const void* plan;
    int64_t rows, groups;
    const void* codes;
    int64_t N, K;
    int group;
    bool swiglu;
    void* Y;
};
enum { kGroupedFp16 = 0, kGroupedE8 = 1, kGroupedBf16 = 2 };
// Workgroups of a launch: one for each tile and block of columns; for tiles of 64 or 128 rows each XCD takes a contiguous run of every class.
constexpr int kNumXcd = 8;
constexpr int64_t kMaxWorkItems = 0xffffffff;           // of a launch
inline int64_t grouped_workgroups(int64_t rows, int64_t groups, int height, int64_t column_blocks)
{
    const int64_t n = most_tiles(rows, groups, height) * column_blocks;
    return height < 64 ? n : (n / kNumXcd + kTileClasses) * kNumXcd;
}
int launch_grouped_few(const GroupedArgs& a, int format, int height, int row_blocks, hipStream_t stream);     // tiles of 16 or 32 rows
int launch_grouped_many(const GroupedArgs& a, int format, int height, int columns, hipStream_t stream);       // tiles of 64 or 128 rows

// Low-rank adapters of rows (see e0m4.h).
struct LoraArgs {
    const void* X;
    int64_t x_ld;
    const void* plan;
    int64_t rows, adapters;
    const void* A;
    const void* B;
    int rank;
    const float* factors;
    int64_t N, K;
    const void* base;
    int64_t base_ld;
    void* out;
    int64_t out_ld;
    int dtype;
};
size_t lora_workspace_bytes(int64_t rows, int64_t adapters, int rank, int64_t N, int64_t K);
int launch_lora(const LoraArgs& a, void* workspace, hipStream_t stream);

}  // namespace e0m4
