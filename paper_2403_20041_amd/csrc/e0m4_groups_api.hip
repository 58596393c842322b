// C entries of the operators of rows that choose their weights: argument checks and the choice of kernels.  Every check happens on the host
// before anything is enqueued.
#include "e0m4_groups.h"

#include <math.h>

namespace e0m4 {

namespace {

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool overlap(const void* a, size_t a_bytes, const void* b, size_t b_bytes)
{
    const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
    return p < q + b_bytes && q < p + a_bytes;
}
// Rows of `bytes`, a_ld and b_ld bytes apart.  Columns of one wider matrix lie between each other without touching.
bool rows_overlap(const void* a, int64_t a_ld, const void* b, int64_t b_ld, int64_t rows, int64_t bytes)
{
    if (!overlap(a, (size_t)((rows - 1) * a_ld + bytes), b, (size_t)((rows - 1) * b_ld + bytes))) return false;
    if (a_ld != b_ld) return true;
    const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
    const int64_t apart = (int64_t)((p > q ? p - q : q - p) % (uintptr_t)a_ld);
    return apart < bytes || apart > a_ld - bytes;
}

// Kernels go where the layout says: results written over one would send those that still read it out of range.
bool overlaps_plan(const void* p, size_t bytes, const void* plan, int64_t rows, int64_t groups)
{
    return overlap(p, bytes, plan, (size_t)plan_words(rows, groups) * 4);
}

int check_groups(int64_t rows, int64_t groups)
{
    return rows < 0 || rows > kMaxGroupRows || groups < 1 || groups > kMaxGroups ? E0M4_ERR_SHAPE : E0M4_OK;
}

// Gathered rows of X are reached by 32-bit offsets from its first byte, a gate's up projection from the gate.
constexpr int64_t kMaxXBytes = 0x7fffffff;

// 8-bit codes: k blocks of 64
int64_t row_block_bytes(int64_t K, int group, int format)
{
    return format == kGroupedE8 ? (K + 63) / 64 * block_bytes(128) : k_blocks(K) * (int64_t)block_bytes(group);
}

int check_grouped(int64_t rows, int64_t groups, int64_t share, int64_t N, int64_t K, int group, int epilogue, int format)
{
    const int rc = check_groups(rows, groups);
    if (rc != E0M4_OK) return rc;
    if (format == kGroupedE8 ? group != 64 && group != 128 : group != 32 && group != 64 && group != 128) return E0M4_ERR_GROUP;
    if (N < 0 || N > (int64_t)1 << 24 || K < 1 || K > (int64_t)1 << (format == kGroupedE8 ? 19 : 20) || K % 32 != 0 || K % group != 0) return E0M4_ERR_SHAPE;
    if (share < 0 || share > kMaxShare || (share > 0 && rows % share != 0)) return E0M4_ERR_SHAPE;
    if (epilogue != E0M4_EPILOGUE_NONE && epilogue != E0M4_EPILOGUE_SWIGLU) return E0M4_ERR_SHAPE;
    if (epilogue == E0M4_EPILOGUE_SWIGLU && (N % 64 != 0 || N / 2 / kBlockRows * row_block_bytes(K, group, format) > kMaxHalfBytes)) return E0M4_ERR_SHAPE;
    if (share > 0 && rows / share * K * 2 > kMaxXBytes) return E0M4_ERR_SHAPE;
    return E0M4_OK;
}

// The forms of the product, and what an estimate of their launches' time goes by, in us: with w the workgroups for each of the 256 compute units, r rows of a
// tile that exist on average and b k blocks of 128 that a part of a workgroup walks,
//     start + b * max(one + one_row r, (full + full_row r) w) + each w,
// one and full each times a factor of bfloat16's or the 8-bit format's own.  Workgroups are counted as if every row chose a group, at random.
// The constants are a least-squares fit (logarithm of the ratio to the measurement, rms 10 - 14 %) to 8803 problems, each timed in all forms: 4 to 128
// groups, 1 to 250 rows to a group, gated and plain, 512 to 27392 columns, 512 to 14080 weights a row, all formats and groups; replays of a graph of 5 or 20 calls on one set of
// inputs, the least of four (430 of them are in tests/golden/grouped_form_timings.txt).  Choosing by the
// estimate costs 1.8 % over the best form of each (geometric mean); without one of the forms 2.1 - 2.5 %, without the second 5.5, without the
// fourth 8.6.  A seventh, 128 x 256 with two parts of K (10 - 15 % less time where the fourth has a workgroup for every second compute unit), would gain 0.2 %
// on all.
struct GroupedForm {
    int height;                                         // rows of a tile
    int columns;                                        // weight rows of a workgroup
    int parts;                                          // of K, side by side
    double start, one, one_row, full, full_row, each;
    double one_bf16, one_e8, full_bf16, full_e8;
};
constexpr GroupedForm kGroupedForms[] = {
    {16, 64, 4, 3.653, 0.6849, 0.0060, 0.7829, 0.0, 0.066, 1.138, 1.121, 1.095, 1.562},
    {16, 32, 4, 3.242, 0.3820, 0.0123, 0.3880, 0.0, 0.112, 1.172, 1.409, 1.056, 1.514},
    {32, 64, 4, 4.058, 0.8297, 0.0028, 0.8736, 0.0040, 0.354, 1.102, 1.082, 1.066, 1.386},
    {128, 256, 1, 4.313, 0.7466, 0.0054, 0.8479, 0.0084, 0.327, 1.168, 1.122, 1.091, 1.386},
    {64, 128, 4, 4.279, 1.1730, 0.0124, 1.5709, 0.0167, 3.818, 1.167, 1.120, 1.123, 1.334},
    {128, 128, 2, 3.982, 0.7367, 0.0077, 0.9139, 0.0105, 2.610, 1.149, 1.131, 1.101, 1.319},
};
constexpr int kGroupedFormCount = sizeof(kGroupedForms) / sizeof(kGroupedForms[0]);
constexpr int kFewestWorkItems = 3;

const GroupedForm& choose_form(int64_t rows, int64_t groups, int64_t N, int64_t K, bool gated, int format)
{
    const int force = knob(Knob::grouped_form);
    if (force >= 1 && force <= kGroupedFormCount) return kGroupedForms[force - 1];
    const double used = fmax(1.0, groups * (1.0 - exp(-(double)rows / groups)));
    const GroupedForm* best = &kGroupedForms[kFewestWorkItems];      // (which refuses the call if no form's grid has room for it)
    double least = INFINITY;
    for (const GroupedForm& f : kGroupedForms) {
        const int64_t columns = gated ? f.columns / 2 : f.columns, out = gated ? N / 2 : N, blocks = (out + columns - 1) / columns;
        const int64_t threads = f.height < 64 ? 64 * f.parts : f.columns * f.parts;
        if (grouped_workgroups(rows, groups, f.height, blocks) * threads > kMaxWorkItems) continue;
        const double tiles = fmax(used, rows / (double)f.height + 0.5 * used), w = tiles * blocks / 256;
        const double one = format == kGroupedBf16 ? f.one_bf16 : format == kGroupedE8 ? f.one_e8 : 1.0;
        const double full = format == kGroupedBf16 ? f.full_bf16 : format == kGroupedE8 ? f.full_e8 : 1.0;
        const double r = rows / tiles, b = K / 128.0 / f.parts;
        const double us = f.start + b * fmax((f.one + f.one_row * r) * one, (f.full + f.full_row * r) * w * full) + f.each * w;
        if (us < least) {
            least = us;
            best = &f;
        }
    }
    return *best;
}

int matmul_grouped(const void* X, int64_t share, const void* plan, int64_t rows, int64_t groups, const void* codes, int64_t N, int64_t K, int group,
                   int epilogue, void* Y, void* stream, int format)
{
    const int rc = check_grouped(rows, groups, share, N, K, group, epilogue, format);
    if (rc != E0M4_OK) return rc;
    if (rows == 0 || N == 0) return E0M4_OK;
    if (!X || !plan || !codes || !Y) return E0M4_ERR_NULL;
    if (!aligned(X, 16) || !aligned(plan, 16) || !aligned(codes, 16) || !aligned(Y, 16)) return E0M4_ERR_ALIGN;
    const int64_t n_out = epilogue == E0M4_EPILOGUE_SWIGLU ? N / 2 : N;
    const size_t y_bytes = (size_t)rows * n_out * 2;
    if (overlap(X, (size_t)(share ? rows / share : rows) * K * 2, Y, y_bytes) || overlaps_plan(Y, y_bytes, plan, rows, groups)) return E0M4_ERR_SHAPE;
    GroupedArgs a;
    a.X = X;
    a.share = share;
    a.plan = plan;
    a.rows = rows;
    a.groups = groups;
    a.codes = codes;
    a.N = N;
    a.K = K;
    a.group = group;
    a.swiglu = epilogue == E0M4_EPILOGUE_SWIGLU;
    a.Y = Y;
    const GroupedForm& f = choose_form(rows, groups, N, K, a.swiglu, format);
    return f.height >= 64 ? launch_grouped_many(a, format, f.height, f.columns, (hipStream_t)stream)
                          : launch_grouped_few(a, format, f.height, f.columns / kBlockRows, (hipStream_t)stream);
}

int check_lora(int64_t rows, int64_t adapters, int rank, int64_t N, int64_t K)
{
    const int rc = check_groups(rows, adapters);
    if (rc != E0M4_OK) return rc;
    if (rank < 8 || rank > 128 || rank % 8 != 0 || N < 0 || N > (int64_t)1 << 24 || N % 8 != 0 || K < 8 || K > (int64_t)1 << 20 || K % 8 != 0) return E0M4_ERR_SHAPE;
    return N * rank * 2 > kMaxXBytes ? E0M4_ERR_SHAPE : E0M4_OK;     // (rows of one adapter's B are reached by 32-bit offsets)
}

}  // namespace

}  // namespace e0m4

using namespace e0m4;

extern "C" {

size_t e0m4_groups_bytes(int64_t rows, int64_t groups)
{
    return check_groups(rows, groups) == E0M4_OK ? (size_t)plan_words(rows, groups) * 4 : 0;
}

int e0m4_groups(const int32_t* index, int64_t rows, int64_t groups, void* plan, void* stream)
{
    const int rc = check_groups(rows, groups);
    if (rc != E0M4_OK) return rc;
    if ((!index && rows) || !plan) return E0M4_ERR_NULL;
    if (!aligned(index, 4) || !aligned(plan, 16)) return E0M4_ERR_ALIGN;
    RouteArgs a = {};
    a.tokens = rows;
    a.groups = (int)groups;
    a.k = 1;
    a.experts = const_cast<int32_t*>(index);
    return launch_route(a, plan, (hipStream_t)stream);
}

int e0m4_route(const void* logits, int dtype, int64_t tokens, int64_t experts, int64_t logits_ld, int k, int scoring, int renormalise, float factor,
               const int32_t* count, int32_t* chosen, float* weights, void* plan, void* stream)
{
    if (tokens < 0 || experts < 1 || experts > kMaxGroups || k < 1 || k > kMaxChoices || k > experts || tokens > kMaxGroupRows / k) return E0M4_ERR_SHAPE;
    if (dtype != E0M4_FP16 && dtype != E0M4_BF16 && dtype != E0M4_FP32) return E0M4_ERR_SHAPE;
    if (scoring != E0M4_ROUTE_SOFTMAX && scoring != E0M4_ROUTE_SIGMOID) return E0M4_ERR_SHAPE;
    if (logits_ld < 0 || logits_ld > (int64_t)1 << 32) return E0M4_ERR_SHAPE;
    if (tokens == 0 && !plan) return E0M4_OK;
    if (tokens && (!logits || !chosen || !weights)) return E0M4_ERR_NULL;
    if (!aligned(logits, dtype == E0M4_FP32 ? 4 : 2) || !aligned(count, 4) || !aligned(chosen, 4) || !aligned(weights, 4) || !aligned(plan, 16)) return E0M4_ERR_ALIGN;
    RouteArgs a;
    a.logits = tokens ? logits : nullptr;
    a.dtype = dtype;
    a.tokens = tokens;
    a.logits_ld = logits_ld;
    a.groups = (int)experts;
    a.k = k;
    a.sigmoid = scoring == E0M4_ROUTE_SIGMOID;
    a.renormalise = renormalise != 0;
    a.factor = factor;
    a.count = count;
    a.experts = chosen;
    a.weights = weights;
    return launch_route(a, plan, (hipStream_t)stream);
}

int e0m4_matmul_grouped(const void* X_f16, int64_t share, const void* plan, int64_t rows, int64_t groups, const void* codes, int64_t N, int64_t K, int group,
                        int epilogue, void* Y_f16, void* stream)
{
    return matmul_grouped(X_f16, share, plan, rows, groups, codes, N, K, group, epilogue, Y_f16, stream, kGroupedFp16);
}

int e0m8_matmul_grouped(const void* X_f16, int64_t share, const void* plan, int64_t rows, int64_t groups, const void* codes, int64_t N, int64_t K, int group,
                        int epilogue, void* Y_f16, void* stream)
{
    return matmul_grouped(X_f16, share, plan, rows, groups, codes, N, K, group, epilogue, Y_f16, stream, kGroupedE8);
}

int e0m4_bf16_matmul_grouped(const void* X_bf16, int64_t share, const void* plan, int64_t rows, int64_t groups, const void* codes, int64_t N, int64_t K,
                             int group, int epilogue, void* Y_bf16, void* stream)
{
    return matmul_grouped(X_bf16, share, plan, rows, groups, codes, N, K, group, epilogue, Y_bf16, stream, kGroupedBf16);
}

int e0m4_combine(const void* Y, int dtype, int64_t N, const float* weights, const void* plan, int64_t tokens, int k, int64_t groups, const void* base,
                 void* out, void* stream)
{
    if (tokens < 0 || k < 1 || k > kMaxShare || tokens > kMaxGroupRows / k || N < 0 || N > (int64_t)1 << 24) return E0M4_ERR_SHAPE;
    const int rc = check_groups(tokens * k, groups);
    if (rc != E0M4_OK) return rc;
    if (dtype != E0M4_FP16 && dtype != E0M4_BF16) return E0M4_ERR_SHAPE;
    if (tokens == 0 || N == 0) return E0M4_OK;
    if (!Y || !weights || !plan || !out) return E0M4_ERR_NULL;
    if (!aligned(Y, 16) || !aligned(weights, 4) || !aligned(plan, 16) || !aligned(base, 16) || !aligned(out, 16)) return E0M4_ERR_ALIGN;
    const size_t bytes = (size_t)tokens * N * 2;
    if (overlap(out, bytes, Y, bytes * k) || (base && base != out && overlap(out, bytes, base, bytes)) || overlap(out, bytes, weights, (size_t)tokens * k * 4) ||
        overlaps_plan(out, bytes, plan, tokens * k, groups))
        return E0M4_ERR_SHAPE;
    return launch_combine(Y, N, weights, plan, tokens, k, groups, base, out, dtype, (hipStream_t)stream);
}

size_t e0m4_lora_workspace_bytes(int64_t rows, int64_t adapters, int rank, int64_t N, int64_t K)
{
    if (check_lora(rows, adapters, rank, N, K) != E0M4_OK || rows == 0 || N == 0) return 0;
    return lora_workspace_bytes(rows, adapters, rank, N, K);
}

int e0m4_lora(const void* X, int64_t x_ld, int dtype, const void* plan, int64_t rows, int64_t adapters, const void* A, const void* B, int rank,
              const float* factors, int64_t N, int64_t K, const void* base, int64_t base_ld, void* out, int64_t out_ld, void* workspace,
              size_t workspace_bytes, void* stream)
{
    const int rc = check_lora(rows, adapters, rank, N, K);
    if (rc != E0M4_OK) return rc;
    if (dtype != E0M4_FP16 && dtype != E0M4_BF16) return E0M4_ERR_SHAPE;
    if (rows == 0 || N == 0) return E0M4_OK;
    if (!X || !plan || !A || !B || !out || !workspace) return E0M4_ERR_NULL;
    if (x_ld < K || out_ld < N || (base && base_ld < N) || x_ld > (int64_t)1 << 24 || out_ld > (int64_t)1 << 32 || base_ld > (int64_t)1 << 32)
        return E0M4_ERR_SHAPE;
    if (base == out && base_ld != out_ld) return E0M4_ERR_SHAPE;
    if (((x_ld | out_ld | (base ? base_ld : 0)) & 7) != 0) return E0M4_ERR_ALIGN;
    if (!aligned(X, 16) || !aligned(plan, 16) || !aligned(A, 16) || !aligned(B, 16) || !aligned(factors, 4) || !aligned(base, 16) || !aligned(out, 16) ||
        !aligned(workspace, 16))
        return E0M4_ERR_ALIGN;
    if (((rows - 1) * x_ld + K) * 2 > kMaxXBytes) return E0M4_ERR_SHAPE;
    if (base && base != out && rows_overlap(base, base_ld * 2, out, out_ld * 2, rows, N * 2)) return E0M4_ERR_SHAPE;
    const size_t ws_bytes = lora_workspace_bytes(rows, adapters, rank, N, K), out_bytes = (size_t)((rows - 1) * out_ld + N) * 2;
    if (overlaps_plan(out, out_bytes, plan, rows, adapters) || overlap(out, out_bytes, workspace, ws_bytes) ||
        overlap(out, out_bytes, B, (size_t)adapters * N * rank * 2))
        return E0M4_ERR_SHAPE;
    if (workspace_bytes < ws_bytes) return E0M4_ERR_WORKSPACE;
    LoraArgs a;
    a.X = X;
    a.x_ld = x_ld;
    a.plan = plan;
    a.rows = rows;
    a.adapters = adapters;
    a.A = A;
    a.B = B;
    a.rank = rank;
    a.factors = factors;
    a.N = N;
    a.K = K;
    a.base = base;
    a.base_ld = base ? base_ld : 0;
    a.out = out;
    a.out_ld = out_ld;
    a.dtype = dtype;
    return launch_lora(a, workspace, (hipStream_t)stream);
}

}  // extern "C"
