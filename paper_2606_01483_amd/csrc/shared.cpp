// C ABI of shared pages and of the attention over shared prefixes
// (include/murmur_shared.h): argument checks, buffer sizes and dispatch.  As in api.cpp,
// every check runs before the first HIP call.
#include <math.h>

#include <algorithm>

#include "internal.h"
#include "murmur_shared.h"

namespace murmur {
namespace {

constexpr int kMaxRows = 65535;  // rows of a block table

// The bookkeeping arguments that every call on shared pages takes.
int check_pages(int32_t B, const int32_t *bt, int32_t max_blocks, const int32_t *ref, int32_t n_blocks,
                const int32_t *stack, const int32_t *top, int32_t capacity) {
    if (!bt || !ref || !stack || !top)
        return fail(MURMUR_EINVAL, "block_table_dev, ref_dev, free_stack_dev and free_top_dev must not be NULL");
    if (B < 1 || B > kMaxRows) return fail(MURMUR_EINVAL, "B must be in [1, %d] (got %d)", kMaxRows, B);
    if (max_blocks < 1) return fail(MURMUR_EINVAL, "max_blocks must be >= 1 (got %d)", max_blocks);
    if ((int64_t)B * max_blocks > (1 << 30)) return fail(MURMUR_EINVAL, "B * max_blocks must be at most 2^30");
    if (n_blocks < 1 || n_blocks > (1 << 30)) return fail(MURMUR_EINVAL, "n_blocks must be in [1, 2^30] (got %d)", n_blocks);
    if (capacity < n_blocks)
        return fail(MURMUR_EINVAL, "capacity (%d) must be at least n_blocks (%d)", capacity, n_blocks);
    if (!aligned(bt, 4) || !aligned(ref, 4) || !aligned(stack, 4) || !aligned(top, 4))
        return fail(MURMUR_EINVAL, "device pointers must be 4-byte aligned");
    return MURMUR_OK;
}

int check_block_size(int32_t block_size, int &log2_bs) {
    if (block_size < 1 || block_size > (1 << 20) || (block_size & (block_size - 1)) != 0)
        return fail(MURMUR_EINVAL, "block_size must be a power of two in [1, 2^20] (got %d)", block_size);
    log2_bs = 0;
    while ((1 << log2_bs) < block_size) ++log2_bs;
    return MURMUR_OK;
}

int check_pool(const murmur_kv *pool, int32_t Hkv, int32_t n_blocks, int32_t block_size) {
    if (!pool->k || !pool->v) return fail(MURMUR_EINVAL, "pool->k and pool->v must not be NULL");
    if (Hkv < 1 || pool->n_layers < 1 || pool->max_len < 1)
        return fail(MURMUR_EINVAL, "Hkv, pool->n_layers and pool->max_len must be >= 1");
    const int64_t strides[3] = {pool->stride_layer, pool->stride_h, pool->stride_pos};
    for (int i = 0; i < 3; ++i)
        if (strides[i] < 0 || strides[i] % 8 != 0)
            return fail(MURMUR_EINVAL, "pool strides must be non-negative multiples of 8 elements");
    if (pool->stride_pos < kHeadDim && pool->max_len > 1)
        return fail(MURMUR_EINVAL, "pool->stride_pos (%lld) must be >= head_dim", (long long)pool->stride_pos);
    if (!aligned(pool->k, 16) || !aligned(pool->v, 16))
        return fail(MURMUR_EINVAL, "pool->k and pool->v must be 16-byte aligned");
    if ((int64_t)n_blocks * block_size > pool->max_len)
        return fail(MURMUR_EINVAL, "pool->max_len (%d) is below n_blocks * block_size (%lld)", pool->max_len,
                    (long long)n_blocks * block_size);
    if ((int64_t)Hkv * block_size > (1 << 26))
        return fail(MURMUR_EINVAL, "Hkv * block_size must be at most 2^26");
    return MURMUR_OK;
}

// The parts of a workspace at `ws`, and the bytes they take.
struct PagesWorkspace {
    ForkWorkspace fork;
    int32_t *moves;
    size_t bytes;
};
PagesWorkspace pages_workspace(void *ws, int32_t B, int32_t max_blocks, int32_t n_blocks) {
    PagesWorkspace p{};
    const size_t entries = (size_t)B * (size_t)max_blocks;
    const size_t lists = (size_t)B * (((size_t)max_blocks + kForkCols - 1) / kForkCols);
    size_t at = 0;
    const auto take = [&](size_t bytes) {
        void *q = (void *)((uintptr_t)ws + at);
        at += round_up(bytes, 256);
        return q;
    };
    p.fork.head = (ForkHead *)take(sizeof(ForkHead));
    p.fork.first = (uint64_t *)take(sizeof(uint64_t) * (size_t)n_blocks);
    p.fork.bits = (uint32_t *)take((entries + 31) / 32 * 4);
    p.moves = (int32_t *)take(0);
    const size_t kept = at;
    p.fork.changes = (ForkChange *)take(sizeof(ForkChange) * lists * kForkCols);
    p.fork.counts = (int32_t *)take(sizeof(int32_t) * lists);
    p.fork.freed = (int32_t *)take(sizeof(int32_t) * ((entries - 1) / kForkPlaces + 1));
    p.fork.block_at = (int32_t *)take(sizeof(int32_t) * entries);
    p.bytes = std::max(at, kept + round_up(sizeof(int32_t) * (1 + 2 * (size_t)(n_blocks / 2)), 256));
    return p;
}

int check_workspace(const void *ws, size_t ws_bytes, size_t needed) {
    if (!ws) return fail(MURMUR_EINVAL, "ws_dev must not be NULL");
    if (!aligned(ws, 256)) return fail(MURMUR_EINVAL, "ws_dev must be 256-byte aligned");
    if (ws_bytes < needed)
        return fail(MURMUR_ENOSPACE, "workspace of %zu bytes is too small (%zu needed)", ws_bytes, needed);
    return MURMUR_OK;
}

int check_shared_sizes(int32_t n_layers, int32_t B, int32_t Hq, int32_t Hkv, int32_t max_keep, int32_t n_groups) {
    if (n_layers < 1 || B < 1 || Hq < 1 || Hkv < 1 || max_keep < 1)
        return fail(MURMUR_EINVAL, "n_layers, B, Hq, Hkv and max_keep must be >= 1");
    if (B > kSharedMaxSeqs)
        return fail(MURMUR_EUNSUPPORTED, "%d sequences exceed %d", B, kSharedMaxSeqs);
    if (n_groups < 1 || n_groups > kSharedMaxSeqs)
        return fail(MURMUR_EINVAL, "n_groups must be in [1, %d] (got %d)", kSharedMaxSeqs, n_groups);
    if (Hq % Hkv != 0) return fail(MURMUR_EINVAL, "Hq (%d) must be a multiple of Hkv (%d)", Hq, Hkv);
    if (Hq / Hkv > kMaxGroup)
        return fail(MURMUR_EUNSUPPORTED, "query heads per KV head %d exceeds %d", Hq / Hkv, kMaxGroup);
    if (max_keep > kMaxKeep) return fail(MURMUR_EUNSUPPORTED, "max_keep %d exceeds %d", max_keep, kMaxKeep);
    if ((int64_t)n_layers * Hkv > 65535 || (int64_t)n_layers * B * Hq > 0x7fffffffLL)
        return fail(MURMUR_EINVAL, "problem too large for one launch (n_layers * Hkv = %lld, B = %d)",
                    (long long)n_layers * Hkv, B);
    const SharedCaps c = shared_caps(n_layers, B, Hq, Hkv, max_keep, n_groups);
    if (c.n_wg > 65535 || c.n_wg < 0 || c.rows > (1 << 24))
        return fail(MURMUR_EINVAL, "problem too large for one launch (B = %d lists of up to %d)", B, max_keep);
    return MURMUR_OK;
}

}  // namespace

// Bounds of any plan for these sizes.  A plan that fits one dispatch round has at
// most per_round workgroups per (layer, KV head) (one on a compute unit), each with
// at most kSharedRows partial rows of a prefix.  Any other is cut at the highest
// level: a group of n sequences has at most n / (sequences per item) + 1 sets of
// rows, each list at most max_keep entries.  Each sequence's rest has a partial per
// workgroup that it touches: one, and one more for every workgroup boundary.
SharedCaps shared_caps(int32_t n_layers, int32_t B, int32_t Hq, int32_t Hkv, int32_t max_keep, int32_t n_groups) {
    SharedCaps c{};
    const int64_t G = Hq / Hkv, heads = (int64_t)n_layers * Hkv;
    const auto div_up = [](int64_t x, int64_t y) { return (x + y - 1) / y; };
    const int64_t passes = div_up(max_keep, kWaveTile);
    const int64_t cuts = div_up(passes, item_passes(kSharedLevels));
    const int64_t chunks = div_up(passes, chunk_passes(kSharedLevels));
    const int64_t sets = n_groups + B / (kSharedRows / G);
    c.per_round = (int32_t)std::max<int64_t>(1, kRoundWorkgroups / heads);
    const int64_t longest = sets * cuts + div_up(B * chunks, kSharedWaves);
    c.n_wg = (int32_t)std::min<int64_t>(std::max<int64_t>(c.per_round, longest), 0x7fffffff);
    c.rows = std::max<int64_t>((int64_t)c.per_round * kSharedRows, B * G * cuts) + G * (B + (int64_t)c.n_wg);
    // Whether lists are left whole (shared_whole_kernel) or cut (shared_attn_kernel and the merge), from what the host
    // knows, in us.  A group's lists come at the memory's rate once at least.  A round of passes, one of each of a
    // workgroup's eight wavefronts, takes 1.2, 2.0 or 2.9 with one, two or three row tiles if a compute unit has nothing
    // but to compute, and 2.4 if its rows come from memory, less the more workgroups share them.  Whole, a workgroup
    // takes a list's rounds one after the other, and 6 besides; cut, they are spread over the chip, and the partials
    // and their join make it 15.  (12 chunks of 8 sequences, lists of 850: 15.4 a layer whole, 16.7 cut; 15 sequences,
    // lists of 2963, next to nothing shared: 32.6 whole, 15.2 cut.)
    const int64_t n = div_up(B, std::max(n_groups, 1)), rounds = div_up(passes, 8);  // sequences of a group
    const double round_us[3] = {1.2, 2.0, 2.9}, wave = (double)kRoundWorkgroups, wg = (double)heads * n_groups;
    const double read_us = (double)heads * std::min(n_groups, B) * max_keep * 512.0 / 5e6;
    double alone_us = 0.0, spread_us = 0.0;
    for (int tiles = 1; tiles <= 3; ++tiles) {
        const int64_t parts = div_up(n, kMaxGroup * tiles / G);
        const double compute = round_us[tiles - 1] * (double)(rounds * parts) * wg / wave;
        const double us = std::max(compute, (double)rounds * std::max(round_us[tiles - 1], 1.2 + 1.2 / (double)std::min<int64_t>(parts, 4)));
        alone_us = tiles == 1 ? us : std::min(alone_us, us);
        spread_us = tiles == 1 ? compute : std::min(spread_us, compute);
    }
    c.whole = 6.0 + std::max(read_us, alone_us) <= 15.0 + std::max(read_us, spread_us);
    c.waves = heads * std::min(n_groups, B) > kRoundWorkgroups ? 4 : 8;
    // The buffers hold either schedule, so that those of the largest batch serve a smaller one that goes the other way.
    const int64_t items = std::min<int64_t>(B, std::max<int64_t>(n_groups + B / (kMaxGroup / G), kRoundWorkgroups / heads));
    c.n_wg = (int32_t)std::max<int64_t>(c.n_wg, items);
    c.grid = c.whole ? (int32_t)items : c.n_wg;
    c.n_scan = (max_keep - 1) / kScanLen + 1;
    c.item_offset = sizeof(PlanHeader) + sizeof(PlanSeq) * (size_t)B;
    c.chunk_offset = c.item_offset + sizeof(PlanItem) * (size_t)c.n_wg;
    c.scan_offset = c.chunk_offset + sizeof(PlanChunk) * (size_t)c.n_wg * kSharedWaves;
    c.plan_bytes = round_up(c.scan_offset + 4 * (size_t)B * c.n_scan, 256);
    c.ws_bytes = round_up((size_t)heads * (size_t)c.rows * (kHeadDim + 2) * sizeof(float) + 1, 256);
    return c;
}

}  // namespace murmur

using namespace murmur;

MURMUR_EXPORT int murmur_paged_workspace(int32_t B, int32_t max_blocks, int32_t n_blocks, size_t *bytes) {
    if (!bytes) return fail(MURMUR_EINVAL, "bytes must not be NULL");
    if (B < 1 || B > kMaxRows || max_blocks < 1 || n_blocks < 1 || n_blocks > (1 << 30) ||
        (int64_t)B * max_blocks > (1 << 30))
        return fail(MURMUR_EINVAL, "B must be in [1, %d], max_blocks >= 1, B * max_blocks and n_blocks at most 2^30",
                    kMaxRows);
    *bytes = pages_workspace(nullptr, B, max_blocks, n_blocks).bytes;
    return ok();
}

MURMUR_EXPORT int murmur_paged_fork(const int32_t *parent_dev, int32_t B, int32_t *block_table_dev,
                                    int32_t max_blocks, int32_t *ref_dev, int32_t n_blocks, int32_t *free_stack_dev,
                                    int32_t *free_top_dev, int32_t capacity, void *ws_dev, size_t ws_bytes,
                                    murmur_stream_t stream) {
    if (!parent_dev) return fail(MURMUR_EINVAL, "parent_dev must not be NULL");
    if (!aligned(parent_dev, 4)) return fail(MURMUR_EINVAL, "device pointers must be 4-byte aligned");
    int rc = check_pages(B, block_table_dev, max_blocks, ref_dev, n_blocks, free_stack_dev, free_top_dev, capacity);
    if (rc == MURMUR_OK) rc = check_workspace(ws_dev, ws_bytes, pages_workspace(nullptr, B, max_blocks, n_blocks).bytes);
    if (rc != MURMUR_OK) return rc;
    const ForkWorkspace ws = pages_workspace(ws_dev, B, max_blocks, n_blocks).fork;
    const int e = launch_paged_fork(parent_dev, B, block_table_dev, max_blocks, ref_dev, n_blocks, free_stack_dev,
                                    free_top_dev, ws, stream);
    if (e != 0) return fail(MURMUR_EHIP, "paged_fork launch failed: %s", hip_error_text(e));
    return ok();
}

MURMUR_EXPORT int murmur_paged_step_shared(const murmur_seg *seg_dev, const murmur_policy *pol_dev,
                                           int32_t pol_per_seq, int32_t B, int32_t *block_table_dev,
                                           int32_t max_blocks, int32_t block_size, int32_t *ref_dev,
                                           int32_t n_blocks, int32_t *free_stack_dev, int32_t *free_top_dev,
                                           int32_t capacity, int32_t full_scan, int32_t *copied_dev,
                                           const murmur_kv *pool, int32_t Hkv, const void *k_new_dev,
                                           const void *v_new_dev, murmur_stream_t stream) {
    if (!seg_dev || !pol_dev || !copied_dev)
        return fail(MURMUR_EINVAL, "seg_dev, pol_dev and copied_dev must not be NULL");
    if (pol_per_seq != 0 && pol_per_seq != 1) return fail(MURMUR_EINVAL, "pol_per_seq must be 0 or 1");
    if (full_scan != 0 && full_scan != 1) return fail(MURMUR_EINVAL, "full_scan must be 0 or 1");
    if (!aligned(seg_dev, 4) || !aligned(pol_dev, 4) || !aligned(copied_dev, 4))
        return fail(MURMUR_EINVAL, "device pointers must be 4-byte aligned");
    int log2_bs = 0;
    int rc = check_pages(B, block_table_dev, max_blocks, ref_dev, n_blocks, free_stack_dev, free_top_dev, capacity);
    if (rc == MURMUR_OK) rc = check_block_size(block_size, log2_bs);
    if (rc != MURMUR_OK) return rc;
    if (pool) {
        if (!k_new_dev || !v_new_dev)
            return fail(MURMUR_EINVAL, "with a pool, k_new_dev and v_new_dev must not be NULL");
        if (!aligned(k_new_dev, 16) || !aligned(v_new_dev, 16))
            return fail(MURMUR_EINVAL, "k_new_dev and v_new_dev must be 16-byte aligned");
        rc = check_pool(pool, Hkv, n_blocks, block_size);
        if (rc != MURMUR_OK) return rc;
        if ((int64_t)B * pool->n_layers * Hkv > ((int64_t)1 << 36))
            return fail(MURMUR_EINVAL, "B * n_layers * Hkv too large");
    }
    int e = launch_paged_step_shared(seg_dev, pol_dev, pol_per_seq, B, block_table_dev, max_blocks, log2_bs, ref_dev,
                                     n_blocks, free_stack_dev, free_top_dev, full_scan, copied_dev, stream);
    if (e != 0) return fail(MURMUR_EHIP, "paged_step_shared launch failed: %s", hip_error_text(e));
    if (pool) {
        e = launch_paged_append_shared(seg_dev, B, block_table_dev, max_blocks, log2_bs, copied_dev, *pool, Hkv,
                                       k_new_dev, v_new_dev, stream);
        if (e != 0) return fail(MURMUR_EHIP, "paged_step_shared append launch failed: %s", hip_error_text(e));
    }
    return ok();
}

MURMUR_EXPORT int murmur_paged_compact(int32_t B, int32_t *block_table_dev, int32_t max_blocks, int32_t block_size,
                                       int32_t *ref_dev, int32_t n_blocks, int32_t *free_stack_dev,
                                       int32_t *free_top_dev, int32_t capacity, int32_t *map_dev,
                                       const murmur_kv *pool, int32_t Hkv, void *ws_dev, size_t ws_bytes,
                                       murmur_stream_t stream) {
    if (!map_dev) return fail(MURMUR_EINVAL, "map_dev must not be NULL");
    if (!aligned(map_dev, 4)) return fail(MURMUR_EINVAL, "device pointers must be 4-byte aligned");
    int log2_bs = 0;
    int rc = check_pages(B, block_table_dev, max_blocks, ref_dev, n_blocks, free_stack_dev, free_top_dev, capacity);
    if (rc == MURMUR_OK) rc = check_block_size(block_size, log2_bs);
    if (rc == MURMUR_OK && pool) rc = check_pool(pool, Hkv, n_blocks, block_size);
    if (rc == MURMUR_OK) rc = check_workspace(ws_dev, ws_bytes, pages_workspace(nullptr, B, max_blocks, n_blocks).bytes);
    if (rc != MURMUR_OK) return rc;
    const int e = launch_paged_compact(B, block_table_dev, max_blocks, log2_bs, ref_dev, n_blocks, free_stack_dev,
                                       free_top_dev, map_dev, pool, Hkv,
                                       pages_workspace(ws_dev, B, max_blocks, n_blocks).moves, stream);
    if (e != 0) return fail(MURMUR_EHIP, "paged_compact launch failed: %s", hip_error_text(e));
    return ok();
}

MURMUR_EXPORT int murmur_decode_attn_shared_workspace(int32_t n_layers, int32_t B, int32_t Hq, int32_t Hkv,
                                                      int32_t max_keep, int32_t n_groups, size_t *ws_bytes,
                                                      size_t *plan_bytes) {
    if (!ws_bytes || !plan_bytes) return fail(MURMUR_EINVAL, "ws_bytes and plan_bytes must not be NULL");
    const int rc = check_shared_sizes(n_layers, B, Hq, Hkv, max_keep, n_groups);
    if (rc != MURMUR_OK) return rc;
    const SharedCaps c = shared_caps(n_layers, B, Hq, Hkv, max_keep, n_groups);
    *ws_bytes = c.ws_bytes;
    *plan_bytes = c.plan_bytes;
    return ok();
}

MURMUR_EXPORT int murmur_shared_plan(const int32_t *idx_dev, const int32_t *ranges_dev, const int32_t *count_dev,
                                     int32_t max_keep, int32_t B, const int32_t *group_dev, int32_t n_groups,
                                     int32_t *shared_dev, int32_t find_shared, int32_t n_layers, int32_t Hq,
                                     int32_t Hkv, void *plan_dev, size_t plan_bytes, murmur_stream_t stream) {
    if (!idx_dev && !ranges_dev) return fail(MURMUR_EINVAL, "one of idx_dev and ranges_dev is required");
    if (!ranges_dev && !count_dev) return fail(MURMUR_EINVAL, "count_dev is required with an index list");
    if (!group_dev || !shared_dev || !plan_dev)
        return fail(MURMUR_EINVAL, "group_dev, shared_dev and plan_dev must not be NULL");
    if (find_shared != 0 && find_shared != 1) return fail(MURMUR_EINVAL, "find_shared must be 0 or 1");
    if (find_shared && ranges_dev)
        return fail(MURMUR_EINVAL, "find_shared compares index lists: ranges_dev must be NULL");
    if (!aligned(idx_dev, 4) || !aligned(ranges_dev, 4) || !aligned(count_dev, 4) || !aligned(group_dev, 4) ||
        !aligned(shared_dev, 4))
        return fail(MURMUR_EINVAL, "device pointers must be 4-byte aligned");
    if (!aligned(plan_dev, 16)) return fail(MURMUR_EINVAL, "plan_dev must be 16-byte aligned");
    const int rc = check_shared_sizes(n_layers, B, Hq, Hkv, max_keep, n_groups);
    if (rc != MURMUR_OK) return rc;
    SharedPlanLaunch p{};
    p.caps = shared_caps(n_layers, B, Hq, Hkv, max_keep, n_groups);
    if (plan_bytes < p.caps.plan_bytes)
        return fail(MURMUR_ENOSPACE, "plan of %zu bytes is too small (%zu needed)", plan_bytes, p.caps.plan_bytes);
    p.idx = idx_dev;
    p.ranges = ranges_dev;
    p.count = count_dev;
    p.group = group_dev;
    p.shared = shared_dev;
    p.max_keep = max_keep;
    p.B = B;
    p.n_groups = n_groups;
    p.find = find_shared;
    p.n_layers = n_layers;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.plan = (uint8_t *)plan_dev;
    const int e = launch_shared_plan(p, stream);
    if (e != 0) return fail(MURMUR_EHIP, "shared_plan launch failed: %s", hip_error_text(e));
    return ok();
}

MURMUR_EXPORT int murmur_decode_attn_shared(const void *q_dev, const murmur_kv *kv, const int32_t *idx_dev,
                                            const int32_t *ranges_dev, int32_t max_keep, int32_t B, int32_t n_groups,
                                            int32_t Hq, int32_t Hkv, int32_t D, float scale, void *out_dev,
                                            int32_t out_dtype, float *lse_dev, const void *plan_dev,
                                            size_t plan_bytes, void *ws_dev, size_t ws_bytes,
                                            murmur_stream_t stream) {
    if (!q_dev || !kv || !out_dev || !plan_dev || !ws_dev)
        return fail(MURMUR_EINVAL, "q_dev, kv, out_dev, plan_dev and ws_dev must not be NULL");
    if (!idx_dev && !ranges_dev) return fail(MURMUR_EINVAL, "one of idx_dev and ranges_dev is required");
    if (!kv->k || !kv->v) return fail(MURMUR_EINVAL, "kv->k and kv->v must not be NULL");
    if (kv->n_layers < 1 || kv->max_len < 1)
        return fail(MURMUR_EINVAL, "kv->n_layers and kv->max_len must be >= 1");
    const int rc = check_shared_sizes(kv->n_layers, B, Hq, Hkv, max_keep, n_groups);
    if (rc != MURMUR_OK) return rc;
    if (D != kHeadDim) return fail(MURMUR_EUNSUPPORTED, "head_dim %d is not supported (only %d)", D, kHeadDim);
    if (out_dtype != MURMUR_DTYPE_BF16 && out_dtype != MURMUR_DTYPE_F32)
        return fail(MURMUR_EINVAL, "out_dtype must be MURMUR_DTYPE_BF16 or MURMUR_DTYPE_F32 (got %d)", out_dtype);
    if (!isfinite(scale)) return fail(MURMUR_EINVAL, "scale must be finite");
    const int64_t strides[4] = {kv->stride_layer, kv->stride_b, kv->stride_h, kv->stride_pos};
    for (int i = 0; i < 4; ++i)
        if (strides[i] < 0 || strides[i] % 8 != 0)
            return fail(MURMUR_EINVAL, "KV strides must be non-negative multiples of 8 elements");
    if (kv->stride_pos < kHeadDim && kv->max_len > 1)
        return fail(MURMUR_EINVAL, "kv->stride_pos (%lld) must be >= head_dim", (long long)kv->stride_pos);
    if (!aligned(q_dev, 16) || !aligned(kv->k, 16) || !aligned(kv->v, 16))
        return fail(MURMUR_EINVAL, "q_dev, kv->k and kv->v must be 16-byte aligned");
    if (!aligned(out_dev, 16) || !aligned(lse_dev, 4))
        return fail(MURMUR_EINVAL, "out_dev must be 16-byte and lse_dev 4-byte aligned");
    if (!aligned(idx_dev, 4) || !aligned(ranges_dev, 4))
        return fail(MURMUR_EINVAL, "idx/ranges pointers must be 4-byte aligned");
    if (!aligned(plan_dev, 16)) return fail(MURMUR_EINVAL, "plan_dev must be 16-byte aligned");
    if (!aligned(ws_dev, 256)) return fail(MURMUR_EINVAL, "ws_dev must be 256-byte aligned");
    const SharedCaps c = shared_caps(kv->n_layers, B, Hq, Hkv, max_keep, n_groups);
    if (plan_bytes < c.plan_bytes)
        return fail(MURMUR_ENOSPACE, "plan of %zu bytes is too small (%zu needed)", plan_bytes, c.plan_bytes);
    if (ws_bytes < c.ws_bytes)
        return fail(MURMUR_ENOSPACE, "workspace of %zu bytes is too small (%zu needed)", ws_bytes, c.ws_bytes);
    SharedAttnLaunch a{};
    a.q = (const uint16_t *)q_dev;
    a.k = (const uint16_t *)kv->k;
    a.v = (const uint16_t *)kv->v;
    a.s_layer = kv->stride_layer;
    a.s_b = kv->stride_b;
    a.s_h = kv->stride_h;
    a.s_pos = kv->stride_pos;
    a.idx = idx_dev;
    a.ranges = ranges_dev;
    a.out = out_dev;
    a.lse = lse_dev;
    a.plan = (const uint8_t *)plan_dev;
    a.item_offset = c.item_offset;
    a.chunk_offset = c.chunk_offset;
    a.part_o = (float *)ws_dev;
    a.part_ml = a.part_o + (size_t)kv->n_layers * Hkv * c.rows * kHeadDim;
    a.rows_cap = c.rows;
    a.max_len = kv->max_len;
    a.max_keep = max_keep;
    a.B = B;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.G = Hq / Hkv;
    a.NL = kv->n_layers;
    a.n_groups = n_groups;
    a.n_wg = c.grid;
    a.waves = c.whole ? c.waves : 0;
    a.kinds = plan_kind(c.whole, false) | (kv->stride_b == 0 ? plan_kind(c.whole, true) : 0);
    a.out_f32 = out_dtype == MURMUR_DTYPE_F32;
    a.magic_g = (uint32_t)((((uint64_t)1 << 32) + a.G - 1) / a.G - 1);
    a.scale_log2 = scale * 1.4426950408889634f;
    const int e = launch_decode_attn_shared(a, stream);
    if (e != 0) return fail(MURMUR_EHIP, "decode_attn_shared launch failed: %s", hip_error_text(e));
    return ok();
}
