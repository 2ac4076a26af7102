// C ABI of requests into a paged pool, rotary positions and trees of drafted tokens
// (include/murmur_draft.h): argument checks, buffer sizes and dispatch.  As in api.cpp,
// every check runs before the first HIP call.
#include <float.h>
#include <math.h>

#include <algorithm>

#include "internal.h"
#include "murmur_draft.h"

namespace murmur {
namespace {

constexpr int kMaxRows = 65535;  // rows of a block table

int check_log2(int32_t block_size, int &log2_bs) {
    if (block_size < 1 || block_size > (1 << 20) || (block_size & (block_size - 1)) != 0)
        return fail(MURMUR_EINVAL, "block_size must be a power of two in [1, 2^20] (got %d)", block_size);
    log2_bs = 0;
    while ((1 << log2_bs) < block_size) ++log2_bs;
    return MURMUR_OK;
}

// A cache that is read or written.
int check_cache(const murmur_kv *kv) {
    if (!kv->k || !kv->v) return fail(MURMUR_EINVAL, "kv->k and kv->v must not be NULL");
    if (kv->n_layers < 1 || kv->max_len < 1) return fail(MURMUR_EINVAL, "kv->n_layers and kv->max_len must be >= 1");
    const int64_t strides[4] = {kv->stride_layer, kv->stride_b, kv->stride_h, kv->stride_pos};
    for (int i = 0; i < 4; ++i)
        if (strides[i] < 0 || strides[i] % 8 != 0)
            return fail(MURMUR_EINVAL, "KV strides must be non-negative multiples of 8 elements");
    if (kv->stride_pos < kHeadDim && kv->max_len > 1)
        return fail(MURMUR_EINVAL, "kv->stride_pos (%lld) must be >= head_dim", (long long)kv->stride_pos);
    if (!aligned(kv->k, 16) || !aligned(kv->v, 16))
        return fail(MURMUR_EINVAL, "kv->k and kv->v must be 16-byte aligned");
    return MURMUR_OK;
}

struct ReserveWorkspace {
    int32_t *top0, *need;
    ReserveSums *sums;
    size_t bytes;
};
ReserveWorkspace reserve_workspace(void *ws, int32_t B) {
    const size_t groups = ((size_t)B + kReserveGroup - 1) / kReserveGroup;
    const size_t need_at = 256, sums_at = need_at + round_up(sizeof(int32_t) * (size_t)B, 256);
    const uintptr_t at = (uintptr_t)ws;
    return ReserveWorkspace{(int32_t *)at, (int32_t *)(at + need_at), (ReserveSums *)(at + sums_at),
                            sums_at + round_up(sizeof(ReserveSums) * groups, 256)};
}

int check_tree(const int32_t *parent, int32_t parent_per_seq, int32_t n_nodes) {
    if (!parent) return fail(MURMUR_EINVAL, "parent_dev must not be NULL");
    if (parent_per_seq != 0 && parent_per_seq != 1) return fail(MURMUR_EINVAL, "parent_per_seq must be 0 or 1");
    if (n_nodes < 1) return fail(MURMUR_EINVAL, "n_nodes must be >= 1 (got %d)", n_nodes);
    if (n_nodes > kMaxNodes) return fail(MURMUR_EUNSUPPORTED, "%d nodes exceed %d", n_nodes, kMaxNodes);
    if (!aligned(parent, 4)) return fail(MURMUR_EINVAL, "device pointers must be 4-byte aligned");
    return MURMUR_OK;
}

int check_tree_sizes(int32_t n_layers, int32_t B, int32_t Hq, int32_t Hkv, int32_t n_nodes, int32_t max_keep) {
    if (n_layers < 1 || B < 1 || Hq < 1 || Hkv < 1 || n_nodes < 1 || max_keep < 1)
        return fail(MURMUR_EINVAL, "n_layers, B, Hq, Hkv, n_nodes and max_keep must be >= 1");
    if (n_nodes > kMaxNodes) return fail(MURMUR_EUNSUPPORTED, "%d nodes exceed %d", n_nodes, kMaxNodes);
    if (Hq % Hkv != 0) return fail(MURMUR_EINVAL, "Hq (%d) must be a multiple of Hkv (%d)", Hq, Hkv);
    if (Hq / Hkv > kMaxGroup)
        return fail(MURMUR_EUNSUPPORTED, "query heads per KV head %d exceeds %d", Hq / Hkv, kMaxGroup);
    if (max_keep > kMaxKeep) return fail(MURMUR_EUNSUPPORTED, "max_keep %d exceeds %d", max_keep, kMaxKeep);
    // 512 threads for each of the row sets of every (layer, sequence, KV head), in 32 bits
    const double groups = (double)n_layers * B * Hkv;
    if (groups * ((n_nodes * (Hq / Hkv) + kTreeRowSet - 1) / kTreeRowSet) > 4194304.0)
        return fail(MURMUR_EINVAL, "problem too large for one launch (n_layers = %d, B = %d, Hq = %d, n_nodes = %d)", n_layers, B,
                    Hq, n_nodes);
    return MURMUR_OK;
}

}  // namespace

// A workgroup has up to 128 rows, of eight wavefronts with a compute unit to itself or
// of four and two on one.  The list is cut into the splits that the following estimate
// (us, fitted to batches of 1 to 128 trees of 2 to 64 nodes over 200 to 20 000 rows)
// finds best, among those that fill the chip once, twice or three times: 7 for the way
// to the first pass and from the last one; a pass of 128 rows 1.3, or 1.9 where
// another workgroup shares the unit, of which 0.55 and 1.25 are the rows of K and V;
// and for a merge 4 and its partials at 4 TB/s, written and read.  (12 trees of 32
// nodes over 4000 rows: two splits on eight wavefronts 80, five on four 71; 32 trees
// of 32 over 900 rows: 42 and 53.)
// Eight wavefronts take one row tile each where a split is short: less is left to join
// at its end, but every tile then reads the rows from LDS again (12 trees of 16 nodes,
// 900 rows: 22.9 and 24.0 with two tiles; 4000 rows: 48.5 and 46.2).
TreePlan tree_plan(int32_t n_layers, int32_t B, int32_t Hq, int32_t Hkv, int32_t n_nodes, int32_t max_keep) {
    TreePlan p{};
    const int64_t rows = (int64_t)n_nodes * (Hq / Hkv), groups = (int64_t)n_layers * B * Hkv;
    const int64_t passes = ((int64_t)max_keep + kWaveTile - 1) / kWaveTile, most = std::min<int64_t>(kMaxTreeSplits, passes / 4);
    p.row_sets = (int32_t)((rows + kTreeRowSet - 1) / kTreeRowSet);
    const int64_t sets = groups * p.row_sets;
    const double full = (double)std::min<int64_t>(rows, kTreeRowSet) / kTreeRowSet;
    double best = 0.0;
    for (int pair = 0; pair < 2; ++pair) {
        const int64_t slots = (pair + 1) * kRoundWorkgroups;
        const double pass_us = pair ? 1.25 + 0.65 * full : 0.55 + 0.75 * full;
        for (int fill = 0; fill <= kTreeFills; ++fill) {
            const int64_t s = std::max<int64_t>(1, std::min(fill * slots / sets, most));
            const double merge_us = s > 1 ? 4.0 + (double)(groups * s * rows) * 2 * (kHeadDim + 2) * sizeof(float) / 4e6 : 0.0;
            const double us = 7.0 + (double)((sets * s + slots - 1) / slots) * (double)((passes + s - 1) / s) * pass_us + merge_us;
            if (best == 0.0 || us < best) {
                best = us;
                p.n_split = (int32_t)s;
                p.shape = pair ? kTreePair : rows <= 64 || passes <= 12 * s ? kTreeFew : kTreeWide;
            }
        }
    }
    // The bytes of calls of these sizes and smaller ones: the estimate may cut the lists of a smaller batch where it leaves
    // those of a larger one whole, so the largest number of partial rows is bounded by what does grow.  A list is cut into
    // at most `most` parts, and only while the parts of all row sets fill the chip's slots at most kTreeFills times.
    const int64_t parts = std::min(groups * rows * std::max<int64_t>(most, 1), kTreeFills * 2 * kRoundWorkgroups * (int64_t)kTreeRowSet);
    p.serves = most > 1 ? round_up((size_t)parts * (kHeadDim + 2) * sizeof(float), 256) : 0;
    p.units = groups * p.n_split;
    if (p.n_split > 1) {
        p.o_bytes = (size_t)p.units * (size_t)rows * kHeadDim * sizeof(float);
        p.total = round_up(p.o_bytes + (size_t)p.units * (size_t)rows * 2 * sizeof(float), 256);
    }
    return p;
}

}  // namespace murmur

using namespace murmur;

MURMUR_EXPORT int murmur_paged_reserve_workspace(int32_t B, size_t *bytes) {
    if (!bytes) return fail(MURMUR_EINVAL, "bytes must not be NULL");
    if (B < 1 || B > kMaxRows) return fail(MURMUR_EINVAL, "B must be in [1, %d] (got %d)", kMaxRows, B);
    *bytes = reserve_workspace(nullptr, B).bytes;
    return ok();
}

MURMUR_EXPORT int murmur_paged_reserve(const int32_t *len_dev, const int32_t *new_dev, int32_t B, int32_t *block_table_dev,
                                       int32_t max_blocks, int32_t block_size, int32_t *ref_dev, int32_t n_blocks,
                                       int32_t *free_stack_dev, int32_t *free_top_dev, int32_t capacity, int32_t per_seq,
                                       int32_t n_tokens, int32_t *start_dev, int32_t *got_dev, int32_t *slot_dev,
                                       int32_t *pos_dev, int32_t *seq_dev, void *ws_dev, size_t ws_bytes,
                                       murmur_stream_t stream) {
    if (!len_dev || !new_dev || !block_table_dev || !free_stack_dev || !free_top_dev)
        return fail(MURMUR_EINVAL, "len_dev, new_dev, block_table_dev, free_stack_dev and free_top_dev must not be NULL");
    if (!start_dev || !got_dev || !slot_dev || !ws_dev)
        return fail(MURMUR_EINVAL, "start_dev, got_dev, slot_dev and ws_dev must not be NULL");
    if (B < 1 || B > kMaxRows) return fail(MURMUR_EINVAL, "B must be in [1, %d] (got %d)", kMaxRows, B);
    if (max_blocks < 1) return fail(MURMUR_EINVAL, "max_blocks must be >= 1 (got %d)", max_blocks);
    if ((int64_t)B * max_blocks > (1 << 30)) return fail(MURMUR_EINVAL, "B * max_blocks must be at most 2^30");
    int log2_bs = 0;
    const int rc = check_log2(block_size, log2_bs);
    if (rc != MURMUR_OK) return rc;
    if (n_blocks < 1 || n_blocks > (1 << 30)) return fail(MURMUR_EINVAL, "n_blocks must be in [1, 2^30] (got %d)", n_blocks);
    if ((int64_t)n_blocks * block_size > ((int64_t)1 << 31))
        return fail(MURMUR_EINVAL, "n_blocks * block_size must be at most 2^31");
    if (capacity < n_blocks) return fail(MURMUR_EINVAL, "capacity (%d) must be at least n_blocks (%d)", capacity, n_blocks);
    if (per_seq < 0) return fail(MURMUR_EINVAL, "per_seq must be >= 0 (got %d)", per_seq);
    if (n_tokens < 1) return fail(MURMUR_EINVAL, "n_tokens must be >= 1 (got %d)", n_tokens);
    if ((int64_t)B * per_seq > n_tokens)
        return fail(MURMUR_EINVAL, "n_tokens (%d) is below B * per_seq (%lld)", n_tokens, (long long)B * per_seq);
    if (!aligned(len_dev, 4) || !aligned(new_dev, 4) || !aligned(block_table_dev, 4) || !aligned(ref_dev, 4) ||
        !aligned(free_stack_dev, 4) || !aligned(free_top_dev, 4) || !aligned(start_dev, 4) || !aligned(got_dev, 4) ||
        !aligned(slot_dev, 4) || !aligned(pos_dev, 4) || !aligned(seq_dev, 4))
        return fail(MURMUR_EINVAL, "device pointers must be 4-byte aligned");
    if (!aligned(ws_dev, 256)) return fail(MURMUR_EINVAL, "ws_dev must be 256-byte aligned");
    const ReserveWorkspace ws = reserve_workspace(ws_dev, B);
    if (ws_bytes < ws.bytes)
        return fail(MURMUR_ENOSPACE, "workspace of %zu bytes is too small (%zu needed)", ws_bytes, ws.bytes);
    ReserveLaunch p{};
    p.len = len_dev;
    p.fresh = new_dev;
    p.bt = block_table_dev;
    p.ref = ref_dev;
    p.stack = free_stack_dev;
    p.top = free_top_dev;
    p.start = start_dev;
    p.got = got_dev;
    p.slot = slot_dev;
    p.pos = pos_dev;
    p.seq = seq_dev;
    p.top0 = ws.top0;
    p.need = ws.need;
    p.sums = ws.sums;
    p.B = B;
    p.max_blocks = max_blocks;
    p.log2_bs = log2_bs;
    p.n_blocks = n_blocks;
    p.per_seq = per_seq;
    p.n_tokens = n_tokens;
    const int e = launch_paged_reserve(p, stream);
    if (e != 0) return fail(MURMUR_EHIP, "paged_reserve launch failed: %s", hip_error_text(e));
    return ok();
}

MURMUR_EXPORT int murmur_rope_freqs_host(int32_t rot_dim, double base, int32_t kind, double factor, double original_len,
                                         double slow_turns, double fast_turns, uint64_t *freq, float *gain) {
    if (!freq || !gain) return fail(MURMUR_EINVAL, "freq and gain must not be NULL");
    if (rot_dim < 2 || rot_dim > kHeadDim || rot_dim % 2 != 0)
        return fail(MURMUR_EINVAL, "rot_dim must be even and in [2, %d] (got %d)", kHeadDim, rot_dim);
    if (kind < MURMUR_ROPE_PLAIN || kind > MURMUR_ROPE_YARN) return fail(MURMUR_EINVAL, "unknown kind %d", kind);
    if (!(base > 1.0) || !isfinite(base)) return fail(MURMUR_EINVAL, "base must be finite and above 1");
    const bool scaled = kind != MURMUR_ROPE_PLAIN, bands = kind == MURMUR_ROPE_BANDS || kind == MURMUR_ROPE_YARN;
    if (scaled && (!(factor >= 1.0) || !isfinite(factor))) return fail(MURMUR_EINVAL, "factor must be finite and at least 1");
    if (bands && (!(original_len > 0.0) || !isfinite(original_len)))
        return fail(MURMUR_EINVAL, "original_len must be finite and positive");
    if (bands && (!(slow_turns >= 0.0) || !(fast_turns > slow_turns) || !isfinite(fast_turns)))
        return fail(MURMUR_EINVAL, "slow_turns must be at least 0 and fast_turns finite and above it");
    // In long double, whose 64 bits keep a turn of up to 1 / (2 pi) to a fraction of the table's step.
    const long double two_pi = 6.283185307179586476925286766559L;
    long double b = base;
    if (kind == MURMUR_ROPE_BASE && rot_dim > 2) b *= powl(factor, rot_dim / (rot_dim - 2.0L));
    if (!(b <= DBL_MAX)) return fail(MURMUR_EINVAL, "base and factor are too large");
    for (int i = 0; i < rot_dim / 2; ++i) {
        long double f = powl(b, -2.0L * i / rot_dim) / two_pi;
        if (kind == MURMUR_ROPE_LINEAR) f /= factor;
        if (bands) {
            const long double keep = std::min(1.0L, std::max(0.0L, (original_len * f - slow_turns) / ((long double)fast_turns - slow_turns)));
            f = f * keep + f / factor * (1.0L - keep);
        }
        freq[i] = (uint64_t)nearbyintl(ldexpl(f, 64));  // f <= 1 / (2 pi)
    }
    *gain = kind == MURMUR_ROPE_YARN ? (float)(1.0 + 0.1 * log(factor)) : 1.f;
    return ok();
}

MURMUR_EXPORT int murmur_rope_append(const murmur_rope *rope, const murmur_qkv *in, const int32_t *pos_dev,
                                     const int32_t *slot_dev, const int32_t *seq_dev, int32_t n_seqs, int32_t n_tokens,
                                     int32_t Hq, int32_t Hkv, int32_t D, void *q_out_dev, const murmur_kv *kv,
                                     murmur_stream_t stream) {
    if (!rope || !in || !pos_dev || !slot_dev || !q_out_dev || !kv)
        return fail(MURMUR_EINVAL, "rope, in, pos_dev, slot_dev, q_out_dev and kv must not be NULL");
    if (rope->rot_dim < 0 || rope->rot_dim > kHeadDim || rope->rot_dim % 2 != 0)
        return fail(MURMUR_EINVAL, "rope->rot_dim must be even and in [0, %d] (got %d)", kHeadDim, rope->rot_dim);
    if (rope->interleaved != 0 && rope->interleaved != 1) return fail(MURMUR_EINVAL, "rope->interleaved must be 0 or 1");
    if (!isfinite(rope->gain)) return fail(MURMUR_EINVAL, "rope->gain must be finite");
    if (rope->rot_dim > 0 && (!rope->freq || !aligned(rope->freq, 8)))
        return fail(MURMUR_EINVAL, "rope->freq must not be NULL and 8-byte aligned");
    if (!in->q || !in->k || !in->v) return fail(MURMUR_EINVAL, "in->q, in->k and in->v must not be NULL");
    if (in->dtype != MURMUR_DTYPE_BF16 && in->dtype != MURMUR_DTYPE_F32)
        return fail(MURMUR_EINVAL, "in->dtype must be MURMUR_DTYPE_BF16 or MURMUR_DTYPE_F32 (got %d)", in->dtype);
    const size_t size = in->dtype == MURMUR_DTYPE_F32 ? 4 : 2;
    if (!aligned(in->q, size) || !aligned(in->k, size) || !aligned(in->v, size))
        return fail(MURMUR_EINVAL, "in->q, in->k and in->v must be aligned to an element");
    if (in->q_layer < 0 || in->q_token < 0 || in->kv_layer < 0 || in->kv_token < 0)
        return fail(MURMUR_EINVAL, "strides of the projections must not be negative");
    if (n_seqs < 1 || n_tokens < 1 || Hq < 1 || Hkv < 1)
        return fail(MURMUR_EINVAL, "n_seqs, n_tokens, Hq and Hkv must be >= 1");
    if (Hq > kMaxRows || Hkv > kMaxRows) return fail(MURMUR_EINVAL, "Hq and Hkv must be at most %d", kMaxRows);
    if (D != kHeadDim) return fail(MURMUR_EUNSUPPORTED, "head_dim %d is not supported (only %d)", D, kHeadDim);
    const int rc = check_cache(kv);
    if (rc != MURMUR_OK) return rc;
    if ((int64_t)kv->n_layers * n_tokens > (1 << 25))
        return fail(MURMUR_EINVAL, "n_layers * n_tokens must be at most 2^25");
    if (!aligned(pos_dev, 4) || !aligned(slot_dev, 4) || !aligned(seq_dev, 4))
        return fail(MURMUR_EINVAL, "device pointers must be 4-byte aligned");
    if (!aligned(q_out_dev, 16)) return fail(MURMUR_EINVAL, "q_out_dev must be 16-byte aligned");
    RopeLaunch p{};
    p.q = in->q;
    p.k = in->k;
    p.v = in->v;
    p.q_layer = in->q_layer;
    p.q_token = in->q_token;
    p.kv_layer = in->kv_layer;
    p.kv_token = in->kv_token;
    p.pos = pos_dev;
    p.slot = slot_dev;
    p.seq = seq_dev;
    p.freq = rope->freq;
    p.q_out = (uint16_t *)q_out_dev;
    p.k_cache = (uint16_t *)kv->k;
    p.v_cache = (uint16_t *)kv->v;
    p.s_layer = kv->stride_layer;
    p.s_b = kv->stride_b;
    p.s_h = kv->stride_h;
    p.s_pos = kv->stride_pos;
    p.gain = rope->gain;
    p.rot = rope->rot_dim;
    p.interleaved = rope->interleaved;
    p.f32 = in->dtype == MURMUR_DTYPE_F32;
    const int64_t wide = 16 / (int64_t)size;
    p.wide = aligned(in->q, 16) && aligned(in->k, 16) && aligned(in->v, 16) &&
             in->q_layer % wide == 0 && in->q_token % wide == 0 && in->kv_layer % wide == 0 && in->kv_token % wide == 0;
    // a token's heads to several wavefronts where the tokens leave most of the chip's 8192 without work
    const int64_t items = (int64_t)kv->n_layers * n_tokens;
    p.parts = p.wide && items <= 1024 && (rope->interleaved || rope->rot_dim % 16 == 0) ? (Hq + 2 * Hkv + 7) / 8 : 1;
    p.n_tokens = n_tokens;
    p.n_seqs = n_seqs;
    p.max_len = kv->max_len;
    p.Hq = Hq;
    p.Hkv = Hkv;
    p.NL = kv->n_layers;
    const int e = launch_rope_append(p, stream);
    if (e != 0) return fail(MURMUR_EHIP, "rope_append launch failed: %s", hip_error_text(e));
    return ok();
}

MURMUR_EXPORT int murmur_decode_attn_tree_workspace(int32_t n_layers, int32_t B, int32_t Hq, int32_t Hkv, int32_t n_nodes,
                                                    int32_t max_keep, size_t *bytes) {
    if (!bytes) return fail(MURMUR_EINVAL, "bytes must not be NULL");
    const int rc = check_tree_sizes(n_layers, B, Hq, Hkv, n_nodes, max_keep);
    if (rc != MURMUR_OK) return rc;
    *bytes = tree_plan(n_layers, B, Hq, Hkv, n_nodes, max_keep).serves;
    return ok();
}

MURMUR_EXPORT int murmur_decode_attn_tree(const murmur_seg *seg_dev, const murmur_policy *pol_dev, int32_t pol_per_seq,
                                          const int32_t *parent_dev, int32_t parent_per_seq, int32_t n_nodes,
                                          const void *q_dev, const murmur_kv *kv, const void *k_tree_dev,
                                          const void *v_tree_dev, const int32_t *block_table_dev, int32_t max_blocks,
                                          int32_t block_size, int32_t max_keep, int32_t B, int32_t Hq, int32_t Hkv,
                                          int32_t D, float scale, void *out_dev, int32_t out_dtype, float *lse_dev,
                                          void *ws_dev, size_t ws_bytes, murmur_stream_t stream) {
    if (!seg_dev || !pol_dev || !q_dev || !kv || !k_tree_dev || !v_tree_dev || !out_dev)
        return fail(MURMUR_EINVAL, "seg_dev, pol_dev, q_dev, kv, k_tree_dev, v_tree_dev and out_dev must not be NULL");
    if (pol_per_seq < 0 || pol_per_seq > 3) return fail(MURMUR_EINVAL, "pol_per_seq must be MURMUR_POL_* bits (got %d)", pol_per_seq);
    int rc = check_tree(parent_dev, parent_per_seq, n_nodes);
    if (rc == MURMUR_OK) rc = check_cache(kv);
    if (rc == MURMUR_OK) rc = check_tree_sizes(kv->n_layers, B, Hq, Hkv, n_nodes, max_keep);
    if (rc != MURMUR_OK) return rc;
    if (D != kHeadDim) return fail(MURMUR_EUNSUPPORTED, "head_dim %d is not supported (only %d)", D, kHeadDim);
    if (out_dtype != MURMUR_DTYPE_BF16 && out_dtype != MURMUR_DTYPE_F32)
        return fail(MURMUR_EINVAL, "out_dtype must be MURMUR_DTYPE_BF16 or MURMUR_DTYPE_F32 (got %d)", out_dtype);
    if (!isfinite(scale)) return fail(MURMUR_EINVAL, "scale must be finite");
    int log2_bs = 0;
    if (block_table_dev) {
        if (max_blocks < 1) return fail(MURMUR_EINVAL, "max_blocks must be >= 1 (got %d)", max_blocks);
        rc = check_log2(block_size, log2_bs);
        if (rc != MURMUR_OK) return rc;
        if (kv->stride_b != 0) return fail(MURMUR_EINVAL, "kv->stride_b must be 0 with a block table");
    } else if (max_blocks != 0 || block_size != 0) {
        return fail(MURMUR_EINVAL, "max_blocks and block_size must be 0 without a block table");
    }
    if (!aligned(seg_dev, 4) || !aligned(pol_dev, 4) || !aligned(block_table_dev, 4) || !aligned(lse_dev, 4))
        return fail(MURMUR_EINVAL, "device pointers must be 4-byte aligned");
    if (!aligned(q_dev, 16) || !aligned(k_tree_dev, 16) || !aligned(v_tree_dev, 16) || !aligned(out_dev, 16))
        return fail(MURMUR_EINVAL, "q_dev, k_tree_dev, v_tree_dev and out_dev must be 16-byte aligned");
    const TreePlan plan = tree_plan(kv->n_layers, B, Hq, Hkv, n_nodes, max_keep);
    if (plan.total > 0) {
        if (!ws_dev) return fail(MURMUR_EINVAL, "ws_dev must not be NULL");
        if (!aligned(ws_dev, 256)) return fail(MURMUR_EINVAL, "ws_dev must be 256-byte aligned");
        if (ws_bytes < plan.total)
            return fail(MURMUR_ENOSPACE, "workspace of %zu bytes is too small (%zu needed)", ws_bytes, plan.total);
    }
    TreeLaunch a{};
    a.seg = (const int32_t *)seg_dev;
    a.pol = (const int32_t *)pol_dev;
    a.parent = parent_dev;
    a.bt = block_table_dev;
    a.q = (const uint16_t *)q_dev;
    a.k = (const uint16_t *)kv->k;
    a.v = (const uint16_t *)kv->v;
    a.k_tree = (const uint16_t *)k_tree_dev;
    a.v_tree = (const uint16_t *)v_tree_dev;
    a.s_layer = kv->stride_layer;
    a.s_b = kv->stride_b;
    a.s_h = kv->stride_h;
    a.s_pos = kv->stride_pos;
    a.out = out_dev;
    a.lse = lse_dev;
    a.part_o = (float *)ws_dev;
    a.part_ml = (float *)((uintptr_t)ws_dev + plan.o_bytes);
    a.pol_mode = pol_per_seq;
    a.parent_per_seq = parent_per_seq;
    a.T = n_nodes;
    a.max_blocks = max_blocks;
    a.log2_bs = log2_bs;
    a.max_len = kv->max_len;
    a.B = B;
    a.Hq = Hq;
    a.Hkv = Hkv;
    a.G = Hq / Hkv;
    a.NL = kv->n_layers;
    a.out_f32 = out_dtype == MURMUR_DTYPE_F32;
    a.n_split = plan.n_split;
    a.row_sets = plan.row_sets;
    a.units = (int32_t)plan.units;
    a.shape = plan.shape;
    const int merge_rows = plan.n_split <= kTreeMergeWhole ? 8 : 2;
    a.merge_sets = (n_nodes * a.G + merge_rows - 1) / merge_rows;
    a.by_sets = DivideBy::of((uint32_t)a.row_sets);
    a.by_split = DivideBy::of((uint32_t)a.n_split);
    a.by_heads = DivideBy::of((uint32_t)Hkv);
    a.by_batch = DivideBy::of((uint32_t)B);
    a.by_merge = DivideBy::of((uint32_t)a.merge_sets);
    a.max_pos = block_table_dev ? (int32_t)std::min<int64_t>((int64_t)max_blocks << log2_bs, 0x7fffffff) : kv->max_len;
    const uint64_t row_bytes = (uint64_t)kv->stride_pos * 2;
    a.near_rows = row_bytes < (1 << 24) && kv->max_len <= (1 << 24) &&
                  (uint64_t)(kv->max_len - 1) * row_bytes + 2 * kHeadDim < ((uint64_t)1 << 32);
    a.magic_g = (65536u + (uint32_t)a.G - 1) / (uint32_t)a.G;
    a.scale_log2 = scale * 1.4426950408889634f;
    const int e = launch_decode_attn_tree(a, stream);
    if (e != 0) return fail(MURMUR_EHIP, "decode_attn_tree launch failed: %s", hip_error_text(e));
    return ok();
}

MURMUR_EXPORT int murmur_tree_accept(const int32_t *parent_dev, int32_t parent_per_seq, int32_t n_nodes,
                                     const int32_t *token_dev, const int32_t *next_dev, const int32_t *slot_dev, int32_t B,
                                     const void *k_tree_dev, const void *v_tree_dev, const murmur_kv *kv, int32_t Hkv,
                                     int32_t *path_dev, int32_t *count_dev, int32_t *last_dev, murmur_stream_t stream) {
    int rc = check_tree(parent_dev, parent_per_seq, n_nodes);
    if (rc != MURMUR_OK) return rc;
    if (!token_dev || !next_dev || !slot_dev || !k_tree_dev || !v_tree_dev || !kv || !path_dev || !count_dev || !last_dev)
        return fail(MURMUR_EINVAL, "token_dev, next_dev, slot_dev, k_tree_dev, v_tree_dev, kv, path_dev, count_dev and last_dev "
                                   "must not be NULL");
    if (B < 1 || B > kMaxRows) return fail(MURMUR_EINVAL, "B must be in [1, %d] (got %d)", kMaxRows, B);
    if (Hkv < 1 || Hkv > kMaxRows) return fail(MURMUR_EINVAL, "Hkv must be in [1, %d] (got %d)", kMaxRows, Hkv);
    rc = check_cache(kv);
    if (rc != MURMUR_OK) return rc;
    if (kv->n_layers > kMaxRows) return fail(MURMUR_EINVAL, "kv->n_layers must be at most %d", kMaxRows);
    if (!aligned(token_dev, 4) || !aligned(next_dev, 4) || !aligned(slot_dev, 4) || !aligned(path_dev, 4) ||
        !aligned(count_dev, 4) || !aligned(last_dev, 4))
        return fail(MURMUR_EINVAL, "device pointers must be 4-byte aligned");
    if (!aligned(k_tree_dev, 16) || !aligned(v_tree_dev, 16))
        return fail(MURMUR_EINVAL, "k_tree_dev and v_tree_dev must be 16-byte aligned");
    AcceptLaunch p{};
    p.parent = parent_dev;
    p.token = token_dev;
    p.next = next_dev;
    p.slot = slot_dev;
    p.k_tree = (const uint16_t *)k_tree_dev;
    p.v_tree = (const uint16_t *)v_tree_dev;
    p.k = (uint16_t *)kv->k;
    p.v = (uint16_t *)kv->v;
    p.s_layer = kv->stride_layer;
    p.s_b = kv->stride_b;
    p.s_h = kv->stride_h;
    p.s_pos = kv->stride_pos;
    p.path = path_dev;
    p.count = count_dev;
    p.last = last_dev;
    p.parent_per_seq = parent_per_seq;
    p.T = n_nodes;
    p.B = B;
    p.Hkv = Hkv;
    p.NL = kv->n_layers;
    p.max_len = kv->max_len;
    const int e = launch_tree_accept(p, stream);
    if (e != 0) return fail(MURMUR_EHIP, "tree_accept launch failed: %s", hip_error_text(e));
    return ok();
}
