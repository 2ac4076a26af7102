// Internal interface between the C ABI layer (api.cpp) and the gfx950 kernels
// (kernels.hip).  Not installed; include/murmur.h is the public surface.
#pragma once

#include <stddef.h>
#include <stdint.h>

#include "murmur.h"

#define MURMUR_EXPORT extern "C" __attribute__((visibility("default")))

namespace murmur {

// Status and error text of an entry point (api.cpp): fail() formats the text of
// murmur_last_error and returns `code`, ok() clears it.
int fail(int code, const char *fmt, ...) __attribute__((format(printf, 2, 3)));
int ok();
inline bool aligned(const void *p, size_t n) { return ((uintptr_t)p % n) == 0; }
inline size_t round_up(size_t x, size_t a) { return (x + a - 1) / a * a; }

constexpr int kHeadDim = 128;     // head_dim supported by the attention kernel
constexpr int kMaxGroup = 16;     // query heads per KV head (MFMA tile height)
constexpr int kWaveTile = 32;     // retained positions one wavefront handles per pass
// The LDS-staged schedule's automatic split counts are chosen in units of 128
// positions: a pass of its four-wavefront workgroup, half a pass of the
// eight-wavefront one that runs them within one dispatch round.
constexpr int kSplitUnit = 4 * kWaveTile;
constexpr int kMaxAutoSplits = 64;
constexpr int kLongSplit = 2048;          // see long_split (api.cpp)
constexpr int kRoundWorkgroups = 256;     // one workgroup per compute unit
// K and V bytes of a layer's retained rows from which a launch streams them past
// the L2s (kernels.hip, kAuxStream).  Below, the rows of all layers of a decoder
// may fit the 256 MB Infinity Cache, and small ones the 32 MB of L2, so the next
// token may find them there, and the normal policy is the faster one.  The line
// is for a decoder of 28 layers; a launch cannot see how many there are, and where
// fewer layers' caches stay in the Infinity Cache, streaming costs up to about
// 30 MiB a layer.  A cache read again and again, a captured call per layer, us a
// launch, normal -> streamed:
//   850 rows a sequence:    8.3 MiB     10.0        13.3        19.9
//     28 layers          6.56 -> 6.48  6.82 -> 6.72  7.52 -> 7.16  8.76 -> 8.30
//     8 layers           6.29 -> 6.37  6.44 -> 6.51  6.84 -> 6.91  7.76 -> 7.88
//     2 layers           5.64 -> 5.94  5.59 -> 5.95  5.69 -> 6.30  7.53 -> 7.16
//   3482 rows a sequence:   6.8 MiB     13.6        20.4        34.0
//     28 layers          6.90 -> 7.71  8.57 -> 8.27  8.82 -> 8.48  13.12 -> 12.25
//     8 layers           6.84 -> 7.58  7.39 -> 7.85  8.20 -> 8.25  12.62 -> 12.02
//     2 layers           6.43 -> 7.32  6.33 -> 7.52  8.23 -> 7.82  12.06 -> 11.34
constexpr int64_t kStreamBytes = 12 << 20;
// Splits one merge can combine: it stages their 2 * n_split * G floats (30 KiB)
// in the workgroup's K/V stages (64 KiB at least).
constexpr int kMaxMergeSplits = 240;
constexpr int kMaxKeep = 1 << 28;  // retained positions per sequence the attention accepts
constexpr int kMergeBatch = 8;  // splits whose partials one merging thread loads at once
// The LDS-staged schedule merges groups of more than 2 * kMergeBatch and at
// most kTwoLevelMax splits in two levels, sets of kSubSplits splits first (so
// that the second level folds at most 16 partials too).
constexpr int kSubSplits = 8;
constexpr int kTwoLevelMax = 128;
// Split-choice model (measured on MI355X): one compute unit streams about 40 GB/s from HBM however many
// wavefronts it runs, and the split-K merge chain (partial stores, ticket, loading the partials) costs
// about 2.3 us on top of the data phase.
constexpr double kCuBytesPerUs = 40e3;
constexpr double kMergeChainUs = 2.3;
// The wide schedule's merge keeps two batches of kMergeBatch partials in flight: every further
// 2 * kMergeBatch partials of a group add one serial load round trip (measured: 14 splits of 192
// positions 8.5 us, 17 of 160 9.0 us on 4 groups of 2592).
constexpr double kMergeRoundTripUs = 0.5;

// Wide schedule: workgroups of kWideWaves wavefronts, each wavefront one pass
// of kWaveTile retained positions, so a split holds at most kWideSplit.
constexpr int kWideWaves = 8;
constexpr int kWideSplit = kWideWaves * kWaveTile;  // 256

// Work of the wide schedule's workgroups, decoded on the device with exact
// multiply-high divisions (values below 2^16, multipliers ceil(2^32 / d), 0
// for d = 1): every (layer, sequence, KV head) group is cut into n splits of
// len positions; the w-th (group, split) in that order goes to the workgroup
// that xcd_order maps to w and, when its group has more than one split,
// leaves its partial in slot w.
struct WideSched {
    uint32_t xcd;       // (per - 1) | tall << 16 for W workgroups: per = ceil(W / 8) and tall = W - 8 (per - 1)
                        // (see xcd_order)
    uint32_t magic_n;   // ceil(2^32 / n)
    uint32_t len;       // len | n << 9 | G << 18 (split lengths <= 256, n <= kMaxMergeSplits, G query heads
                        // per KV head); the launch adds the policy mode (MURMUR_POL_* bits) << 23, at
                        // bit 25 whether stride_pos < kRunRowLimit and at bit 26 whether every group's
                        // first K/V element lies below 2^31 elements
    uint32_t hkv_b;     // Hkv | B << 16
    uint32_t magic_hkv;
    uint32_t magic_b;
};

// Row strides (elements) below this let a pass of kWaveTile consecutive rows
// address its K/V rows with 32-bit byte offsets from its first row.
constexpr int64_t kRunRowLimit = (int64_t)1 << 23;

// Launch description of one decode_attn call, fully validated by the caller.
// Where the attention takes the retained sets from (see AttnLaunch::src0/src1).
enum SrcMode : int32_t { kSrcIndex = 0, kSrcRanges = 1, kSrcLayout = 2, kSrcRing = 3 };

struct AttnLaunch {
    // kSrcIndex / kSrcRanges: src0 = counts [B], src1 = range tables [B][6][2]
    // (kSrcRanges); kSrcLayout and kSrcRing: src0 = layouts (murmur_seg [B]),
    // src1 = policies (murmur_policy [1] or [B], pol_per_seq).
    const int32_t *src0;
    const int32_t *src1;
    int32_t src_mode, pol_per_seq;
    int32_t *idx_out, *count_out, *ranges_out;  // kSrcLayout / kSrcRing: optional evict_compact outputs
    // kSrcRing: output ring rows, and the current token's K/V [NL][B][Hkv][D]
    // (read instead of its ring row, then appended there).
    int32_t ring_cap;
    const uint16_t *k_new;
    const uint16_t *v_new;
    const uint16_t *q;
    const uint16_t *k;
    const uint16_t *v;
    int64_t s_layer, s_b, s_h, s_pos;
    const int32_t *idx;
    void *out;
    float *lse;
    int32_t *ticket;   // [groups][kTicketStride]: one counter per group (layer, sequence, KV head), then
                       // for a two-level merge one per set of kSubSplits splits, [groups][n_sub]
    float *part_ml;    // [groups][n_split][G][2]  (running max in log2 units, sum)
    float *part_o;     // [groups][n_split][G][128]
    uint32_t part_ml_bytes, part_o_bytes;  // extents of the two partial arrays (< 2^31)
    int32_t max_len, max_keep, B, Hq, Hkv, G, NL;
    int32_t split_len, n_split, out_f32;
    int32_t stream_count;  // retained positions per sequence from which K/V rows are streamed (kStreamBytes)
    float scale_log2;  // logit scale times log2(e)
    int32_t wide_wg;   // > 0: the wide schedule with this many workgroups (sched)
    WideSched sched;
};

struct WorkspacePlan {
    int32_t split_len;
    int32_t n_split;  // splits per group (the wide schedule: of the groups with the most)
    int32_t wide_wg;  // > 0: the wide schedule's workgroups
    WideSched sched;
    int64_t groups;
    int64_t tickets;  // ticket counters the launch uses
    size_t ml_bytes, o_bytes, total;
};

// Ticket counters sit kTicketStride int32 apart (one 128-byte cache line
// each), so that the atomics of different groups do not queue on one line.
constexpr int kTicketStride = 32;
// Bytes at the start of a workspace of ws_bytes that hold the tickets (the
// partials follow): 128 bytes per KiB, rounded up to 256, room for a ticket
// per KiB.  Depends on the size alone, so calls of different shapes that share
// a workspace place their tickets alike, and never where another call left
// partials.
size_t ticket_region(size_t ws_bytes);

// Whether an automatic split length cuts long sequences in grids of more than
// one dispatch round too (see long_split, api.cpp): never (such a launch needs no
// partials: for workspaces that cannot hold them), where the lengths alone say
// so, or as for a call with policies per layer (wherever kByLength does, and
// more).
enum class LongCut { kNone, kByLength, kPerLayer };

// Split choice and workspace layout; deterministic in its arguments.
WorkspacePlan plan_workspace(int32_t n_layers, int32_t B, int32_t Hq, int32_t Hkv, int32_t max_keep,
                             int32_t split_len, LongCut cut_long);

// Kernel launchers (kernels.hip).  They return a hipError_t value as int.
int launch_evict_compact(const murmur_seg *seg, const murmur_policy *pol, int32_t pol_per_seq, int32_t B,
                         int32_t *idx, int32_t max_keep, int32_t *count, int32_t *ranges, const int32_t *bt,
                         int32_t max_blocks, int32_t log2_bs, murmur_stream_t stream);
int launch_decode_attn(const AttnLaunch &a, murmur_stream_t stream);
int launch_workspace_init(int32_t *ticket, int64_t n, murmur_stream_t stream);
// Device address of the current device's scratch array (MURMUR_STATIC_SCRATCH_BYTES,
// 256-byte aligned), looked up once per device; *fresh is true on that first
// lookup, when the caller must zero the ticket region.  Returns a hipError_t value.
int static_scratch(void **ptr, bool *fresh);
int launch_read_probe(const void *buf, int64_t n16, int32_t n_workgroups, int32_t threads, int32_t depth, bool lds,
                      uint32_t *sink, murmur_stream_t stream);
int launch_paged_step(const murmur_seg *seg, const murmur_policy *pol, int32_t pol_per_seq, int32_t B, int32_t *bt,
                      int32_t max_blocks, int32_t log2_bs, int32_t *stack, int32_t *top, int32_t capacity,
                      int32_t full_scan, murmur_stream_t stream);
int launch_paged_append(const murmur_seg *seg, int32_t B, const int32_t *bt, int32_t max_blocks, int32_t log2_bs,
                        const murmur_kv &pool, int32_t Hkv, const void *k_new, const void *v_new,
                        murmur_stream_t stream);

// ---- shared pages and shared prefixes (shared.cpp; pages.hpp and shared_attn.hpp) ----

// Workspace of murmur_paged_fork and murmur_paged_compact: fork's header, the place
// of every block's first entry, and a bit per place (zero between calls); then what a
// call leaves to no other: fork's lists of changes (one per kForkCols columns of a
// row) and the freed blocks by place, or compact's number of moves and the source
// and destination blocks of at most n_blocks / 2.
constexpr int kForkCols = 256;
constexpr int kForkPlaces = 1 << 15;  // places of a workgroup that pushes
struct ForkHead {
    int32_t call;  // calls so far
    int32_t top;   // the stack's, before the call's pushes
    int32_t unused[62];
};
struct ForkChange {
    uint32_t place;
    int32_t fresh, old;
};
struct ForkWorkspace {
    ForkHead *head;
    uint64_t *first;      // [n_blocks]
    ForkChange *changes;  // [lists][kForkCols]
    int32_t *counts;      // [lists]
    int32_t *freed;       // [B * max_blocks / kForkPlaces]: bits set
    int32_t *block_at;    // [B * max_blocks]
    uint32_t *bits;       // [B * max_blocks / 32]
};
int launch_paged_fork(const int32_t *parent, int32_t B, int32_t *bt, int32_t max_blocks, int32_t *ref,
                      int32_t n_blocks, int32_t *stack, int32_t *top, const ForkWorkspace &ws,
                      murmur_stream_t stream);
int launch_paged_step_shared(const murmur_seg *seg, const murmur_policy *pol, int32_t pol_per_seq, int32_t B,
                             int32_t *bt, int32_t max_blocks, int32_t log2_bs, int32_t *ref, int32_t n_blocks,
                             int32_t *stack, int32_t *top, int32_t full_scan, int32_t *copied,
                             murmur_stream_t stream);
int launch_paged_append_shared(const murmur_seg *seg, int32_t B, const int32_t *bt, int32_t max_blocks,
                               int32_t log2_bs, const int32_t *copied, const murmur_kv &pool, int32_t Hkv,
                               const void *k_new, const void *v_new, murmur_stream_t stream);
int launch_paged_compact(int32_t B, int32_t *bt, int32_t max_blocks, int32_t log2_bs, int32_t *ref, int32_t n_blocks,
                         int32_t *stack, int32_t *top, int32_t *map, const murmur_kv *pool, int32_t Hkv, int32_t *ws,
                         murmur_stream_t stream);

// The schedule of an attention over shared prefixes, written by
// murmur_shared_plan into the caller's plan buffer (in this order):
//   PlanHeader;
//   PlanSeq [B]: where a sequence's partials lie;
//   PlanItem [n_wg]: what a workgroup does;
//   PlanChunk [n_wg][kSharedWaves]: the wavefronts' parts where it does remainders;
//   first differing rank [B][n_scan] of each sequence's list against its group's
//     first one, per kScanLen entries.
// n_wg bounds the workgroups of a (layer, KV head) whatever the lists hold (see
// shared_caps).
constexpr int kSharedWaves = 8;       // of a workgroup, which has a compute unit to itself
constexpr int kSharedRows = 48;       // query rows of one prefix item: three MFMA row tiles
constexpr int kSharedMaxSeqs = 4096;  // sequences of a batch (the planner's LDS)
// A cut of the work at level j = 4 .. kSharedLevels gives the wavefronts of a prefix
// item j / 4 passes of kWaveTile positions on average and one of a rest up to 3 j / 8
// (it has one row tile).
constexpr int kSharedLevels = 64;
constexpr int item_passes(int level) { return kSharedWaves * level / 4; }
constexpr int chunk_passes(int level) { return level * 3 / 8; }
constexpr int kScanLen = 4096;
constexpr int32_t kPlanMagic = 0x6d75726d;
struct PlanHeader {
    int32_t magic, n_work, bad, kind;     // bad: the groups are not in order; every output is NaN; kind: see plan_kind
    int32_t B, max_keep, n_layers, Hq, Hkv, n_groups;  // what the plan was made for
    int32_t rows, level, unused[4];       // partial rows per (layer, KV head); the cut (below 0: no list is cut)
};
// A plan's kind, one bit of four: whether lists are cut or whole, and whether lists of
// several sequences were found to begin alike (then they name the same rows in one
// cache only, and the plan does not serve caches of the sequences' own).
constexpr int32_t plan_kind(bool whole, bool found) { return (whole ? 2 : 1) << (found ? 2 : 0); }
struct PlanSeq {
    int32_t state;  // 0: not there or in no group (outputs untouched), 1: computed, 2: invalid count (NaN outputs)
    int32_t pre_row, pre_stride, n_pre;  // partials over the prefix: rows pre_row + i * pre_stride + head
    int32_t rest_row, n_rest;            // over the rest: rows rest_row + i * G + head
    int32_t rest, unused;                // length of the rest (plans without cuts)
};
struct PlanItem {
    int32_t seq0, n_seq, list, r0, r1, row;  // n_seq 0: remainders; list: the sequence whose list is read; row: partial row
    int32_t stream, unused;                  // stream: the rows are read once, in a large launch
};
struct PlanChunk {
    int32_t seq, r0, r1, row;  // seq -1: none
};
struct SharedCaps {
    int32_t per_round;  // workgroups per (layer, KV head) of one dispatch round
    int32_t n_wg, n_scan;
    int32_t grid;       // workgroups that are launched, at most n_wg
    bool whole;         // no list is cut (see shared_caps)
    int32_t waves;      // of a workgroup then
    int64_t rows;       // partial rows per (layer, KV head)
    size_t plan_bytes, ws_bytes, scan_offset, chunk_offset, item_offset;
};
SharedCaps shared_caps(int32_t n_layers, int32_t B, int32_t Hq, int32_t Hkv, int32_t max_keep, int32_t n_groups);

struct SharedPlanLaunch {
    const int32_t *idx, *ranges, *count, *group;
    int32_t *shared;
    int32_t max_keep, B, n_groups, find, n_layers, Hq, Hkv;
    uint8_t *plan;
    SharedCaps caps;
};
int launch_shared_plan(const SharedPlanLaunch &p, murmur_stream_t stream);

struct SharedAttnLaunch {
    const uint16_t *q, *k, *v;
    int64_t s_layer, s_b, s_h, s_pos;
    const int32_t *idx, *ranges;
    void *out;
    float *lse;
    const uint8_t *plan;
    size_t item_offset, chunk_offset;
    float *part_o;   // [layers * KV heads][rows][128], then the pairs
    float *part_ml;  // [layers * KV heads][rows][2]  (running max in log2 units, sum)
    int64_t rows_cap;
    int32_t max_len, max_keep, B, Hq, Hkv, G, NL, n_groups, n_wg, out_f32;
    int32_t kinds;     // plans that serve the call, bits of plan_kind (16 bytes with n_wg: one load at a kernel's
                       // start; behind magic_g and scale_log2 it came later, 0.3 us a launch)
    uint32_t magic_g;  // magic16(G): row / G for rows below 2^16
    float scale_log2;
    int32_t waves;     // SharedCaps::waves, 0 where lists are cut
};
int launch_decode_attn_shared(const SharedAttnLaunch &a, murmur_stream_t stream);

int read_and_clear_device_error(murmur_stream_t stream, int32_t *code);
const char *hip_error_text(int err);

}  // namespace murmur
