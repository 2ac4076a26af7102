// Device code of the shared pages of a paged cache (included by kernels.hip):
// block tables whose rows may name the same blocks, with a reference count per
// block.
//
//   fork_compare_kernel, fork_apply_kernel, fork_push_kernel
//                            rows of the table become copies of other rows
//   step_shared_kernel       the block manager's step with reference counts and
//                            copies on write
//   append_shared_kernel     the copied rows and the current token's K/V
//   compact_plan_kernel, compact_move_kernel
//                            the blocks in use move to the front of the pool
//
// Counts change by integer atomics, whose order does not matter.  What does
// matter is where a block that nobody names any more lands on the free stack:
// every entry that gave it up has a place (row, column), and the block is pushed by
// its first one, found with atomic minima or maxima, whatever the timing.  So the
// stack is the same on every run.
#pragma once

namespace murmur {

// Sums over the wavefront's lanes up to each one, all lanes active: shifts within the
// rows of 16 lanes, then the sums of the row and of the two rows before (DPP operands
// of the adds, where a shuffle is a round trip to LDS).
static __device__ __forceinline__ int wave_inclusive_scan(int x) {
    x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);  // row_shr:1
    x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
    x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);  // row_bcast:15
    x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);  // row_bcast:31
    return x;
}
static __device__ __forceinline__ int wave_sum(int x) { return __builtin_amdgcn_readlane(wave_inclusive_scan(x), 63); }
// The maximum of values that are not negative.
static __device__ __forceinline__ int wave_max(int x) {
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
    x = max(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
    return __builtin_amdgcn_readlane(x, 63);
}

static __device__ __forceinline__ void add_ref(int32_t *ref, int32_t n) {
    __hip_atomic_fetch_add(ref, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// Exclusive scan of one int per thread over a workgroup of kThreads; `total` in
// every thread.  s: one int per wavefront (two barriers).
template <int kThreads>
static __device__ __forceinline__ int wg_exclusive_scan(int v, int *s, int tid, int &total) {
    const int lane = tid & 63, wave = tid >> 6;
    const int x = wave_inclusive_scan(v);
    if (lane == 63) s[wave] = x;
    __syncthreads();
    int before = 0;
    total = 0;
#pragma unroll
    for (int w = 0; w < kThreads / 64; ++w) {
        const int n = s[w];
        before += w < wave ? n : 0;
        total += n;
    }
    __syncthreads();
    return before + x - v;
}

// ---------------------------------------------------------------------------
// fork, in three launches; the first two have a wavefront per 256 columns of a row.
//   fork_compare_kernel  Each entry that differs from the parent's moves the two
//     counts, enters its place for the block that it gives up (`first`: a maximum of
//     (call number, 2^30 - place), so that nothing has to be reset between calls),
//     and goes on the wavefront's list of changes, marked if it took the count to
//     zero.  No table entry is written while another wavefront may read it.
//   fork_apply_kernel  The counts are final.  The changes are written, and a marked
//     one whose block is free sets a bit at the block's first entry's place.
//   fork_push_kernel  The blocks are pushed in the order of their bits.
// Nothing but the comparison looks at the whole table: hypotheses differ from their
// parents in the blocks of their last tokens only.  Bound by round trips to memory.
// 96 rows of 215 blocks 11.4 us, 1024 rows of 311 20.2.  In one launch,
// with the list left to the workgroup that ends last, 11.0 and 58.8: a compute unit
// has only so many scattered loads on their way.
// ---------------------------------------------------------------------------
constexpr int kForkThreads = 1024;
constexpr int kForkWaves = kForkThreads / 64;
constexpr uint32_t kForkEmptied = 1u << 31;  // mark of a change's place (places are below 2^30)

// The wavefront's row and first column (its lane's), or none.
struct ForkUnit {
    int64_t at;
    int b, col;
};
static __device__ __forceinline__ ForkUnit fork_unit(int32_t B, int32_t max_blocks, int wave, int lane) {
    const int segs = (max_blocks + kForkCols - 1) / kForkCols;
    const int64_t unit = (int64_t)blockIdx.x * kForkWaves + wave;
    if (unit >= (int64_t)B * segs) return ForkUnit{-1, 0, 0};
    const int b = (int)(unit / segs);
    return ForkUnit{unit, b, (int)(unit - (int64_t)b * segs) * kForkCols + lane};
}

__global__ __launch_bounds__(kForkThreads) void fork_compare_kernel(const int32_t *__restrict__ parent, int32_t B,
                                                                    const int32_t *__restrict__ bt,
                                                                    int32_t max_blocks, int32_t *ref,
                                                                    int32_t n_blocks, const ForkWorkspace ws) {
    const int lane = threadIdx.x & 63;
    const ForkUnit u = fork_unit(B, max_blocks, __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane);
    if (u.at < 0) return;
    if (lane == 0 && u.at < ((int64_t)B * max_blocks - 1) / kForkPlaces + 1) ws.freed[u.at] = 0;
    const uint32_t call = (uint32_t)ws.head->call + 1;
    int err = 0;
    int32_t p = parent[u.b];
    if (p < -1 || p >= B) {
        err |= MURMUR_DEVERR_PARENT;
        p = u.b;
    }
    int32_t old[4], fresh[4];
    const int32_t *mine = bt + (int64_t)u.b * max_blocks, *from = bt + (int64_t)(p < 0 ? 0 : p) * max_blocks;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const int c = u.col + 64 * j;
        old[j] = c < max_blocks ? mine[c] : -1;
        fresh[j] = c < max_blocks && p >= 0 ? from[c] : -1;
    }
    ForkChange *list = ws.changes + u.at * kForkCols;
    int n = 0;
    int32_t was[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        was[j] = 0;
        if (old[j] == fresh[j]) continue;
        if (fresh[j] >= n_blocks || old[j] >= n_blocks) err |= MURMUR_DEVERR_BLOCK;
        if (fresh[j] >= 0 && fresh[j] < n_blocks) add_ref(ref + fresh[j], 1);
        if (old[j] >= 0 && old[j] < n_blocks) {
            const uint32_t place = (uint32_t)(u.b * max_blocks + u.col + 64 * j);
            was[j] = __hip_atomic_fetch_add(ref + old[j], -1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
            __hip_atomic_fetch_max(ws.first + old[j], (uint64_t)call << 32 | ((1u << 30) - place), __ATOMIC_RELAXED,
                                   __HIP_MEMORY_SCOPE_AGENT);
        }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint64_t differs = __ballot(old[j] != fresh[j]);
        if (old[j] != fresh[j]) {
            const uint32_t place = (uint32_t)(u.b * max_blocks + u.col + 64 * j);
            list[n + __popcll(differs & ((1ull << lane) - 1))] =
                ForkChange{place | (was[j] == 1 ? kForkEmptied : 0u), fresh[j], old[j]};
        }
        n += __popcll(differs);
    }
    if (lane == 0) ws.counts[u.at] = n;
    if (err) raise_device_error(err);
}

__global__ __launch_bounds__(kForkThreads) void fork_apply_kernel(int32_t B, int32_t *__restrict__ bt,
                                                                  int32_t max_blocks, const int32_t *__restrict__ ref,
                                                                  const int32_t *__restrict__ top,
                                                                  const ForkWorkspace ws) {
    const int tid = threadIdx.x, lane = tid & 63;
    const ForkUnit u = fork_unit(B, max_blocks, __builtin_amdgcn_readfirstlane(tid >> 6), lane);
    if (blockIdx.x == 0 && tid == 0) ws.head->top = *top;
    if (u.at < 0) return;
    const ForkChange *list = ws.changes + u.at * kForkCols;
    const int n = ws.counts[u.at];
    ForkChange c[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) c[j] = list[lane + 64 * j];  // past the end: of an earlier call, not used
    int32_t left[4];
    uint64_t first[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        left[j] = 1;
        first[j] = 0;
        if (lane + 64 * j >= n) continue;
        bt[c[j].place & ~kForkEmptied] = c[j].fresh;
        if (c[j].place & kForkEmptied) {
            left[j] = ref[c[j].old];
            first[j] = ws.first[c[j].old];
        }
    }
    // One atomic per word of bits: a wavefront's places are neighbours, and the atomics of one word, or of one
    // count, queue (one per block: 59 us for 1024 rows, not 10).
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const uint32_t place = (1u << 30) - (uint32_t)first[j];
        if (left[j] == 0) ws.block_at[place] = c[j].old;  // else not marked, or named again by another row
        uint64_t todo = __ballot(left[j] == 0);
        while (todo) {
            const uint32_t word = __builtin_amdgcn_readlane(place, (int)__ffsll((unsigned long long)todo) - 1) >> 5;
            const bool here = left[j] == 0 && place >> 5 == word;
            uint32_t bits = here ? 1u << (place & 31) : 0u;
#pragma unroll
            for (int x = 32; x >= 1; x /= 2) bits |= __shfl_xor(bits, x);
            if (lane == 0) {
                const uint32_t had = __hip_atomic_fetch_or(ws.bits + word, bits, __ATOMIC_RELAXED,
                                                           __HIP_MEMORY_SCOPE_AGENT);
                add_ref(ws.freed + word / (kForkPlaces / 32), __popc(bits & ~had));  // a block may be marked twice
            }
            todo &= ~__ballot(here);
        }
    }
}

// Workgroup w: the freed blocks of places [w, w + 1) * kForkPlaces.
__global__ __launch_bounds__(kForkThreads) void fork_push_kernel(int64_t places, int32_t n_blocks,
                                                                 int32_t *__restrict__ stack,
                                                                 int32_t *__restrict__ top, const ForkWorkspace ws) {
    constexpr int kWindow = 8192;  // pushes that LDS orders at a time
    static_assert(kForkPlaces == 32 * kForkThreads, "a word of bits per thread");
    __shared__ int32_t s_place[kWindow];
    __shared__ int s_scan[kForkWaves];
    const int tid = threadIdx.x;
    const int64_t w = (int64_t)blockIdx.x * kForkThreads + tid, words = (places + 31) / 32;
    const uint32_t bits = w < words ? ws.bits[w] : 0u;
    int32_t tp = ws.head->top;
    tp = tp < 0 ? 0 : (tp > n_blocks ? n_blocks : tp);
    int before = 0, all = 0;
    for (int g = tid; g < (int)gridDim.x; g += kForkThreads) {
        const int f = ws.freed[g];
        before += g < (int)blockIdx.x ? f : 0;
        all += f;
    }
    wg_exclusive_scan<kForkThreads>(before, s_scan, tid, before);
    int total;
    const int mine = wg_exclusive_scan<kForkThreads>(__popc(bits), s_scan, tid, total);
    if (blockIdx.x == 0) {
        wg_exclusive_scan<kForkThreads>(all, s_scan, tid, all);
        if (tid == 0) {
            *top = tp + all < n_blocks ? tp + all : n_blocks;
            ws.head->call += 1;
            if (tp + all > n_blocks) raise_device_error(MURMUR_DEVERR_POOL);
        }
    }
    if (bits) ws.bits[w] = 0;  // zero between calls
    const int32_t *block_at = ws.block_at + (int64_t)blockIdx.x * kForkPlaces;
    for (int r0 = 0; r0 < total; r0 += kWindow) {
        int rank = mine - r0;
        for (uint32_t x = bits; x; x &= x - 1, ++rank)
            if (rank >= 0 && rank < kWindow) s_place[rank] = 32 * tid + __ffs(x) - 1;
        __syncthreads();
        for (int i = tid; i < min(total - r0, kWindow); i += kForkThreads) {
            const int64_t to = (int64_t)tp + before + r0 + i;
            if (to < n_blocks) stack[to] = block_at[s_place[i]];
        }
        __syncthreads();
    }
}

// ---------------------------------------------------------------------------
// step_shared: paged_step's two passes with counts, by one workgroup.  Every entry
// given up takes one off its block's count.  Where that empties a block, each
// entry of it offers its place with an atomic minimum on the count itself (offers
// are negative), and the first one pushes the block; steps in which nothing empties
// (all but one in block-size many, and those of hypotheses that share what they
// give up) pass over that.  Then each sequence finds whether its current token's
// block is missing, its own, or held by others too: of R holders, the k sequences
// of the batch that are about to write there are ranked by (position, index), and
// the one of rank i copies if i < R - 1, as if they went one after the other: the
// last one keeps the block when nobody else holds it.  It is the one furthest
// ahead, so what it writes lies behind every row that the others copy.
// Round trips to memory bound it, so a sequence's layout, policy and current block
// stay in registers where a thread has only one, and the counts in its XCD's L2: 4.6
// us for 4 sequences, 11.2 for 96 of which 35 copy (17.0 with the counts past the L2;
// 3.5 of the 11 rank the writers).  The ranking compares every row that may have to
// copy with every row of the batch, one workgroup for all: with seven of eight
// copying, timed around the call, 13 us for 96 sequences, 88 for 1024, 1222 for 4096.
// ---------------------------------------------------------------------------
// The counts are this workgroup's alone while it runs: atomics in its XCD's L2, where
// those that other XCDs see go past it.
static __device__ __forceinline__ int32_t load_count(const int32_t *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
static __device__ __forceinline__ void store_count(int32_t *p, int32_t x) {
    __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
}
static __device__ __forceinline__ int32_t place_key(int32_t at) { return (int32_t)(0x80000000u + (uint32_t)at); }
static __device__ __forceinline__ int64_t seq_position(const murmur_seg &s) {  // of the current token
    return (int64_t)s.prompt_pre + s.speech_len + s.prompt_mid + s.out_len - 1;
}

// What step_shared needs of a sequence: its freeable columns and where its token goes.
struct StepSeq {
    PagedSeq q;
    int32_t pos;  // valid sequences: of the current token
    int32_t x;    // the block there (-1: none, or past the table)
};

template <int kThreads>
__global__ __launch_bounds__(kThreads) void step_shared_kernel(const murmur_seg *__restrict__ seg,
                                                               const murmur_policy *__restrict__ pol,
                                                               int32_t pol_per_seq, int32_t B, int32_t *bt,
                                                               int32_t max_blocks, int32_t log2_bs, int32_t *ref,
                                                               int32_t n_blocks, int32_t *stack, int32_t *top,
                                                               int32_t full_scan, int32_t *copied) {
    __shared__ int s_scan[kThreads / 64];
    __shared__ int2 s_writer[kThreads];
    constexpr int32_t kTakeBlock = -3;
    const int tid = threadIdx.x;
    const bool one_each = B <= kThreads;
    int32_t tp = *top;
    tp = tp < 0 ? 0 : (tp > n_blocks ? n_blocks : tp);
    int err = 0;
    const auto load_seq = [&](int b) {
        int bad = 0;
        StepSeq s{paged_seq(seg, pol, pol_per_seq, b, B, max_blocks, log2_bs, full_scan, bad), 0, -1};
        // a sequence that is not there gives up, takes and writes nothing, and is no error
        if (bad && !layout_absent(seg[b].prompt_pre, seg[b].speech_len, seg[b].prompt_mid, seg[b].out_len)) err |= bad;
        if (s.q.valid) {
            s.pos = (int32_t)seq_position(seg[b]);
            if (s.q.cur < max_blocks) s.x = bt[(int64_t)b * max_blocks + s.q.cur];
        }
        return s;
    };
    const StepSeq mine = load_seq(tid);
    const auto seq_of = [&](int b) { return one_each ? mine : load_seq(b); };
    // every entry of sequence b to give up, with its place
    const auto each_freed = [&](int b, const StepSeq &s, auto f) {
        int32_t *row = bt + (int64_t)(s.q.valid ? b : 0) * max_blocks;
#pragma unroll
        for (int k = 0; k < 2; ++k)
            for (int32_t blk = s.q.lo[k]; blk < s.q.hi[k]; ++blk) {
                const int32_t phys = row[blk];
                if (phys >= 0) f(row + blk, phys, b * max_blocks + blk);
            }
    };
    int emptied = 0;
    for (int b = tid; b < B; b += kThreads)
        each_freed(b, seq_of(b), [&](int32_t *, int32_t phys, int32_t) {
            if (phys < n_blocks)
                emptied |= __hip_atomic_fetch_add(ref + phys, -1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP) == 1;
            else
                err |= MURMUR_DEVERR_BLOCK;
        });
    emptied = __syncthreads_or(emptied);
    if (emptied) {
        for (int b = tid; b < B; b += kThreads)
            each_freed(b, seq_of(b), [&](int32_t *, int32_t phys, int32_t at) {
                if (phys < n_blocks && load_count(ref + phys) <= 0)
                    __hip_atomic_fetch_min(ref + phys, place_key(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            });
        wait_vmem();
        __syncthreads();
    }
    for (int b0 = 0; b0 < B; b0 += kThreads) {
        const StepSeq s = seq_of(b0 + tid);
        int to = tp, seen = 0;
        uint32_t won = 0;  // of the first 32 entries, those that push their blocks
        const auto wins = [&](int32_t phys, int32_t at) { return phys < n_blocks && load_count(ref + phys) == place_key(at); };
        if (emptied) {
            int n = 0, pushed;
            each_freed(b0 + tid, s, [&](int32_t *, int32_t phys, int32_t at) {
                const bool win = wins(phys, at);
                n += win;
                won |= win && seen < 32 ? 1u << seen : 0u;
                ++seen;
            });
            seen = 0;
            to = tp + wg_exclusive_scan<kThreads>(n, s_scan, tid, pushed);
            tp = tp + pushed < n_blocks ? tp + pushed : n_blocks;
        }
        each_freed(b0 + tid, s, [&](int32_t *entry, int32_t phys, int32_t at) {
            if (emptied && (seen < 32 ? won >> seen & 1u : wins(phys, at))) {
                if (to < n_blocks) stack[to] = phys;
                else err |= MURMUR_DEVERR_POOL;
                ++to;
                store_count(ref + phys, 0);
            }
            ++seen;
            *entry = -1;
        });
    }
    if (emptied) {
        wait_vmem();
        __syncthreads();  // the stack and the counts before the pops
    }
    // What each sequence needs, before any table entry or count changes: kTakeBlock, -1 for nothing, -2 if it is not
    // valid, else a copy of the block named.
    const auto need_of = [&](int b0) {
        const StepSeq s = seq_of(b0 + tid);
        int32_t what = s.q.valid ? -1 : -2;
        int holders = 0;
        if (s.q.valid && s.q.cur >= max_blocks) {
            err |= MURMUR_DEVERR_BLOCK;
        } else if (s.q.valid && s.x < 0) {
            what = kTakeBlock;
        } else if (s.q.valid && s.x >= n_blocks) {
            what = -2;  // a caller's pool may be larger than its blocks: no rows behind them are written
            err |= MURMUR_DEVERR_BLOCK;
        } else if (s.q.valid) {
            holders = load_count(ref + s.x);
        }
        if (!__syncthreads_or(holders > 1)) return what;
        int before = 0;
        for (int o0 = 0; o0 < B; o0 += kThreads) {  // all sequences that write to a block, kThreads at a time
            const StepSeq o = seq_of(o0 + tid);
            s_writer[tid] = o.q.valid && o.q.cur < max_blocks ? int2{o.x, o.pos} : int2{-1, 0};
            __syncthreads();
            if (holders > 1)
#pragma unroll 8
                for (int i = 0; i < (min(kThreads, B - o0) + 7) / 8 * 8; ++i) {  // behind the last sequence none writes
                    const int2 y = s_writer[i];
                    // (position, index) before this one's; no short cuts, which would be branches
                    before += (int)(y.x == s.x) & (int)((y.y >> log2_bs) == s.q.cur) &
                              (int)(y.y <= s.pos - (int)(o0 + i >= b0 + tid));
                }
            __syncthreads();
        }
        return holders > 1 && before < holders - 1 ? s.x : what;
    };
    int32_t need_mine = 0;
    for (int b0 = 0; b0 < B; b0 += kThreads) {
        need_mine = need_of(b0);
        if (!one_each && b0 + tid < B) copied[b0 + tid] = need_mine;
    }
    __syncthreads();  // every count is read
    for (int b0 = 0; b0 < B; b0 += kThreads) {
        const int b = b0 + tid;
        const int32_t what = b >= B ? -2 : (one_each ? need_mine : copied[b]);
        const bool need = what >= 0 || what == kTakeBlock;
        int taken;
        const int off = wg_exclusive_scan<kThreads>(need, s_scan, tid, taken);
        int32_t from_block = what;
        if (need) {
            const int32_t cur = one_each ? mine.q.cur : (int32_t)(seq_position(seg[b]) >> log2_bs);
            const int from = tp - 1 - off;
            const int32_t got = from >= 0 ? stack[from] : -1;
            const bool good = got >= 0 && got < n_blocks;
            if (good) store_count(ref + got, 1);
            else err |= MURMUR_DEVERR_POOL;
            if (what >= 0) __hip_atomic_fetch_add(ref + what, -1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
            bt[(int64_t)b * max_blocks + cur] = good ? got : -1;
            from_block = good ? (what >= 0 ? what : -1) : -2;
        }
        if (b < B) copied[b] = from_block;
        tp = tp - taken > 0 ? tp - taken : 0;
    }
    if (tid == 0) *top = tp;
    if (err) raise_device_error(err);
}

// A workgroup per sequence and some of its (layer, K or V) planes: the rows of the
// current block before the token from the block it was copied from, then the
// token's own rows.  A thread has a 16-byte chunk of a row in each plane, and its
// loads of kAppendPlanes planes are on their way at once (96 sequences, 28 layers, 181
// rows copied for 35 of them: 31.8 MB read and written in 9.4 us, 10.0 with a plane at
// a time).
constexpr int kAppendPlanes = 4;
__global__ __launch_bounds__(256) void append_shared_kernel(const murmur_seg *__restrict__ seg, int32_t B,
                                                            const int32_t *__restrict__ bt, int32_t max_blocks,
                                                            int32_t log2_bs, const int32_t *__restrict__ copied,
                                                            uint16_t *k, uint16_t *v, int64_t s_layer, int64_t s_h,
                                                            int64_t s_pos, int64_t rows,
                                                            const uint16_t *__restrict__ k_new,
                                                            const uint16_t *__restrict__ v_new, int32_t NL,
                                                            int32_t Hkv) {
    const int b = blockIdx.x;
    const int32_t from = copied[b];
    const int64_t p = seq_position(seg[b]);
    const int64_t blk = p >> log2_bs;
    if (p < 0 || blk >= max_blocks) return;
    const int32_t phys = bt[(int64_t)b * max_blocks + blk];
    if (phys < 0 || from < -1) return;
    const int32_t slot = (int32_t)(p & ((1 << log2_bs) - 1));
    const int64_t row0 = (int64_t)phys << log2_bs, src0 = (int64_t)from << log2_bs;
    if (row0 + slot >= rows || src0 + slot > rows) return;
    const int planes = 2 * NL, copies = from >= 0 ? slot * Hkv * 16 : 0;
    for (int t = threadIdx.x; t < copies + Hkv * 16; t += 256) {
        const bool copy = t < copies;
        const int r = (copy ? t : t - copies) >> 4, j = copy ? r / Hkv : slot, h = copy ? r - j * Hkv : r;
        const int64_t to = (row0 + j) * s_pos + h * s_h + 8 * (t & 15);
        // the source of a copied chunk and of a new one, each with its step from layer to layer
        const int64_t at = copy ? (src0 + j) * s_pos + h * s_h + 8 * (t & 15) : ((int64_t)b * Hkv + h) * kHeadDim + 8 * (t & 15);
        const int64_t step = copy ? s_layer : (int64_t)B * Hkv * kHeadDim;
        const uint16_t *from_k = copy ? k : k_new, *from_v = copy ? v : v_new;
        for (int lv0 = (int)blockIdx.y * kAppendPlanes; lv0 < planes; lv0 += (int)gridDim.y * kAppendPlanes) {
            u32x4 x[kAppendPlanes];
#pragma unroll
            for (int i = 0; i < kAppendPlanes; ++i) {
                const int lv = min(lv0 + i, planes - 1);
                x[i] = load16((lv & 1 ? from_v : from_k) + (lv >> 1) * step + at);
            }
#pragma unroll
            for (int i = 0; i < kAppendPlanes; ++i) {
                const int lv = lv0 + i;
                if (lv < planes) *reinterpret_cast<u32x4 *>((lv & 1 ? v : k) + (lv >> 1) * s_layer + to) = x[i];
            }
        }
    }
}

// ---------------------------------------------------------------------------
// compact.  n blocks are in use (count > 0): those at n and behind move, in
// ascending order, into the free ones before n, so no block is both read and
// written.  One workgroup ranks them with scans over the counts (2650 blocks: 5.0 us);
// then the chip copies the blocks and renames the table's entries.
// ---------------------------------------------------------------------------
constexpr int kCompactThreads = 1024;
constexpr int kCompactEach = 4;  // consecutive blocks of a thread

__global__ __launch_bounds__(kCompactThreads) void compact_plan_kernel(int32_t *__restrict__ ref, int32_t n_blocks,
                                                                       int32_t *__restrict__ stack,
                                                                       int32_t *__restrict__ top, int32_t *map,
                                                                       int32_t *ws) {
    __shared__ int s_scan[kCompactThreads / 64];
    constexpr int kRound = kCompactThreads * kCompactEach;
    const int tid = threadIdx.x;
    int32_t *src = ws + 1, *dst = src + n_blocks / 2;
    const auto load = [&](int i0, int32_t (&r)[kCompactEach]) {
#pragma unroll
        for (int j = 0; j < kCompactEach; ++j) r[j] = i0 + j < n_blocks ? ref[i0 + j] : 0;
    };
    int32_t r[kCompactEach];
    int used = 0;
    for (int i0 = 0; i0 < n_blocks; i0 += kRound) {
        load(i0 + tid * kCompactEach, r);
        int n = 0, total;
#pragma unroll
        for (int j = 0; j < kCompactEach; ++j) n += r[j] > 0;
        wg_exclusive_scan<kCompactThreads>(n, s_scan, tid, total);
        used += total;
    }
    int moves = 0, holes = 0;
    for (int i0 = 0; i0 < n_blocks; i0 += kRound) {
        const int first = i0 + tid * kCompactEach;
        if (n_blocks > kRound) load(first, r);  // one round: still in registers
        // movers and holes in one scan: at most kRound each, 16 bits apart
        static_assert(kRound < 1 << 16, "two counts in one word");
        int n = 0, total;
#pragma unroll
        for (int j = 0; j < kCompactEach; ++j) {
            const int i = first + j;
            n += i < n_blocks && i >= used && r[j] > 0 ? 1 : 0;
            n += i < used && r[j] <= 0 ? 1 << 16 : 0;
        }
        const int at = wg_exclusive_scan<kCompactThreads>(n, s_scan, tid, total);
        int am = moves + (at & 0xffff), ah = holes + (at >> 16);
#pragma unroll
        for (int j = 0; j < kCompactEach; ++j) {
            const int i = first + j;
            if (i >= n_blocks) break;
            const bool live = r[j] > 0;
            if (live && i >= used) src[am++] = i;
            if (!live && i < used) dst[ah++] = i;
            map[i] = live && i < used ? i : -1;
            if (i < n_blocks - used) stack[i] = n_blocks - 1 - i;
        }
        moves += total & 0xffff;
        holes += total >> 16;
    }
    __syncthreads();
    for (int j = tid; j < moves; j += kCompactThreads) {
        const int32_t s = src[j], d = dst[j];
        map[s] = d;
        ref[d] = ref[s];
        ref[s] = 0;
    }
    if (tid == 0) {
        ws[0] = moves;
        *top = n_blocks - used;
    }
}

// Workgroups 0 .. gridDim.x - 1 of y = 0 rename the table, those of y > 0 copy: K and V of every (move, layer),
// each by one workgroup in 16-byte units.  Bound by memory: 1.15 GB read and written in 251 us (4.6 TB/s; a plain copy
// of 4 GiB reaches 4.8).
__global__ __launch_bounds__(256) void compact_move_kernel(int32_t *__restrict__ bt, int64_t entries,
                                                           const int32_t *__restrict__ map, int32_t n_blocks,
                                                           const int32_t *__restrict__ ws, int32_t log2_bs,
                                                           uint16_t *k, uint16_t *v, int64_t s_layer, int64_t s_h,
                                                           int64_t s_pos, int32_t NL, int32_t Hkv) {
    if (blockIdx.y == 0) {
        int err = 0;
        for (int64_t i = blockIdx.x * (int64_t)256 + threadIdx.x; i < entries; i += (int64_t)gridDim.x * 256) {
            const int32_t x = bt[i];
            if (x < 0) continue;
            if (x >= n_blocks) {
                err |= MURMUR_DEVERR_BLOCK;
                continue;
            }
            const int32_t to = map[x];
            if (to < 0) err |= MURMUR_DEVERR_BLOCK;
            if (to != x) bt[i] = to;
        }
        if (err) raise_device_error(err);
        return;
    }
    const int32_t *src = ws + 1, *dst = src + n_blocks / 2;
    const int64_t items = (int64_t)ws[0] * NL * 2;
    const int units = (Hkv * 16) << log2_bs;
    for (int64_t it = (int64_t)(blockIdx.y - 1) * gridDim.x + blockIdx.x; it < items;
         it += (int64_t)(gridDim.y - 1) * gridDim.x) {
        const int64_t j = it / (2 * NL), lv = it - j * 2 * NL;
        uint16_t *base = ((lv & 1) ? v : k) + (lv >> 1) * s_layer;
        const int64_t from = ((int64_t)src[j] << log2_bs) * s_pos, to = ((int64_t)dst[j] << log2_bs) * s_pos;
        for (int t = threadIdx.x; t < units; t += 256) {
            const int c = t & 15, h = (t >> 4) % Hkv, r = (t >> 4) / Hkv;
            const int64_t at = h * s_h + r * s_pos + 8 * c;
            *reinterpret_cast<u32x4 *>(base + to + at) = load16(base + from + at);
        }
    }
}

// ---- launchers ----

int launch_paged_fork(const int32_t *parent, int32_t B, int32_t *bt, int32_t max_blocks, int32_t *ref,
                      int32_t n_blocks, int32_t *stack, int32_t *top, const ForkWorkspace &ws,
                      murmur_stream_t stream) {
    const int64_t units = (int64_t)B * ((max_blocks + kForkCols - 1) / kForkCols);
    const dim3 grid((unsigned)((units + kForkWaves - 1) / kForkWaves)), threads(kForkThreads);
    hipLaunchKernelGGL(fork_compare_kernel, grid, threads, 0, (hipStream_t)stream, parent, B, bt, max_blocks, ref,
                       n_blocks, ws);
    int e = (int)hipGetLastError();
    if (e != 0) return e;
    hipLaunchKernelGGL(fork_apply_kernel, grid, threads, 0, (hipStream_t)stream, B, bt, max_blocks, ref, top, ws);
    e = (int)hipGetLastError();
    if (e != 0) return e;
    const int64_t places = (int64_t)B * max_blocks;
    hipLaunchKernelGGL(fork_push_kernel, dim3((unsigned)((places - 1) / kForkPlaces + 1)), threads, 0,
                       (hipStream_t)stream, places, n_blocks, stack, top, ws);
    return (int)hipGetLastError();
}

int launch_paged_step_shared(const murmur_seg *seg, const murmur_policy *pol, int32_t pol_per_seq, int32_t B,
                             int32_t *bt, int32_t max_blocks, int32_t log2_bs, int32_t *ref, int32_t n_blocks,
                             int32_t *stack, int32_t *top, int32_t full_scan, int32_t *copied,
                             murmur_stream_t stream) {
    // a thread per sequence up to 1024; a small batch takes fewer wavefronts through the barriers
    if (B <= 256)
        hipLaunchKernelGGL(step_shared_kernel<256>, dim3(1), dim3(256), 0, (hipStream_t)stream, seg, pol, pol_per_seq,
                           B, bt, max_blocks, log2_bs, ref, n_blocks, stack, top, full_scan, copied);
    else
        hipLaunchKernelGGL(step_shared_kernel<1024>, dim3(1), dim3(1024), 0, (hipStream_t)stream, seg, pol,
                           pol_per_seq, B, bt, max_blocks, log2_bs, ref, n_blocks, stack, top, full_scan, copied);
    return (int)hipGetLastError();
}

int launch_paged_append_shared(const murmur_seg *seg, int32_t B, const int32_t *bt, int32_t max_blocks,
                               int32_t log2_bs, const int32_t *copied, const murmur_kv &pool, int32_t Hkv,
                               const void *k_new, const void *v_new, murmur_stream_t stream) {
    const unsigned y = (unsigned)std::min<int64_t>((2 * (int64_t)pool.n_layers + kAppendPlanes - 1) / kAppendPlanes, 65535);
    hipLaunchKernelGGL(append_shared_kernel, dim3((unsigned)B, y), dim3(256), 0, (hipStream_t)stream, seg, B, bt,
                       max_blocks, log2_bs, copied, (uint16_t *)pool.k, (uint16_t *)pool.v, pool.stride_layer,
                       pool.stride_h, pool.stride_pos, (int64_t)pool.max_len, (const uint16_t *)k_new,
                       (const uint16_t *)v_new, pool.n_layers, Hkv);
    return (int)hipGetLastError();
}

int launch_paged_compact(int32_t B, int32_t *bt, int32_t max_blocks, int32_t log2_bs, int32_t *ref, int32_t n_blocks,
                         int32_t *stack, int32_t *top, int32_t *map, const murmur_kv *pool, int32_t Hkv, int32_t *ws,
                         murmur_stream_t stream) {
    hipLaunchKernelGGL(compact_plan_kernel, dim3(1), dim3(kCompactThreads), 0, (hipStream_t)stream, ref, n_blocks,
                       stack, top, map, ws);
    const int e = (int)hipGetLastError();
    if (e != 0) return e;
    const unsigned y = pool ? 1 + 32 : 1;
    hipLaunchKernelGGL(compact_move_kernel, dim3(64, y), dim3(256), 0, (hipStream_t)stream, bt,
                       (int64_t)B * max_blocks, map, n_blocks, ws, log2_bs, pool ? (uint16_t *)pool->k : nullptr,
                       pool ? (uint16_t *)pool->v : nullptr, pool ? pool->stride_layer : 0, pool ? pool->stride_h : 0,
                       pool ? pool->stride_pos : 0, pool ? pool->n_layers : 0, Hkv);
    return (int)hipGetLastError();
}

}  // namespace murmur
