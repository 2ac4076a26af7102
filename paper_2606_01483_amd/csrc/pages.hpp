// Device code of the shared pages of a paged cache (included by kernels.hip):
// block tables whose rows may name the same blocks, with a reference count per
// block.
//
//   fork_kernel              rows of the table become copies of other rows
//   step_shared_kernel       the block manager's step with reference counts and
//                            copies on write
//   append_shared_kernel     the copied rows and the current token's K/V
//   compact_plan_kernel, compact_move_kernel
//                            the blocks in use move to the front of the pool
//
// Counts change by integer atomics, whose order does not matter.  What does
// matter is where a block that nobody names any more lands on the free stack:
// every entry that gave it up offers its place (row, column) with an atomic
// minimum on the count itself, which is zero by then, so that the block is
// pushed by its first entry whatever the timing, and the stack is the same on
// every run.
#pragma once

namespace murmur {

// Loads and stores of words that other workgroups of the launch, or atomics of
// this one, write: past the caches that are not coherent between XCDs.
static __device__ __forceinline__ int32_t load_shared_word(const int32_t *p) {
    return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
static __device__ __forceinline__ void store_shared_word(int32_t *p, int32_t x) {
    __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
static __device__ __forceinline__ void add_ref(int32_t *ref, int32_t n) {
    __hip_atomic_fetch_add(ref, n, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
// Offers place `at` (below 2^30) as the one that pushes a block whose count is
// zero; counts that are offered for are negative.
static __device__ __forceinline__ int32_t place_key(int32_t at) { return (int32_t)(0x80000000u + (uint32_t)at); }
static __device__ __forceinline__ void offer_place(int32_t *ref, int32_t at) {
    if (load_shared_word(ref) <= 0)
        __hip_atomic_fetch_min(ref, place_key(at), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// Exclusive scan of one int per thread over a workgroup of kThreads; `total` in
// every thread.  s: one int per wavefront (two barriers).
template <int kThreads>
static __device__ __forceinline__ int wg_exclusive_scan(int v, int *s, int tid, int &total) {
    const int lane = tid & 63, wave = tid >> 6;
    int x = v;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
        const int y = __shfl_up(x, off);
        x += lane >= off ? y : 0;
    }
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
// fork.  A workgroup per row compares it with its parent's, moves the counts of
// the blocks that differ and lists the entries that change, in column order; no
// table entry is written while another workgroup may read it as a parent's.  The
// workgroup that ends last takes all rows' lists, 1024 entries at a time: it
// pushes the blocks whose count went to zero (see above) and writes the table.
// Beams differ from their parents in the blocks of their last tokens only, so
// the lists are short and the comparison, which reads the table twice, is the
// work; it is spread over the chip.
// ---------------------------------------------------------------------------
constexpr int kForkThreads = 512;

__global__ __launch_bounds__(kForkThreads) void fork_kernel(const int32_t *__restrict__ parent, int32_t B,
                                                            int32_t *bt, int32_t max_blocks, int32_t *ref,
                                                            int32_t n_blocks, int32_t *stack, int32_t *top,
                                                            int32_t *ws) {
    __shared__ int s_scan[kForkThreads / 64];
    __shared__ int s_first[kForkThreads + 1];
    __shared__ int s_last;
    const int tid = threadIdx.x, b = blockIdx.x;
    int32_t *ticket = ws, *count = ws + kForkHeader;
    ForkEntry *lists = reinterpret_cast<ForkEntry *>(ws + kForkHeader + ((B + 63) & ~63));
    int err = 0;
    int32_t p = parent[b];
    if (p < -1 || p >= B) {
        err |= MURMUR_DEVERR_PARENT;
        p = b;
    }
    int n = 0;
    if (p != b) {
        const int32_t *from = bt + (int64_t)(p < 0 ? 0 : p) * max_blocks;
        const int32_t *mine = bt + (int64_t)b * max_blocks;
        ForkEntry *list = lists + (int64_t)b * max_blocks;
        for (int c0 = 0; c0 < max_blocks; c0 += kForkThreads) {
            const int c = c0 + tid;
            const bool in = c < max_blocks;
            const int32_t old = in ? mine[c] : -1;
            const int32_t fresh = in && p >= 0 ? from[c] : -1;
            const bool differs = old != fresh;
            if (differs) {
                if (fresh >= n_blocks || old >= n_blocks) err |= MURMUR_DEVERR_BLOCK;
                if (fresh >= 0 && fresh < n_blocks) add_ref(ref + fresh, 1);
                if (old >= 0 && old < n_blocks) add_ref(ref + old, -1);
            }
            int total;
            const int at = n + wg_exclusive_scan<kForkThreads>(differs, s_scan, tid, total);
            if (differs) {
                store_shared_word(&list[at].col, c);
                store_shared_word(&list[at].fresh, fresh);
                store_shared_word(&list[at].old, old);
            }
            n += total;
        }
    }
    if (err) raise_device_error(err);
    if (tid == 0) store_shared_word(count + b, n);
    wait_vmem();
    __syncthreads();
    if (tid == 0) {
        const int prev = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        s_last = prev == B - 1;
        if (s_last) store_shared_word(ticket, 0);
    }
    __syncthreads();
    if (!s_last) return;

    // Entry e of the rows b0 .. b0 + kForkThreads - 1, of which s_first holds each row's first.
    const auto entry_of = [&](int e, int b0, int &row, ForkEntry &x) {
        int lo = 0, hi = kForkThreads;  // the last row whose first entry is at or before e
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (s_first[mid] <= e) lo = mid;
            else hi = mid;
        }
        row = b0 + lo;
        const ForkEntry *l = lists + (int64_t)row * max_blocks + (e - s_first[lo]);
        x.col = load_shared_word(&l->col);
        x.fresh = load_shared_word(&l->fresh);
        x.old = load_shared_word(&l->old);
    };
    int32_t tp = *top;
    tp = tp < 0 ? 0 : (tp > n_blocks ? n_blocks : tp);
    err = 0;
    for (int pass = 0; pass < 2; ++pass) {  // every place is offered before the first block is pushed
        for (int b0 = 0; b0 < B; b0 += kForkThreads) {
            int total;
            const int c = b0 + tid < B ? load_shared_word(count + b0 + tid) : 0;
            const int first = wg_exclusive_scan<kForkThreads>(c, s_scan, tid, total);
            s_first[tid] = first;
            __syncthreads();
            for (int e0 = 0; e0 < total; e0 += kForkThreads) {
                const int e = e0 + tid;
                int row = 0;
                ForkEntry x{0, -1, -1, 0};
                if (e < total) entry_of(e, b0, row, x);
                const int32_t at = row * max_blocks + x.col;
                const bool block = x.old >= 0 && x.old < n_blocks;
                if (pass == 0) {
                    if (block) offer_place(ref + x.old, at);
                    continue;
                }
                const bool mine = block && load_shared_word(ref + x.old) == place_key(at);
                int pushed;
                const int to = tp + wg_exclusive_scan<kForkThreads>(mine, s_scan, tid, pushed);
                if (mine) {
                    if (to < n_blocks) stack[to] = x.old;
                    else err |= MURMUR_DEVERR_POOL;
                    store_shared_word(ref + x.old, 0);
                }
                tp = tp + pushed < n_blocks ? tp + pushed : n_blocks;
                if (e < total) bt[at] = x.fresh;
            }
            __syncthreads();  // s_first is read
        }
        wait_vmem();
        __syncthreads();
    }
    if (tid == 0) *top = tp;
    if (err) raise_device_error(err);
}

// ---------------------------------------------------------------------------
// step_shared: paged_step's two passes with counts.  Freeing takes three rounds
// over the sequences (the counts, the places, the pushes).  Then each sequence
// finds whether its current token's block is missing, its own, or held by others
// too: of R holders, the k sequences of the batch that are about to write there
// are ranked by (position, index), and the one of rank i copies if i < R - 1, as
// if they went one after the other: the last one keeps the block when nobody
// else holds it.  It is the one furthest ahead, so what it writes lies behind
// every row that the others copy.
// ---------------------------------------------------------------------------
static __device__ __forceinline__ int64_t seq_position(const murmur_seg &s) {  // of the current token
    return (int64_t)s.prompt_pre + s.speech_len + s.prompt_mid + s.out_len - 1;
}

__global__ __launch_bounds__(256) void step_shared_kernel(const murmur_seg *__restrict__ seg,
                                                          const murmur_policy *__restrict__ pol, int32_t pol_per_seq,
                                                          int32_t B, int32_t *bt, int32_t max_blocks, int32_t log2_bs,
                                                          int32_t *ref, int32_t n_blocks, int32_t *stack, int32_t *top,
                                                          int32_t full_scan, int32_t *copied) {
    __shared__ int s_scan[4];
    __shared__ int2 s_writer[256];
    constexpr int32_t kTakeBlock = -3;
    const int tid = threadIdx.x;
    int32_t tp = *top;
    tp = tp < 0 ? 0 : (tp > n_blocks ? n_blocks : tp);
    int err = 0;
    // every entry of sequence b to give up, with its place
    const auto each_freed = [&](int b, int &e, auto f) {
        const PagedSeq q = paged_seq(seg, pol, pol_per_seq, b, B, max_blocks, log2_bs, full_scan, e);
        int32_t *row = bt + (int64_t)(q.valid ? b : 0) * max_blocks;
#pragma unroll
        for (int k = 0; k < 2; ++k)
            for (int32_t blk = q.lo[k]; blk < q.hi[k]; ++blk) {
                const int32_t phys = row[blk];
                if (phys >= 0) f(row + blk, phys, b * max_blocks + blk);
            }
    };
    // where a sequence writes its token: its position, that position's column and the block there
    struct Writer {
        bool valid;
        int32_t blk, x;
        int64_t pos;
    };
    const auto writer_of = [&](int b, int &e) {
        const PagedSeq q = paged_seq(seg, pol, pol_per_seq, b, B, max_blocks, log2_bs, 1, e);
        Writer w{q.valid, q.cur, -1, 0};
        if (q.valid) {
            w.pos = seq_position(seg[b]);
            if (q.cur < max_blocks) w.x = bt[(int64_t)b * max_blocks + q.cur];
        }
        return w;
    };
    int ignore = 0;
    for (int b = tid; b < B; b += 256)
        each_freed(b, err, [&](int32_t *, int32_t phys, int32_t) {
            if (phys < n_blocks) add_ref(ref + phys, -1);
            else err |= MURMUR_DEVERR_BLOCK;
        });
    wait_vmem();
    __syncthreads();
    for (int b = tid; b < B; b += 256)
        each_freed(b, ignore, [&](int32_t *, int32_t phys, int32_t at) {
            if (phys < n_blocks) offer_place(ref + phys, at);
        });
    wait_vmem();
    __syncthreads();
    for (int b0 = 0; b0 < B; b0 += 256) {
        int n = 0, pushed;
        each_freed(b0 + tid, ignore, [&](int32_t *, int32_t phys, int32_t at) {
            n += phys < n_blocks && load_shared_word(ref + phys) == place_key(at);
        });
        int to = tp + wg_exclusive_scan<256>(n, s_scan, tid, pushed);
        each_freed(b0 + tid, ignore, [&](int32_t *entry, int32_t phys, int32_t at) {
            if (phys < n_blocks && load_shared_word(ref + phys) == place_key(at)) {
                if (to < n_blocks) stack[to] = phys;
                else err |= MURMUR_DEVERR_POOL;
                ++to;
                store_shared_word(ref + phys, 0);
            }
            *entry = -1;
        });
        tp = tp + pushed < n_blocks ? tp + pushed : n_blocks;
    }
    wait_vmem();
    __syncthreads();
    // What each sequence needs, before any table entry or count changes: kTakeBlock, -1 for nothing, -2 if it is not
    // valid, else a copy of the block named.
    for (int b0 = 0; b0 < B; b0 += 256) {
        const Writer w = writer_of(b0 + tid, err);
        int32_t what = w.valid ? -1 : -2;
        int holders = 0;
        if (w.valid && w.blk >= max_blocks) {
            err |= MURMUR_DEVERR_BLOCK;
        } else if (w.valid && w.x < 0) {
            what = kTakeBlock;
        } else if (w.valid && w.x >= n_blocks) {
            err |= MURMUR_DEVERR_BLOCK;
        } else if (w.valid) {
            holders = load_shared_word(ref + w.x);
        }
        int before = 0;
        for (int o0 = 0; o0 < B; o0 += 256) {  // all sequences that write to a block, 256 at a time
            const Writer o = writer_of(o0 + tid, ignore);
            s_writer[tid] = o.valid && o.blk < max_blocks ? int2{o.x, (int)o.pos} : int2{-1, 0};
            __syncthreads();
            if (holders > 1)
                for (int i = 0; i < 256; ++i) {
                    const int2 y = s_writer[i];
                    before += y.x == w.x && (y.y >> log2_bs) == w.blk &&
                              (y.y < (int)w.pos || (y.y == (int)w.pos && o0 + i < b0 + tid));
                }
            __syncthreads();
        }
        if (holders > 1 && before < holders - 1) what = w.x;
        if (b0 + tid < B) copied[b0 + tid] = what;
    }
    __syncthreads();
    for (int b0 = 0; b0 < B; b0 += 256) {
        const int b = b0 + tid;
        const int32_t what = b < B ? copied[b] : -1;
        const bool need = what >= 0 || what == kTakeBlock;
        int taken;
        const int off = wg_exclusive_scan<256>(need, s_scan, tid, taken);
        if (need) {
            const int64_t blk = seq_position(seg[b]) >> log2_bs;
            const int from = tp - 1 - off;
            const int32_t got = from >= 0 ? stack[from] : -1;
            const bool good = got >= 0 && got < n_blocks;
            if (good) store_shared_word(ref + got, 1);
            else err |= MURMUR_DEVERR_POOL;
            if (what >= 0) add_ref(ref + what, -1);
            bt[(int64_t)b * max_blocks + blk] = good ? got : -1;
            copied[b] = good ? (what >= 0 ? what : -1) : -2;
        }
        tp = tp - taken > 0 ? tp - taken : 0;
    }
    if (tid == 0) *top = tp;
    if (err) raise_device_error(err);
}

// A workgroup per (sequence, layer, K or V): the rows of the current block before
// the token from the block it was copied from, then the token's own rows.
__global__ __launch_bounds__(256) void append_shared_kernel(const murmur_seg *__restrict__ seg, int32_t B,
                                                            const int32_t *__restrict__ bt, int32_t max_blocks,
                                                            int32_t log2_bs, const int32_t *__restrict__ copied,
                                                            uint16_t *k, uint16_t *v, int64_t s_layer, int64_t s_h,
                                                            int64_t s_pos, int64_t rows,
                                                            const uint16_t *__restrict__ k_new,
                                                            const uint16_t *__restrict__ v_new, int32_t NL,
                                                            int32_t Hkv) {
    const int b = blockIdx.x;
    const int64_t p = seq_position(seg[b]);
    const int64_t blk = p >> log2_bs;
    if (p < 0 || blk >= max_blocks) return;
    const int32_t phys = bt[(int64_t)b * max_blocks + blk], from = copied[b];
    if (phys < 0 || from < -1) return;
    const int32_t slot = (int32_t)(p & ((1 << log2_bs) - 1));
    const int64_t row0 = (int64_t)phys << log2_bs, src0 = (int64_t)from << log2_bs;
    if (row0 + slot >= rows || src0 + slot > rows) return;
    for (int64_t lv = blockIdx.y; lv < 2 * (int64_t)NL; lv += gridDim.y) {
        const int64_t layer = lv >> 1;
        uint16_t *base = ((lv & 1) ? v : k) + layer * s_layer;
        const uint16_t *fresh = ((lv & 1) ? v_new : k_new) + (layer * B + b) * Hkv * kHeadDim;
        if (from >= 0)
            for (int t = threadIdx.x; t < slot * Hkv * 16; t += 256) {
                const int c = t & 15, h = (t >> 4) % Hkv, j = (t >> 4) / Hkv;
                const int64_t at = h * s_h + j * s_pos + 8 * c;
                *reinterpret_cast<u32x4 *>(base + row0 * s_pos + at) = load16(base + src0 * s_pos + at);
            }
        for (int t = threadIdx.x; t < Hkv * 16; t += 256)
            *reinterpret_cast<u32x4 *>(base + (row0 + slot) * s_pos + (t >> 4) * s_h + 8 * (t & 15)) = load16(fresh + 8 * t);
    }
}

// ---------------------------------------------------------------------------
// compact.  n blocks are in use (count > 0): those at n and behind move, in
// ascending order, into the free ones before n, so no block is both read and
// written.  One workgroup ranks them with scans over the counts; then the chip copies the blocks and renames the table's entries.
// ---------------------------------------------------------------------------
constexpr int kCompactThreads = 1024;

__global__ __launch_bounds__(kCompactThreads) void compact_plan_kernel(int32_t *__restrict__ ref, int32_t n_blocks,
                                                                       int32_t *__restrict__ stack,
                                                                       int32_t *__restrict__ top, int32_t *map,
                                                                       int32_t *ws) {
    __shared__ int s_scan[kCompactThreads / 64];
    const int tid = threadIdx.x;
    int32_t *src = ws + kForkHeader, *dst = src + n_blocks / 2;
    int used = 0;
    for (int i0 = 0; i0 < n_blocks; i0 += kCompactThreads) {
        const int i = i0 + tid;
        int total;
        wg_exclusive_scan<kCompactThreads>(i < n_blocks && ref[i] > 0, s_scan, tid, total);
        used += total;
    }
    int moves = 0, holes = 0;
    for (int i0 = 0; i0 < n_blocks; i0 += kCompactThreads) {
        const int i = i0 + tid;
        const bool in = i < n_blocks, live = in && ref[i] > 0;
        const bool mover = live && i >= used, hole = in && !live && i < used;
        int nm, nh;
        const int am = moves + wg_exclusive_scan<kCompactThreads>(mover, s_scan, tid, nm);
        const int ah = holes + wg_exclusive_scan<kCompactThreads>(hole, s_scan, tid, nh);
        if (mover) src[am] = i;
        if (hole) dst[ah] = i;
        if (in) map[i] = live && !mover ? i : -1;
        moves += nm;
        holes += nh;
        if (in && i < n_blocks - used) stack[i] = n_blocks - 1 - i;
    }
    __syncthreads();
    for (int j = tid; j < moves; j += kCompactThreads) {
        const int32_t s = src[j], d = dst[j];
        map[s] = d;
        ref[d] = ref[s];
        ref[s] = 0;
    }
    if (tid == 0) {
        ws[1] = moves;  // ws[0] is the ticket of a fork
        *top = n_blocks - used;
    }
}

// Workgroups 0 .. gridDim.x - 1 of y = 0 rename the table, those of y > 0 copy: K and V of every (move, layer),
// each by one workgroup in 16-byte units.
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
    const int32_t *src = ws + kForkHeader, *dst = src + n_blocks / 2;
    const int64_t items = (int64_t)ws[1] * NL * 2;
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
                      int32_t n_blocks, int32_t *stack, int32_t *top, int32_t *ws, murmur_stream_t stream) {
    hipLaunchKernelGGL(fork_kernel, dim3((unsigned)B), dim3(kForkThreads), 0, (hipStream_t)stream, parent, B, bt,
                       max_blocks, ref, n_blocks, stack, top, ws);
    return (int)hipGetLastError();
}

int launch_paged_step_shared(const murmur_seg *seg, const murmur_policy *pol, int32_t pol_per_seq, int32_t B,
                             int32_t *bt, int32_t max_blocks, int32_t log2_bs, int32_t *ref, int32_t n_blocks,
                             int32_t *stack, int32_t *top, int32_t full_scan, int32_t *copied,
                             murmur_stream_t stream) {
    hipLaunchKernelGGL(step_shared_kernel, dim3(1), dim3(256), 0, (hipStream_t)stream, seg, pol, pol_per_seq, B, bt,
                       max_blocks, log2_bs, ref, n_blocks, stack, top, full_scan, copied);
    return (int)hipGetLastError();
}

int launch_paged_append_shared(const murmur_seg *seg, int32_t B, const int32_t *bt, int32_t max_blocks,
                               int32_t log2_bs, const int32_t *copied, const murmur_kv &pool, int32_t Hkv,
                               const void *k_new, const void *v_new, murmur_stream_t stream) {
    const unsigned y = (unsigned)(pool.n_layers < 32768 ? 2 * pool.n_layers : 65535);
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
