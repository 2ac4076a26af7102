// Device code of the attention over shared prefixes (included by kernels.hip):
//
//   shared_scan_kernel   where each list leaves the first one of its group
//   shared_plan_kernel   what the groups share, and the work of every workgroup
//   shared_attn_kernel   partial softmax sums of the prefixes and of the rests
//   shared_merge_kernel  their log-sum-exp join
//
// out = sum_i softmax_i(s q.K_i) V_i over a list R = P ++ T is
// (e^(mP-m) OP + e^(mT-m) OT) / (e^(mP-m) lP + e^(mT-m) lT), m = max(mP, mT), for
// the (max, sum, unscaled sum) of each part, so the part P that the sequences of
// a group have in common is read once for all of their query rows: a workgroup
// multiplies a pass of 32 positions with up to 64 rows (four MFMA row tiles) from
// the same K and V registers.  Bound: the K/V bytes, each distinct row once.
#pragma once

namespace murmur {

// ---------------------------------------------------------------------------
// The schedule
// ---------------------------------------------------------------------------
static __device__ __forceinline__ int list_count(const int32_t *ranges, const int32_t *count, int b) {
    if (!ranges) return count[b];
    int c = 0;
#pragma unroll
    for (int k = 0; k < kPieces; ++k) c += ranges[(int64_t)b * 2 * kPieces + 2 * k + 1];
    return c;
}

// Workgroup (x, b) compares entries [kScanLen x, kScanLen (x + 1)) of list b with
// those of the first list of its group: the first rank that differs, or max_keep.
constexpr int kScanThreads = 256;
__global__ __launch_bounds__(kScanThreads) void shared_scan_kernel(const int32_t *__restrict__ idx,
                                                                   const int32_t *__restrict__ count,
                                                                   const int32_t *__restrict__ group,
                                                                   int32_t n_groups, int32_t max_keep, int32_t B,
                                                                   int32_t *__restrict__ scan) {
    __shared__ int s_min;
    const int tid = threadIdx.x, b = blockIdx.y;
    int lead = -1;  // the last group start at or before b
    for (int g0 = 0; g0 < n_groups; g0 += kScanThreads) {
        const int32_t start = g0 + tid < n_groups ? group[g0 + tid] : 0x7fffffff;
        if (tid == 0) s_min = -1;
        __syncthreads();
        if (start >= 0 && start <= b) atomicMax(&s_min, start);
        __syncthreads();
        lead = s_min > lead ? s_min : lead;
        __syncthreads();
    }
    if (tid == 0) s_min = max_keep;
    __syncthreads();
    if (lead >= 0 && lead < b) {
        const int n = min(min(count[b], count[lead]), max_keep);
        const int32_t *mine = idx + (int64_t)b * max_keep, *first = idx + (int64_t)lead * max_keep;
        const int r0 = (int)blockIdx.x * kScanLen, r1 = min(r0 + kScanLen, n);
        int at = max_keep;
        for (int r = r0 + tid; r < r1; r += kScanThreads) at = mine[r] != first[r] ? min(at, r) : at;
        if (at < max_keep) atomicMin(&s_min, at);
    }
    __syncthreads();
    if (tid == 0) scan[(int64_t)b * gridDim.x + blockIdx.x] = s_min;
}

constexpr int kPlanThreads = 1024;

static __device__ __forceinline__ int tiles_of(int n_seq, int per_tile) { return (n_seq + per_tile - 1) / per_tile; }
static __device__ __forceinline__ int passes_of(int n) { return (n + kWaveTile - 1) / kWaveTile; }

// One workgroup.  Passes per wavefront (k) decide the cut: a prefix takes
// ceil(passes / 8k) workgroups per row tile and a rest ceil(passes / k)
// wavefronts.  The smallest k whose workgroups fit one dispatch round is taken,
// each of the sixteen wavefronts trying one.
__global__ __launch_bounds__(kPlanThreads) void shared_plan_kernel(const SharedPlanLaunch p) {
    __shared__ int s_scan[kPlanThreads / 64];
    __shared__ int s_wg[kSharedMaxPasses + 1];
    __shared__ int s_bad;
    static_assert(kSharedMaxPasses == kPlanThreads / 64, "a wavefront per candidate");
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int B = p.B, n_groups = p.n_groups, max_keep = p.max_keep;
    const int G = p.Hq / p.Hkv, per_tile = kSharedRows / G;
    PlanHeader *h = reinterpret_cast<PlanHeader *>(p.plan);
    PlanSeq *seqs = reinterpret_cast<PlanSeq *>(p.plan + sizeof(PlanHeader));
    PlanItem *items = reinterpret_cast<PlanItem *>(p.plan + p.caps.item_offset);
    PlanChunk *chunks = reinterpret_cast<PlanChunk *>(p.plan + p.caps.chunk_offset);
    const int32_t *scan = reinterpret_cast<const int32_t *>(p.plan + p.caps.scan_offset);
    const int n_scan = p.caps.n_scan;

    if (tid == 0) s_bad = 0;
    __syncthreads();
    for (int g = tid; g < n_groups; g += kPlanThreads) {
        const int lo = p.group[g], hi = p.group[g + 1];
        if (lo < 0 || lo > hi || hi > B || (g == 0 && lo != 0)) s_bad = 1;
    }
    for (int b = tid; b < B; b += kPlanThreads) seqs[b].state = 0;
    __syncthreads();
    if (tid == 0) {
        h->magic = kPlanMagic;
        h->bad = s_bad;
        h->B = B;
        h->max_keep = max_keep;
        h->n_layers = p.n_layers;
        h->Hq = p.Hq;
        h->Hkv = p.Hkv;
        h->n_groups = n_groups;
        if (s_bad) {
            h->n_items = h->n_rest = h->rows = 0;
            raise_device_error(MURMUR_DEVERR_GROUP);
        }
    }
    if (s_bad) return;

    // What each group shares: a wavefront per group, a lane per sequence.  rest_row
    // holds the rest's length and pre_stride the group's for the moment.
    int err = 0;
    for (int g = wave; g < n_groups; g += kPlanThreads / 64) {
        const int lo = p.group[g], hi = p.group[g + 1];
        int common = p.find ? max_keep : p.shared[g];
        if (p.find) {
            for (int b = lo + lane; b < hi; b += 64) {
                const int c = list_count(p.ranges, p.count, b);
                if (c < 1 || c > max_keep) {
                    if (b == lo) common = 0;
                    continue;
                }
                common = min(common, c);
                for (int x = 0; x < n_scan; ++x) common = min(common, scan[(int64_t)b * n_scan + x]);
            }
#pragma unroll
            for (int x = 32; x >= 1; x /= 2) common = min(common, __shfl_xor(common, x));
            if (lo == hi) common = 0;
            if (lane == 0) p.shared[g] = common;
        }
        // the first sequence's list is the one that is read, so it has to hold what is shared
        const int c_lead = lo < hi ? list_count(p.ranges, p.count, lo) : 0;
        const bool usable = common == 0 || (common > 0 && common <= c_lead && c_lead <= max_keep);
        for (int b = lo + lane; b < hi; b += 64) {
            const int c = list_count(p.ranges, p.count, b);
            const bool good = c >= 1 && c <= max_keep && usable && c >= common;
            if (!good) err |= MURMUR_DEVERR_COUNT;
            seqs[b].state = good ? 1 : 2;
            seqs[b].n_pre = usable ? common : 0;
            seqs[b].rest_row = good ? c - common : 0;
        }
    }
    if (err) raise_device_error(err);
    __syncthreads();

    {
        const int k = wave + 1;
        int wg = 0, waves = 0;
        for (int g = lane; g < n_groups; g += 64) {
            const int lo = p.group[g], hi = p.group[g + 1];
            const int pre = lo < hi ? passes_of(seqs[lo].n_pre) : 0;
            wg += tiles_of(hi - lo, per_tile) * ((pre + kSharedWaves * k - 1) / (kSharedWaves * k));
        }
        for (int b = lane; b < B; b += 64)
            if (seqs[b].state == 1) waves += (passes_of(seqs[b].rest_row) + k - 1) / k;
#pragma unroll
        for (int x = 32; x >= 1; x /= 2) {
            wg += __shfl_xor(wg, x);
            waves += __shfl_xor(waves, x);
        }
        if (lane == 0) s_wg[k] = wg + (waves + kSharedWaves - 1) / kSharedWaves;
    }
    __syncthreads();
    int k = 1;
    while (k < kSharedMaxPasses && s_wg[k] > p.caps.per_round) ++k;

    // Prefix work: the groups' items one after the other, the row tiles of one stretch side by side.
    int items_done = 0, rows_done = 0;
    for (int g0 = 0; g0 < n_groups; g0 += kPlanThreads) {
        const int g = g0 + tid;
        const int lo = g < n_groups ? p.group[g] : 0, hi = g < n_groups ? p.group[g + 1] : 0;
        const int n_seq = hi - lo, common = n_seq > 0 ? seqs[lo].n_pre : 0, pre = passes_of(common);
        const int tiles = tiles_of(n_seq, per_tile), cuts = (pre + kSharedWaves * k - 1) / (kSharedWaves * k);
        int total, total_rows;
        const int at = items_done + wg_exclusive_scan<kPlanThreads>(tiles * cuts, s_scan, tid, total);
        const int row = rows_done + wg_exclusive_scan<kPlanThreads>(cuts * n_seq * G, s_scan, tid, total_rows);
        for (int i = 0; i < cuts; ++i) {
            const int r0 = (int)((int64_t)pre * i / cuts) * kWaveTile;
            const int r1 = min((int)((int64_t)pre * (i + 1) / cuts) * kWaveTile, common);
            for (int t = 0; t < tiles; ++t) {
                const int s0 = t * per_tile;
                items[at + i * tiles + t] = PlanItem{lo + s0, min(per_tile, n_seq - s0), lo, r0, r1,
                                                     row + (i * n_seq + s0) * G, {0, 0}};
            }
        }
        for (int b = lo; b < hi; ++b) {
            seqs[b].pre_row = row + (b - lo) * G;
            seqs[b].pre_stride = n_seq * G;
            seqs[b].n_pre = cuts;
            seqs[b].common = common;
        }
        items_done += total;
        rows_done += total_rows;
    }
    __syncthreads();
    // The rests: a wavefront's chunk each, the sequences one after the other; a
    // workgroup's chunks of one sequence end in one partial.
    int chunks_done = 0;
    for (int b0 = 0; b0 < B; b0 += kPlanThreads) {
        const int b = b0 + tid;
        const bool on = b < B && seqs[b].state == 1;
        const int rest = on ? seqs[b].rest_row : 0, common = on ? seqs[b].common : 0, pre = passes_of(rest);
        const int n = (pre + k - 1) / k;
        int total;
        const int at = chunks_done + wg_exclusive_scan<kPlanThreads>(n, s_scan, tid, total);
        const int parts = n > 0 ? (at + n - 1) / kSharedWaves - at / kSharedWaves + 1 : 0;
        int total_rows;
        const int row = rows_done + wg_exclusive_scan<kPlanThreads>(parts * G, s_scan, tid, total_rows);
        for (int i = 0; i < n; ++i) {
            const int r0 = (int)((int64_t)pre * i / n) * kWaveTile;
            const int r1 = min((int)((int64_t)pre * (i + 1) / n) * kWaveTile, rest);
            chunks[at + i] = PlanChunk{b, common + r0, common + r1,
                                       row + ((at + i) / kSharedWaves - at / kSharedWaves) * G};
        }
        if (on) {
            seqs[b].rest_row = row;
            seqs[b].n_rest = parts;
            seqs[b].first_chunk = at;
        }
        chunks_done += total;
        rows_done += total_rows;
    }
    const int rest_wg = (chunks_done + kSharedWaves - 1) / kSharedWaves;
    for (int c = chunks_done + tid; c < rest_wg * kSharedWaves; c += kPlanThreads) chunks[c] = PlanChunk{-1, 0, 0, 0};
    if (tid == 0) {
        h->n_items = items_done;
        h->n_rest = rest_wg;
        h->rows = rows_done;
        h->passes = k;
    }
}

// ---------------------------------------------------------------------------
// The passes of one wavefront.  K and V have a tile each in its LDS stage.  Once
// a pass's K operands are in registers the next pass's K rows start into their
// tile, and V likewise, so 8 KiB at least are on their way at any time; the waits
// count the loads issued after the ones awaited (loads complete in order).
// ---------------------------------------------------------------------------
template <int kAux>
static __device__ __forceinline__ void dma_rows(uint8_t *tile, const uint16_t *base, int64_t s_pos,
                                                const int32_t (&pos)[8], int lane) {
    const int q = lane >> 4, sl = lane & 15;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int c = sl ^ ((4 * j + q) & 15);
        __builtin_amdgcn_global_load_lds(base + (int64_t)pos[j] * s_pos + 8 * c, (lds_void_t *)(tile + j * 1024), 16,
                                         0, kAux);
    }
}

static __device__ __forceinline__ void read_k_operands(u32x4 (&kf)[8], uint32_t kt, int n16, int c4) {
    uint32_t ka[4];
#pragma unroll
    for (int kc = 0; kc < 4; ++kc) ka[kc] = kt + n16 * kTileRowBytes + (((4 * kc + c4) ^ n16) << 4);
    asm volatile(
        "ds_read_b128 %0, %8\n\t"
        "ds_read_b128 %1, %9\n\t"
        "ds_read_b128 %2, %10\n\t"
        "ds_read_b128 %3, %11\n\t"
        "ds_read_b128 %4, %8 offset:4096\n\t"
        "ds_read_b128 %5, %9 offset:4096\n\t"
        "ds_read_b128 %6, %10 offset:4096\n\t"
        "ds_read_b128 %7, %11 offset:4096\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(kf[0]), "=&v"(kf[1]), "=&v"(kf[2]), "=&v"(kf[3]), "=&v"(kf[4]), "=&v"(kf[5]), "=&v"(kf[6]),
          "=&v"(kf[7])
        : "v"(ka[0]), "v"(ka[1]), "v"(ka[2]), "v"(ka[3])
        : "memory");
}

static __device__ __forceinline__ void read_v_operands(u32x2 (&vf)[16], uint32_t vt, int n16, int c4) {
    const int vr = 4 * c4 + (n16 >> 2);
    uint32_t va[8];
#pragma unroll
    for (int db = 0; db < 8; ++db)
        va[db] = vt + vr * kTileRowBytes + (((2 * db + ((n16 & 3) >> 1)) ^ vr) << 4) + (n16 & 1) * 8;
    asm volatile(
        "ds_read_b64_tr_b16 %0, %16\n\t"
        "ds_read_b64_tr_b16 %1, %16 offset:4096\n\t"
        "ds_read_b64_tr_b16 %2, %17\n\t"
        "ds_read_b64_tr_b16 %3, %17 offset:4096\n\t"
        "ds_read_b64_tr_b16 %4, %18\n\t"
        "ds_read_b64_tr_b16 %5, %18 offset:4096\n\t"
        "ds_read_b64_tr_b16 %6, %19\n\t"
        "ds_read_b64_tr_b16 %7, %19 offset:4096\n\t"
        "ds_read_b64_tr_b16 %8, %20\n\t"
        "ds_read_b64_tr_b16 %9, %20 offset:4096\n\t"
        "ds_read_b64_tr_b16 %10, %21\n\t"
        "ds_read_b64_tr_b16 %11, %21 offset:4096\n\t"
        "ds_read_b64_tr_b16 %12, %22\n\t"
        "ds_read_b64_tr_b16 %13, %22 offset:4096\n\t"
        "ds_read_b64_tr_b16 %14, %23\n\t"
        "ds_read_b64_tr_b16 %15, %23 offset:4096\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(vf[0]), "=&v"(vf[1]), "=&v"(vf[2]), "=&v"(vf[3]), "=&v"(vf[4]), "=&v"(vf[5]), "=&v"(vf[6]),
          "=&v"(vf[7]), "=&v"(vf[8]), "=&v"(vf[9]), "=&v"(vf[10]), "=&v"(vf[11]), "=&v"(vf[12]), "=&v"(vf[13]),
          "=&v"(vf[14]), "=&v"(vf[15])
        : "v"(va[0]), "v"(va[1]), "v"(va[2]), "v"(va[3]), "v"(va[4]), "v"(va[5]), "v"(va[6]), "v"(va[7])
        : "memory");
}

// Query rows of an item in LDS, laid out as a K tile (16-byte chunk c of row r at
// slot c ^ (r & 15)): B operands of row tile t.
static __device__ __forceinline__ void read_q_operands(u32x4 (&qf)[4], uint32_t qt, int t, int n16, int c4) {
    const uint32_t row = qt + (16 * t + n16) * kTileRowBytes;
    uint32_t qa[4];
#pragma unroll
    for (int kc = 0; kc < 4; ++kc) qa[kc] = row + (((4 * kc + c4) ^ n16) << 4);
    asm volatile(
        "ds_read_b128 %0, %4\n\t"
        "ds_read_b128 %1, %5\n\t"
        "ds_read_b128 %2, %6\n\t"
        "ds_read_b128 %3, %7\n\t"
        "s_waitcnt lgkmcnt(0)"
        : "=&v"(qf[0]), "=&v"(qf[1]), "=&v"(qf[2]), "=&v"(qf[3])
        : "v"(qa[0]), "v"(qa[1]), "v"(qa[2]), "v"(qa[3])
        : "memory");
}

// What a wavefront reads from: the list or range table of one sequence, and the
// K/V of one (layer, KV head) of it.
struct Rows {
    RangeTab tab;
    __amdgpu_buffer_rsrc_t list;
    const uint16_t *k, *v;
    int64_t s_pos;
    int max_len;
};

// Ranks r, r + step, ... below r_end, 32 at a time, against kTiles row tiles whose
// queries are in LDS (kQLds) or, one tile, in registers.
template <int kSrc, int kTiles, bool kQLds>
static __device__ __forceinline__ void run_passes(const Rows &in, int r, int r_end, int step, uint8_t *stage,
                                                  uint8_t (*slots)[kIdxSlotBytes], uint32_t q_lds, const u32x4 (&qreg)[4],
                                                  float scale, WaveAcc (&w)[kTiles], int lane) {
    static_assert(kQLds || kTiles == 1, "one row tile's queries fit registers");
    if (r >= r_end) return;
    const int n16 = lane & 15, c4 = lane >> 4;
    const uint32_t kt = lds_addr(stage), vt = kt + kTileBytes;
    int32_t pos[8];
    int bad = 0;
    const auto positions = [&](int r0, int slot) {
        if (kSrc == kSrcIndex) dma_pos_index(slots[slot], r0, r_end, in.max_len, c4, pos, bad);
        else dma_pos_ranges(in.tab, r0, r_end, in.max_len, c4, pos, bad);
    };
    if (kSrc == kSrcIndex) {
        dma_idx(slots[0], in.list, r, lane);
        dma_idx(slots[1], in.list, r + step, lane);
        wait_vm<1>();
    }
    positions(r, 0);
    dma_rows<0>(stage, in.k, in.s_pos, pos, lane);
    dma_rows<0>(stage + kTileBytes, in.v, in.s_pos, pos, lane);
    for (int it = 0;; r += step, ++it) {
        const bool more = r + step < r_end;
        const int valid = min(kWaveTile, r_end - r);
        u32x4 kf[8];
        wait_vm<8>();  // this pass's K rows; its V rows came after them
        read_k_operands(kf, kt, n16, c4);
        if (more) {
            positions(r + step, (it + 1) & 1);  // entries that were loaded before this pass's K rows
            if (kSrc == kSrcIndex) dma_idx(slots[it & 1], in.list, r + 2 * step, lane);
            dma_rows<0>(stage, in.k, in.s_pos, pos, lane);
        }
        u32x4 p_hi[kTiles], p_lo[kTiles];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            u32x4 qf[4];
            if (kQLds) {
                read_q_operands(qf, q_lds, t, n16, c4);
            } else {
#pragma unroll
                for (int kc = 0; kc < 4; ++kc) qf[kc] = qreg[kc];
            }
            f32x4 s[2];
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                s[blk] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kc = 0; kc < 4; ++kc) s[blk] = mfma16x16x32(kf[4 * blk + kc], qf[kc], s[blk]);
            }
            softmax_step<true>(s, valid, scale, w[t], c4, p_hi[t], p_lo[t]);
        }
        u32x2 vf[16];
        if (more) wait_vm<8>();  // this pass's V rows; the next pass's K rows came after them
        else wait_vm<0>();
        read_v_operands(vf, vt, n16, c4);
        if (more) dma_rows<0>(stage + kTileBytes, in.v, in.s_pos, pos, lane);
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            const u32x4 av = u32x4{vf[2 * db][0], vf[2 * db][1], vf[2 * db + 1][0], vf[2 * db + 1][1]};
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                w[t].acc[db] = mfma16x16x32(av, p_hi[t], w[t].acc[db]);
                w[t].acc[db] = mfma16x16x32(av, p_lo[t], w[t].acc[db]);
            }
        }
        if (!more) break;
    }
    w[0].bad_pos |= bad;
}

// ---------------------------------------------------------------------------
// Workgroup (layer and KV head, i): item i, or the chunks of workgroup
// i - n_items.  An item's eight wavefronts share its rows and take its passes in
// turn; a chunk's wavefront works on a sequence of its own.
// ---------------------------------------------------------------------------
struct SharedLds {
    uint8_t stages[kSharedWaves][kStageBytes];
    uint8_t slots[kSharedWaves][2][kIdxSlotBytes];
    uint8_t q[kSharedRows * kTileRowBytes];
    CombineLdsT<kSharedWaves> cl;
    int flag[kSharedWaves];
    int seq[kSharedWaves + 1], row[kSharedWaves];
};

template <int kSrc>
static __device__ __forceinline__ Rows rows_of(const SharedAttnLaunch &a, int list, int layer, int g) {
    Rows in;
    if (kSrc == kSrcIndex) {
        in.list = raw_buffer(a.idx + (int64_t)list * a.max_keep, (uint32_t)a.max_keep * 4u);
    } else {
        int32_t rg[2 * kPieces];
#pragma unroll
        for (int k = 0; k < 2 * kPieces; ++k) rg[k] = a.ranges[(int64_t)list * 2 * kPieces + k];
        in.tab = make_tab(rg);
    }
    const int64_t off = layer * a.s_layer + list * a.s_b + g * a.s_h;
    in.k = a.k + off;
    in.v = a.v + off;
    in.s_pos = a.s_pos;
    in.max_len = a.max_len;
    return in;
}

// The state of head h, head dims d0 .. d0+3 over wavefronts [w0, w1) of the
// workgroup into partial row `row` of this (layer, KV head).
static __device__ __forceinline__ void store_partial(const SharedLds &l, float *part_o, float *part_ml, int w0, int w1,
                                                     int h, int d0, int64_t row, bool bad) {
    const float *o = reinterpret_cast<const float *>(&l.stages[0][0]);
    float M = kNegInf, L = 0.f;
    for (int w = w0; w < w1; ++w) M = fmaxf(M, l.cl.ml[h][w][0]);
    f32x4 O = {0.f, 0.f, 0.f, 0.f};
    for (int w = w0; w < w1; ++w) {
        const float m = l.cl.ml[h][w][0];
        const float f = m == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m - M);
        L += l.cl.ml[h][w][1] * f;
        O += f * *reinterpret_cast<const f32x4 *>(&o[w * (kStageBytes / 4) + h * kOStride + d0]);
    }
    if (bad) L = __builtin_nanf("");
    *reinterpret_cast<f32x4 *>(part_o + row * kHeadDim + d0) = O;
    if (d0 == 0) {
        part_ml[2 * row] = M;
        part_ml[2 * row + 1] = L;
    }
}

template <int kSrc, int kTiles>
static __device__ __forceinline__ void item_work(const SharedAttnLaunch &a, const PlanItem &it, SharedLds &l, int layer,
                                                 int g, float *part_o, float *part_ml, int tid) {
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, c4 = lane >> 4;
    const int rows = it.n_seq * a.G;
    // the queries, past the last row its copies (their results are not stored)
    for (int t = tid; t < kTiles * 16 * 16; t += kSharedWaves * 64) {
        const int r = t >> 4, c = t & 15, rr = min(r, rows - 1);
        const int s = rr / a.G, hh = rr - s * a.G;
        u32x4 x = load16(a.q + (((int64_t)layer * a.B + it.seq0 + s) * a.Hq + g * a.G + hh) * kHeadDim + 8 * c);
        const uint32_t bits = __builtin_bit_cast(uint32_t, a.scale_log2);
        if ((int32_t)bits <= 0) x = (bits & 0x7fffffffu) ? x ^ 0x80008000u : u32x4{0u, 0u, 0u, 0u};
        *reinterpret_cast<u32x4 *>(&l.q[r * kTileRowBytes + ((c ^ (r & 15)) << 4)]) = x;
    }
    __syncthreads();
    const uint32_t mag = __builtin_bit_cast(uint32_t, a.scale_log2) & 0x7fffffffu;
    const float scale = __builtin_bit_cast(float, mag ? mag : 0x3f800000u);
    WaveAcc w[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) wave_acc_reset(w[t]);
    const Rows in = rows_of<kSrc>(a, it.list, layer, g);
    const u32x4 none[4] = {};
    run_passes<kSrc, kTiles, true>(in, it.r0 + wave * kWaveTile, it.r1, kSharedWaves * kWaveTile, l.stages[wave],
                                   l.slots[wave], lds_addr(l.q), none, scale, w, lane);
    float *o_w = reinterpret_cast<float *>(&l.stages[wave][0]);
    int bad = 0;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        if (t > 0) __syncthreads();  // the rows of the tile before are stored
        w[t].m_run *= scale;
        publish_wave(w[t], o_w, l.cl, wave, n16, c4);
        if (t == 0) bad = barrier_or<kSharedWaves>(w[0].bad_pos, l.flag, wave, lane);
        else __syncthreads();
        const int h = tid >> 5, d0 = (tid & 31) * 4;
        if (16 * t + h < rows) store_partial(l, part_o, part_ml, 0, kSharedWaves, h, d0, it.row + 16 * t + h, bad);
    }
    if (bad && tid == 0) raise_device_error(MURMUR_DEVERR_POSITION);
}

template <int kSrc>
static __device__ __forceinline__ void chunk_work(const SharedAttnLaunch &a, const PlanChunk &c, SharedLds &l, int layer,
                                                  int g, float *part_o, float *part_ml, int tid) {
    const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n16 = lane & 15, c4 = lane >> 4;
    WaveAcc w[1];
    wave_acc_reset(w[0]);
    float scale = 1.f;
    if (c.seq >= 0) {
        u32x4 qf[4];
        load_q(qf, a.q, ((int64_t)layer * a.B + c.seq) * a.Hq + g * a.G, a.G, n16, c4);
        scale = signed_scale(qf, a.scale_log2);
        const Rows in = rows_of<kSrc>(a, c.seq, layer, g);
        run_passes<kSrc, 1, false>(in, c.r0, c.r1, kWaveTile, l.stages[wave], l.slots[wave], 0u, qf, scale, w, lane);
    }
    w[0].m_run *= scale;
    publish_wave(w[0], reinterpret_cast<float *>(&l.stages[wave][0]), l.cl, wave, n16, c4);
    const int any_bad = __ballot(w[0].bad_pos != 0) != 0;
    if (lane == 0) {
        l.seq[wave] = c.seq;
        l.row[wave] = c.row;
        l.flag[wave] = any_bad;
    }
    if (tid == 0) l.seq[kSharedWaves] = -2;
    __syncthreads();
    // consecutive wavefronts of one sequence are one partial
    for (int t = tid; t < kSharedWaves * a.G * (kHeadDim / 4); t += kSharedWaves * 64) {
        const int row = t / (kHeadDim / 4), d0 = (t % (kHeadDim / 4)) * 4;
        const int w0 = row / a.G, h = row - w0 * a.G, s = l.seq[w0];
        if (s < 0 || (w0 > 0 && l.seq[w0 - 1] == s)) continue;
        int w1 = w0, bad = 0;
        do bad |= l.flag[w1];
        while (l.seq[++w1] == s);
        store_partial(l, part_o, part_ml, w0, w1, h, d0, l.row[w0] + h, bad);
        if (bad && h == 0 && d0 == 0) raise_device_error(MURMUR_DEVERR_POSITION);
    }
}

// Whether a plan was made for a call of these sizes.
static __device__ __forceinline__ bool plan_fits(const SharedAttnLaunch &a, const PlanHeader &h) {
    return h.magic == kPlanMagic && !h.bad && h.B == a.B && h.max_keep == a.max_keep && h.n_layers == a.NL &&
           h.Hq == a.Hq && h.Hkv == a.Hkv && h.n_groups == a.n_groups && h.rows <= a.rows_cap;
}

template <int kSrc>
__global__ __launch_bounds__(kSharedWaves * 64, 2) void shared_attn_kernel(const SharedAttnLaunch a) {
    __shared__ __attribute__((aligned(16))) SharedLds l;
    const int tid = threadIdx.x;
    const PlanHeader h = *reinterpret_cast<const PlanHeader *>(a.plan);
    if (!plan_fits(a, h)) return;
    const int i = blockIdx.y;
    if (i >= h.n_items + h.n_rest) return;
    const int layer = (int)blockIdx.x / a.Hkv, g = (int)blockIdx.x - layer * a.Hkv;
    float *part_o = a.part_o + (int64_t)blockIdx.x * h.rows * kHeadDim;
    float *part_ml = a.part_ml + (int64_t)blockIdx.x * h.rows * 2;
    if (i < h.n_items) {
        const PlanItem it = reinterpret_cast<const PlanItem *>(a.plan + a.item_offset)[i];
        switch ((it.n_seq * a.G + 15) / 16) {
        case 1: item_work<kSrc, 1>(a, it, l, layer, g, part_o, part_ml, tid); break;
        case 2: item_work<kSrc, 2>(a, it, l, layer, g, part_o, part_ml, tid); break;
        case 3: item_work<kSrc, 3>(a, it, l, layer, g, part_o, part_ml, tid); break;
        default: item_work<kSrc, 4>(a, it, l, layer, g, part_o, part_ml, tid); break;
        }
        return;
    }
    const int c = (i - h.n_items) * kSharedWaves + __builtin_amdgcn_readfirstlane(tid >> 6);
    const PlanChunk ch = reinterpret_cast<const PlanChunk *>(a.plan + a.chunk_offset)[c];
    chunk_work<kSrc>(a, ch, l, layer, g, part_o, part_ml, tid);
}

// Half a wavefront per query row: the pairs of up to 32 partials at a time, one
// per lane, then the partials' rows weighted, four head dims per lane.
__global__ __launch_bounds__(256) void shared_merge_kernel(const SharedAttnLaunch a) {
    const PlanHeader h = *reinterpret_cast<const PlanHeader *>(a.plan);
    const int64_t row = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int64_t n_rows = (int64_t)a.NL * a.B * a.Hq;
    if (row >= n_rows) return;
    const int lane = threadIdx.x & 31, d0 = lane * 4;
    const bool fits = plan_fits(a, h);
    const int64_t lb = row / a.Hq;
    const int hq = (int)(row - lb * a.Hq), layer = (int)(lb / a.B), b = (int)(lb - (int64_t)layer * a.B);
    const int g = hq / a.G, hh = hq - g * a.G;
    PlanSeq s{2, 0, 0, 0, 0, 0, 0, 0};
    if (fits) s = reinterpret_cast<const PlanSeq *>(a.plan + sizeof(PlanHeader))[b];
    else if (row == 0 && lane == 0) raise_device_error(MURMUR_DEVERR_GROUP);
    if (s.state == 0) return;
    float M = kNegInf, L = s.state == 1 ? 0.f : __builtin_nanf("");
    f32x4 O = {0.f, 0.f, 0.f, 0.f};
    const int n = s.state == 1 ? s.n_pre + s.n_rest : 0;
    const int64_t base = ((int64_t)layer * a.Hkv + g) * h.rows;
    const auto row_of = [&](int i) {
        return base + hh + (i < s.n_pre ? s.pre_row + i * s.pre_stride : s.rest_row + (i - s.n_pre) * a.G);
    };
    for (int i0 = 0; i0 < n; i0 += 32) {
        float m = kNegInf, sum = 0.f;
        if (i0 + lane < n) {
            const int64_t r = row_of(i0 + lane);
            m = a.part_ml[2 * r];
            sum = a.part_ml[2 * r + 1];
        }
        float top = m;
#pragma unroll
        for (int x = 16; x >= 1; x /= 2) top = fmaxf(top, __shfl_xor(top, x, 32));
        top = fmaxf(top, M);
        const float before = M == kNegInf ? 0.f : __builtin_amdgcn_exp2f(M - top);
        const float weight = m == kNegInf && sum == 0.f ? 0.f : __builtin_amdgcn_exp2f(m - top);
        float total = sum * weight;
#pragma unroll
        for (int x = 16; x >= 1; x /= 2) total += __shfl_xor(total, x, 32);
        L = L * before + total;
        O *= before;
        M = top;
        const int here = min(32, n - i0);
        for (int i = 0; i < here; ++i) {
            const f32x4 o = *reinterpret_cast<const f32x4 *>(a.part_o + row_of(i0 + i) * kHeadDim + d0);
            O += o * __shfl(weight, i, 32);
        }
    }
    const float inv = 1.f / L;
    if (a.out_f32)
        *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.out) + row * kHeadDim + d0) = O * inv;
    else
        *reinterpret_cast<u32x2 *>(reinterpret_cast<uint16_t *>(a.out) + row * kHeadDim + d0) =
            u32x2{pack_bf16(O[0] * inv, O[1] * inv), pack_bf16(O[2] * inv, O[3] * inv)};
    if (lane == 0 && a.lse) a.lse[row] = (M + __builtin_log2f(L)) * 0.69314718055994530942f;
}

// ---- launchers ----

int launch_shared_plan(const SharedPlanLaunch &p, murmur_stream_t stream) {
    if (p.find) {
        hipLaunchKernelGGL(shared_scan_kernel, dim3((unsigned)p.caps.n_scan, (unsigned)p.B), dim3(kScanThreads), 0,
                           (hipStream_t)stream, p.idx, p.count, p.group, p.n_groups, p.max_keep, p.B,
                           reinterpret_cast<int32_t *>(p.plan + p.caps.scan_offset));
        const int e = (int)hipGetLastError();
        if (e != 0) return e;
    }
    hipLaunchKernelGGL(shared_plan_kernel, dim3(1), dim3(kPlanThreads), 0, (hipStream_t)stream, p);
    return (int)hipGetLastError();
}

int launch_decode_attn_shared(const SharedAttnLaunch &a, murmur_stream_t stream) {
    const dim3 grid((unsigned)(a.NL * a.Hkv), (unsigned)a.n_wg);
    if (a.ranges)
        hipLaunchKernelGGL(shared_attn_kernel<kSrcRanges>, grid, dim3(kSharedWaves * 64), 0, (hipStream_t)stream, a);
    else
        hipLaunchKernelGGL(shared_attn_kernel<kSrcIndex>, grid, dim3(kSharedWaves * 64), 0, (hipStream_t)stream, a);
    const int e = (int)hipGetLastError();
    if (e != 0) return e;
    const int64_t rows = (int64_t)a.NL * a.B * a.Hq;
    hipLaunchKernelGGL(shared_merge_kernel, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}

}  // namespace murmur
