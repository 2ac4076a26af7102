// Device code of the attention over shared prefixes (included by kernels.hip):
//
//   shared_scan_kernel   where each list leaves the first one of its group
//   shared_plan_kernel   what the groups share, and the work of every workgroup
//   shared_whole_kernel  the attention, each list left whole; or
//   shared_attn_kernel   partial softmax sums of the prefixes and of the rests
//   shared_merge_kernel  and their log-sum-exp join
//
// out = sum_i softmax_i(s q.K_i) V_i over a list R = P ++ T is
// (e^(mP-m) OP + e^(mT-m) OT) / (e^(mP-m) lP + e^(mT-m) lT), m = max(mP, mT), for
// the (max, sum, unscaled sum) of each part, so the part P that the sequences of
// a group have in common is read once for all of their query rows: a workgroup
// multiplies each pass of 32 positions with up to 48 rows (three MFMA row tiles).
// Bound: the K/V bytes, each distinct row once.
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
// those of the first list of its group that is there: the first rank that differs, or
// max_keep.  Three round trips: the groups, the counts, the entries (16 a thread at
// once); two more where the group's first sequence is not there.
constexpr int kScanThreads = 256;
constexpr int kScanEach = kScanLen / kScanThreads;
__global__ __launch_bounds__(kScanThreads) void shared_scan_kernel(const int32_t *__restrict__ idx,
                                                                   const int32_t *__restrict__ count,
                                                                   const int32_t *__restrict__ group,
                                                                   int32_t n_groups, int32_t max_keep, int32_t B,
                                                                   int32_t *__restrict__ scan) {
    __shared__ int s_lead, s_min, s_first;
    const int tid = threadIdx.x, b = blockIdx.y;
    if (tid == 0) {
        s_lead = -1;
        s_min = max_keep;
        s_first = b;
    }
    __syncthreads();
    int start = -1;  // the last group start at or before b
    for (int g = tid; g < n_groups; g += kScanThreads) {
        const int32_t at = group[g];
        start = at <= b && at > start ? at : start;
    }
    if (start >= 0) atomicMax(&s_lead, start);
    __syncthreads();
    const int lead = s_lead;
    if (lead >= 0 && lead < b) {
        int n = min(min(count[b], count[lead]), max_keep);
        const int32_t *mine = idx + (int64_t)b * max_keep, *first = idx + (int64_t)lead * max_keep;
        const int r0 = (int)blockIdx.x * kScanLen + tid, last = max_keep - 1;
        int32_t x[kScanEach], y[kScanEach];
#pragma unroll
        for (int j = 0; j < kScanEach; ++j) {
            const int r = min(r0 + j * kScanThreads, last);
            x[j] = mine[r];
            y[j] = first[r];
        }
        if (__builtin_expect(count[lead] == kAbsent, 0)) {  // uniform
            for (int i = lead + 1 + tid; i < b; i += kScanThreads)
                if (count[i] != kAbsent) {
                    atomicMin(&s_first, i);
                    break;
                }
            __syncthreads();
            n = min(min(count[b], count[s_first]), max_keep);  // itself, if none before it is there: nothing differs
            first = idx + (int64_t)s_first * max_keep;
#pragma unroll
            for (int j = 0; j < kScanEach; ++j) y[j] = first[min(r0 + j * kScanThreads, last)];
        }
        int at = max_keep;
#pragma unroll
        for (int j = kScanEach - 1; j >= 0; --j) {
            const int r = r0 + j * kScanThreads;
            at = r < n && x[j] != y[j] ? r : at;
        }
        if (at < max_keep) atomicMin(&s_min, at);
    }
    __syncthreads();
    if (tid == 0) scan[(int64_t)b * gridDim.x + blockIdx.x] = s_min;
}

static __device__ __forceinline__ int div_up(int x, int y) { return (x + y - 1) / y; }

// x / y for 0 <= x < 2^22 and y >= 1: the estimate is off by one at most.
static __device__ __forceinline__ int small_div(int x, int y) {
    int q = (int)((float)x * __builtin_amdgcn_rcpf((float)y));
    const int r = x - q * y;
    q += r >= y ? 1 : 0;
    return r < 0 ? q - 1 : q;
}
static __device__ __forceinline__ int small_div_up(int x, int y) { return small_div(x + y - 1, y); }
// n things dealt to `parts` parts in runs: the first of part i.
struct Dealt {
    int per, more;
    __device__ __forceinline__ Dealt(int n, int parts) : per((int)((unsigned)n / (unsigned)parts)), more(n - per * parts) {}
    __device__ __forceinline__ int start(int i) const { return per * i + min(i, more); }
};

// SharedPlanLaunch::find where the planner compares the lists itself: few entries, a
// load or two of a thread, are cheaper than another launch (4 lists of 192: 15.0 us for
// plan and attention, 17.6 with it).
constexpr int kFindHere = 2;
constexpr int kFindHereEntries = 4096;

// One workgroup; what it needs of every sequence and group is in LDS, so that the
// global round trips are the counts with the groups, the scans, and the stores.  It
// runs each line once, on code that no cache holds yet, so what bounds it is the
// size of the code (loops are not unrolled, divisions are by reciprocal, sums over
// lanes go by DPP): 5.6 us for 4 sequences, 7.0 for 96 in whole lists, 8.3 to 11.5 with
// cuts.
// The lowest level of cut whose workgroups fit one dispatch round is taken, or the
// highest; the wavefronts add up eight levels side by side, then the eight between
// two of them.
struct PlanLds {
    int rest[kSharedMaxSeqs];           // by sequence: length of the rest, or one of the two below
    uint16_t of[kSharedMaxSeqs];        // its group
    int lo[kSharedMaxSeqs + 1];         // by group: first sequence
    int lead[kSharedMaxSeqs];           // the first one that is there, whose list is read (the next group's first: none)
    int common[kSharedMaxSeqs];         // what it shares
    int row[kSharedMaxSeqs], item[kSharedMaxSeqs];  // its first partial row and item
    int cuts[kSharedMaxSeqs];
    int scan[16], work[2][8], bad, found;
    unsigned positions;
};
constexpr int kInvalid = -1, kNotThere = -2;  // PlanLds::rest: the count is invalid; kAbsent
static __device__ __forceinline__ int32_t seq_state(int rest) { return rest >= 0 ? 1 : (rest == kInvalid ? 2 : 0); }

// Workgroups that read the same rows should share an L2.  Workgroup w of a launch runs
// on XCD w mod 8, and the (layer, KV head) is the fastest index of the grid, so with
// `heads` of them item i of a head runs on one of 8 / gcd(8, heads) XCDs in turn.  Item
// number q of n, in an order with neighbours that share rows, goes to the place that
// gives every such XCD a run of neighbours (a bijection of [0, n)).
static __device__ __forceinline__ int item_place(int q, int n, int heads) {
    const int log2 = 3 - min(3, __ffs(heads) - 1), xcds = 1 << log2;
    const int per = (n + xcds - 1) >> log2, tall = n - xcds * (per - 1);  // the first `tall` runs have `per`, the others one less
    const int x = q < tall * per ? small_div(q, per) : tall + small_div(q - tall * per, max(per - 1, 1));
    const int first = x * (per - 1) + min(x, tall);
    return (q - first) * xcds + x;
}

// The plan where no list is cut: a workgroup per (layer, KV head) and some sequences
// of a group: as many as fill one, two or three row tiles, or a half, a quarter, ... of
// what fills one, whichever is estimated fastest (in tenths of a pass with one tile;
// measured: a pass takes half as long again with each further tile, and a workgroup
// about six passes besides).  The prefix is read by all, the rests one after the other.
// The last choice that the launch has no workgroups for is that of one tile.
template <int kPlanThreads>
static __device__ __forceinline__ void plan_whole(const SharedPlanLaunch &p, PlanLds &l, PlanHeader *h, PlanSeq *seqs,
                                                  PlanItem *items, int end, int stream, int tid) {
    const int n_groups = p.n_groups, G = small_div(p.Hq, p.Hkv), lane = tid & 63, wave = tid >> 6;
    const int heads = p.n_layers * p.Hkv, waves = p.caps.waves, slots = waves == 8 ? kRoundWorkgroups : 2 * kRoundWorkgroups;
#pragma unroll 1
    for (int g = tid; g < n_groups; g += kPlanThreads) l.row[g] = 0;
    __syncthreads();
#pragma unroll 1
    for (int b = tid; b < p.B; b += kPlanThreads) {
        const int rest = b < end ? max(l.rest[b], 0) : 0;
        if (b < end) {
            PlanSeq s = {};
            s.state = seq_state(l.rest[b]);
            s.rest = rest;
            seqs[b] = s;
            atomicAdd(&l.row[l.of[b]], div_up(rest, kWaveTile));
        }
    }
    __syncthreads();
    const int one_tile = small_div(16, G), choices = 3 + 31 - __clz(one_tile);
    const auto per_of = [&](int c) { return c < 3 ? small_div(16 * (c + 1), G) : one_tile >> (c - 2); };
    for (int c = wave; c < choices; c += kPlanThreads / 64) {
        const int per = per_of(c), extra = c < 3 ? 5 * c : 0;
        int wg = 0, sum = 0, most = 0;
#pragma unroll 1
        for (int g = lane; g < n_groups; g += 64) {
            const int n = l.lo[g + 1] - l.lo[g], parts = small_div_up(n, per);
            if (n == 0) continue;
            const int passes = div_up(max(l.common[g], 0), kWaveTile) + (int)((unsigned)(l.row[g] + parts - 1) / (unsigned)parts);
            const int cost = 60 + (10 + extra) * (waves == 8 ? div_up(passes, 8) : div_up(passes, 4));
            wg += parts;
            sum += parts * min(cost, 1 << 18);
            most = max(most, cost);
        }
        wg = wave_sum(wg);
        sum = wave_sum(sum);
        most = wave_max(most);
        const int64_t all = (int64_t)(((uint64_t)sum * (uint64_t)heads) / kRoundWorkgroups >> (waves == 8 ? 0 : 1));
        const int64_t time = most + ((int64_t)wg * heads > slots ? all : 0);
        if (lane == 0) l.work[0][c] = wg > p.caps.grid ? 0x7fffffff : (int)min<int64_t>(time, 0x7ffffffe);
    }
    __syncthreads();
    int choice = 0;
#pragma unroll 1
    for (int c = 1; c < choices; ++c) choice = l.work[0][c] < l.work[0][choice] ? c : choice;
    const int per = per_of(choice);
    int work = 0;
#pragma unroll 1
    for (int g0 = 0; g0 < n_groups; g0 += kPlanThreads) {
        const int g = g0 + tid, n = g < n_groups ? l.lo[g + 1] - l.lo[g] : 0;
        int total;
        const int at = work + wg_exclusive_scan<kPlanThreads>(small_div_up(n, per), l.scan, tid, total);
        work += total;
        if (g < n_groups) l.item[g] = at;
    }
    __syncthreads();
#pragma unroll 1
    for (int g = wave; g < n_groups; g += kPlanThreads / 64) {
        const int lo = l.lo[g], lead = l.lead[g], n = l.lo[g + 1] - lo, parts = small_div_up(n, per);
        const Dealt dealt(n, max(parts, 1));
#pragma unroll 1
        for (int i = lane; i < parts; i += 64) {
            const int s0 = dealt.start(i), s1 = dealt.start(i + 1);
            items[item_place(l.item[g] + i, work, heads)] =
                PlanItem{lo + s0, s1 - s0, lead, 0, max(l.common[g], 0), 0, stream && parts <= 2, 0};
        }
    }
    if (tid == 0) {
        h->n_work = work;
        h->kind = plan_kind(true, l.found);
        h->rows = 0;
        h->level = -per;
    }
}

template <int kPlanThreads>
__global__ __launch_bounds__(kPlanThreads) void shared_plan_kernel(const SharedPlanLaunch p) {
    __shared__ PlanLds l;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const int B = p.B, n_groups = p.n_groups, max_keep = p.max_keep;
    const int G = small_div(p.Hq, p.Hkv), per_item = small_div(kSharedRows, G);
    PlanHeader *h = reinterpret_cast<PlanHeader *>(p.plan);
    PlanSeq *seqs = reinterpret_cast<PlanSeq *>(p.plan + sizeof(PlanHeader));
    PlanItem *items = reinterpret_cast<PlanItem *>(p.plan + p.caps.item_offset);
    PlanChunk *chunks = reinterpret_cast<PlanChunk *>(p.plan + p.caps.chunk_offset);
    const int32_t *scan = reinterpret_cast<const int32_t *>(p.plan + p.caps.scan_offset);
    const int n_scan = p.caps.n_scan;

    // the groups, and every sequence's count (in `rest` for now)
    if (tid == 0) l.bad = l.found = l.positions = 0;
#pragma unroll 1
    for (int b = tid; b < B; b += kPlanThreads) l.rest[b] = list_count(p.ranges, p.count, b);
#pragma unroll 1
    for (int g = tid; g <= n_groups; g += kPlanThreads) l.lo[g] = p.group[g];
#pragma unroll 1
    for (int g = tid; g < n_groups; g += kPlanThreads) l.common[g] = p.find ? max_keep + 1 : p.shared[g];
    __syncthreads();
#pragma unroll 1
    for (int g = tid; g < n_groups; g += kPlanThreads) {
        const int lo = l.lo[g], hi = l.lo[g + 1];
        int lead = lo;
        if (lo < 0 || lo > hi || hi > B || (g == 0 && lo != 0)) l.bad = 1;
        else
            while (lead < hi && l.rest[lead] == kAbsent) ++lead;
        l.lead[g] = lead;
    }
    __syncthreads();
    const int bad = l.bad, end = bad ? 0 : l.lo[n_groups];
    if (tid == 0) {
        h->magic = kPlanMagic;
        h->bad = bad;
        h->B = B;
        h->max_keep = max_keep;
        h->n_layers = p.n_layers;
        h->Hq = p.Hq;
        h->Hkv = p.Hkv;
        h->n_groups = n_groups;
        if (bad) {
            h->n_work = h->rows = 0;
            raise_device_error(MURMUR_DEVERR_GROUP);
        }
    }
    if (bad) return;

    // a sequence's group: the last one that starts at or before it and is not empty
#pragma unroll 1
    for (int b = tid; b < end; b += kPlanThreads) {
        int lo = 0, hi = n_groups;  // l.lo[lo] <= b < l.lo[hi]
#pragma unroll 1
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (l.lo[mid] <= b) lo = mid;
            else hi = mid;
        }
        l.of[b] = (uint16_t)lo;
        const int c = l.rest[b];
        if (p.find && ((c >= 1 && c <= max_keep) || b == l.lead[lo])) atomicMin(&l.common[lo], max(c, 0));
    }
    __syncthreads();
    if (p.find == kFindHere) {
        // entries side by side, four of a thread in flight
        const int n = end * max_keep;
#pragma unroll 1
        for (int t0 = tid; t0 < n; t0 += 4 * kPlanThreads) {
            int b[4], r[4], x[4], y[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int t = min(t0 + j * kPlanThreads, n - 1);
                b[j] = small_div(t, max_keep);
                r[j] = t - b[j] * max_keep;
                x[j] = p.idx[t];
                y[j] = p.idx[min(l.lead[l.of[b[j]]], b[j]) * max_keep + r[j]];  // a list that is not there: any one
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const int c = l.rest[b[j]];
                if (r[j] < c && c <= max_keep && x[j] != y[j]) atomicMin(&l.common[l.of[b[j]]], r[j]);
            }
        }
        __syncthreads();
    } else if (p.find) {
#pragma unroll 1
        for (int t = tid; t < end * n_scan; t += kPlanThreads) {  // below 2^29
            const int b = (int)((unsigned)t / (unsigned)n_scan), c = l.rest[b];
            if (c >= 1 && c <= max_keep) atomicMin(&l.common[l.of[b]], scan[t]);
        }
        __syncthreads();
    }
    // what is shared has to be in the list that is read, the first one that is there (-1: it is not)
#pragma unroll 1
    for (int g = tid; g < n_groups; g += kPlanThreads) {
        const int lead = l.lead[g];
        const bool some = lead < l.lo[g + 1];
        int common = some ? l.common[g] : 0;
        if (p.find) p.shared[g] = common = common <= max_keep ? common : 0;  // above: none has a valid count
        else if (common != 0 && some && !(common > 0 && common <= l.rest[lead] && l.rest[lead] <= max_keep)) common = -1;
        l.common[g] = common;
    }
    __syncthreads();
    int err = 0;
#pragma unroll 1
    for (int b = tid; b < B; b += kPlanThreads) {
        const int c = l.rest[b], common = b < end ? l.common[l.of[b]] : 0;
        const bool good = c >= 1 && c <= max_keep && common >= 0 && c >= common;
        const int rest = b >= end || c == kAbsent ? kNotThere : (good ? c - common : kInvalid);
        if (rest == kInvalid) err |= MURMUR_DEVERR_COUNT;
        if (p.find && rest >= 0 && common > 0 && b != l.lead[l.of[b]]) l.found = 1;
        seqs[b].state = seq_state(rest);
        l.rest[b] = rest;
    }
    if (err) raise_device_error(err);
    __syncthreads();

    // Rows that are read once or twice go past the caches where a layer reads kStreamBytes or more, so that they do not
    // push out what several workgroups read (us with and without: an hour of five hypotheses 706 and 744, 16 x 6 drafted
    // tokens 485 and 524; small lists of their own behind a long shared prefix lose, 64 chunks 121 and 115, 23 ragged
    // groups 64 and 61; all rows past the caches: 706, 485, 122, 65).
    int stream;
    {  // positions that a layer reads
        int n = 0;
#pragma unroll 1
        for (int g = tid; g < n_groups; g += kPlanThreads) n += max(l.common[g], 0);
#pragma unroll 1
        for (int b = tid; b < end; b += kPlanThreads) n += max(l.rest[b], 0);
        n = wave_sum(n);
        if (lane == 0) atomicAdd(&l.positions, (unsigned)min(n, 1 << 24));
        __syncthreads();
        stream = (int64_t)l.positions * p.Hkv * 2 * kTileRowBytes >= kStreamBytes;
    }
    if (p.caps.whole) {
        plan_whole<kPlanThreads>(p, l, h, seqs, items, end, stream, tid);
        return;
    }

    int level = 0;
#pragma unroll 1
    for (int round = 0; round < 2; ++round) {
        const auto candidate = [&](int k) { return min(round == 0 ? 4 + 8 * k : max(level - 7 + k, 4), kSharedLevels); };
#pragma unroll 1
        for (int k = wave; k < 8; k += kPlanThreads / 64) {
            const unsigned item = item_passes(candidate(k)), chunk = chunk_passes(candidate(k));
            int wg = 0, waves = 0;
#pragma unroll 1
            for (int g = lane; g < n_groups; g += 64) {
                const int n = l.lo[g + 1] - l.lo[g], pre = div_up(max(l.common[g], 0), kWaveTile);
                wg += small_div_up(n, per_item) * (int)((pre + item - 1) / item);
            }
#pragma unroll 1
            for (int b = lane; b < end; b += 64) waves += (int)((div_up(max(l.rest[b], 0), kWaveTile) + chunk - 1) / chunk);
            wg = wave_sum(wg);
            waves = wave_sum(waves);
            if (lane == 0) l.work[round][k] = wg + div_up(waves, kSharedWaves);
        }
        __syncthreads();
        int k = 0;
#pragma unroll 1
        while (k < 8 && l.work[round][k] > p.caps.per_round) ++k;
        level = round == 0 ? 4 + 8 * k : candidate(min(k, 7));
    }

    // Prefix work: the groups' items one after the other, the row tiles of one stretch side by side.
    int work = 0, rows = 0;
#pragma unroll 1
    for (int g0 = 0; g0 < n_groups; g0 += kPlanThreads) {
        const int g = g0 + tid;
        const int n = g < n_groups ? l.lo[g + 1] - l.lo[g] : 0, pre = n > 0 ? div_up(max(l.common[g], 0), kWaveTile) : 0;
        const int cuts = (int)((unsigned)(pre + item_passes(level) - 1) / (unsigned)item_passes(level));
        int total;
        const int at = work + wg_exclusive_scan<kPlanThreads>(small_div_up(n, per_item) * cuts, l.scan, tid, total);
        work += total;
        const int row = rows + wg_exclusive_scan<kPlanThreads>(cuts * n * G, l.scan, tid, total);
        rows += total;
        if (g < n_groups) {
            l.item[g] = at;
            l.row[g] = row;
            l.cuts[g] = cuts;
        }
    }
    __syncthreads();
    const int heads = p.n_layers * p.Hkv;
#pragma unroll 1
    for (int g = wave; g < n_groups; g += kPlanThreads / 64) {
        const int lo = l.lo[g], n = l.lo[g + 1] - lo, common = max(l.common[g], 0), pre = n > 0 ? div_up(common, kWaveTile) : 0;
        const int cuts = l.cuts[g], parts = small_div_up(n, per_item);
        const Dealt to_parts(n, max(parts, 1)), to_cuts(pre, max(cuts, 1));
#pragma unroll 1
        for (int i = lane; i < cuts * parts; i += 64) {
            const int cut = small_div(i, parts), part = i - cut * parts;
            const int s0 = to_parts.start(part), s1 = to_parts.start(part + 1);
            const int r0 = to_cuts.start(cut) * kWaveTile, r1 = min(to_cuts.start(cut + 1) * kWaveTile, common);
            items[item_place(l.item[g] + i, work, heads)] = PlanItem{lo + s0, s1 - s0, l.lead[g], r0, r1, l.row[g] + (cut * n + s0) * G,
                         stream && parts <= 2, 0};
        }
    }
    // The rests: a wavefront's chunk each, the sequences one after the other; a
    // workgroup's chunks of one sequence end in one partial.
    const int chunk0 = work * kSharedWaves, each = chunk_passes(level);
    int done = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < B; b0 += kPlanThreads) {
        const int b = b0 + tid;
        const int rest = b < end ? max(l.rest[b], 0) : 0, pre = div_up(rest, kWaveTile);
        const int n = (int)((unsigned)(pre + each - 1) / (unsigned)each);
        int total;
        const int at = done + wg_exclusive_scan<kPlanThreads>(n, l.scan, tid, total);
        done += total;
        const int parts = n > 0 ? (at + n - 1) / kSharedWaves - at / kSharedWaves + 1 : 0;
        const int row = rows + wg_exclusive_scan<kPlanThreads>(parts * G, l.scan, tid, total);
        rows += total;
        if (b >= end) continue;
        const int g = l.of[b], lo = l.lo[g], n_seq = l.lo[g + 1] - lo, common = max(l.common[g], 0);
        const Dealt dealt(pre, max(n, 1));
#pragma unroll 1
        for (int i = 0; i < n; ++i) {
            const int r0 = dealt.start(i) * kWaveTile, r1 = min(dealt.start(i + 1) * kWaveTile, rest);
            chunks[chunk0 + at + i] = PlanChunk{b, common + r0, common + r1,
                                                row + ((at + i) / kSharedWaves - at / kSharedWaves) * G};
        }
        PlanSeq s = {};
        s.state = seq_state(l.rest[b]);
        s.pre_row = l.row[g] + (b - lo) * G;
        s.pre_stride = n_seq * G;
        s.n_pre = l.cuts[g];
        s.rest_row = row;
        s.n_rest = parts;
        seqs[b] = s;
    }
    const int rest_wg = div_up(done, kSharedWaves);
#pragma unroll 1
    for (int c = done + tid; c < rest_wg * kSharedWaves; c += kPlanThreads) chunks[chunk0 + c] = PlanChunk{-1, 0, 0, 0};
#pragma unroll 1
    for (int w = tid; w < rest_wg; w += kPlanThreads) items[work + w] = PlanItem{0, 0, 0, 0, 0, 0, stream, 0};
    if (tid == 0) {
        h->n_work = work + rest_wg;
        h->kind = plan_kind(false, l.found);
        h->rows = rows;
        h->level = level;
    }
}

// ---------------------------------------------------------------------------
// The passes of one wavefront.  K and V have a tile each in its LDS stage.  Once
// a pass's K operands are in registers the next pass's K rows start into their
// tile, and V likewise, so 8 KiB at least are on their way at any time; the waits
// count the loads issued after the ones awaited (loads complete in order).
// ---------------------------------------------------------------------------
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

// The 16-byte loads of one pass's K or V rows straight into LDS, laid out as for
// dma_pass.  kNear: every row of the cache lies within 2^32 bytes of its first, so
// that a row is a 32-bit offset, the same for K and V, and the buffer's size bounds
// it; else 64-bit addresses.
template <bool kNear>
struct RowSource;
template <>
struct RowSource<true> {
    __amdgpu_buffer_rsrc_t base;
    __device__ __forceinline__ void init(const uint16_t *p, int64_t s_pos, int max_len) {
        base = raw_buffer(p, (uint32_t)(max_len - 1) * ((uint32_t)s_pos * 2u) + kTileRowBytes);
    }
    template <int kAux>
    __device__ __forceinline__ void load(uint8_t *tile, const uint32_t (&at)[8]) const {
#pragma unroll
        for (int j = 0; j < 8; ++j)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(base, (lds_void_t *)(tile + j * 1024), 16, at[j], 0, 0, kAux);
    }
};
template <>
struct RowSource<false> {
    const uint16_t *base;
    int64_t s_pos;
    __device__ __forceinline__ void init(const uint16_t *p, int64_t s, int) {
        base = p;
        s_pos = s;
    }
    template <int kAux>
    __device__ __forceinline__ void load(uint8_t *tile, const int32_t (&pos)[8], int lane) const {
        const int q = lane >> 4, sl = lane & 15;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            __builtin_amdgcn_global_load_lds(base + (int64_t)pos[j] * s_pos + 8 * (sl ^ ((4 * j + q) & 15)),
                                             (lds_void_t *)(tile + j * 1024), 16, 0, kAux);
    }
};

// The K/V of one (layer, KV head) of a sequence, and its list or range table.
template <bool kNear>
struct Rows {
    RowSource<kNear> k, v;
};
template <bool kNear>
static __device__ __forceinline__ Rows<kNear> rows_of(const SharedAttnLaunch &a, int list, int layer, int g) {
    Rows<kNear> in;
    const int64_t off = layer * a.s_layer + list * a.s_b + g * a.s_h;
    in.k.init(a.k + off, a.s_pos, a.max_len);
    in.v.init(a.v + off, a.s_pos, a.max_len);
    return in;
}
static __device__ __forceinline__ __amdgpu_buffer_rsrc_t list_of(const SharedAttnLaunch &a, int list) {
    return raw_buffer(a.idx + (int64_t)list * a.max_keep, (uint32_t)a.max_keep * 4u);
}
static __device__ __forceinline__ RangeTab table_of(const SharedAttnLaunch &a, int list) {
    int32_t rg[2 * kPieces];
#pragma unroll
    for (int k = 0; k < 2 * kPieces; ++k) rg[k] = a.ranges[(int64_t)list * 2 * kPieces + k];
    return make_tab(rg);
}

// Positions of a pass from its index slot (dma_idx), as dma_pos_index, which a pass
// that is not full or names a position outside the cache goes to: a full one needs
// no clamping once all of its positions are known to be inside (5 instructions for
// the eight of a lane, not 80, in a loop that instruction issue bounds).
static __device__ __forceinline__ void slot_positions(const uint8_t *slot, int r, int r_end, int max_len, int q,
                                                      int32_t (&pos)[8], int &bad) {
    if (r_end - r >= kWaveTile) {
        u32x4 e0, e1;
        asm volatile("ds_read_b128 %0, %2\n\tds_read_b128 %1, %2 offset:16\n\ts_waitcnt lgkmcnt(0)"
                     : "=&v"(e0), "=&v"(e1)
                     : "v"(lds_addr(slot) + 32u * q)
                     : "memory");
        uint32_t most = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            pos[j] = (int32_t)(j < 4 ? e0[j] : e1[j - 4]);
            most = max(most, (uint32_t)pos[j]);
        }
        if (__builtin_expect(__ballot(most >= (uint32_t)max_len) == 0, 1)) return;
    }
    dma_pos_index(slot, r, r_end, max_len, q, pos, bad);
}

// A pass: ranks r .. min(r + 32, r_end) - 1 of a sequence's list, for the rows of
// every sequence of the item, or (only >= 0) of one.
struct Pass {
    int list, r, r_end, only;
};

// Where a wavefront's passes come from; next() is false behind the last one.
struct OneList {  // ranks r, r + step, ... below r_end of one list
    static constexpr bool kOne = true;
    int list, r, r_end, step;
    __device__ __forceinline__ bool next(Pass &p) {
        p = Pass{list, r, r_end, -1};
        r += step;
        return p.r < r_end;
    }
};
struct WholeLists {  // every step-th pass of an item: those of the prefix, then its sequences' rests
    static constexpr bool kOne = false;
    int list, seq0, n_seq, common, pre, total;  // passes of the prefix, of everything
    int at, step;
    int rest, first;  // of the lane's sequence: length, first pass of the rests
    __device__ __forceinline__ bool next(Pass &p) {
        const int i = at;
        at += step;
        p = Pass{list, i * kWaveTile, common, -1};
        if (i < pre) return true;
        const int q = i - pre;
        // the last sequence that starts at or before pass q (sequences without a rest start where the next one does)
        const uint64_t begun = __ballot((int)(threadIdx.x & 63) < n_seq && first <= q);
        const int s = max(__popcll(begun) - 1, 0);
        const int r = common + (q - __builtin_amdgcn_readlane(first, s)) * kWaveTile;
        p = Pass{seq0 + s, r, common + __builtin_amdgcn_readlane(rest, s), s};
        return i < total;
    }
};

// A running max that is below every logit and finite, so that a row which a pass
// leaves out entirely (every logit -inf) stays as it is: exp2 of -inf, not of NaN.
constexpr float kNoRows = -3.0e38f;
static __device__ __forceinline__ void start_rows(WaveAcc &w) {
    wave_acc_reset(w);
    w.m_run = kNoRows;
}

// A pass of one sequence's rest is multiplied with the rows of other sequences too,
// whose weights are zero, but zero times an infinity or a NaN is NaN.  Where the
// values hold one (the product with zeros tells), they are taken out of the tile
// and added to the sums of the sequence itself, whose result is not finite there
// whatever its weights.
template <int kTiles>
static __device__ __forceinline__ void keep_apart(u32x2 (&vf)[16], uint8_t *tile, int valid, int only,
                                                  const int (&row_seq)[kTiles], WaveAcc (&w)[kTiles], int lane) {
    const int c4 = lane >> 4;
    f32x4 zero = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int db = 0; db < 8; ++db)
        zero = mfma16x16x32(u32x4{vf[2 * db][0], vf[2 * db][1], vf[2 * db + 1][0], vf[2 * db + 1][1]}, u32x4{0u, 0u, 0u, 0u}, zero);
    if (__builtin_expect(__ballot(zero[0] + zero[1] + zero[2] + zero[3] != 0.f) == 0, 1)) return;
    // 0xffff in the halves of x whose exponent is all ones
    const auto not_finite = [](uint32_t x) { return ((((x & 0x7f807f80u) + 0x00800080u) >> 15) & 0x00010001u) * 0xffffu; };
#pragma unroll
    for (int db = 0; db < 8; ++db) {
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
        for (int r = 0; r < valid; ++r) {
            u32x2 e = *reinterpret_cast<const u32x2 *>(tile + r * kTileRowBytes + (((2 * db + (c4 >> 1)) ^ (r & 15)) << 4) +
                                                       8 * (c4 & 1));
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                e[i] &= not_finite(e[i]);
                sum[2 * i] += __builtin_bit_cast(float, e[i] << 16);
                sum[2 * i + 1] += __builtin_bit_cast(float, e[i] & 0xffff0000u);
            }
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t)
#pragma unroll
            for (int i = 0; i < 4; ++i) w[t].acc[db][i] += row_seq[t] == only ? sum[i] : 0.f;
    }
#pragma unroll 1
    for (int i = lane; i < kTileBytes / 16; i += 64) {
        u32x4 e = *reinterpret_cast<const u32x4 *>(tile + 16 * i);
#pragma unroll
        for (int x = 0; x < 4; ++x) e[x] &= ~not_finite(e[x]);
        *reinterpret_cast<u32x4 *>(tile + 16 * i) = e;
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    read_v_operands(vf, lds_addr(tile), lane & 15, c4);
}

// softmax_step of a pass that is one of many, with the weights as the sums of kTerms
// bf16 parts, each the rounding of what the ones before leave: two for bf16 outputs
// (2^-17 of a weight at most, against an output's 2^-9) and three for fp32 ones (what
// is left is below fp32's own rounding: over 35 096 positions outputs are 2.5e-7 off,
// relative, where two parts gave 1.8e-6; 28 layers 700 us instead of 670).
template <int kTerms>
static __device__ __forceinline__ void softmax_pass(f32x4 (&s)[2], int valid, float scale, WaveAcc &w, int c4,
                                                    u32x4 (&p)[kTerms]) {
    if (valid < kWaveTile) {  // uniform
#pragma unroll
        for (int blk = 0; blk < 2; ++blk)
#pragma unroll
            for (int i = 0; i < 4; ++i) s[blk][i] = 16 * blk + 4 * c4 + i < valid ? s[blk][i] : kNegInf;
    }
    const float lane_max = fmaxf(fmaxf(fmaxf(s[0][0], s[0][1]), fmaxf(s[0][2], s[0][3])),
                                 fmaxf(fmaxf(s[1][0], s[1][1]), fmaxf(s[1][2], s[1][3])));
    if (__ballot(lane_max > w.m_run)) {
        const float m_new = fmaxf(w.m_run, max_over_c4(lane_max));
        const float alpha = __builtin_amdgcn_exp2f((w.m_run - m_new) * scale);  // 0 while the state is empty
        w.l_run *= alpha;
#pragma unroll
        for (int db = 0; db < 8; ++db) w.acc[db] *= alpha;
        w.m_run = m_new;
    }
    float pr[2][4];
#pragma unroll
    for (int blk = 0; blk < 2; ++blk)
#pragma unroll
        for (int i = 0; i < 4; ++i) pr[blk][i] = __builtin_amdgcn_exp2f((s[blk][i] - w.m_run) * scale);
    w.l_run += ((pr[0][0] + pr[0][1]) + (pr[0][2] + pr[0][3])) + ((pr[1][0] + pr[1][1]) + (pr[1][2] + pr[1][3]));
#pragma unroll
    for (int wd = 0; wd < 4; ++wd) {
        float e0 = pr[wd >> 1][(wd & 1) * 2], e1 = pr[wd >> 1][(wd & 1) * 2 + 1];
#pragma unroll
        for (int k = 0; k < kTerms; ++k) {
            p[k][wd] = pack_bf16(e0, e1);
            e0 -= __builtin_bit_cast(float, p[k][wd] << 16);
            e1 -= __builtin_bit_cast(float, p[k][wd] & 0xffff0000u);
        }
    }
}

// The passes of `feed` against kTiles row tiles.  load_queries starts the loads of
// the queries (4 kTiles of them) into qf.  row_seq: which of the item's sequences
// the lane's row of a tile belongs to (several lists only).  on_bad(pass) is called
// for a pass with a position outside the cache.  Returns the positive scale
// (signed_scale).
template <int kTerms, int kSrc, bool kNear, int kTiles, typename Feed, typename LoadQ, typename OnBad>
static __device__ __forceinline__ float run_passes(const SharedAttnLaunch &a, int layer, int g, bool stream, Feed &feed,
                                                   uint8_t *stage, uint8_t (*slots)[kIdxSlotBytes],
                                                   u32x4 (&qf)[kTiles][4], LoadQ load_queries,
                                                   const int (&row_seq)[kTiles], WaveAcc (&w)[kTiles], int lane,
                                                   OnBad on_bad) {
    Pass cur, nxt;
    if (!feed.next(cur)) return 1.f;
    bool more = feed.next(nxt);
    const int n16 = lane & 15, c4 = lane >> 4;
    const uint32_t kt = lds_addr(stage), vt = kt + kTileBytes;
    int32_t pos[8];
    uint32_t at[8];
    int bad = 0;
    const uint32_t row_bytes = (uint32_t)a.s_pos * 2u;
    RangeTab tab;
    const auto positions = [&](const Pass &p, int slot) {
        if (kSrc == kSrcIndex) slot_positions(slots[slot], p.r, p.r_end, a.max_len, c4, pos, bad);
        else dma_pos_ranges(tab, p.r, p.r_end, a.max_len, c4, pos, bad);
        if (__builtin_expect(__ballot(bad) != 0, 0)) {
            on_bad(p);
            bad = 0;
        }
        if constexpr (kNear) {  // positions and row bytes are below 2^24 (see launch_shared_attn)
#pragma unroll
            for (int j = 0; j < 8; ++j)
                at[j] = __umul24((uint32_t)pos[j], row_bytes) + 16u * (uint32_t)(n16 ^ ((4 * j + c4) & 15));
        }
    };
    const auto load_as = [&](const RowSource<kNear> &from, uint8_t *tile, auto aux) {
        if constexpr (kNear) from.template load<decltype(aux)::value>(tile, at);
        else from.template load<decltype(aux)::value>(tile, pos, lane);
    };
    const auto load = [&](const RowSource<kNear> &from, uint8_t *tile) {  // uniform
        if (stream) load_as(from, tile, std::integral_constant<int, kAuxStream>{});
        else load_as(from, tile, std::integral_constant<int, 0>{});
    };
    if (kSrc == kSrcIndex) {
        dma_idx(slots[0], list_of(a, cur.list), cur.r, lane);
        dma_idx(slots[1], list_of(a, more ? nxt.list : cur.list), more ? nxt.r : cur.r, lane);
    } else {
        tab = table_of(a, cur.list);
    }
    Rows<kNear> in = rows_of<kNear>(a, cur.list, layer, g);
    asm volatile("" ::: "memory");  // the queries' loads stay behind the entries'
    load_queries();
    // the first slot: the second slot's load and then the queries' came after it
    if (kSrc == kSrcIndex) wait_vm<1 + 4 * kTiles>();
    positions(cur, 0);
    load(in.k, stage);
    load(in.v, stage + kTileBytes);
    float scale = 1.f;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) scale = signed_scale(qf[t], a.scale_log2);
    for (int it = 0;; ++it) {
        u32x4 kf[8];
        wait_vm<8>();  // this pass's K rows; its V rows came after them
        read_k_operands(kf, kt, n16, c4);
        Pass after;
        bool more_after = false;
        if (more) {
            if (!Feed::kOne) {  // uniform
                if (kSrc != kSrcIndex && nxt.list != cur.list) tab = table_of(a, nxt.list);
                in = rows_of<kNear>(a, nxt.list, layer, g);
            }
            positions(nxt, (it + 1) & 1);  // entries that were loaded before this pass's K rows
            more_after = feed.next(after);
            if (kSrc == kSrcIndex) {
                const Pass &x = more_after ? after : nxt;
                dma_idx(slots[it & 1], list_of(a, x.list), x.r, lane);
            }
            load(in.k, stage);
        }
        const int valid = min(kWaveTile, cur.r_end - cur.r);
        u32x4 p[kTiles][kTerms];
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            f32x4 s[2];
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                s[blk] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kc = 0; kc < 4; ++kc) s[blk] = mfma16x16x32(kf[4 * blk + kc], qf[t][kc], s[blk]);
            }
            if (!Feed::kOne && cur.only >= 0) {
                asm volatile("");  // a branch, which few passes take, rather than selects in every pass
                const bool mine = row_seq[t] == cur.only;
#pragma unroll
                for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s[blk][i] = mine ? s[blk][i] : kNegInf;
            }
            softmax_pass<kTerms>(s, valid, scale, w[t], c4, p[t]);
        }
        u32x2 vf[16];
        if (more) wait_vm<8>();  // this pass's V rows; the next pass's K rows came after them
        else wait_vm<0>();
        read_v_operands(vf, vt, n16, c4);
        if (!Feed::kOne && cur.only >= 0) keep_apart<kTiles>(vf, stage + kTileBytes, valid, cur.only, row_seq, w, lane);
        if (more) load(in.v, stage + kTileBytes);
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            const u32x4 av = u32x4{vf[2 * db][0], vf[2 * db][1], vf[2 * db + 1][0], vf[2 * db + 1][1]};
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int k = 0; k < kTerms; ++k) w[t].acc[db] = mfma16x16x32(av, p[t][k], w[t].acc[db]);
        }
        if (!more) break;
        cur = nxt;
        nxt = after;
        more = more_after;
    }
    return scale;
}

// The queries of an item's rows as B operands of its row tiles, past the last row
// its copies (their results are not stored); row_seq: each lane's sequence.
template <int kTiles>
static __device__ __forceinline__ void load_item_queries(const SharedAttnLaunch &a, const PlanItem &it, int layer, int g,
                                                         int n16, int c4, u32x4 (&qf)[kTiles][4], int (&row_seq)[kTiles]) {
    const int rows = it.n_seq * a.G;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const uint32_t rr = (uint32_t)min(16 * t + n16, rows - 1);
        const uint32_t s = div16(rr, a.magic_g);
        row_seq[t] = (int)s;
        const int64_t row = ((int64_t)layer * a.B + it.seq0 + (int)s) * a.Hq + g * a.G + (int)(rr - s * (uint32_t)a.G);
#pragma unroll
        for (int kc = 0; kc < 4; ++kc) qf[t][kc] = load16(a.q + row * kHeadDim + 8 * c4 + 32 * kc);
    }
}

// ---------------------------------------------------------------------------
// Workgroup (layer and KV head, i) does item i of the plan: a stretch of a prefix,
// whose passes its wavefronts take in turn, each for all of the item's query rows;
// or remainders, each wavefront a chunk of some sequence's.  Eight wavefronts and
// 134 KiB of LDS, a compute unit for a workgroup: with four, two on one, there are
// twice the partials to write and to join (35 096 positions, 5 hypotheses, 4 KV
// heads: 21.8 + 4.0 us a layer, 22.5 + 5.1 with four; 21.1 + 4.0 since the levels go
// by quarters of a pass).  Two thirds of it is the read: 73 MB at 5.5 TB/s.
// Two wavefronts on a SIMD leave 256 vector registers each, which three row tiles fill:
// none is spilled with index lists within 32-bit offsets, 17 with range tables and fp32
// outputs (none with bf16 ones), 14 and 57 where rows go by 64-bit addresses.
// ---------------------------------------------------------------------------
constexpr int kSharedThreads = kSharedWaves * 64;
constexpr size_t kComputeUnitLds = 160 * 1024;
template <int kWaves>
struct SharedLds {
    uint8_t stages[kWaves][kStageBytes];
    uint8_t slots[kWaves][2][kIdxSlotBytes];
    float ml[kWaves][32][2];  // per wavefront and row of a round: max (log2 units), sum
    int flag[kWaves];
    int seq[kWaves + 1], row[kWaves];
    unsigned long long bad;   // sequences of the item with a position outside the cache or an invalid count
    unsigned long long gone;  // those that are not there
};

// Up to two of a wavefront's tiles into its own stage and the pairs, for the sums
// over the wavefronts: row r, 16-byte chunk c at slot c ^ (r & 7) (the lanes of a
// store hold 16 rows of one chunk).
template <int kFirst, int kTiles, int kWaves, int kAll>
static __device__ __forceinline__ void publish_tiles(SharedLds<kWaves> &l, WaveAcc (&w)[kAll], float scale, int wave, int n16,
                                                     int c4) {
    static_assert(kTiles <= 2, "two tiles fit a stage");
    float *o = reinterpret_cast<float *>(&l.stages[wave][0]);
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        const float sum = sum_over_c4(w[kFirst + t].l_run);
        const int r = 16 * t + n16;
        if (c4 == 0) *reinterpret_cast<float2 *>(&l.ml[wave][r][0]) = float2{w[kFirst + t].m_run * scale, sum};
#pragma unroll
        for (int db = 0; db < 8; ++db)
            *reinterpret_cast<f32x4 *>(&o[r * kHeadDim + 4 * ((4 * db + c4) ^ (r & 7))]) = w[kFirst + t].acc[db];
    }
}

// The state of row r, head dims 4 c .. 4 c + 3, over n wavefronts (at most kMost)
// from w0 on.
template <int kMost, int kWaves>
static __device__ __forceinline__ void gather_row(const SharedLds<kWaves> &l, int w0, int n, int r, int c, float &M, float &L,
                                                  f32x4 &O) {
    float2 ml[kMost];
    f32x4 o[kMost];
#pragma unroll
    for (int w = 0; w < kMost; ++w) {
        const int wv = w0 + min(w, n - 1);
        ml[w] = *reinterpret_cast<const float2 *>(&l.ml[wv][r][0]);
        o[w] = *reinterpret_cast<const f32x4 *>(&l.stages[wv][(r * kHeadDim + 4 * (c ^ (r & 7))) * 4]);
    }
    M = ml[0].x;
    L = 0.f;
#pragma unroll
    for (int w = 1; w < kMost; ++w) M = fmaxf(M, ml[w].x);
    O = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int w = 0; w < kMost; ++w) {
        const float f = w >= n || ml[w].x == kNegInf ? 0.f : __builtin_amdgcn_exp2f(ml[w].x - M);
        L += ml[w].y * f;
        O += f * o[w];
    }
}

// The same into partial row `row` of this (layer, KV head).
template <int kMost>
static __device__ __forceinline__ void store_partial(const SharedLds<kSharedWaves> &l, float *part_o, float *part_ml, int w0,
                                                     int n, int r, int c, int64_t row, bool bad) {
    float M, L;
    f32x4 O;
    gather_row<kMost>(l, w0, n, r, c, M, L, O);
    if (bad) L = __builtin_nanf("");
    *reinterpret_cast<f32x4 *>(part_o + row * kHeadDim + 4 * c) = O;
    if (c == 0) *reinterpret_cast<float2 *>(part_ml + 2 * row) = float2{M, L};
}

// Normalised output of four head dims of query row `row`, and the lse (c == 0).
static __device__ __forceinline__ void store_row(const SharedAttnLaunch &a, int64_t row, int c, f32x4 O, float M, float L) {
    const float inv = 1.f / L;
    if (a.out_f32)
        *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.out) + row * kHeadDim + 4 * c) = O * inv;
    else
        *reinterpret_cast<u32x2 *>(reinterpret_cast<uint16_t *>(a.out) + row * kHeadDim + 4 * c) =
            u32x2{pack_bf16(O[0] * inv, O[1] * inv), pack_bf16(O[2] * inv, O[3] * inv)};
    if (c == 0 && a.lse) a.lse[row] = (M + __builtin_log2f(L)) * 0.69314718055994530942f;
}

template <int kTerms, int kSrc, bool kNear, int kTiles>
static __device__ __forceinline__ void item_work(const SharedAttnLaunch &a, const PlanItem &it, SharedLds<kSharedWaves> &l,
                                                 int layer, int g, float *part_o, float *part_ml, int tid, int wave) {
    const int lane = tid & 63, n16 = lane & 15, c4 = lane >> 4;
    const int rows = it.n_seq * a.G;
    u32x4 qf[kTiles][4];
    int row_seq[kTiles];
    WaveAcc w[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) start_rows(w[t]);
    OneList feed{it.list, it.r0 + wave * kWaveTile, it.r1, kSharedWaves * kWaveTile};
    int wave_bad = 0;
    const float scale = run_passes<kTerms, kSrc, kNear, kTiles>(
        a, layer, g, it.stream, feed, l.stages[wave], l.slots[wave], qf,
        [&] { load_item_queries<kTiles>(a, it, layer, g, n16, c4, qf, row_seq); }, row_seq, w, lane,
        [&](const Pass &) { wave_bad = 1; });
    const auto store = [&](int t0, int n_tiles, bool bad) {
#pragma unroll 1
        for (int j = tid >> 5; j < min(16 * n_tiles, rows - 16 * t0); j += kSharedThreads / 32)
            store_partial<kSharedWaves>(l, part_o, part_ml, 0, kSharedWaves, j, tid & 31, it.row + 16 * t0 + j, bad);
    };
    constexpr int kFirstTiles = kTiles < 2 ? 1 : 2;
    publish_tiles<0, kFirstTiles>(l, w, scale, wave, n16, c4);
    const int bad = barrier_or<kSharedWaves>(wave_bad, l.flag, wave, lane);
    store(0, kFirstTiles, bad);
    if constexpr (kTiles > 2) {
        __syncthreads();  // the rows of the tiles before are read
        publish_tiles<2, 1>(l, w, scale, wave, n16, c4);
        __syncthreads();
        store(2, 1, bad);
    }
    if (bad && tid == 0) raise_device_error(MURMUR_DEVERR_POSITION);
}

template <int kTerms, int kSrc, bool kNear>
static __device__ __forceinline__ void chunk_work(const SharedAttnLaunch &a, const PlanChunk &c, bool stream,
                                                  SharedLds<kSharedWaves> &l, int layer, int g, float *part_o, float *part_ml,
                                                  int tid, int wave) {
    const int lane = tid & 63, n16 = lane & 15, c4 = lane >> 4;
    WaveAcc w[1];
    start_rows(w[0]);
    u32x4 qf[1][4];
    int row_seq[1], wave_bad = 0;
    OneList feed{c.seq, c.r0, c.r1, kWaveTile};  // none: r0 == r1
    const PlanItem one{c.seq, 1, c.seq, 0, 0, 0, 0, 0};
    const float scale = run_passes<kTerms, kSrc, kNear, 1>(
        a, layer, g, stream, feed, l.stages[wave], l.slots[wave], qf,
        [&] { load_item_queries<1>(a, one, layer, g, n16, c4, qf, row_seq); }, row_seq, w, lane,
        [&](const Pass &) { wave_bad = 1; });
    publish_tiles<0, 1>(l, w, scale, wave, n16, c4);
    if (lane == 0) {
        l.seq[wave] = c.seq;
        l.row[wave] = c.row;
        l.flag[wave] = wave_bad;
    }
    if (tid == 0) l.seq[kSharedWaves] = -2;
    __syncthreads();
    // consecutive wavefronts of one sequence are one partial
    for (int t = tid; t < kSharedWaves * a.G * (kHeadDim / 4); t += kSharedThreads) {
        const uint32_t row = (uint32_t)t / (kHeadDim / 4);
        const int w0 = (int)div16(row, a.magic_g), h = (int)row - w0 * a.G, s = l.seq[w0];
        if (s < 0 || (w0 > 0 && l.seq[w0 - 1] == s)) continue;
        int w1 = w0, bad = 0;
        do bad |= l.flag[w1];
        while (l.seq[++w1] == s);
        if (w1 - w0 == 1)
            store_partial<1>(l, part_o, part_ml, w0, 1, h, t & 31, l.row[w0] + h, bad);
        else
            store_partial<kSharedWaves>(l, part_o, part_ml, w0, w1 - w0, h, t & 31, l.row[w0] + h, bad);
        if (bad && h == 0 && (t & 31) == 0) raise_device_error(MURMUR_DEVERR_POSITION);
    }
}

// Whether a plan was made for a call of these sizes.
static __device__ __forceinline__ bool plan_fits(const SharedAttnLaunch &a, const PlanHeader &h) {
    return h.magic == kPlanMagic && !h.bad && h.B == a.B && h.max_keep == a.max_keep && h.n_layers == a.NL &&
           h.Hq == a.Hq && h.Hkv == a.Hkv && h.n_groups == a.n_groups && h.rows <= a.rows_cap && h.n_work <= a.n_wg &&
           (h.kind & a.kinds);
}

static_assert(sizeof(SharedLds<8>) <= kComputeUnitLds && 2 * sizeof(SharedLds<4>) <= kComputeUnitLds,
              "eight wavefronts on a compute unit");

template <int kTerms, int kSrc, bool kNear>
__global__ __launch_bounds__(kSharedThreads, 2) void shared_attn_kernel(const SharedAttnLaunch a) {
    __shared__ __attribute__((aligned(16))) SharedLds<kSharedWaves> l;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = blockIdx.y;
    // the header, the item and the wavefront's chunk in one round trip, whichever of the two it will be
    const PlanHeader h = *reinterpret_cast<const PlanHeader *>(a.plan);
    const PlanItem it = reinterpret_cast<const PlanItem *>(a.plan + a.item_offset)[i];
    const PlanChunk c = reinterpret_cast<const PlanChunk *>(a.plan + a.chunk_offset)[i * kSharedWaves + wave];
    materialize(h.magic, h.n_work, h.rows, it.seq0, it.n_seq, it.list, it.r0, it.r1, it.row, it.stream, c.seq, c.r0, c.r1, c.row);
    if (!plan_fits(a, h) || i >= h.n_work) return;
    const int layer = (int)blockIdx.x / a.Hkv, g = (int)blockIdx.x - layer * a.Hkv;
    float *part_o = a.part_o + (int64_t)blockIdx.x * h.rows * kHeadDim;
    float *part_ml = a.part_ml + (int64_t)blockIdx.x * h.rows * 2;
    const int rows = it.n_seq * a.G;
    if (rows == 0)
        chunk_work<kTerms, kSrc, kNear>(a, c, it.stream, l, layer, g, part_o, part_ml, tid, wave);
    else if (rows <= 16)
        item_work<kTerms, kSrc, kNear, 1>(a, it, l, layer, g, part_o, part_ml, tid, wave);
    else if (rows <= 32)
        item_work<kTerms, kSrc, kNear, 2>(a, it, l, layer, g, part_o, part_ml, tid, wave);
    else
        item_work<kTerms, kSrc, kNear, 3>(a, it, l, layer, g, part_o, part_ml, tid, wave);
}

// ---------------------------------------------------------------------------
// The attention without cuts (SharedCaps::whole): a workgroup takes the whole lists
// of some sequences of one group, up to 48 query rows, the prefix once for all of
// them and each rest with the other sequences' rows masked, and writes the outputs.
// No partials, no second launch.  Workgroups of one group read the same prefix
// (from the L2s, mostly).  Eight wavefronts and a compute unit each where there are
// about as many workgroups as compute units, else four, two workgroups on one, whose
// prologues and epilogues overlap.  12 groups of 8, lists of 850, 4 KV heads: 16.4 us a
// layer, of which 5 are the first round trips (plan, entries, rows) and 4 the passes,
// at 91 bytes a nanosecond and compute unit; 28 layers of 16 groups of 6 drafted tokens
// in one launch: 2.67 GB in 482 us (5.5 TB/s).
// Every instance fills the 256 vector registers of its wavefronts.  With index lists
// within 32-bit offsets 1 (bf16 outputs) or 5 (fp32) are spilled, with range tables 16
// or 26 (the table is live through the passes), with 64-bit row addresses 20, or 48 to 53
// with range tables too.
// ---------------------------------------------------------------------------
template <int kTerms, int kSrc, bool kNear, int kTiles, int kWaves>
static __device__ __forceinline__ void whole_work(const SharedAttnLaunch &a, const PlanItem &it, SharedLds<kWaves> &l,
                                                  int layer, int g, int tid, int wave) {
    const int lane = tid & 63, n16 = lane & 15, c4 = lane >> 4;
    const int rows = it.n_seq * a.G;
    const PlanSeq *seqs = reinterpret_cast<const PlanSeq *>(a.plan + sizeof(PlanHeader)) + it.seq0;
    int rest = 0, state = 1;
    if (lane < it.n_seq) {
        rest = seqs[lane].rest;
        state = seqs[lane].state;
    }
    if (tid == 0) l.bad = 0;
    __syncthreads();
    if (wave == 0) {
        const uint64_t invalid = __ballot(state == 2), gone = __ballot(state == 0);
        if (lane == 0) {
            if (invalid) atomicOr(&l.bad, invalid);
            l.gone = gone;
        }
    }
    const int passes = (rest + kWaveTile - 1) / kWaveTile;
    int upto = passes;
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
        const int y = __shfl_up(upto, x);
        upto += lane >= x ? y : 0;
    }
    const int pre = (it.r1 + kWaveTile - 1) / kWaveTile;
    WholeLists feed{it.list, it.seq0, it.n_seq, it.r1, pre, pre + __builtin_amdgcn_readlane(upto, 63), wave, kWaves, rest,
                    upto - passes};
    u32x4 qf[kTiles][4];
    int row_seq[kTiles];
    WaveAcc w[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) start_rows(w[t]);
    const float scale = run_passes<kTerms, kSrc, kNear, kTiles>(
        a, layer, g, it.stream, feed, l.stages[wave], l.slots[wave], qf,
        [&] { load_item_queries<kTiles>(a, it, layer, g, n16, c4, qf, row_seq); }, row_seq, w, lane,
        [&](const Pass &p) {
            if (lane == 0) {
                atomicOr(&l.bad, p.only < 0 ? ~0ull : 1ull << p.only);
                raise_device_error(MURMUR_DEVERR_POSITION);
            }
        });
    const auto store = [&](int t0, int n_tiles) {
        const uint64_t bad = l.bad, gone = l.gone;
#pragma unroll 1
        for (int j = tid >> 5; j < min(16 * n_tiles, rows - 16 * t0); j += kWaves * 2) {
            const uint32_t rr = (uint32_t)(16 * t0 + j), s = div16(rr, a.magic_g);
            if (gone >> s & 1) continue;
            float M, L;
            f32x4 O;
            gather_row<kWaves>(l, 0, kWaves, j, tid & 31, M, L, O);
            if (bad >> s & 1) L = __builtin_nanf("");
            store_row(a, ((int64_t)layer * a.B + it.seq0 + (int)s) * a.Hq + g * a.G + (int)(rr - s * (uint32_t)a.G), tid & 31,
                      O, M, L);
        }
    };
    constexpr int kFirstTiles = kTiles < 2 ? 1 : 2;
    publish_tiles<0, kFirstTiles>(l, w, scale, wave, n16, c4);
    __syncthreads();
    store(0, kFirstTiles);
    if constexpr (kTiles > 2) {
        __syncthreads();  // the rows of the tiles before are read
        publish_tiles<2, 1>(l, w, scale, wave, n16, c4);
        __syncthreads();
        store(2, 1);
    }
}

template <int kTerms, int kSrc, bool kNear, int kWaves>
__global__ __launch_bounds__(kWaves * 64, 2) void shared_whole_kernel(const SharedAttnLaunch a) {
    __shared__ __attribute__((aligned(16))) SharedLds<kWaves> l;
    const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), i = blockIdx.y;
    const PlanHeader h = *reinterpret_cast<const PlanHeader *>(a.plan);
    const PlanItem it = reinterpret_cast<const PlanItem *>(a.plan + a.item_offset)[i];
    materialize(h.magic, h.n_work, it.seq0, it.n_seq, it.list, it.r1, it.stream);
    if (!plan_fits(a, h)) {  // every output is NaN
        const int64_t rows = (int64_t)a.NL * a.B * a.Hq, step = (int64_t)gridDim.x * gridDim.y * (kWaves * 2);
        const float nan = __builtin_nanf("");
        for (int64_t row = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * (kWaves * 2) + (tid >> 5); row < rows; row += step)
            store_row(a, row, tid & 31, f32x4{nan, nan, nan, nan}, nan, nan);
        if (blockIdx.x == 0 && i == 0 && tid == 0) raise_device_error(MURMUR_DEVERR_GROUP);
        return;
    }
    if (i >= h.n_work) return;
    const int layer = (int)blockIdx.x / a.Hkv, g = (int)blockIdx.x - layer * a.Hkv;
    const int rows = it.n_seq * a.G;
    if (rows <= 16)
        whole_work<kTerms, kSrc, kNear, 1, kWaves>(a, it, l, layer, g, tid, wave);
    else if (rows <= 32)
        whole_work<kTerms, kSrc, kNear, 2, kWaves>(a, it, l, layer, g, tid, wave);
    else
        whole_work<kTerms, kSrc, kNear, 3, kWaves>(a, it, l, layer, g, tid, wave);
}

// kPer half wavefronts per query row, each folding every kPer-th partial: the pairs
// of all of them, one per lane, 32 at a time, then the rows of its own, four head
// dims per lane, kMergeBatch loads in flight.
template <int kPer>
__global__ __launch_bounds__(256) void shared_merge_kernel(const SharedAttnLaunch a) {
    __shared__ f32x4 s_o[kPer > 1 ? 8 : 1][32];
    const PlanHeader h = *reinterpret_cast<const PlanHeader *>(a.plan);
    const int lane = threadIdx.x & 31, who = (threadIdx.x >> 5) % kPer;
    const int64_t n_rows = (int64_t)a.NL * a.B * a.Hq;
    const int64_t row = min((int64_t)blockIdx.x * (8 / kPer) + (threadIdx.x >> 5) / kPer, n_rows - 1);
    const int64_t lb = row / a.Hq;
    const int hq = (int)(row - lb * a.Hq), layer = (int)(lb / a.B), b = (int)(lb - (int64_t)layer * a.B);
    const int g = (int)div16((uint32_t)hq, a.magic_g), hh = hq - g * a.G;
    PlanSeq s = reinterpret_cast<const PlanSeq *>(a.plan + sizeof(PlanHeader))[b];
    if (!plan_fits(a, h)) {
        s.state = 2;
        if (row == 0 && threadIdx.x == 0) raise_device_error(MURMUR_DEVERR_GROUP);
    }
    float M = kNegInf, L = s.state == 1 ? 0.f : __builtin_nanf("");
    f32x4 O = {0.f, 0.f, 0.f, 0.f};
    const int n = s.state == 1 ? s.n_pre + s.n_rest : 0;
    const int64_t base = ((int64_t)layer * a.Hkv + g) * h.rows + hh;
    const auto row_of = [&](int i) {
        return base + (i < s.n_pre ? s.pre_row + i * s.pre_stride : s.rest_row + (i - s.n_pre) * a.G);
    };
    f32x4 o[kMergeBatch];
    const auto load_rows = [&](int i0, int i, int here) {
#pragma unroll
        for (int j = 0; j < kMergeBatch; ++j) {
            const int x = i + j * kPer;
            o[j] = *reinterpret_cast<const f32x4 *>(a.part_o + row_of(i0 + (x < here ? x : 0)) * kHeadDim + 4 * lane);
        }
    };
    for (int i0 = 0; i0 < n; i0 += 32) {
        const int here = min(32, n - i0);
        float2 ml = {kNegInf, 0.f};
        if (lane < here) ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * row_of(i0 + lane));
        load_rows(i0, who, here);
        float top = ml.x;
#pragma unroll
        for (int x = 16; x >= 1; x /= 2) top = fmaxf(top, __shfl_xor(top, x, 32));
        top = fmaxf(top, M);
        const float before = M == kNegInf ? 0.f : __builtin_amdgcn_exp2f(M - top);
        const float weight = ml.x == kNegInf && ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
        float total = ml.y * weight;
#pragma unroll
        for (int x = 16; x >= 1; x /= 2) total += __shfl_xor(total, x, 32);
        L = L * before + total;
        O *= before;
        M = top;
        for (int i = who; i < here; i += kPer * kMergeBatch) {
            if (i != who) load_rows(i0, i, here);
#pragma unroll
            for (int j = 0; j < kMergeBatch; ++j) {
                const int x = i + j * kPer;
                const float f = __shfl(weight, x & 31, 32);
                O += o[j] * (x < here ? f : 0.f);
            }
        }
    }
    if constexpr (kPer > 1) {
        s_o[threadIdx.x >> 5][lane] = O;
        __syncthreads();
        if (who != 0) return;
        const int first = threadIdx.x >> 5;
#pragma unroll
        for (int x = 1; x < kPer; ++x) O += s_o[first + x][lane];
    }
    if (s.state == 0 || (int64_t)blockIdx.x * (8 / kPer) + (threadIdx.x >> 5) / kPer >= n_rows) return;
    store_row(a, row, lane, O, M, L);
}

// ---- launchers ----

int launch_shared_plan(const SharedPlanLaunch &call, murmur_stream_t stream) {
    SharedPlanLaunch p = call;
    if (p.find && (int64_t)p.B * p.max_keep <= kFindHereEntries) {
        p.find = kFindHere;
    } else if (p.find) {
        hipLaunchKernelGGL(shared_scan_kernel, dim3((unsigned)p.caps.n_scan, (unsigned)p.B), dim3(kScanThreads), 0,
                           (hipStream_t)stream, p.idx, p.count, p.group, p.n_groups, p.max_keep, p.B,
                           reinterpret_cast<int32_t *>(p.plan + p.caps.scan_offset));
        const int e = (int)hipGetLastError();
        if (e != 0) return e;
    }
    // small batches take fewer wavefronts through the barriers
    if (p.B <= 256 && p.n_groups <= 256)
        hipLaunchKernelGGL(shared_plan_kernel<256>, dim3(1), dim3(256), 0, (hipStream_t)stream, p);
    else
        hipLaunchKernelGGL(shared_plan_kernel<1024>, dim3(1), dim3(1024), 0, (hipStream_t)stream, p);
    return (int)hipGetLastError();
}

template <int kTerms, int kSrc, bool kNear>
static void launch_shared_attn_near(const SharedAttnLaunch &a, hipStream_t stream) {
    const dim3 grid((unsigned)(a.NL * a.Hkv), (unsigned)a.n_wg);
    if (a.waves == 8)
        hipLaunchKernelGGL((shared_whole_kernel<kTerms, kSrc, kNear, 8>), grid, dim3(8 * 64), 0, stream, a);
    else if (a.waves == 4)
        hipLaunchKernelGGL((shared_whole_kernel<kTerms, kSrc, kNear, 4>), grid, dim3(4 * 64), 0, stream, a);
    else
        hipLaunchKernelGGL((shared_attn_kernel<kTerms, kSrc, kNear>), grid, dim3(kSharedThreads), 0, stream, a);
}

template <int kTerms>
static void launch_shared_attn(const SharedAttnLaunch &a, hipStream_t stream) {
    // rows of at least 256 bytes (one if the cache has one row) within 2^32: positions below 2^24
    const bool near = a.s_pos < kRunRowLimit && (a.s_pos >= kHeadDim || a.max_len == 1) &&
                      (__int128)(a.max_len - 1) * a.s_pos * 2 + kTileRowBytes < ((__int128)1 << 32);
    if (a.ranges && near) launch_shared_attn_near<kTerms, kSrcRanges, true>(a, stream);
    else if (a.ranges) launch_shared_attn_near<kTerms, kSrcRanges, false>(a, stream);
    else if (near) launch_shared_attn_near<kTerms, kSrcIndex, true>(a, stream);
    else launch_shared_attn_near<kTerms, kSrcIndex, false>(a, stream);
}

int launch_decode_attn_shared(const SharedAttnLaunch &a, murmur_stream_t stream) {
    if (a.out_f32) launch_shared_attn<3>(a, (hipStream_t)stream);
    else launch_shared_attn<2>(a, (hipStream_t)stream);
    const int e = (int)hipGetLastError();
    if (e != 0 || a.waves > 0) return e;
    // Half wavefronts per row: as many as keep the rows' workgroups below two per compute unit; few rows have many
    // partials (a dispatch round's workgroups are shared out among them).
    const int64_t rows = (int64_t)a.NL * a.B * a.Hq;
    const dim3 threads(256);
    if (rows <= 2 * kRoundWorkgroups)
        hipLaunchKernelGGL(shared_merge_kernel<8>, dim3((unsigned)rows), threads, 0, (hipStream_t)stream, a);
    else if (rows <= 8 * kRoundWorkgroups)
        hipLaunchKernelGGL(shared_merge_kernel<2>, dim3((unsigned)((rows + 3) / 4)), threads, 0, (hipStream_t)stream, a);
    else
        hipLaunchKernelGGL(shared_merge_kernel<1>, dim3((unsigned)((rows + 7) / 8)), threads, 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}

}  // namespace murmur
