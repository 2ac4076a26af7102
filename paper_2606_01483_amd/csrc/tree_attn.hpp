// Device code of the attention of trees of drafted tokens (included by kernels.hip).
//
//   tree_attn_kernel   the query rows of a tree (nodes x the heads of a KV head) over
//                      a part of what its nodes retain together
//   tree_merge_kernel  joins the parts by log-sum-exp
//
// What node t of depth d retains at its step out_len + d differs from node to node only
// where a window moves: at the two ends of the speech window, at the old end of the
// output window, and in the tree itself.  The cached positions that any node retains
// make one list, by rank: six pieces as in retained_pieces, the windows as long as the
// deepest node's step moves them, then the nodes.  A row leaves out at most three
// stretches of ranks
//   [a0, a0 + a)   speech that its window has left,
//   [b1 - b, b1)   speech that its window has not reached,
//   [c0, c0 + c)   outputs that its window has left,
// and the nodes that are not its ancestors (a bit each).  Only the passes that touch
// one of these stretches look at the rules.
#pragma once

namespace murmur {

struct TreeRule {
    int32_t a, b, c, depth;
    uint32_t lo, hi;  // the nodes that a node attends to
};

// One sequence's list: the cached pieces, then the nodes from rank n0 on.
struct TreeList {
    RangeTab tab;
    int32_t n0, count;
    int32_t a0, a_most, b1, b_most, c0, c_most;
    int32_t live;       // nodes up to the last that is there
    uint64_t there;
    int32_t err;        // device error bits of the layout, policy or tree
};

// The tree of a sequence by one wavefront, lane i for node i, and the list.
static __device__ __forceinline__ TreeList tree_list(const murmur_seg &s, const murmur_policy &p,
                                                     const int32_t *__restrict__ parent, int T, int lane, TreeRule &rule) {
    TreeList l{};
    int par = lane < T ? parent[lane] : -2;
    const uint64_t there = __ballot(par != -2);
    l.there = there;
    l.live = there ? 64 - __builtin_clzll(there) : 0;
    const bool ok = par == -2 || (lane == 0 ? par == -1 : par >= 0 && par < lane && (there >> (par & 63) & 1));
    if (__ballot(!ok)) l.err |= MURMUR_DEVERR_TREE;
    // ancestors and itself, twice as far up in every round
    uint64_t up = 1ull << lane;
    int hop = ok && par >= 0 ? par : lane;
    for (int reach = 1; reach < T; reach *= 2) {
        const uint32_t lo = __shfl((uint32_t)up, hop), hi = __shfl((uint32_t)(up >> 32), hop);
        up |= (uint64_t)hi << 32 | lo;
        hop = __shfl(hop, hop);
    }
    const int depth = __popcll(up) - 1;
    const int deepest = wave_max(par != -2 ? depth : 0);
    const int32_t pre = s.prompt_pre, ls = s.speech_len, mid = s.prompt_mid, j = s.out_len;
    if (!layout_valid(pre, ls, mid, j, p.speech_window, p.speech_delay, p.speech_sink, p.out_window, p.out_sink) ||
        (int64_t)pre + ls + mid + j + 64 > 0x7fffffffLL)
        l.err |= MURMUR_DEVERR_POLICY;
    if (l.err) return l;

    const int32_t ws = p.speech_window, wo = p.out_window;
    const int32_t first = p.speech_delay > 1 ? p.speech_delay : 1;
    const int32_t ns = min(p.speech_sink, ls), c = j - 1;
    int32_t rg[2 * kPieces];
    rg[0] = 0;
    rg[1] = pre;
    rg[2] = pre;
    rg[3] = ls;
    rg[4] = pre + ls;
    rg[5] = 0;
    int32_t from = 0, most = 0;  // first speech token behind the sinks that any node retains; the window's last start
    const bool moves = ws != -1 && ws < ls;
    const auto start = [&](int e) { return max(0, min(j + e - first + 1, ls - ws)); };
    if (moves) {
        const int32_t l0 = start(0);
        most = start(deepest);
        from = max(l0, ns);
        if (l0 > ns) {
            rg[3] = ns;
            rg[4] = pre + l0;
            rg[5] = most + ws - l0;
        } else {
            rg[3] = max(ns, most + ws);
        }
        rule.a = max(start(depth), from) - from;
        rule.b = max(ns, most + ws) - max(ns, start(depth) + ws);
        l.a_most = max(most, from) - from;  // the deepest node's
        l.b_most = max(ns, most + ws) - max(ns, l0 + ws);  // the root's
    } else {
        rule.a = rule.b = 0;
    }
    rg[6] = pre + ls;
    rg[7] = mid;
    const int32_t out0 = pre + ls + mid, sinks = min(p.out_sink, c);
    rg[8] = out0;
    rg[9] = c;
    rg[10] = out0 + c;
    rg[11] = 0;
    rule.c = 0;
    if (wo != -1) {
        const int32_t base = min(max(p.out_sink, j - wo), c);
        if (j - wo > p.out_sink) {
            rg[9] = sinks;
            rg[10] = out0 + base;
            rg[11] = c - base;
        }
        rule.c = max(0, min(j + depth - wo, c) - base);
        l.c_most = max(0, min(j + deepest - wo, c) - base);
        if (wo <= deepest) {  // ancestors that the output window has left, unless they are sinks
            uint64_t near = 1ull << lane;
            const int to = par >= 0 ? par : lane;
            int above = to;
            for (int e = 1; e < wo; ++e) {
                near |= 1ull << above;
                above = __shfl(to, above);
            }
            up &= near | __ballot(c + depth < p.out_sink);
        }
    }
    rule.depth = depth;
    rule.lo = (uint32_t)up;
    rule.hi = (uint32_t)(up >> 32);
    l.tab = make_tab(rg);
    l.a0 = pre + ns;
    l.b1 = pre + rg[3] + rg[5];
    l.c0 = l.b1 + mid + sinks;
    l.n0 = l.b1 + mid + rg[9] + rg[11];
    if (l.n0 > 0x7fffffff - kMaxNodes - kWaveTile) l.err |= MURMUR_DEVERR_POLICY;  // ranks, to the end of the last pass, are 32 bits
    l.count = l.n0 + l.live;
    return l;
}

// The ranks r0 .. r0 + 31 that a row attends to, a bit each.
static __device__ __forceinline__ uint32_t tree_allows(const TreeList &l, const TreeRule &x, int r0) {
    const auto below = [](int n) { return (uint32_t)((1ull << min(max(n, 0), 32)) - 1); };  // ranks before r0 + n
    const auto stretch = [&](int from, int to) { return below(to - r0) & ~below(from - r0); };
    const uint32_t out = stretch(l.a0, l.a0 + x.a) | stretch(l.b1 - x.b, l.b1) | stretch(l.c0, l.c0 + x.c);
    const uint64_t nodes = (uint64_t)x.hi << 32 | x.lo;
    const int n = r0 - l.n0;
    // bits of nodes past the last are clear, which masks the list's end too
    const uint32_t in = n >= 0 ? (n < 64 ? (uint32_t)(nodes >> n) : 0u) : (uint32_t)(nodes << min(-n, 63)) | below(-n);
    return in & ~out;
}

// Rows of a pass for each lane: kTreeRows ranks four apart, as cache rows (>= 0) or
// ~node; ~0, the root's, wherever none is to be read.
constexpr int kTreeRows = 4;  // of a lane in a half pass of 16 rows
struct TreeRows {
    int32_t pos[kTreeRows], entry[kTreeRows];
    bool plain;  // uniform: consecutive cached positions, all within the table
    // positions, and the block table's entries on their way
    __device__ __forceinline__ void begin(const TreeList &l, const TreeLaunch &a, const int32_t *bt_row, int r0, int c4) {
        int p0;
        plain = r0 + 16 <= l.n0 && tab_run(l.tab, r0, 16, a.max_pos, p0);
        if (plain) {
#pragma unroll
            for (int i = 0; i < kTreeRows; ++i) pos[i] = p0 + 4 * i + c4;
        } else {
#pragma unroll
            for (int i = 0; i < kTreeRows; ++i) {
                const int r = r0 + 4 * i + c4;
                int piece;
                const int p = tab_pos(l.tab, r, piece);
                pos[i] = r < l.n0 ? p : (r < l.count ? ~(r - l.n0) : ~0);
            }
        }
        if (bt_row) {  // uniform
#pragma unroll
            for (int i = 0; i < kTreeRows; ++i)
                entry[i] = bt_row[plain ? pos[i] >> a.log2_bs : min(max(pos[i], 0) >> a.log2_bs, a.max_blocks - 1)];
        }
    }
    // cache rows; a position that has none is an error and becomes the root's row
    __device__ __forceinline__ void finish(const TreeLaunch &a, const int32_t *bt_row, int &err) {
        if (plain && !bt_row) return;
        const uint32_t last = (uint32_t)(a.max_len - 1), last_block = last >> a.log2_bs, in_block = (1u << a.log2_bs) - 1;
        uint32_t row[kTreeRows];
        bool wrong[kTreeRows], any = false;
#pragma unroll
        for (int i = 0; i < kTreeRows; ++i) {
            row[i] = (uint32_t)pos[i];
            wrong[i] = false;
            if (bt_row) {
                row[i] = (uint32_t)entry[i] << a.log2_bs | (row[i] & in_block);
                wrong[i] = ((uint32_t)entry[i] > last_block) | (!plain & (pos[i] >> a.log2_bs >= a.max_blocks));
            }
            wrong[i] = (wrong[i] | (row[i] > last)) & (plain | (pos[i] >= 0));
            any |= wrong[i];
        }
        if (plain && __builtin_expect(__ballot(any) == 0, 1)) {
#pragma unroll
            for (int i = 0; i < kTreeRows; ++i) pos[i] = (int32_t)row[i];
            return;
        }
        plain = false;
#pragma unroll
        for (int i = 0; i < kTreeRows; ++i) {
            if (wrong[i])
                err |= bt_row && (entry[i] < 0 || pos[i] >> a.log2_bs >= a.max_blocks) ? MURMUR_DEVERR_BLOCK : MURMUR_DEVERR_POSITION;
            pos[i] = wrong[i] ? ~0 : (pos[i] >= 0 ? (int32_t)row[i] : pos[i]);
        }
    }
};

// The values of a pass that some rows leave out: zero times an infinity or a NaN is
// NaN, so where the values hold one (the product with zeros tells), those are added
// to the sums of the rows that attend to them, whose result is not finite there
// whatever their weights, and taken out of the operands.
template <int kTiles>
static __device__ __forceinline__ void tree_keep_apart(u32x2 (&vf)[16], const uint8_t *tile, const uint32_t (&allows)[kTiles],
                                                       WaveAcc (&w)[kTiles], int lane) {
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
#pragma unroll 1
        for (int r = 0; r < kWaveTile; ++r) {
            u32x2 e = *reinterpret_cast<const u32x2 *>(tile + r * kTileRowBytes + (((2 * db + (c4 >> 1)) ^ (r & 15)) << 4) +
                                                       8 * (c4 & 1));
#pragma unroll
            for (int i = 0; i < 2; ++i) e[i] &= not_finite(e[i]);
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                const bool mine = allows[t] >> r & 1;
#pragma unroll
                for (int i = 0; i < 2; ++i) {
                    w[t].acc[db][2 * i] += mine ? __builtin_bit_cast(float, e[i] << 16) : 0.f;
                    w[t].acc[db][2 * i + 1] += mine ? __builtin_bit_cast(float, e[i] & 0xffff0000u) : 0.f;
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int x = 0; x < 2; ++x) vf[i][x] &= ~not_finite(vf[i][x]);
}

// Softmax update of a pass for all row tiles, as softmax_pass, but the running max of
// a row follows only where a logit exceeds it by more than kTreeLag (in log2 units of
// the weight): weights are then at most 2^kTreeLag, which costs their sums in fp32 and
// their bf16 parts nothing, and after a list's first passes next to no pass rescales.
constexpr float kTreeLag = 8.f;
template <int kTerms, int kTiles>
static __device__ __forceinline__ void tree_softmax(const f32x4 (&s)[kTiles][2], float scale, WaveAcc (&w)[kTiles],
                                                    u32x4 (&p)[kTiles][kTerms]) {
    float top[kTiles];
    bool rises = false;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        top[t] = fmaxf(fmaxf(fmaxf(s[t][0][0], s[t][0][1]), fmaxf(s[t][0][2], s[t][0][3])),
                       fmaxf(fmaxf(s[t][1][0], s[t][1][1]), fmaxf(s[t][1][2], s[t][1][3])));
        rises |= (top[t] - w[t].m_run) * scale > kTreeLag;
    }
    if (__ballot(rises)) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const float m_new = fmaxf(w[t].m_run, max_over_c4(top[t]));
            const float alpha = __builtin_amdgcn_exp2f((w[t].m_run - m_new) * scale);  // 0 while the state is empty
            w[t].l_run *= alpha;
#pragma unroll
            for (int db = 0; db < 8; ++db) w[t].acc[db] *= alpha;
            w[t].m_run = m_new;
        }
    }
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        float pr[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) pr[i] = __builtin_amdgcn_exp2f((s[t][i >> 2][i & 3] - w[t].m_run) * scale);
        w[t].l_run += ((pr[0] + pr[1]) + (pr[2] + pr[3])) + ((pr[4] + pr[5]) + (pr[6] + pr[7]));
#pragma unroll
        for (int wd = 0; wd < 4; ++wd) {
            float e0 = pr[2 * wd], e1 = pr[2 * wd + 1];
#pragma unroll
            for (int k = 0; k < kTerms; ++k) {
                p[t][k][wd] = pack_bf16(e0, e1);
                e0 -= __builtin_bit_cast(float, p[t][k][wd] << 16);
                e1 -= __builtin_bit_cast(float, p[t][k][wd] & 0xffff0000u);
            }
        }
    }
}

// Normalised output of four head dims of a row, and the lse (c == 0).
static __device__ __forceinline__ void tree_store(const TreeLaunch &a, int64_t row, int c, f32x4 O, float M, float L) {
    const float inv = 1.f / L;
    if (a.out_f32)
        *reinterpret_cast<f32x4 *>(reinterpret_cast<float *>(a.out) + row * kHeadDim + 4 * c) = O * inv;
    else
        *reinterpret_cast<u32x2 *>(reinterpret_cast<uint16_t *>(a.out) + row * kHeadDim + 4 * c) =
            u32x2{pack_bf16(O[0] * inv, O[1] * inv), pack_bf16(O[2] * inv, O[3] * inv)};
    if (c == 0 && a.lse) a.lse[row] = (M + __builtin_log2f(L)) * 0.69314718055994530942f;
}

// ---------------------------------------------------------------------------
// Workgroup: up to 128 query rows of one (layer, sequence, KV head) over one split of
// the list.  Its wavefronts take the list kWaves / 2 passes (a round) at a time:
// together they load a round's rows into one of two buffers while they compute the
// other.  They are `ways` ways by rows and the rest by passes, as the rows that are
// there ask for; groups by passes are joined by way of LDS at the end.
// Large trees are bound by the vector and matrix units: 64 trees of 64 nodes over 2000
// rows, two layers, 489 to 500 us, 488 to 477 TFLOP/s (an 8192^3 product reaches 1102), where a pass
// of two row tiles is 212 vector and 48 matrix instructions, a third of these for the
// weights' second part.  One tile a wavefront reads K and V from LDS twice as often (64
// chunks of 64 nodes 807 us, 612 with two); three, at two wavefronts a SIMD, do not fit
// the registers.  Small ones are bound by latency: of 10 us (16 nodes, 160 rows,
// clocked in an earlier form) 3.4 pass before the first rows are on their way (layout,
// policy and tree; the table's entries; code that is fetched), 0.8 before they are
// there, 4.5 in six passes, 0.9 in the outputs.  The table's row in LDS, loaded at the
// start, gained nothing, and loads that pass the L2s by cost 7 to 9 % of the 64 chunks
// of 64 nodes.  A raised wavefront priority around the values' products: 31 nodes over
// 35 000 rows 2 % faster, the others 0.5 to 2 % slower.
// ---------------------------------------------------------------------------
template <int kWaves>
struct TreeLds {
    uint8_t stages[2][kWaves / 2][kStageBytes];
    TreeRule rule[64];
    float2 ml[kWaves][2][64];
    int err;
};

template <int kTerms, int kTiles, int kWaves>
__global__ __launch_bounds__(kWaves * 64, 2) void tree_attn_kernel(const TreeLaunch a) {
    constexpr int kAll = 128, kThreads = kWaves * 64, kRound = kWaves / 2;
    static_assert(kAll <= kWaves * kTiles * 16, "a wavefront's tiles for all rows");
    __shared__ __attribute__((aligned(16))) TreeLds<kWaves> lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n16 = lane & 15, c4 = lane >> 4;
    // The workgroups of one split's row sets follow each other on one XCD.  An XCD's go to its shader engines in turn,
    // so the sets start with another one for every split: otherwise (with as many sets as engines) one engine has every
    // first set, and another every last one, where trees of few nodes have no rows.
    const int x = blockIdx.x, eight = a.by_sets(x >> 3), turned = (x >> 3) - eight * a.row_sets + eight;
    const int set = turned - a.by_sets(turned) * a.row_sets, unit = eight * 8 + (x & 7);
    if (unit >= a.units) return;
    const int group = a.by_split(unit), split = unit - group * a.n_split;
    const int lb = a.by_heads(group), g = group - lb * a.Hkv, layer = a.by_batch(lb), b = lb - layer * a.B;
    const murmur_seg s = reinterpret_cast<const murmur_seg *>(a.seg)[b];
    const int rec = ((a.pol_mode & MURMUR_POL_PER_LAYER) ? layer * ((a.pol_mode & MURMUR_POL_PER_SEQ) ? a.B : 1) : 0) +
                    ((a.pol_mode & MURMUR_POL_PER_SEQ) ? b : 0);
    const murmur_policy p = reinterpret_cast<const murmur_policy *>(a.pol)[rec];
    TreeRule mine{};
    const TreeList l = tree_list(s, p, a.parent + (a.parent_per_seq ? (int64_t)b * a.T : 0), a.T, lane, mine);
    if (layout_absent(s.prompt_pre, s.speech_len, s.prompt_mid, s.out_len)) return;
    const int row0 = set * kAll, rows_live = l.live * a.G;
    if (row0 >= rows_live) return;
    const int wanted = (min(rows_live - row0, kAll) + 16 * kTiles - 1) / (16 * kTiles);
    const int ways = wanted <= 1 ? 1 : wanted <= 2 ? 2 : wanted <= 4 ? 4 : 8, groups = min(kWaves / ways, kRound);
    const int way = wave & (ways - 1), grp = wave / ways;
    // the lane's row of every tile
    int node[kTiles], row[kTiles];
    u32x4 qf[kTiles][4];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        row[t] = row0 + (way * kTiles + t) * 16 + n16;
        const int r = min(row[t], a.T * a.G - 1);
        node[t] = (int)((uint32_t)r * a.magic_g >> 16);
        const uint16_t *q = a.q + ((((int64_t)lb * a.T + node[t]) * a.Hq + g * a.G + r - node[t] * a.G) * kHeadDim + 8 * c4);
#pragma unroll
        for (int kc = 0; kc < 4; ++kc) qf[t][kc] = load16(q + 32 * kc);
    }
    const int passes = l.err ? 0 : (l.count + kWaveTile - 1) / kWaveTile;
    const int p0 = (int)((int64_t)passes * split / a.n_split), p1 = (int)((int64_t)passes * (split + 1) / a.n_split);
    const int rounds = (p1 - p0 + kRound - 1) / kRound;
    const int32_t *bt_row = a.bt ? a.bt + (int64_t)b * a.max_blocks : nullptr;
    const int64_t cache_at = layer * a.s_layer + b * a.s_b + g * a.s_h;
    const uint16_t *kc = a.k + cache_at, *vc = a.v + cache_at;
    const int64_t tree_at = ((int64_t)lb * a.T * a.Hkv + g) * kHeadDim;
    // this wavefront loads the half `wave & 1` of a round's pass `wave >> 1`
    const int half = wave & 1, chunk = 16 * (n16 ^ c4);
    const uint32_t row_bytes = (uint32_t)a.s_pos * 2u;
    int err = 0;
    TreeRows rows;
    const auto mine_in = [&](int it) { return p0 + it * kRound + (wave >> 1) < p1; };
    if (wave == 0) lds.rule[lane] = mine;
    if (tid == 0) {
        lds.err = l.err;
        if (l.err) raise_device_error(l.err);
    }
    float scale = 1.f;  // of the softmax, set with the queries' sign before the first pass
    WaveAcc w[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) start_rows(w[t]);
    const bool idle = grp >= groups || row0 + way * kTiles * 16 >= rows_live;  // uniform: a wavefront without rows
    // Step `it` looks up the rows of round it + 2, loads round it + 1 and computes round it, so that there is one copy
    // of each part's code: fetching it costs a short launch more than running it.
#pragma unroll 1
    for (int it = -2; it < rounds; ++it) {
        if (it >= 0) {
            wait_vm<0>();
            asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // the round's rows are in, and the other buffer is read
        }
        if (it >= -1 && mine_in(it + 1)) {
            rows.finish(a, bt_row, err);
            uint8_t *stage = lds.stages[(it + 1) & 1][wave >> 1] + 4096 * half;
            if (rows.plain && a.near_rows) {  // uniform: offsets of 32 bits, the same for K and V, from scalar bases
                uint32_t at[kTreeRows];
#pragma unroll
                for (int i = 0; i < kTreeRows; ++i)
                    at[i] = __umul24((uint32_t)rows.pos[i], row_bytes) + (uint32_t)(chunk ^ 64 * i);
#pragma unroll
                for (int i = 0; i < kTreeRows; ++i) {
                    __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint8_t *>(kc) + at[i], (lds_void_t *)(stage + i * 1024), 16, 0, 0);
                    __builtin_amdgcn_global_load_lds(reinterpret_cast<const uint8_t *>(vc) + at[i],
                                                     (lds_void_t *)(stage + kTileBytes + i * 1024), 16, 0, 0);
                }
                asm volatile("" ::: "memory");  // the two paths' last loads are not one load of a 64-bit address
            } else {
#pragma unroll
                for (int i = 0; i < kTreeRows; ++i) {
                    const bool node_row = rows.pos[i] < 0;
                    const int64_t at = (node_row ? tree_at + (int64_t)~rows.pos[i] * (a.Hkv * kHeadDim) : rows.pos[i] * a.s_pos) +
                                       (chunk ^ 64 * i) / 2;
                    __builtin_amdgcn_global_load_lds((node_row ? a.k_tree : kc) + at, (lds_void_t *)(stage + i * 1024), 16, 0, 0);
                    __builtin_amdgcn_global_load_lds((node_row ? a.v_tree : vc) + at, (lds_void_t *)(stage + kTileBytes + i * 1024),
                                                     16, 0, 0);
                }
            }
        }
        if (mine_in(it + 2)) rows.begin(l, a, bt_row, (p0 + (it + 2) * kRound + (wave >> 1)) * kWaveTile + 16 * half, c4);
        if (it < 0) continue;
        if (it == 0) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t) scale = signed_scale(qf[t], a.scale_log2);
        }
        if (idle) continue;
#pragma unroll 1
        for (int i = grp; i < kRound; i += groups) {
            const int pass = p0 + it * kRound + i, r0 = pass * kWaveTile;
            if (pass >= p1) break;
            const uint8_t *stage = lds.stages[it & 1][i];
            u32x4 kf[8];
            read_k_operands(kf, lds_addr(stage), n16, c4);
            const int r1 = r0 + kWaveTile;
            const bool ruled = r1 > l.n0 || (r1 > l.a0 && r0 < l.a0 + l.a_most) || (r1 > l.b1 - l.b_most && r0 < l.b1) ||
                               (r1 > l.c0 && r0 < l.c0 + l.c_most);
            u32x4 pr[kTiles][kTerms];
            uint32_t allows[kTiles];
            f32x4 sc[kTiles][2];
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int blk = 0; blk < 2; ++blk) {
                    sc[t][blk] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                    for (int kk = 0; kk < 4; ++kk) sc[t][blk] = mfma16x16x32(kf[4 * blk + kk], qf[t][kk], sc[t][blk]);
                }
            if (ruled) {
                asm volatile("");  // a branch, which few passes take
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    allows[t] = tree_allows(l, lds.rule[node[t]], r0);
                    const uint32_t mine = allows[t] >> (4 * c4);
#pragma unroll
                    for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                        for (int e = 0; e < 4; ++e) sc[t][blk][e] = mine & (1u << (16 * blk + e)) ? sc[t][blk][e] : kNegInf;
                }
            }
            tree_softmax<kTerms, kTiles>(sc, scale, w, pr);
            u32x2 vf[16];
            read_v_operands(vf, lds_addr(stage + kTileBytes), n16, c4);
            if (ruled) tree_keep_apart<kTiles>(vf, stage + kTileBytes, allows, w, lane);
#pragma unroll
            for (int k = 0; k < kTerms; ++k)  // a sum's products apart, since each waits for the one before
#pragma unroll
                for (int db = 0; db < 8; ++db)
#pragma unroll
                    for (int t = 0; t < kTiles; ++t)
                        w[t].acc[db] = mfma16x16x32(u32x4{vf[2 * db][0], vf[2 * db][1], vf[2 * db + 1][0], vf[2 * db + 1][1]},
                                                    pr[t][k], w[t].acc[db]);
        }
    }
    if (__ballot(err != 0)) {
        if (err) {
            raise_device_error(err);
            atomicOr(&lds.err, err);
        }
    }
    __syncthreads();
    const bool bad = lds.err != 0;

    // The groups' states by way of the buffers, register by register: a lane's share of a row's sum, its part of O and
    // the row's max stand in the same lane of every group.
    const int groups_here = min(groups, p1 - p0);  // those that had a pass
    if (groups_here > 1) {
        constexpr int kWords = 8 * kTiles;
        f32x4 *o = reinterpret_cast<f32x4 *>(&lds.stages[0][0][0]);
        static_assert(sizeof(lds.stages) >= kWaves * kWords * 64 * sizeof(f32x4), "the sums of every wavefront");
        if (grp > 0 && grp < groups_here) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t) {
                lds.ml[wave][t][lane] = float2{w[t].m_run, w[t].l_run};
#pragma unroll
                for (int db = 0; db < 8; ++db) o[(wave * kWords + 8 * t + db) * 64 + lane] = w[t].acc[db];
            }
        }
        __syncthreads();
        if (grp == 0) {
#pragma unroll 1
            for (int e = 1; e < groups_here; ++e) {
                const int wv = e * ways + way;
#pragma unroll
                for (int t = 0; t < kTiles; ++t) {
                    const float2 ml = lds.ml[wv][t][lane];
                    const float m = fmaxf(w[t].m_run, ml.x);
                    const float f0 = __builtin_amdgcn_exp2f((w[t].m_run - m) * scale), f1 = __builtin_amdgcn_exp2f((ml.x - m) * scale);
                    w[t].l_run = w[t].l_run * f0 + ml.y * f1;
#pragma unroll
                    for (int db = 0; db < 8; ++db)
                        w[t].acc[db] = w[t].acc[db] * f0 + o[(wv * kWords + 8 * t + db) * 64 + lane] * f1;
                    w[t].m_run = m;
                }
            }
        }
    }
    if (grp > 0) return;
    // rows to the outputs, or to the split's partials
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        float M = w[t].m_run * scale, L = sum_over_c4(w[t].l_run);
        if (bad) {
            M = 0.f;
            L = __builtin_nanf("");
        }
        const bool there = row[t] < rows_live && (l.there >> node[t] & 1);
        if (!there) continue;
        if (a.n_split > 1) {
            const int64_t at = ((int64_t)group * a.n_split + split) * (a.T * a.G) + row[t];
#pragma unroll
            for (int db = 0; db < 8; ++db)
                *reinterpret_cast<f32x4 *>(a.part_o + at * kHeadDim + 16 * db + 4 * c4) = w[t].acc[db];
            if (c4 == 0) *reinterpret_cast<float2 *>(a.part_ml + 2 * at) = float2{M, L};
        } else {
            const int64_t at = ((int64_t)lb * a.T + node[t]) * a.Hq + g * a.G + row[t] - node[t] * a.G;
#pragma unroll
            for (int db = 0; db < 8; ++db) tree_store(a, at, 4 * db + c4, w[t].acc[db], M, L);
        }
    }
}

// A row by 32 threads, four head dims each, kParts times: each takes every kParts-th
// split.  868 rows of 64 splits 7.4 us (29 MB of partials, the launch), 5376 of five 5.0.
template <int kParts>
__global__ __launch_bounds__(256) void tree_merge_kernel(const TreeLaunch a) {
    constexpr int kRows = 8 / kParts, kBatch = 8;
    __shared__ f32x4 s_o[kParts > 1 ? 8 : 1][32];
    __shared__ float2 s_ml[8];
    const int rows = a.T * a.G, slice = threadIdx.x >> 5, c = threadIdx.x & 31, part = slice / kRows;
    const int group = a.by_merge(blockIdx.x), r0 = ((int)blockIdx.x - group * a.merge_sets) * kRows;
    const int lb = a.by_heads(group), g = group - lb * a.Hkv, b = lb - a.by_batch(lb) * a.B;
    const int r = min(r0 + slice % kRows, rows - 1), n = (int)((uint32_t)r * a.magic_g >> 16);
    const murmur_seg s = reinterpret_cast<const murmur_seg *>(a.seg)[b];
    const int32_t parent = a.parent[(a.parent_per_seq ? (int64_t)b * a.T : 0) + n];
    float M = kNegInf, L = 0.f;
    f32x4 O = {0.f, 0.f, 0.f, 0.f};
    {  // of rows that are not there too: whatever the workspace holds is not stored
        const int64_t part0 = (int64_t)group * a.n_split * rows + r;
        for (int i0 = part; i0 < a.n_split; i0 += kBatch * kParts) {
            float2 ml[kBatch];
            f32x4 o[kBatch];
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {  // behind the last split: the last one again, which weighs nothing
                const int64_t p = part0 + (int64_t)min(i0 + j * kParts, a.n_split - 1) * rows;
                ml[j] = *reinterpret_cast<const float2 *>(a.part_ml + 2 * p);
                o[j] = *reinterpret_cast<const f32x4 *>(a.part_o + p * kHeadDim + 4 * c);
            }
            float m = M;
#pragma unroll
            for (int j = 0; j < kBatch; ++j) m = fmaxf(m, ml[j].x);
            const float f0 = M == kNegInf ? 0.f : __builtin_amdgcn_exp2f(M - m);
            L *= f0;
            O *= f0;
#pragma unroll
            for (int j = 0; j < kBatch; ++j) {
                const bool counts = i0 + j * kParts < a.n_split && ml[j].x != kNegInf;
                const float f = counts ? __builtin_amdgcn_exp2f(ml[j].x - m) : 0.f;
                L += counts ? ml[j].y * f : 0.f;
#pragma unroll
                for (int e = 0; e < 4; ++e) O[e] += counts ? o[j][e] * f : 0.f;
            }
            M = m;
        }
    }
    if constexpr (kParts > 1) {
        s_o[slice][c] = O;
        if (c == 0) s_ml[slice] = float2{M, L};
        __syncthreads();
        if (part > 0) return;
        float m = kNegInf;
#pragma unroll
        for (int e = 0; e < kParts; ++e) m = fmaxf(m, s_ml[e * kRows + slice].x);
        L = 0.f;
        O = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int e = 0; e < kParts; ++e) {
            const float2 ml = s_ml[e * kRows + slice];
            const float f = ml.x == kNegInf ? 0.f : __builtin_amdgcn_exp2f(ml.x - m);
            L += ml.y * f;
            O += f * s_o[e * kRows + slice][c];
        }
        M = m;
    }
    const bool there = parent != -2 && !layout_absent(s.prompt_pre, s.speech_len, s.prompt_mid, s.out_len);
    if (there && r0 + slice % kRows < rows) tree_store(a, ((int64_t)lb * a.T + n) * a.Hq + g * a.G + r - n * a.G, c, O, M, L);
}

template <int kTerms, int kTiles, int kWaves>
static int launch_tree_as(const TreeLaunch &a, hipStream_t stream) {
    const unsigned grid = (unsigned)((a.units + 7) / 8 * 8 * a.row_sets);
    hipLaunchKernelGGL((tree_attn_kernel<kTerms, kTiles, kWaves>), dim3(grid), dim3(kWaves * 64), 0, stream, a);
    return (int)hipGetLastError();
}

template <int kTerms>
static int launch_tree(const TreeLaunch &a, hipStream_t stream) {
    switch (a.shape) {
        case kTreeFew: return launch_tree_as<kTerms, 1, 8>(a, stream);
        case kTreeWide: return launch_tree_as<kTerms, 2, 8>(a, stream);
        default: return launch_tree_as<kTerms, 2, 4>(a, stream);
    }
}

int launch_decode_attn_tree(const TreeLaunch &a, murmur_stream_t stream) {
    const int e = a.out_f32 ? launch_tree<3>(a, (hipStream_t)stream) : launch_tree<2>(a, (hipStream_t)stream);
    if (e != 0 || a.n_split == 1) return e;
    const unsigned grid = (unsigned)(a.units / a.n_split) * (unsigned)a.merge_sets;
    if (a.n_split <= kTreeMergeWhole)
        hipLaunchKernelGGL(tree_merge_kernel<1>, dim3(grid), dim3(256), 0, (hipStream_t)stream, a);
    else
        hipLaunchKernelGGL(tree_merge_kernel<4>, dim3(grid), dim3(256), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}

}  // namespace murmur
