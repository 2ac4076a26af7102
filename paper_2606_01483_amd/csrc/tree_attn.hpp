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
#pragma unroll
    for (int round = 0; round < 6; ++round) {
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
    l.count = l.n0 + l.live;
    const bool is = par != -2;
    l.a_most = wave_max(is ? rule.a : 0);
    l.b_most = wave_max(is ? rule.b : 0);
    l.c_most = wave_max(is ? rule.c : 0);
    return l;
}

// Whether rank r of the list is one that a row attends to.
static __device__ __forceinline__ bool tree_allows(const TreeList &l, const TreeRule &x, int r) {
    const int n = r - l.n0;
    const uint32_t bits = n < 32 ? x.lo >> (n & 31) : x.hi >> (n & 31);
    return r < l.count && (uint32_t)(r - l.a0) >= (uint32_t)x.a && (uint32_t)(l.b1 - 1 - r) >= (uint32_t)x.b &&
           (uint32_t)(r - l.c0) >= (uint32_t)x.c && (n < 0 || (bits & 1u));
}

// Where ranks lie: the cache rows of a (layer, KV head) of a sequence, and the nodes.
// kRows rows of a pass for each lane; a row is one of the cache (>= 0) or ~node, and
// ~0, the root's, wherever none is to be read.
template <int kRows>
struct TreeRows {
    int32_t pos[kRows], entry[kRows];
    // positions, and the block table's entries on their way
    __device__ __forceinline__ void begin(const TreeList &l, const int32_t *bt_row, int32_t max_blocks, int32_t log2_bs,
                                          int r0) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int r = r0 + 4 * i;
            int piece;
            const int p = tab_pos(l.tab, r, piece);
            pos[i] = r < l.n0 ? p : (r < l.count ? ~(r - l.n0) : ~0);
            if (bt_row) entry[i] = bt_row[pos[i] < 0 ? 0 : min(pos[i] >> log2_bs, max_blocks - 1)];  // uniform
        }
    }
    __device__ __forceinline__ void finish(const int32_t *bt_row, int32_t max_blocks, int32_t log2_bs, int32_t max_len,
                                           int &err) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            if (pos[i] < 0) continue;
            int64_t row = pos[i];
            if (bt_row) {
                const bool blocked = entry[i] < 0 || (pos[i] >> log2_bs) >= max_blocks;
                row = ((int64_t)entry[i] << log2_bs) | (pos[i] & ((1 << log2_bs) - 1));
                if (blocked) {
                    err |= MURMUR_DEVERR_BLOCK;
                    pos[i] = ~0;
                    continue;
                }
            }
            if (row >= max_len) {
                err |= MURMUR_DEVERR_POSITION;
                row = ~0;
            }
            pos[i] = (int32_t)row;
        }
    }
};

// The values of a pass that some rows leave out: zero times an infinity or a NaN is
// NaN, so where the values hold one (the product with zeros tells), those are added
// to the sums of the rows that attend to them, whose result is not finite there
// whatever their weights, and taken out of the operands.
template <int kTiles>
static __device__ __forceinline__ void tree_keep_apart(u32x2 (&vf)[16], const uint8_t *tile, int r0, const TreeList &l,
                                                       const TreeRule (&rule)[kTiles], WaveAcc (&w)[kTiles], int lane) {
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
                const bool mine = tree_allows(l, rule[t], r0 + r);
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
// Workgroup: kWays * kTiles * 16 query rows of one (layer, sequence, KV head) over one
// split of the list.  Its four wavefronts are kWays ways by rows and 4 / kWays groups
// by passes: the wavefronts of a group share the K and V rows of a pass, which they
// load together into one of the group's two stages while they compute the other.
// ---------------------------------------------------------------------------
constexpr int kTreeThreads = 256;
template <int kWays>
struct TreeLds {
    static constexpr int kGroups = 4 / kWays;
    uint8_t stages[kGroups][2][kStageBytes];
    TreeRule rule[64];
    float ml[4][32][2];
    int err;
};

template <int kTerms, int kTiles, int kWays>
__global__ __launch_bounds__(kTreeThreads, 2) void tree_attn_kernel(const TreeLaunch a) {
    constexpr int kGroups = 4 / kWays, kRows = 8 / kWays, kAll = kWays * kTiles * 16;
    __shared__ __attribute__((aligned(16))) TreeLds<kWays> lds;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int way = wave % kWays, grp = wave / kWays, n16 = lane & 15, c4 = lane >> 4;
    // the workgroups of one split's row sets follow each other on one XCD
    const int x = blockIdx.x, set = (x >> 3) % a.row_sets, unit = (x >> 3) / a.row_sets * 8 + (x & 7);
    if (unit >= a.units) return;
    const int split = unit % a.n_split, group = unit / a.n_split;
    const int g = group % a.Hkv, lb = group / a.Hkv, b = lb % a.B, layer = lb / a.B;
    const murmur_seg s = reinterpret_cast<const murmur_seg *>(a.seg)[b];
    if (layout_absent(s.prompt_pre, s.speech_len, s.prompt_mid, s.out_len)) return;
    const int rec = ((a.pol_mode & MURMUR_POL_PER_LAYER) ? layer * ((a.pol_mode & MURMUR_POL_PER_SEQ) ? a.B : 1) : 0) +
                    ((a.pol_mode & MURMUR_POL_PER_SEQ) ? b : 0);
    const murmur_policy p = reinterpret_cast<const murmur_policy *>(a.pol)[rec];
    TreeRule mine{};
    const TreeList l = tree_list(s, p, a.parent + (a.parent_per_seq ? (int64_t)b * a.T : 0), a.T, lane, mine);
    const int row0 = set * kAll;
    if (row0 >= l.live * a.G) return;
    if (wave == 0) lds.rule[lane] = mine;
    if (tid == 0) {
        lds.err = l.err;
        if (l.err) raise_device_error(l.err);
    }
    __syncthreads();

    // the lane's row of every tile
    int node[kTiles], row[kTiles];
    u32x4 qf[kTiles][4];
    float scale = 1.f;
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        row[t] = row0 + (way * kTiles + t) * 16 + n16;
        const int r = min(row[t], a.T * a.G - 1);
        node[t] = (int)((uint32_t)r * a.magic_g >> 16);
        const uint16_t *q = a.q + ((((int64_t)lb * a.T + node[t]) * a.Hq + g * a.G + r - node[t] * a.G) * kHeadDim + 8 * c4);
#pragma unroll
        for (int kc = 0; kc < 4; ++kc) qf[t][kc] = load16(q + 32 * kc);
    }
    WaveAcc w[kTiles];
#pragma unroll
    for (int t = 0; t < kTiles; ++t) {
        scale = signed_scale(qf[t], a.scale_log2);
        start_rows(w[t]);
    }
    const int passes = l.err ? 0 : (l.count + kWaveTile - 1) / kWaveTile;
    const int p0 = (int)((int64_t)passes * split / a.n_split), p1 = (int)((int64_t)passes * (split + 1) / a.n_split);
    const int rounds = (p1 - p0 + kGroups - 1) / kGroups;
    const int32_t *bt_row = a.bt ? a.bt + (int64_t)b * a.max_blocks : nullptr;
    const uint16_t *kc = a.k + layer * a.s_layer + b * a.s_b + g * a.s_h, *vc = a.v + layer * a.s_layer + b * a.s_b + g * a.s_h;
    const int64_t tree_at = ((int64_t)lb * a.T * a.Hkv + g) * kHeadDim;
    const int first = way * kRows;  // of the eight loads of a tile this wavefront has [first, first + kRows)
    int err = 0;
    TreeRows<kRows> rows;
    const auto pass_of = [&](int it) { return p0 + it * kGroups + grp; };
    const auto begin = [&](int it) {
        rows.begin(l, bt_row, a.max_blocks, a.log2_bs, pass_of(it) * kWaveTile + 4 * first + c4);
    };
    const auto load = [&](int it) {
        rows.finish(bt_row, a.max_blocks, a.log2_bs, a.max_len, err);
        uint8_t *stage = lds.stages[grp][it & 1];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const int j = first + i, c = n16 ^ ((4 * j + c4) & 15);
            const bool is_node = rows.pos[i] < 0;
            const int64_t at = (is_node ? tree_at + (int64_t)~rows.pos[i] * a.Hkv * kHeadDim : rows.pos[i] * a.s_pos) + 8 * c;
            __builtin_amdgcn_global_load_lds((is_node ? a.k_tree : kc) + at, (lds_void_t *)(stage + j * 1024), 16, 0, 0);
            __builtin_amdgcn_global_load_lds((is_node ? a.v_tree : vc) + at, (lds_void_t *)(stage + kTileBytes + j * 1024), 16, 0, 0);
        }
    };
    if (rounds > 0) {
        begin(0);
        load(0);
        begin(1);
    }
#pragma unroll 1
    for (int it = 0; it < rounds; ++it) {
        wait_vm<0>();
        __syncthreads();  // the group's rows are in, and its other stage is read
        if (it + 1 < rounds) {
            load(it + 1);
            begin(it + 2);
        }
        const int r0 = pass_of(it) * kWaveTile;
        if (pass_of(it) >= p1) continue;  // uniform: the last round of a group without one
        const uint32_t kt = lds_addr(lds.stages[grp][it & 1]), vt = kt + kTileBytes;
        u32x4 kf[8];
        read_k_operands(kf, kt, n16, c4);
        const int r1 = r0 + kWaveTile;
        const bool ruled = r1 > l.n0 || (r1 > l.a0 && r0 < l.a0 + l.a_most) || (r1 > l.b1 - l.b_most && r0 < l.b1) ||
                           (r1 > l.c0 && r0 < l.c0 + l.c_most);
        u32x4 pr[kTiles][kTerms];
        TreeRule rule[kTiles];
        if (ruled) {
#pragma unroll
            for (int t = 0; t < kTiles; ++t) rule[t] = lds.rule[node[t]];
        }
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            f32x4 sc[2];
#pragma unroll
            for (int blk = 0; blk < 2; ++blk) {
                sc[blk] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int kk = 0; kk < 4; ++kk) sc[blk] = mfma16x16x32(kf[4 * blk + kk], qf[t][kk], sc[blk]);
            }
            if (ruled) {
                asm volatile("");  // a branch, which few passes take
#pragma unroll
                for (int blk = 0; blk < 2; ++blk)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        sc[blk][i] = tree_allows(l, rule[t], r0 + 16 * blk + 4 * c4 + i) ? sc[blk][i] : kNegInf;
            }
            softmax_pass<kTerms>(sc, kWaveTile, scale, w[t], c4, pr[t]);
        }
        u32x2 vf[16];
        read_v_operands(vf, vt, n16, c4);
        if (ruled) tree_keep_apart<kTiles>(vf, lds.stages[grp][it & 1] + kTileBytes, r0, l, rule, w, lane);
#pragma unroll
        for (int db = 0; db < 8; ++db) {
            const u32x4 av = u32x4{vf[2 * db][0], vf[2 * db][1], vf[2 * db + 1][0], vf[2 * db + 1][1]};
#pragma unroll
            for (int t = 0; t < kTiles; ++t)
#pragma unroll
                for (int k = 0; k < kTerms; ++k) w[t].acc[db] = mfma16x16x32(av, pr[t][k], w[t].acc[db]);
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

    // Rows to the outputs, or to the split's partials
    const auto put = [&](int r, int c, f32x4 O, float M, float L) {
        if (r >= l.live * a.G) return;
        if (bad) L = __builtin_nanf("");
        if (a.n_split > 1) {
            const int64_t at = ((int64_t)group * a.n_split + split) * (a.T * a.G) + r;
            *reinterpret_cast<f32x4 *>(a.part_o + at * kHeadDim + 4 * c) = O;
            if (c == 0) *reinterpret_cast<float2 *>(a.part_ml + 2 * at) = float2{M, L};
        } else {
            const int n = (int)((uint32_t)r * a.magic_g >> 16);
            if (l.there >> n & 1) tree_store(a, ((int64_t)lb * a.T + n) * a.Hq + g * a.G + r - n * a.G, c, O, M, L);
        }
    };
    if constexpr (kGroups == 1) {
#pragma unroll
        for (int t = 0; t < kTiles; ++t) {
            const float sum = sum_over_c4(w[t].l_run);
#pragma unroll
            for (int db = 0; db < 8; ++db) put(row[t], 4 * db + c4, w[t].acc[db], w[t].m_run * scale, sum);
        }
    } else {
        // the groups' states by way of LDS, two tiles of every wavefront at a time
        float *o = reinterpret_cast<float *>(&lds.stages[0][0][0]) + wave * 32 * kHeadDim;
        static_assert(sizeof(lds.stages) >= 4 * 32 * kHeadDim * sizeof(float), "two tiles of each wavefront");
#pragma unroll
        for (int t0 = 0; t0 < kTiles; t0 += 2) {
            if (t0 > 0) __syncthreads();
#pragma unroll
            for (int t = t0; t < t0 + 2 && t < kTiles; ++t) {
                const float sum = sum_over_c4(w[t].l_run);
                const int r = 16 * (t - t0) + n16;
                if (c4 == 0) *reinterpret_cast<float2 *>(&lds.ml[wave][r][0]) = float2{w[t].m_run * scale, sum};
#pragma unroll
                for (int db = 0; db < 8; ++db)
                    *reinterpret_cast<f32x4 *>(&o[r * kHeadDim + 4 * ((4 * db + c4) ^ (r & 7))]) = w[t].acc[db];
            }
            __syncthreads();
            const int n = min(2, kTiles - t0) * 16;  // rows of a way in this turn
            for (int i = tid; i < kWays * n * 32; i += kTreeThreads) {
                const int c = i & 31, wy = (i >> 5) / n, r = (i >> 5) % n;
                float M = kNegInf, L = 0.f;
#pragma unroll
                for (int e = 0; e < kGroups; ++e) M = fmaxf(M, lds.ml[e * kWays + wy][r][0]);
                f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
                for (int e = 0; e < kGroups; ++e) {
                    const int wv = e * kWays + wy;
                    const float m = lds.ml[wv][r][0], f = m == kNegInf ? 0.f : __builtin_amdgcn_exp2f(m - M);
                    const f32x4 part = *reinterpret_cast<const f32x4 *>(
                        reinterpret_cast<const float *>(&lds.stages[0][0][0]) + (wv * 32 + r) * kHeadDim + 4 * (c ^ (r & 7)));
                    L += lds.ml[wv][r][1] * f;
                    O += f * part;
                }
                put(row0 + (wy * kTiles + t0) * 16 + r, c, O, M, L);
            }
        }
    }
}

// A row by 32 threads, four head dims each.
__global__ __launch_bounds__(256) void tree_merge_kernel(const TreeLaunch a) {
    const int rows = a.T * a.G;
    const int64_t at = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
    const int c = threadIdx.x & 31;
    if (at >= (int64_t)a.NL * a.B * a.Hkv * rows) return;
    const int64_t group = at / rows;
    const int r = (int)(at - group * rows), n = (int)((uint32_t)r * a.magic_g >> 16);
    const int64_t lb = group / a.Hkv;
    const int g = (int)(group - lb * a.Hkv), b = (int)(lb % a.B);
    const murmur_seg s = reinterpret_cast<const murmur_seg *>(a.seg)[b];
    if (layout_absent(s.prompt_pre, s.speech_len, s.prompt_mid, s.out_len)) return;
    if (a.parent[(a.parent_per_seq ? (int64_t)b * a.T : 0) + n] == -2) return;
    const int64_t part0 = group * a.n_split * rows + r;
    float M = kNegInf, L = 0.f;
    for (int i = 0; i < a.n_split; ++i) M = fmaxf(M, a.part_ml[2 * (part0 + (int64_t)i * rows)]);
    f32x4 O = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int i = 0; i < a.n_split; ++i) {
        const int64_t p = part0 + (int64_t)i * rows;
        const float2 ml = *reinterpret_cast<const float2 *>(a.part_ml + 2 * p);
        const f32x4 part = *reinterpret_cast<const f32x4 *>(a.part_o + p * kHeadDim + 4 * c);
        const float f = ml.x == kNegInf ? 0.f : __builtin_amdgcn_exp2f(ml.x - M);
        L += ml.y * f;
        O += f * part;
    }
    tree_store(a, (lb * a.T + n) * a.Hq + g * a.G + r - n * a.G, c, O, M, L);
}

template <int kTerms, int kTiles, int kWays>
static int launch_tree_as(const TreeLaunch &a, hipStream_t stream) {
    const unsigned grid = (unsigned)((a.units + 7) / 8 * 8 * a.row_sets);
    hipLaunchKernelGGL((tree_attn_kernel<kTerms, kTiles, kWays>), dim3(grid), dim3(kTreeThreads), 0, stream, a);
    return (int)hipGetLastError();
}

template <int kTerms>
static int launch_tree(const TreeLaunch &a, hipStream_t stream) {
    switch (a.shape) {
        case kTree16: return launch_tree_as<kTerms, 1, 1>(a, stream);
        case kTree32: return launch_tree_as<kTerms, 2, 1>(a, stream);
        case kTree64: return launch_tree_as<kTerms, 2, 2>(a, stream);
        default: return launch_tree_as<kTerms, 2, 4>(a, stream);
    }
}

int launch_decode_attn_tree(const TreeLaunch &a, murmur_stream_t stream) {
    const int e = a.out_f32 ? launch_tree<3>(a, (hipStream_t)stream) : launch_tree<2>(a, (hipStream_t)stream);
    if (e != 0 || a.n_split == 1) return e;
    const int64_t rows = (int64_t)a.NL * a.B * a.Hkv * a.T * a.G;
    hipLaunchKernelGGL(tree_merge_kernel, dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, (hipStream_t)stream, a);
    return (int)hipGetLastError();
}

}  // namespace murmur
