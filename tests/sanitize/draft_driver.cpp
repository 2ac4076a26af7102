// Drives the checks and buffer sizes of requests, rotary positions and drafted trees
// under the sanitizers: every entry point with random and extreme arguments, on
// launchers that check what they are given against the sizes the library asked for and
// against the limits of a launch.
#include <limits.h>
#include <math.h>
#include <stdio.h>
#include <stdlib.h>

#include <algorithm>
#include <random>

#include "internal.h"
#include "murmur_draft.h"

static std::mt19937 rng(11);
static void check(bool ok, const char *what) {
    if (!ok) {
        fprintf(stderr, "failed: %s\n", what);
        abort();
    }
}
static size_t g_ws;  // bytes of the workspace of the call

namespace murmur {
int launch_paged_reserve(const ReserveLaunch &p, murmur_stream_t) {
    const uint8_t *base = (const uint8_t *)p.top0;
    check((const uint8_t *)(p.need + p.B) <= (const uint8_t *)p.sums, "reserve: needs");
    check((const uint8_t *)(p.sums + (p.B + kReserveGroup - 1) / kReserveGroup) <= base + g_ws, "reserve: sums");
    check((int64_t)p.B * p.per_seq <= p.n_tokens && p.B <= 65535 && p.log2_bs >= 0 && p.log2_bs <= 20, "reserve: launch");
    check(((int64_t)p.n_blocks << p.log2_bs) <= (int64_t)1 << 31, "reserve: rows");
    return 0;
}
int launch_rope_append(const RopeLaunch &p, murmur_stream_t) {
    check(((int64_t)p.NL * p.n_tokens * p.parts + 3) / 4 * 256 < (int64_t)1 << 32, "rope: threads");
    check(p.parts >= 1 && (p.parts == 1 || p.parts * 8 >= p.Hq + 2 * p.Hkv), "rope: heads");
    check(p.parts == 1 || (p.wide && (p.interleaved || p.rot % 16 == 0)), "rope: parts");
    return 0;
}
int launch_decode_attn_tree(const TreeLaunch &a, murmur_stream_t) {
    const int64_t rows = (int64_t)a.T * a.G, groups = (int64_t)a.NL * a.B * a.Hkv;
    check(a.n_split >= 1 && a.n_split <= kMaxTreeSplits && a.units == groups * a.n_split, "tree: units");
    check((int64_t)a.row_sets * kTreeRowSet >= rows && (int64_t)(a.row_sets - 1) * kTreeRowSet < rows, "tree: rows");
    check(((int64_t)a.units + 7) / 8 * 8 * a.row_sets * 512 < (int64_t)1 << 32, "tree: threads");
    check(groups * a.merge_sets * 256 < (int64_t)1 << 32 || a.n_split == 1, "tree: threads of the merge");
    check(groups * a.merge_sets < INT_MAX, "tree: workgroups of the merge");
    if (a.n_split > 1)
        check((uint8_t *)(a.part_ml + 2 * (size_t)a.units * rows) <= (uint8_t *)a.part_o + g_ws && a.part_ml >= a.part_o + (size_t)a.units * rows * 128,
              "tree: partials");
    const auto divides = [](const DivideBy &by, int64_t d, int64_t most) {
        for (int i = 0; i < 4; ++i) {
            const int64_t x = i == 0 ? most : i == 1 ? 0 : (int64_t)(rng() % (uint64_t)(most + 1));
            check(by((int)x) == x / d, "tree: division");
        }
    };
    divides(a.by_split, a.n_split, a.units);
    divides(a.by_heads, a.Hkv, groups);
    divides(a.by_batch, a.B, groups);
    divides(a.by_sets, a.row_sets, a.units);
    divides(a.by_merge, a.merge_sets, INT_MAX);
    for (int r = 0; r < rows; ++r) check((int)((uint32_t)r * a.magic_g >> 16) == r / a.G, "tree: rows of a node");
    check(a.max_pos >= 1 && a.G >= 1 && a.G <= 16, "tree: launch");
    return 0;
}
int launch_tree_accept(const AcceptLaunch &p, murmur_stream_t) {
    check(p.T >= 1 && p.T <= 64 && p.B <= 65535 && p.NL <= 65535 && (int64_t)p.Hkv * 16 * 64 < INT_MAX, "accept: launch");
    return 0;
}
}  // namespace murmur

static int32_t pick(std::initializer_list<int64_t> extremes, int32_t most) {
    if (rng() % 6 == 0) return (int32_t)*(extremes.begin() + rng() % extremes.size());
    const int bits = 1 + (int)(rng() % 20);
    return 1 + (int32_t)(rng() % (uint32_t)std::min<int64_t>(most, (int64_t)1 << bits));
}

int main() {
    void *const fake = (void *)4096;
    int32_t *const ints = (int32_t *)fake;
    int launched[4] = {0, 0, 0, 0}, refused[4] = {0, 0, 0, 0};
    const auto count = [&](int call, int rc) { (rc == MURMUR_OK ? launched : refused)[call] += 1; };
    for (int i = 0; i < 120000; ++i) {
        murmur_kv kv{};
        kv.k = kv.v = fake;
        kv.n_layers = pick({0, 1, 65535, 65536, INT_MAX, INT_MIN}, 80);
        kv.max_len = pick({0, 1, INT_MAX}, 1 << 20);
        kv.stride_pos = 128 * (int64_t)(rng() % 9);
        kv.stride_h = rng() % 9 ? 128 : INT64_MAX / 8 * 8;
        if (rng() % 9 == 0) kv.stride_pos = (int64_t)1 << (7 + rng() % 50);
        const int32_t B = pick({0, -1, 1, 65535, 65536, INT_MAX, INT_MIN}, 4096), hkv = pick({0, 1, 65535, 65536, INT_MAX}, 16);
        const int32_t hq = rng() % 8 ? (int32_t)((int64_t)hkv * (1 + rng() % 17) % INT_MAX) : pick({0, -3, INT_MAX}, 300);

        const int32_t nodes = pick({0, 64, 65, INT_MAX, INT_MIN}, 64), keep = pick({0, 1, 1 << 28, INT_MAX, INT_MIN}, 200000);
        size_t ws = 0;
        const int rc = murmur_decode_attn_tree_workspace(kv.n_layers, B, hq, hkv, nodes, keep, &ws);
        g_ws = ws;
        const int32_t blocks = pick({0, 1, INT_MAX}, 1 << 18), bs = 1 << (rng() % 22);
        const bool paged = rng() % 2;
        int r = murmur_decode_attn_tree((murmur_seg *)fake, (murmur_policy *)fake, (int32_t)(rng() % 5), ints, 1, nodes, fake, &kv, fake, fake,
                                        paged ? ints : nullptr, paged ? blocks : 0, paged ? bs : 0, keep, B, hq, hkv, 128, 0.1f, fake,
                                        MURMUR_DTYPE_BF16, nullptr, fake, ws, nullptr);
        check(r != MURMUR_OK || rc == MURMUR_OK, "tree agrees with its size");
        count(0, r);

        size_t bytes = 0;
        const int pr = murmur_paged_reserve_workspace(B, &bytes);
        g_ws = bytes;
        const int32_t n = pick({0, 1, 1 << 30, INT_MAX}, 1 << 20), per = (int32_t)(rng() % 3 ? 0 : rng() % 200);
        const int32_t tokens = pick({0, 1, INT_MAX}, INT_MAX);
        r = murmur_paged_reserve(ints, ints, B, ints, blocks, bs, rng() % 2 ? ints : nullptr, n, ints, ints, n, per, tokens, ints, ints, ints,
                                 rng() % 2 ? ints : nullptr, nullptr, fake, bytes, nullptr);
        check(r != MURMUR_OK || pr == MURMUR_OK, "reserve agrees with its size");
        count(1, r);

        murmur_rope rope{(int32_t)(rng() % 140) - 4, (int32_t)(rng() % 3), 1.f, (const uint64_t *)fake};
        murmur_qkv in{fake, fake, fake, (int32_t)(rng() % 4), (int64_t)(rng() % 5), (int64_t)(rng() % 100000), INT64_MAX, (int64_t)(rng() % 64) * 8};
        count(2, murmur_rope_append(&rope, &in, ints, ints, nullptr, pick({0, 1, INT_MAX}, 100), pick({0, 1, INT_MAX}, 1 << 20), hq, hkv, 128, fake,
                                    &kv, nullptr));
        count(3, murmur_tree_accept(ints, (int32_t)(rng() % 2), nodes, ints, ints, ints, B, fake, fake, &kv, hkv, ints, ints, ints, nullptr));

        uint64_t freq[64];
        float gain = 0.f;
        const double extremes[] = {0.0, 1.0, 1e4, 1e300, HUGE_VAL, -HUGE_VAL, NAN, 1e-300, 4096.0, 1.5};
        const auto value = [&] { return extremes[rng() % 10]; };
        (void)murmur_rope_freqs_host((int32_t)(rng() % 70) * 2 - 2, value(), (int32_t)(rng() % 7) - 1, value(), value(), value(), value(), freq,
                                     &gain);
    }
    for (int i = 0; i < 4; ++i) check(launched[i] > 1000 && refused[i] > 1000, "both kinds of calls");
    printf("draft driver: ok (%d %d %d %d launched)\n", launched[0], launched[1], launched[2], launched[3]);
    return 0;
}
