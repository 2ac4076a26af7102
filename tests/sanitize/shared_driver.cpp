// Drives the checks and buffer sizes of shared pages and shared prefixes under the
// sanitizers: every entry point with random and extreme arguments, on launchers that
// check what they are given against the sizes the library asked for.
#include <limits.h>
#include <stdio.h>
#include <stdlib.h>

#include <random>

#include "internal.h"
#include "murmur_shared.h"

static std::mt19937 rng(7);
static void check(bool ok, const char *what) {
    if (!ok) {
        fprintf(stderr, "failed: %s\n", what);
        abort();
    }
}
static size_t g_ws, g_plan;  // bytes of the buffers of the call

namespace murmur {
int launch_paged_fork(const int32_t *, int32_t B, int32_t *, int32_t max_blocks, int32_t *, int32_t n_blocks, int32_t *,
                      int32_t *, const ForkWorkspace &ws, murmur_stream_t) {
    const size_t entries = (size_t)B * max_blocks, base = (size_t)(uintptr_t)ws.head;
    check((size_t)(uintptr_t)(ws.block_at + entries) <= base + g_ws, "fork: block_at");
    check((size_t)(uintptr_t)(ws.bits + (entries + 31) / 32) <= base + g_ws, "fork: bits");
    check((size_t)(uintptr_t)(ws.first + n_blocks) <= base + g_ws, "fork: first");
    return 0;
}
int launch_paged_step_shared(const murmur_seg *, const murmur_policy *, int32_t, int32_t, int32_t *, int32_t, int32_t log2_bs,
                             int32_t *, int32_t, int32_t *, int32_t *, int32_t, int32_t *, murmur_stream_t) {
    check(log2_bs >= 0 && log2_bs <= 20, "step: block size");
    return 0;
}
int launch_paged_append_shared(const murmur_seg *, int32_t, const int32_t *, int32_t, int32_t, const int32_t *,
                               const murmur_kv &, int32_t, const void *, const void *, murmur_stream_t) {
    return 0;
}
int launch_paged_compact(int32_t, int32_t *, int32_t, int32_t, int32_t *, int32_t n_blocks, int32_t *, int32_t *, int32_t *,
                         const murmur_kv *, int32_t, int32_t *ws, murmur_stream_t) {
    check((size_t)(uintptr_t)(ws + 1 + 2 * (size_t)(n_blocks / 2)) <= 4096 + g_ws, "compact: moves");
    return 0;
}
static void check_caps(const SharedCaps &c, int32_t B) {
    check(c.grid >= 1 && c.grid <= c.n_wg && c.n_wg <= 65535, "grid");
    check(c.rows >= 0 && c.rows <= 1 << 24, "rows");
    check(c.item_offset >= sizeof(PlanHeader) + sizeof(PlanSeq) * (size_t)B, "items");
    check(c.chunk_offset >= c.item_offset + sizeof(PlanItem) * (size_t)c.n_wg, "chunks");
    check(c.scan_offset >= c.chunk_offset + sizeof(PlanChunk) * (size_t)c.n_wg * kSharedWaves, "scan");
    check(c.scan_offset + 4 * (size_t)B * c.n_scan <= c.plan_bytes && c.plan_bytes <= g_plan, "plan");
    check(c.waves == 4 || c.waves == 8, "waves");
}
int launch_shared_plan(const SharedPlanLaunch &p, murmur_stream_t) {
    check_caps(p.caps, p.B);
    return 0;
}
int launch_decode_attn_shared(const SharedAttnLaunch &a, murmur_stream_t) {
    const size_t rows = (size_t)a.NL * a.Hkv * a.rows_cap;
    check((uint8_t *)(a.part_ml + rows * 2) <= (uint8_t *)a.part_o + g_ws, "partials");
    check(a.n_wg >= 1 && a.n_wg <= 65535 && a.G >= 1 && a.G <= 16, "launch");
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
    int launched = 0, refused = 0;
    for (int i = 0; i < 300000; ++i) {
        const int32_t B = pick({0, -1, 1, 4096, 4097, INT_MAX, INT_MIN}, 4096), hkv = pick({0, 1, 65535, INT_MAX}, 16);
        const int32_t hq = rng() % 8 ? (int32_t)((int64_t)hkv * (1 + rng() % 17) % INT_MAX) : pick({0, -3, INT_MAX}, 300);
        const int32_t keep = pick({0, 1, 1 << 28, INT_MAX, INT_MIN}, 200000), groups = pick({0, 1, 4096, INT_MAX}, 4096);
        murmur_kv kv{};
        kv.k = kv.v = fake;
        kv.n_layers = pick({0, 1, 65535, INT_MAX, INT_MIN}, 80);
        kv.max_len = pick({0, 1, INT_MAX}, 1 << 20);
        kv.stride_pos = 128 * (int64_t)(rng() % 9);
        kv.stride_h = 128;
        size_t ws = 0, plan = 0;
        const int rc = murmur_decode_attn_shared_workspace(kv.n_layers, B, hq, hkv, keep, groups, &ws, &plan);
        if (rc == MURMUR_OK) {
            size_t ws2 = 0, plan2 = 0;
            const int32_t B2 = B + (int32_t)(rng() % 3), keep2 = keep + (int32_t)(rng() % 2000), groups2 = groups + (int32_t)(rng() % 3);
            if (murmur_decode_attn_shared_workspace(kv.n_layers, B2, hq, hkv, keep2, groups2, &ws2, &plan2) == MURMUR_OK)
                check(ws2 >= ws && plan2 >= plan, "sizes grow with the batch");
        }
        g_ws = ws;
        g_plan = plan;
        const int32_t find = (int32_t)(rng() % 2);
        int r = murmur_shared_plan((const int32_t *)fake, nullptr, (const int32_t *)fake, keep, B, (const int32_t *)fake,
                                   groups, (int32_t *)fake, find, kv.n_layers, hq, hkv, fake, plan, nullptr);
        check((r == MURMUR_OK) == (rc == MURMUR_OK), "plan agrees with its size");
        r = murmur_decode_attn_shared(fake, &kv, (const int32_t *)fake, nullptr, keep, B, groups, hq, hkv, 128, 0.1f, fake,
                                      MURMUR_DTYPE_F32, nullptr, fake, plan, fake, ws, nullptr);
        check(r != MURMUR_OK || rc == MURMUR_OK, "attention agrees with its size");
        (r == MURMUR_OK ? launched : refused) += 1;

        const int32_t rows = pick({0, 65535, 65536, INT_MAX}, 65535), blocks = pick({0, 1, 1 << 20, INT_MAX}, 1 << 18);
        const int32_t n = pick({0, 1, 1 << 30, INT_MAX}, 1 << 20), bs = 1 << (rng() % 22);
        size_t bytes = 0;
        const int pr = murmur_paged_workspace(rows, blocks, n, &bytes);
        g_ws = bytes;
        r = murmur_paged_fork((const int32_t *)fake, rows, (int32_t *)fake, blocks, (int32_t *)fake, n, (int32_t *)fake,
                              (int32_t *)fake, n, fake, bytes, nullptr);
        check((r == MURMUR_OK) == (pr == MURMUR_OK), "fork agrees with its size");
        (void)murmur_paged_compact(rows, (int32_t *)fake, blocks, bs, (int32_t *)fake, n, (int32_t *)fake, (int32_t *)fake, n,
                                   (int32_t *)fake, rng() % 2 ? &kv : nullptr, hkv, fake, bytes, nullptr);
        (void)murmur_paged_step_shared((const murmur_seg *)fake, (const murmur_policy *)fake, 1, rows, (int32_t *)fake, blocks,
                                       bs, (int32_t *)fake, n, (int32_t *)fake, (int32_t *)fake, n, 0, (int32_t *)fake,
                                       rng() % 2 ? &kv : nullptr, hkv, fake, fake, nullptr);
    }
    check(launched > 1000 && refused > 1000, "both kinds of calls");
    printf("shared driver: ok (%d launched, %d refused)\n", launched, refused);
    return 0;
}
