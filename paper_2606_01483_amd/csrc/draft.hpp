// Device code of requests into a paged pool, rotary positions and accepted paths
// (included by kernels.hip).
//
//   reserve_group_kernel, reserve_count_kernel, reserve_long_kernel
//                                              blocks and slot maps for new tokens
//   rope_wide_kernel, rope_mixed_kernel, rope_pair_kernel
//                                              q and k rotated, K and V into the cache
//   tree_accept_kernel                         the accepted path into the cache
#pragma once

namespace murmur {

// ---------------------------------------------------------------------------
// reserve.  Sequences are served in order, so a sequence's blocks are found from the
// number that those before it need.  Up to kReserveGroup sequences are one workgroup's
// work, a wavefront each; more take two launches: the first counts (a wavefront per
// sequence, and sums over kReserveGroup of them), the second pops and writes the maps,
// a wavefront per sequence or (long prompts) a workgroup.  A sequence is refused where
// its blocks end behind the stack, or its tokens behind the maps; then so is every
// later one that needs a block, so those that are served pop without holes and the top
// is the minimum of what they leave (an integer atomic, whose order does not matter).
// Bound by round trips to memory: lengths, entries, stack, maps.
// ---------------------------------------------------------------------------
constexpr int kReserveThreads = 64 * kReserveGroup;

static __device__ __forceinline__ int64_t wave_sum64(int64_t x) {
#pragma unroll
    for (int d = 32; d >= 1; d /= 2) x += __shfl_xor(x, d);
    return x;
}

// What sequence b asks for, by a wavefront: its blocks, or -1 and the device error.
struct ReserveAsk {
    int32_t len, fresh;  // fresh: 0 where either is negative
    int32_t need, err;
    int32_t entry;  // the lane's of the first 64 columns
};
static __device__ __forceinline__ ReserveAsk reserve_ask(const ReserveLaunch &p, int b, int lane) {
    ReserveAsk a{p.len[b], p.fresh[b], 0, 0, 0};
    if (a.len < 0 || a.fresh < 0) {
        a.err = MURMUR_DEVERR_COUNT;
        a.fresh = 0;
    } else if (a.fresh > 0) {
        const int64_t last = ((int64_t)a.len + a.fresh - 1) >> p.log2_bs;
        if (last >= p.max_blocks) a.err = MURMUR_DEVERR_BLOCK;
        else if (p.per_seq > 0 && a.fresh > p.per_seq) a.err = MURMUR_DEVERR_OVERFLOW;
        else {
            const int32_t *row = p.bt + (int64_t)b * p.max_blocks;
            for (int c0 = a.len >> p.log2_bs; c0 <= (int)last; c0 += 64) {
                const bool in = c0 + lane <= (int)last;
                const int32_t x = in ? row[c0 + lane] : 0;
                if (c0 == a.len >> p.log2_bs) a.entry = x;
                a.need += __popcll(__ballot(in && x < 0));
                const bool wrong = in && (x >= p.n_blocks || (p.ref && x >= 0 && p.ref[x] > 1));
                if (__ballot(wrong)) a.err = MURMUR_DEVERR_BLOCK;
            }
        }
    }
    if (a.err) a.need = -1;
    return a;
}

// Takes the blocks of sequence b and writes its maps, by kThreads threads (a wavefront,
// or a workgroup with s_scan and s_bad).  tokens, blocks: of the sequences before it;
// all: tokens of all of them.  Returns the top that it leaves, or INT32_MAX.
template <int kThreads>
static __device__ __forceinline__ int32_t reserve_take(const ReserveLaunch &p, int b, const ReserveAsk &ask, int32_t top, int64_t tokens,
                                                    int blocks, int64_t all, int tid, int *s_scan, int *s_bad) {
    const auto start_at = [&](int64_t packed, int q) {
        return (int32_t)min(p.per_seq > 0 ? (int64_t)q * p.per_seq : packed, (int64_t)0x7fffffff);
    };
    const int32_t len = ask.len, fresh = ask.fresh, need = ask.need;
    const int64_t at = p.per_seq > 0 ? (int64_t)b * p.per_seq : tokens;
    int err = 0;
    bool served = need >= 0;
    if (served && at + fresh > p.n_tokens) {
        served = false;
        err |= MURMUR_DEVERR_OVERFLOW;
    } else if (served && need > 0 && (int64_t)blocks + need > top) {
        served = false;
        err |= MURMUR_DEVERR_POOL;
    }
    int32_t *row = p.bt + (int64_t)b * p.max_blocks;
    const int first = len >> p.log2_bs, last = fresh > 0 ? (int)(((int64_t)len + fresh - 1) >> p.log2_bs) : first;
    const bool held = kThreads == 64 && last - first < 64;  // every entry stands in a lane
    int32_t entry = ask.entry, left = 0x7fffffff;
    // the blocks: the k-th that is missing is the k-th from the top behind those of the sequences before
    if (served && need > 0) {
        int k = top - 1 - blocks;
        left = k + 1 - need;
        bool bad = false;
        for (int c0 = first; c0 <= last; c0 += kThreads) {
            const int c = c0 + tid;
            const bool missing = c <= last && (held ? entry : row[c]) < 0;
            int total, off;
            if constexpr (kThreads == 64) {
                const uint64_t those = __ballot(missing);
                total = __popcll(those);
                off = __popcll(those & ((1ull << tid) - 1));
            } else {
                off = wg_exclusive_scan<kThreads>(missing, s_scan, tid, total);
            }
            if (missing) {
                const int32_t x = p.stack[k - off];
                if (x >= 0 && x < p.n_blocks) {
                    row[c] = x;
                    if (p.ref) p.ref[x] = 1;
                    entry = x;
                } else {
                    bad = true;
                }
            }
            k -= total;
        }
        if constexpr (kThreads == 64) {
            if (!held) wait_vmem();  // the entries before they are read again
            bad = __ballot(bad) != 0;
        } else {
            if (bad) *s_bad = 1;
            __syncthreads();
            bad = *s_bad;
        }
        if (bad) {
            served = false;
            err |= MURMUR_DEVERR_POOL;
        }
    }
    // the maps, kBatch entries of a thread at a time
    constexpr int kBatch = 4;
    const int64_t end = min(p.per_seq > 0 ? at + p.per_seq : at + fresh, (int64_t)p.n_tokens);
    for (int64_t i0 = at; i0 < end; i0 += kBatch * kThreads) {
        int32_t block[kBatch];
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int64_t i = i0 + j * kThreads + tid, of = min(i - at, max((int64_t)fresh - 1, (int64_t)0));
            const int c = (int)((len + of) >> p.log2_bs);
            if (held) block[j] = __shfl(entry, c - first);
            else block[j] = served && fresh > 0 && i < end ? row[c] : 0;
        }
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int64_t i = i0 + j * kThreads + tid, pos = len + (i - at);
            if (i >= end) break;
            const bool there = i - at < fresh;
            p.slot[i] = there && served ? (block[j] << p.log2_bs) | (int32_t)(pos & ((1 << p.log2_bs) - 1)) : -1;
            if (p.pos) p.pos[i] = there ? (int32_t)min(pos, (int64_t)0x7fffffff) : -1;
            if (p.seq) p.seq[i] = there ? b : -1;
        }
    }
    // the entries that no sequence has, between all of them
    for (int64_t i = (p.per_seq > 0 ? (int64_t)p.B * p.per_seq : all) + (int64_t)b * kThreads + tid; i < p.n_tokens;
         i += (int64_t)p.B * kThreads) {
        p.slot[i] = -1;
        if (p.pos) p.pos[i] = -1;
        if (p.seq) p.seq[i] = -1;
    }
    if (tid == 0) {
        p.got[b] = served ? fresh : -1;
        p.start[b] = start_at(tokens, b);
        if (b == p.B - 1) p.start[p.B] = start_at(all, p.B);
        if (err | ask.err) raise_device_error(err | ask.err);
    }
    return left;
}

static __device__ __forceinline__ int32_t reserve_top(const ReserveLaunch &p, int32_t top) { return min(max(top, 0), p.n_blocks); }

__global__ __launch_bounds__(kReserveThreads) void reserve_count_kernel(const ReserveLaunch p) {
    __shared__ ReserveSums s_sums[kReserveGroup];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = blockIdx.x * kReserveGroup + wave;
    ReserveAsk ask{0, 0, 0, 0, 0};
    if (b < p.B) ask = reserve_ask(p, b, lane);
    if (lane == 0) {
        s_sums[wave] = ReserveSums{ask.fresh, max(ask.need, 0), 0};
        if (b < p.B) p.need[b] = ask.need;
        if (ask.err) raise_device_error(ask.err);
    }
    __syncthreads();
    if (tid == 0) {
        ReserveSums t{0, 0, 0};
        for (int w = 0; w < kReserveGroup; ++w) {
            t.tokens += s_sums[w].tokens;
            t.blocks += s_sums[w].blocks;
        }
        p.sums[blockIdx.x] = t;
        if (blockIdx.x == 0) *p.top0 = *p.top;
    }
}

// kReserveGroup sequences, a wavefront each; all there are, or (kMany) those of one
// workgroup behind reserve_count_kernel.
template <bool kMany>
__global__ __launch_bounds__(kReserveThreads) void reserve_group_kernel(const ReserveLaunch p) {
    __shared__ int s_need[kReserveGroup], s_fresh[kReserveGroup], s_blocks[kReserveGroup];
    __shared__ int64_t s_tokens[2][kReserveGroup];
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int b = blockIdx.x * kReserveGroup + wave;
    const int32_t top = reserve_top(p, kMany ? *p.top0 : *p.top);
    ReserveAsk ask{0, 0, 0, 0, 0};
    if (b < p.B) ask = reserve_ask(p, b, lane);
    ask.err = kMany ? 0 : ask.err;  // reported
    int64_t tokens = 0, all = 0;
    int blocks = 0;
    if (kMany) {
        for (int i = tid; i < (int)gridDim.x; i += kReserveThreads) {
            const ReserveSums t = p.sums[i];
            tokens += i < (int)blockIdx.x ? t.tokens : 0;
            blocks += i < (int)blockIdx.x ? t.blocks : 0;
            all += t.tokens;
        }
        tokens = wave_sum64(tokens);
        all = wave_sum64(all);
        blocks = wave_sum(blocks);
    }
    if (lane == 0) {
        s_need[wave] = max(ask.need, 0);
        s_fresh[wave] = ask.fresh;
        s_tokens[0][wave] = tokens;
        s_tokens[1][wave] = all;
        s_blocks[wave] = blocks;
    }
    __syncthreads();
    const int w = lane & (kReserveGroup - 1);
    const bool one = lane < kReserveGroup, before = one && w < wave;
    const int64_t fresh = s_fresh[w];
    tokens = wave_sum64((one ? s_tokens[0][w] : 0) + (before ? fresh : 0));
    blocks = wave_sum((one ? s_blocks[w] : 0) + (before ? s_need[w] : 0));
    all = wave_sum64(one ? (kMany ? s_tokens[1][w] : fresh) : 0);
    int32_t left = 0x7fffffff;
    if (b < p.B) left = reserve_take<64>(p, b, ask, top, tokens, blocks, all, lane, nullptr, nullptr);
    __syncthreads();  // the sums are read, and so is the top
    if (lane == 0) s_need[wave] = left;
    __syncthreads();
    if (tid == 0) {
#pragma unroll
        for (int i = 0; i < kReserveGroup; ++i) left = min(left, s_need[i]);
        if (left != 0x7fffffff) __hip_atomic_fetch_min(p.top, left, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
}

// Long prompts: a workgroup per sequence, behind reserve_count_kernel.
__global__ __launch_bounds__(kReserveThreads) void reserve_long_kernel(const ReserveLaunch p) {
    constexpr int kWaves = kReserveThreads / 64;
    __shared__ int64_t s_tokens[2][kWaves];
    __shared__ int s_blocks[kWaves];
    __shared__ int s_bad;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, b = blockIdx.x;
    const int groups = (p.B + kReserveGroup - 1) / kReserveGroup, mine = b / kReserveGroup;
    ReserveAsk ask{p.len[b], p.fresh[b], p.need[b], 0, 0};
    if (ask.len < 0 || ask.fresh < 0) ask.fresh = 0;
    const int32_t top = reserve_top(p, *p.top0);
    if (tid == 0) s_bad = 0;
    // tokens and blocks of the sequences before this one, and all tokens
    int64_t tokens = 0, all = 0;
    int blocks = 0;
    if (tid < b - mine * kReserveGroup) {
        const int o = mine * kReserveGroup + tid;
        blocks = max(p.need[o], 0);
        tokens = p.len[o] >= 0 ? max(p.fresh[o], 0) : 0;
    }
    for (int i = tid; i < groups; i += kReserveThreads) {
        const ReserveSums t = p.sums[i];
        tokens += i < mine ? t.tokens : 0;
        blocks += i < mine ? t.blocks : 0;
        all += t.tokens;
    }
    tokens = wave_sum64(tokens);
    all = wave_sum64(all);
    blocks = wave_sum(blocks);
    if (lane == 0) {
        s_tokens[0][wave] = tokens;
        s_tokens[1][wave] = all;
        s_blocks[wave] = blocks;
    }
    __syncthreads();
    tokens = all = blocks = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
        tokens += s_tokens[0][w];
        all += s_tokens[1][w];
        blocks += s_blocks[w];
    }
    __syncthreads();
    const int32_t left = reserve_take<kReserveThreads>(p, b, ask, top, tokens, blocks, all, tid, s_blocks, &s_bad);
    if (tid == 0 && left != 0x7fffffff) __hip_atomic_fetch_min(p.top, left, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// ---------------------------------------------------------------------------
// rope.  Position p turns pair i by the fraction p * freq[i] mod 2^64, an integer
// product that is exact at any position; its nearest quarter turn is taken off and the
// rest, at most pi / 4, goes through the Taylor series of sine and cosine.
// ---------------------------------------------------------------------------
static __device__ __forceinline__ void turn_of(uint64_t freq, int32_t p, float gain, float &cos, float &sin) {
    const uint64_t turn = freq * (uint64_t)(uint32_t)p;
    const uint32_t t = (uint32_t)(turn >> 32), quarter = (t + 0x20000000u) >> 30;
    const float x = (float)(int32_t)(t - (quarter << 30)) * 1.4629180792671596e-9f;  // 2 pi / 2^32: at most pi / 4
    const float x2 = x * x;
    // what is left off is below 2^-28: x^11 / 11! and x^12 / 12!
    float s = fmaf(x2, fmaf(x2, fmaf(x2, 2.7557319e-6f, -1.9841270e-4f), 8.3333333e-3f), -1.6666667e-1f);
    s = fmaf(x * x2, s, x);
    float c = fmaf(x2, fmaf(x2, fmaf(x2, fmaf(x2, -2.7557319e-7f, 2.4801587e-5f), -1.3888889e-3f), 4.1666667e-2f), -0.5f);
    c = fmaf(x2, c, 1.f);
    const bool swap = quarter & 1;
    const float cs = swap ? s : c, sn = swap ? c : s;
    // quarters 1 and 2 negate the cosine, 2 and 3 the sine
    cos = ((quarter + 1) & 2 ? -cs : cs) * gain;
    sin = (quarter & 2 ? -sn : sn) * gain;
}

// Where a token's heads go: q, then k, then v.
struct RopeToken {
    int layer, t;
    int32_t pos;
    int64_t cache;  // of its K and V in the cache, or -1
};
// The position of token x.t and where its K and V go; false if it is not there.
static __device__ __forceinline__ bool rope_token(const RopeLaunch &p, bool raise, RopeToken &x) {
    x.pos = p.pos[x.t];
    const int32_t slot = p.slot[x.t], seq = p.seq ? p.seq[x.t] : 0;
    if (x.pos < 0) return false;
    const bool good = slot < p.max_len && (uint32_t)seq < (uint32_t)p.n_seqs;
    x.cache = slot >= 0 && good ? x.layer * p.s_layer + seq * p.s_b + slot * p.s_pos : -1;
    if (slot >= 0 && !good && raise) raise_device_error(MURMUR_DEVERR_POSITION);
    return true;
}
template <typename T>
static __device__ __forceinline__ const T *rope_source(const RopeLaunch &p, const RopeToken &x, int h) {
    const int64_t kv = x.layer * p.kv_layer + x.t * p.kv_token;
    if (h < p.Hq) return reinterpret_cast<const T *>(p.q) + x.layer * p.q_layer + x.t * p.q_token + (int64_t)h * kHeadDim;
    if (h < p.Hq + p.Hkv) return reinterpret_cast<const T *>(p.k) + kv + (int64_t)(h - p.Hq) * kHeadDim;
    return reinterpret_cast<const T *>(p.v) + kv + (int64_t)(h - p.Hq - p.Hkv) * kHeadDim;
}
// null: not kept
static __device__ __forceinline__ uint16_t *rope_target(const RopeLaunch &p, const RopeToken &x, int h) {
    if (h < p.Hq) return p.q_out + (((int64_t)x.layer * p.n_tokens + x.t) * p.Hq + h) * kHeadDim;
    if (x.cache < 0) return nullptr;
    return h < p.Hq + p.Hkv ? p.k_cache + x.cache + (h - p.Hq) * p.s_h : p.v_cache + x.cache + (h - p.Hq - p.Hkv) * p.s_h;
}

// Eight values of a head as floats.
static __device__ __forceinline__ void load8(const uint16_t *from, float (&x)[8]) {
    const u32x4 y = load16(from);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __builtin_bit_cast(float, y[i] << 16);
        x[2 * i + 1] = __builtin_bit_cast(float, y[i] & 0xffff0000u);
    }
}
static __device__ __forceinline__ void load8(const float *from, float (&x)[8]) {
    const f32x4 y0 = *reinterpret_cast<const f32x4 *>(from), y1 = *reinterpret_cast<const f32x4 *>(from + 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[i] = y0[i];
        x[4 + i] = y1[i];
    }
}
static __device__ __forceinline__ void store8(uint16_t *to, const float (&x)[8]) {
    *reinterpret_cast<u32x4 *>(to) = u32x4{pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]), pack_bf16(x[4], x[5]), pack_bf16(x[6], x[7])};
}

// A wavefront per (layer, token), or kRopeHeads heads of one (p.parts of them), which
// takes fewer round trips to memory where there are few tokens: the current token of
// 12 sequences 4.0 us, 5.0 with a wavefront each (of bf16 a lane then loads a second
// head, which is another wavefront's to store).  A head is eight units
// of two 16-byte (bf16) chunks, a lane has one of them in every eighth head: eight
// pairs that turn alike in all heads, so the sines are computed once.  Bound by memory:
// 27 396 tokens of 36 heads, 505 MB, 98 us, 5.2 TB/s (a plain copy of 4 GiB reaches 4.7).
constexpr int kRopeHeads = 8;
template <typename T, bool kInterleaved>
__global__ __launch_bounds__(256) void rope_wide_kernel(const RopeLaunch p) {
    constexpr int kBatch = sizeof(T) == 2 ? 2 : 1;  // heads of a lane whose loads are on their way at once
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int u = lane & 7, heads = p.Hq + 2 * p.Hkv;
    const int64_t task = (int64_t)blockIdx.x * 4 + wave, item = task / p.parts;
    if (item >= (int64_t)p.NL * p.n_tokens) return;
    const int part = (int)(task - item * p.parts);
    const int h0 = part * kRopeHeads, h_end = p.parts > 1 ? min(h0 + kRopeHeads, heads) : heads;
    const int turns = kInterleaved ? min(max(p.rot / 2 - 8 * u, 0), 8) : (16 * u < p.rot ? 8 : 0);  // pairs that do
    const int at0 = kInterleaved || !turns ? 16 * u : 8 * u, at1 = kInterleaved || !turns ? 16 * u + 8 : p.rot / 2 + 8 * u;
    RopeToken x;
    x.layer = (int)(item / p.n_tokens);
    x.t = (int)(item - (int64_t)x.layer * p.n_tokens);
    float a[kBatch][8], b[kBatch][8];
    const auto load = [&](int h) {
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const T *from = rope_source<T>(p, x, min(h + 8 * j, heads - 1));
            load8(from + at0, a[j]);
            load8(from + at1, b[j]);
        }
    };
    uint64_t freq[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) freq[i] = i < turns ? p.freq[8 * u + i] : 0;
    const int first = h0 + (lane >> 3);
    if (p.parts > 1) load(first);  // before it is known whether the token is there: one round trip fewer
    if (!rope_token(p, part == 0 && lane == 0, x)) return;
    float cos[8], sin[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) turn_of(freq[i], x.pos, p.gain, cos[i], sin[i]);
    for (int h = first; h < h_end; h += 8 * kBatch) {
        if (p.parts == 1) load(h);
#pragma unroll
        for (int j = 0; j < kBatch; ++j) {
            const int hj = h + 8 * j;
            uint16_t *to = hj < h_end ? rope_target(p, x, hj) : nullptr;
            if (!to) continue;
            if (turns && hj < p.Hq + p.Hkv) {
                if (kInterleaved) {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        float &e = i < 4 ? a[j][2 * i] : b[j][2 * i - 8], &o = i < 4 ? a[j][2 * i + 1] : b[j][2 * i - 7];
                        const float y = fmaf(e, cos[i], -(o * sin[i])), z = fmaf(e, sin[i], o * cos[i]);
                        e = i < turns ? y : e;
                        o = i < turns ? z : o;
                    }
                } else {
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const float y = fmaf(a[j][i], cos[i], -(b[j][i] * sin[i]));
                        b[j][i] = fmaf(a[j][i], sin[i], b[j][i] * cos[i]);
                        a[j][i] = y;
                    }
                }
            }
            store8(to + at0, a[j]);
            store8(to + at1, b[j]);
        }
    }
}

// The half layout where the pairs' second elements do not start at a 16-byte chunk: a
// lane loads, turns and stores the eight elements of a chunk and finds the other one of
// each pair in LDS.  Lane i computes pair i's sines for the wavefront.  (26 880 tokens
// of 36 heads, 50 of 128 elements rotated: 98 us, 143 by pairs.)
template <typename T>
__global__ __launch_bounds__(256) void rope_mixed_kernel(const RopeLaunch p) {
    __shared__ float s_head[4][4][kHeadDim];  // four heads a wavefront
    __shared__ float2 s_turn[4][64];
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int heads = p.Hq + 2 * p.Hkv, half = p.rot / 2, mine = lane >> 4, c0 = 8 * (lane & 15);
    const int64_t item = (int64_t)blockIdx.x * 4 + wave;
    if (item >= (int64_t)p.NL * p.n_tokens) return;
    RopeToken x;
    x.layer = (int)(item / p.n_tokens);
    x.t = (int)(item - (int64_t)x.layer * p.n_tokens);
    if (!rope_token(p, lane == 0, x)) return;
    // LDS between the lanes of one wavefront, whose accesses are done in order
    const auto ordered = [] { asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory"); };
    if (lane < half) turn_of(p.freq[lane], x.pos, p.gain, s_turn[wave][lane].x, s_turn[wave][lane].y);
    ordered();
    float2 turn[8];  // cosine, and the sine that the other element takes
    int other[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int e = c0 + i;
        other[i] = e < half ? e + half : e - half;
        if (e >= p.rot) other[i] = e;
        turn[i] = e < p.rot ? s_turn[wave][min(e, other[i])] : float2{1.f, 0.f};
        if (e < half) turn[i].y = -turn[i].y;
    }
    for (int h0 = 0; h0 < heads; h0 += 4) {
        const int h = h0 + mine;
        float a[8];
        load8(rope_source<T>(p, x, min(h, heads - 1)) + c0, a);
        float *head = s_head[wave][mine];
        *reinterpret_cast<f32x4 *>(head + c0) = f32x4{a[0], a[1], a[2], a[3]};
        *reinterpret_cast<f32x4 *>(head + c0 + 4) = f32x4{a[4], a[5], a[6], a[7]};
        ordered();
        if (h < p.Hq + p.Hkv) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float y = fmaf(a[i], turn[i].x, head[other[i]] * turn[i].y);
                a[i] = c0 + i < p.rot ? y : a[i];
            }
        }
        ordered();
        uint16_t *to = h < heads ? rope_target(p, x, h) : nullptr;
        if (to) store8(to + c0, a);
    }
}

// The same for any rot_dim and alignment: a lane has a pair of elements of every head.
template <typename T>
__global__ __launch_bounds__(256) void rope_pair_kernel(const RopeLaunch p) {
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int64_t item = (int64_t)blockIdx.x * 4 + wave;
    if (item >= (int64_t)p.NL * p.n_tokens) return;
    RopeToken x;
    x.layer = (int)(item / p.n_tokens);
    x.t = (int)(item - (int64_t)x.layer * p.n_tokens);
    if (!rope_token(p, lane == 0, x)) return;
    const int half = p.rot / 2;
    const bool turns = lane < half;
    const int at0 = p.interleaved || !turns ? 2 * lane : lane, at1 = p.interleaved || !turns ? 2 * lane + 1 : half + lane;
    float cos = 1.f, sin = 0.f;
    if (turns) turn_of(p.freq[lane], x.pos, p.gain, cos, sin);
    const auto value = [](auto y) {
        if constexpr (sizeof(y) == 2) return __builtin_bit_cast(float, (uint32_t)y << 16);
        else return (float)y;
    };
    const int heads = p.Hq + 2 * p.Hkv;
#pragma unroll 4
    for (int h = 0; h < heads; ++h) {
        uint16_t *to = rope_target(p, x, h);
        if (!to) continue;
        const T *from = rope_source<T>(p, x, h);
        float a = value(from[at0]), b = value(from[at1]);
        if (turns && h < p.Hq + p.Hkv) {
            const float y = fmaf(a, cos, -(b * sin));
            b = fmaf(a, sin, b * cos);
            a = y;
        }
        const uint32_t both = pack_bf16(a, b);
        to[at0] = (uint16_t)both;
        to[at1] = (uint16_t)(both >> 16);
    }
}

// ---------------------------------------------------------------------------
// accept.  A wavefront follows the path from the root, a step a ballot; every
// workgroup of a sequence does so for itself, then they copy the path's rows.  Bound by
// round trips: a workgroup's planes one after the other, since a store may be to what
// the next load reads (64 sequences, 56 planes, 3.3 rows each: 10.0 us, 2.4 TB/s).
// ---------------------------------------------------------------------------
constexpr int kAcceptPlanes = 4;  // (layer, K or V) planes of a workgroup

__global__ __launch_bounds__(256) void tree_accept_kernel(const AcceptLaunch p) {
    const int tid = threadIdx.x, lane = tid & 63, b = blockIdx.x, T = p.T;
    const int par = lane < T ? p.parent[(p.parent_per_seq ? (int64_t)b * T : 0) + lane] : -2;
    const int32_t token = lane < T ? p.token[(int64_t)b * T + lane] : -1, next = lane < T ? p.next[(int64_t)b * T + lane] : -1;
    const int32_t slot = lane < T ? p.slot[(int64_t)b * T + lane] : -1;
    const uint64_t there = __ballot(par != -2);
    const bool ok = par == -2 || (lane == 0 ? par == -1 : par >= 0 && par < lane && (there >> (par & 63) & 1));
    const bool invalid = __ballot(!ok) != 0;
    int n = 0, at = 0;
    int32_t mine = -1, last = -1;  // lane i: the path's node i
    if (!invalid && (there & 1) && __builtin_amdgcn_readfirstlane(token) >= 0) {
        for (;;) {
            if (lane == n) mine = at;
            ++n;
            last = __builtin_amdgcn_readlane(next, at);
            const uint64_t child = __ballot(par == at && token == last && token >= 0);
            if (!child) break;
            at = __builtin_ctzll(child);
        }
    }
    const bool far = lane < n && slot >= p.max_len;
    if (blockIdx.y == 0 && tid < 64) {
        if (lane < T) p.path[(int64_t)b * T + lane] = mine;
        if (lane == 0) {
            p.count[b] = n;
            p.last[b] = last;
        }
        const int err = (invalid ? MURMUR_DEVERR_TREE : 0) | (__ballot(far) ? MURMUR_DEVERR_POSITION : 0);
        if (lane == 0 && err) raise_device_error(err);
    }
    const int chunks = p.Hkv * 16, planes = 2 * p.NL;
    for (int lv = blockIdx.y * kAcceptPlanes; lv < min((int)blockIdx.y * kAcceptPlanes + kAcceptPlanes, planes); ++lv) {
        const int layer = lv >> 1;
        const uint16_t *from = ((lv & 1) ? p.v_tree : p.k_tree) + ((int64_t)layer * p.B + b) * T * p.Hkv * kHeadDim;
        uint16_t *to = ((lv & 1) ? p.v : p.k) + layer * p.s_layer + b * p.s_b;
        for (int i0 = 0; i0 < n * chunks; i0 += 256) {  // every lane goes along: it may hold what another one needs
            const int i = i0 + tid, step = min(i / chunks, n - 1), c = i - step * chunks;
            const int32_t node = __shfl(mine, step), row = __shfl(slot, step);
            if (i < n * chunks && row >= 0 && row < p.max_len)
                *reinterpret_cast<u32x4 *>(to + row * p.s_pos + (c >> 4) * p.s_h + 8 * (c & 15)) =
                    load16(from + (int64_t)node * p.Hkv * kHeadDim + 8 * c);
        }
    }
}

// ---- launchers ----

int launch_paged_reserve(const ReserveLaunch &p, murmur_stream_t stream) {
    const hipStream_t s = (hipStream_t)stream;
    const dim3 groups((unsigned)((p.B + kReserveGroup - 1) / kReserveGroup)), threads(kReserveThreads);
    // 12 prompts of 2283 tokens: 6.1 us behind the count's 3.3; in one launch, a wavefront each, 14.2.  The map's length
    // stands for the sequences', which only the device knows: a long prompt among short requests is one wavefront's work
    // (27 000 tokens and 127 single ones 98 us, and 8 single ones, a workgroup each, 20).
    const bool few = p.n_tokens / p.B <= 256;
    if (few && groups.x == 1) {
        hipLaunchKernelGGL(reserve_group_kernel<false>, groups, threads, 0, s, p);
        return (int)hipGetLastError();
    }
    hipLaunchKernelGGL(reserve_count_kernel, groups, threads, 0, s, p);
    const int e = (int)hipGetLastError();
    if (e != 0) return e;
    if (few) hipLaunchKernelGGL(reserve_group_kernel<true>, groups, threads, 0, s, p);
    else hipLaunchKernelGGL(reserve_long_kernel, dim3((unsigned)p.B), threads, 0, s, p);
    return (int)hipGetLastError();
}

int launch_rope_append(const RopeLaunch &p, murmur_stream_t stream) {
    const dim3 grid((unsigned)(((int64_t)p.NL * p.n_tokens * p.parts + 3) / 4)), threads(256);
    const hipStream_t s = (hipStream_t)stream;
    if (p.wide && !p.interleaved && p.rot % 16 != 0) {
        if (p.f32) hipLaunchKernelGGL(rope_mixed_kernel<float>, grid, threads, 0, s, p);
        else hipLaunchKernelGGL(rope_mixed_kernel<uint16_t>, grid, threads, 0, s, p);
    } else if (!p.wide) {
        if (p.f32) hipLaunchKernelGGL(rope_pair_kernel<float>, grid, threads, 0, s, p);
        else hipLaunchKernelGGL(rope_pair_kernel<uint16_t>, grid, threads, 0, s, p);
    } else if (p.f32) {
        if (p.interleaved) hipLaunchKernelGGL((rope_wide_kernel<float, true>), grid, threads, 0, s, p);
        else hipLaunchKernelGGL((rope_wide_kernel<float, false>), grid, threads, 0, s, p);
    } else {
        if (p.interleaved) hipLaunchKernelGGL((rope_wide_kernel<uint16_t, true>), grid, threads, 0, s, p);
        else hipLaunchKernelGGL((rope_wide_kernel<uint16_t, false>), grid, threads, 0, s, p);
    }
    return (int)hipGetLastError();
}

int launch_tree_accept(const AcceptLaunch &p, murmur_stream_t stream) {
    const unsigned y = (unsigned)((2 * (int64_t)p.NL + kAcceptPlanes - 1) / kAcceptPlanes);
    hipLaunchKernelGGL(tree_accept_kernel, dim3((unsigned)p.B, y), dim3(256), 0, (hipStream_t)stream, p);
    return (int)hipGetLastError();
}

}  // namespace murmur
