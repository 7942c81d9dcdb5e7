// The gradient of attention (hq_attention_fwd.cu): the probabilities are recomputed from the scores and the row statistic.
//
//   P_ij = exp(scale q_i . k_j - lse_i),  dP = dout V^T,  D_i = dout_i . out_i,  dS = P o (dP - D)
//   dq = scale dS K,   dk = scale sum over the heads that share k of dS^T Q,   dv = sum of P^T dout
//
// A first kernel leaves -lse log2(e) and -D of every query.  Then two kinds of item in one launch, each with the sums it owns in tensor
// memory from its first step to its last, so that nothing is added up in memory and the same inputs give the same bits:
//   keys     a tile of 128 keys of one (sample, key head) walks the queries of every head of its group: S^T = K Q^T, dP^T = V dout^T
//            with the keys along the lanes, P^T and dS^T as bf16 over the columns they were computed from, dv += P^T dout,
//            dk += dS^T Q;
//   queries  a tile of 128 queries of one (sample, head) walks the keys: S = Q K^T, dP = dout V^T, dq += dS K.
// The scores are computed twice (seven products a pair of tiles where five would do); what that buys is that P and dS never leave
// tensor memory (as operands of the second products they are read where they were written), no fp32 partial dq in memory and no
// order of additions that changes from run to run.  Where tiles of keys are few and long each is cut into shares whose sums a last
// kernel adds in their order (bwd_parts).  P and dS are rounded to bf16 (the products' type); all sums are fp32.
//
// Up to 64 channels an item is a CTA of its own, two an SM (attention_bwd_small_kernel); above, persistent CTAs take item after item
// (attention_bwd_kernel).  Measured, the statistics' kernel included: 64 x 1024 tokens, 8 heads of 64 (481 GFLOP in seven products)
// 684 us in a run of calls, which the power limit holds to 1.6 GHz (650 in a short one), 239 us of it two passes of exponentials (16 a
// clock in an SM); 2 x 4096 causal, 16 / 2 heads of 128 501 us (460); 8 x 4096 queries on 77 keys, 8 heads of 40 86 us; 2 x 64 tokens, 8 heads
// of 64 12.1 us a call.
#include "hq_attention_tile.cuh"

namespace hq {
namespace {

constexpr int32_t kStatusBwdWait = 0x710, kStatusBwdTma = 0x711, kStatusBwdSmem = 0x712;
constexpr int kBwdWarps = 16, kBwdFirst = 4;                   // of the probabilities; in front of them the others (the issuing warp
                                                               // is the oldest of its scheduler's)
constexpr int kBwdThreads = (kBwdFirst + kBwdWarps) * 32;
constexpr uint32_t kStatBytes = kAttnTile * 4;                 // of one query tile: -lse * log2(e), and as many for -D

// Rings of the kernel above 64 channels: tiles of 32 KB, of which two kept ones, three and two take all but 3 KB of the 227 KB of shared
// memory; the statistics of the ring's tiles and the barriers take 2.75 KB of those.
struct BwdRings {
    static constexpr int kParts = 2, kB0 = 3, kB1 = 2;         // kParts: of 64 channels
    static constexpr int kTile = kParts * kAttnPart;
    static constexpr int kTiles = (2 + kB0 + kB1) * kTile, kStats = (kB0 + kB1) * int(kStatBytes);
};

struct BwdParams {
    AttnShape s;
    const float* stats;                            // [Nb * heads][q_tiles][2][128]
    unsigned* taken;                               // items taken beyond the first of every CTA
    __nv_bfloat16 *dq, *dk, *dv;
    int64_t lddq, lddk, lddv;
    int q_tiles, k_tiles;
    unsigned key_items, items, key_chunk, chunk;   // tiles of keys (each in `parts` items), items; their order (attn_order)
    int parts;                                     // shares of a tile of keys' steps, each an item; 1: no shares
    float* partial;                                // [parts][key_items][dk, dv][16 a part of 64 channels][128][4] sums of the shares
    int ragged;                                    // rows outside the lengths may lie in a tile
    int32_t* dev_status;
};
struct BwdMaps { CUtensorMap q, k, v, dout, dq, dk, dv; };

struct BwdBars {
    using R = BwdRings;
    uint64_t keep_full, keep_empty, b0_full[R::kB0], b0_empty[R::kB0], b1_full[R::kB1], b1_empty[R::kB1];
    // dP and dS of a step alternate between two barriers: where the next dP does not wait for this dS, one could come round twice
    // before a slow warp has looked at it
    uint64_t s, p, dp[2], ds[2], acc, drain, staged, item_full[2], item_empty[2];
    uint32_t item[2], tmem_slot;
};
constexpr size_t kBwdSmem = size_t(BwdRings::kTiles + BwdRings::kStats) + sizeof(BwdBars);
static_assert(kBwdSmem <= 227 * 1024, "the rings, their statistics and the barriers fit the shared memory of an SM");

// What an item is: a tile of keys of one (sample, key head) or of queries of one (sample, head), and the other side's tiles it walks.
struct BwdItem {
    bool keys;
    int n, head, tile, row0;
    AttnSample sm;
    int first, last, begin, total, whole;          // tiles [first, last) of each of its heads; its steps of the `whole` over all of them
    unsigned part, base;                           // which share of which tile of keys
};
// `block_rows`: of the other side's tiles.
__device__ __forceinline__ BwdItem bwd_item(const BwdParams& p, unsigned index, int block_rows = kAttnTile) {
    const AttnShape& s = p.s;
    BwdItem t;
    // tiles of keys first (they walk every head of their group); under the causal mask the first keys and the last queries walk the most
    t.keys = index < p.key_items * unsigned(p.parts);
    t.base = t.keys ? index / unsigned(p.parts) : index - p.key_items * unsigned(p.parts);
    t.part = t.keys ? index - t.base * unsigned(p.parts) : 0u;
    const unsigned heads = unsigned(t.keys ? s.kv_heads : s.heads);
    unsigned block, bh;
    attn_order(t.base, unsigned(t.keys ? p.k_tiles : p.q_tiles), unsigned(s.Nb) * heads, t.keys ? p.key_chunk : p.chunk, block, bh);
    t.n = int(bh / heads);
    t.head = int(bh - unsigned(t.n) * heads);
    t.tile = !t.keys && s.causal ? p.q_tiles - 1 - int(block) : int(block);
    t.row0 = t.tile * kAttnTile;
    t.sm = attn_sample(s, t.n);
    if (t.keys) {
        t.first = max(t.sm.q_lo, s.causal ? t.row0 - t.sm.shift : 0) / block_rows;
        t.last = t.row0 < t.sm.kl ? (t.sm.q_hi + block_rows - 1) / block_rows : 0;
    } else {
        const int end = min(t.row0 + kAttnTile, t.sm.q_hi) - 1;
        t.first = 0;
        t.last = t.row0 > end || end < t.sm.q_lo ? 0 : (attn_key_limit(s, t.sm, end) + block_rows - 1) / block_rows;
    }
    t.whole = t.total = max(0, t.last - t.first) * (t.keys ? s.heads / s.kv_heads : 1);
    t.begin = 0;
    if (t.keys && p.parts > 1) {
        t.begin = int(int64_t(t.whole) * t.part / p.parts);
        t.total = int(int64_t(t.whole) * (t.part + 1) / p.parts) - t.begin;
    }
    return t;
}

// ---- above 64 channels: persistent CTAs, one an SM; an item, then the next that no other has taken.  Warp 0 issues, warp 1 takes items
// and loads, warp 2 stores; warps 4-19: thread = lane, four warps per quarter of the 128 columns.  The tile an item keeps (K and V, or Q
// and dout) stays in shared memory, where its gradient is staged at the end; the other side's two kinds of tiles come through a ring each.

// Rows of a landed tile outside [lo, hi) become zeros (one warp): they belong to tokens outside the lengths, whose values may be
// infinite or not numbers, and would meet zero weights in a product.
__device__ __forceinline__ void clear_rows(unsigned char* tile, int lo, int hi, int lane) {
    for (int h = 0; h < BwdRings::kParts; ++h)
        for (int f = lane; f < kAttnTile * 8; f += 32) {
            const int row = f >> 3;
            if (row < lo || row >= hi) *reinterpret_cast<uint4*>(tile + h * kAttnPart + f * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
}

// A place in a ring and how often it has come round.
template <int N> struct RingAt {
    int slot = 0;
    uint32_t phase = 0;
    __device__ __forceinline__ void next() { if (++slot == N) { slot = 0; phase ^= 1u; } }
};

// ---- warp 1, one lane: takes items, tells the others, loads their tiles
__device__ __forceinline__ void bwd_load(const BwdMaps& m, const BwdParams& p, unsigned char* smem, float* stat0, float* stat1, BwdBars& bar) {
    using R = BwdRings;
    unsigned char *sB0 = smem + 2 * R::kTile, *sB1 = sB0 + R::kB0 * R::kTile;
    const int group = p.s.heads / p.s.kv_heads;
    uint32_t keep = 0;
    RingAt<R::kB0> b0;
    RingAt<R::kB1> b1;
    RingAt<2> told;
    int n0 = 0, n1 = 0;                 // begun so far
    bool ok = true, kept = false;
    unsigned index = blockIdx.x;
    while (ok) {
        ok = mbar_wait_lane(&bar.item_empty[told.slot], told.phase ^ 1u, p.dev_status, kStatusBwdWait);
        if (!ok) break;
        bar.item[told.slot] = index;
        mbar_arrive(&bar.item_full[told.slot]);
        told.next();
        if (index >= p.items) break;
        const unsigned following = gridDim.x + atomicAdd(p.taken, 1u);
        const BwdItem t = bwd_item(p, index);
        index = following;
        if (t.total == 0) continue;
        ok = mbar_wait_lane(&bar.keep_empty, keep ^ 1u, p.dev_status, kStatusBwdWait);
        if (!ok) break;
        mbar_expect_tx(&bar.keep_full, 2 * R::kTile);
        load_tile<BwdRings::kParts>(smem, t.keys ? &m.k : &m.q, &bar.keep_full, t.head, t.row0, t.n);
        load_tile<BwdRings::kParts>(smem + R::kTile, t.keys ? &m.v : &m.dout, &bar.keep_full, t.head, t.row0, t.n);
        keep ^= 1u;
        kept = true;
        const int per_head = t.last - t.first;
        int head = t.keys ? t.head * group + t.begin / per_head : t.head / group, tile = t.first + t.begin % per_head;
        for (int i = 0; i < t.total; ++i) {
            const float* stats = p.stats + (int64_t(t.n * p.s.heads + head) * p.q_tiles + tile) * (2 * kAttnTile);
            ok = mbar_wait_lane(&bar.b0_empty[b0.slot], b0.phase ^ 1u, p.dev_status, kStatusBwdWait);
            if (!ok) break;
            mbar_expect_tx(&bar.b0_full[b0.slot], R::kTile + (t.keys ? kStatBytes : 0));
            load_tile<BwdRings::kParts>(sB0 + b0.slot * R::kTile, t.keys ? &m.q : &m.k, &bar.b0_full[b0.slot], head, tile * kAttnTile, t.n);
            if (t.keys) bulk_load(stat0 + b0.slot * kAttnTile, stats, kStatBytes, &bar.b0_full[b0.slot]);
            b0.next();
            ++n0;
            ok = mbar_wait_lane(&bar.b1_empty[b1.slot], b1.phase ^ 1u, p.dev_status, kStatusBwdWait);
            if (!ok) break;
            mbar_expect_tx(&bar.b1_full[b1.slot], R::kTile + (t.keys ? kStatBytes : 0));
            load_tile<BwdRings::kParts>(sB1 + b1.slot * R::kTile, t.keys ? &m.dout : &m.v, &bar.b1_full[b1.slot], head, tile * kAttnTile, t.n);
            if (t.keys) bulk_load(stat1 + b1.slot * kAttnTile, stats + kAttnTile, kStatBytes, &bar.b1_full[b1.slot]);
            b1.next();
            ++n1;
            if (++tile == t.last) { tile = t.first; ++head; }
        }
    }
    // what was requested lands before the CTA's shared memory is given up, on every way out
    if (kept) mbar_wait_lane(&bar.keep_full, keep ^ 1u, nullptr, 0);
    for (int i = max(0, n0 - R::kB0); i < n0; ++i) mbar_wait_lane(&bar.b0_full[i % R::kB0], uint32_t(i / R::kB0) & 1u, nullptr, 0);
    for (int i = max(0, n1 - R::kB1); i < n1; ++i) mbar_wait_lane(&bar.b1_full[i % R::kB1], uint32_t(i / R::kB1) & 1u, nullptr, 0);
}

// The next item's number (p.items and beyond: none, or a wait ran out), the same in every lane.
__device__ __forceinline__ unsigned bwd_next(const BwdParams& p, BwdBars& bar, RingAt<2>& told, int lane) {
    if (!mbar_wait_warp(&bar.item_full[told.slot], told.phase, p.dev_status, kStatusBwdWait)) return 0xffffffffu;
    const unsigned index = *const_cast<volatile uint32_t*>(&bar.item[told.slot]);
    __syncwarp();
    if (lane == 0) mbar_arrive(&bar.item_empty[told.slot]);
    told.next();
    return index;
}

// ---- warp 0: products.  Tensor memory: S at columns 0, dP at 128; keys: dv at 256, dk at 384; queries: dP's second buffer at 256,
// dq at 384.  Products run in the order of their issue: one that overwrites another's operand or result in tensor memory, or an
// accumulator that the other warps have read before they handed over the operand it waits for, is issued behind it.
__device__ __forceinline__ void bwd_issue(const BwdParams& p, unsigned char* smem, BwdBars& bar, uint32_t tmem_base, int lane) {
    using R = BwdRings;
    const AttnShape& s = p.s;
    unsigned char *sB0 = smem + 2 * R::kTile, *sB1 = sB0 + R::kB0 * R::kTile;
    const uint32_t idesc_s = make_idesc_bf16(kAttnTile, kAttnTile, false);
    const uint32_t idesc_acc = make_idesc_bf16(kAttnTile, (s.dh + 15) & ~15, true);
    const int ksteps = (s.dh + 15) / 16;
    const uint64_t dA = make_sw128_kmajor_desc(smem_u32(smem));
    const uint64_t dB0 = make_sw128_kmajor_desc(smem_u32(sB0)), dB1 = make_sw128_kmajor_desc(smem_u32(sB1));
    const uint64_t dB0t = make_sw128_mnmajor_desc(smem_u32(sB0), kAttnPart), dB1t = make_sw128_mnmajor_desc(smem_u32(sB1), kAttnPart);
    constexpr uint64_t kTileUnits = R::kTile >> 4;
    auto score_product = [&](uint64_t a, uint64_t b, uint32_t column) {
        for (int k = 0; k < ksteps; ++k) {
            const uint64_t step = uint64_t((k >> 2) * (kAttnPart >> 4) + 2 * (k & 3));
            mma_bf16(tmem_base + column, a + step, b + step, idesc_s, k != 0 ? 1u : 0u);
        }
    };
    // bf16 operand of each quarter in the first half of its 32 columns
    auto acc_product = [&](uint32_t column, uint64_t b, uint32_t acc, bool add) {
#pragma unroll
        for (int k = 0; k < kAttnTile / 16; ++k)
            mma_bf16_ts(tmem_base + acc, tmem_base + column + uint32_t((k >> 1) * 32 + (k & 1) * 8), b + uint64_t(k * 128), idesc_acc,
                        add || k != 0 ? 1u : 0u);
    };
    auto wait = [&](uint64_t* b, uint32_t parity, int32_t code) { return mbar_wait_warp(b, parity, p.dev_status, code); };
    uint32_t keep = 0;
    RingAt<R::kB0> s0, a0;                         // B0's tile of the next score product / of the next sum
    RingAt<R::kB1> s1, a1;
    RingAt<2> told;
    uint32_t step = 0;                             // over all items
    for (;;) {
        const unsigned index = bwd_next(p, bar, told, lane);
        if (index >= p.items) return;
        const BwdItem t = bwd_item(p, index);
        if (t.total == 0) continue;
        // rows of tokens outside the lengths (zero as they come behind the last row of the matrix) are made zero where they would
        // meet zero probabilities in a sum: queries and their gradients, or keys
        int tile = t.first + t.begin % (t.last - t.first);
        const int outer_lo = t.keys ? t.sm.q_lo : 0, outer_hi = t.keys ? t.sm.q_hi : t.sm.kl, exist = t.keys ? s.Lq : s.Lk;
        auto clear = [&](unsigned char* at, int which_tile) {
            const int r0 = which_tile * kAttnTile;
            if (outer_lo > r0 || outer_hi < min(r0 + kAttnTile, exist)) {
                clear_rows(at, outer_lo - r0, outer_hi - r0, lane);
                fence_proxy_async_smem();
                __syncwarp();
            }
        };
        if (!wait(&bar.keep_full, keep, kStatusBwdTma)) return;
        keep ^= 1u;
        auto scores = [&](int which_tile) {        // S of the next tile
            if (!wait(&bar.b0_full[s0.slot], s0.phase, kStatusBwdTma)) return false;
            clear(sB0 + s0.slot * R::kTile, which_tile);
            if (elect_one()) {
                tc_fence_after();
                score_product(dA, dB0 + uint64_t(s0.slot) * kTileUnits, 0u);
                mma_commit(&bar.s);
            }
            __syncwarp();
            s0.next();
            return true;
        };
        auto dprobs = [&](int which_tile, uint32_t column, uint32_t of) {  // dP of the next tile, step `of`
            if (!wait(&bar.b1_full[s1.slot], s1.phase, kStatusBwdTma)) return false;
            if (t.keys) clear(sB1 + s1.slot * R::kTile, which_tile);
            if (elect_one()) {
                tc_fence_after();
                score_product(dA + kTileUnits, dB1 + uint64_t(s1.slot) * kTileUnits, column);
                mma_commit(&bar.dp[of & 1u]);
                if (!t.keys) mma_commit(&bar.b1_empty[s1.slot]);
            }
            __syncwarp();
            s1.next();
            return true;
        };
        if (!scores(tile) || !dprobs(tile, 128u, step)) return;
        for (int i = 0; i < t.total; ++i) {
            const bool more = i + 1 < t.total;
            if (++tile == t.last) tile = t.first;
            if (!wait(&bar.p, step & 1u, kStatusBwdWait)) return;
            if (t.keys) {
                if (elect_one()) {
                    tc_fence_after();
                    acc_product(0u, dB1t + uint64_t(a1.slot) * kTileUnits, 256u, i != 0);
                }
                __syncwarp();
                if (more && !scores(tile)) return;
            } else if (more) {
                if (!scores(tile) || !dprobs(tile, 128u + 128u * uint32_t((i + 1) & 1), step + 1u)) return;
            }
            if (!wait(&bar.ds[step & 1u], (step >> 1) & 1u, kStatusBwdWait)) return;
            if (elect_one()) {
                tc_fence_after();
                acc_product(t.keys || !(i & 1) ? 128u : 256u, dB0t + uint64_t(a0.slot) * kTileUnits, 384u, i != 0);
                mma_commit(&bar.b0_empty[a0.slot]);
                if (t.keys) mma_commit(&bar.b1_empty[a1.slot]);        // its statistics have been read by now
                if (!more) mma_commit(&bar.acc);
            }
            __syncwarp();
            a0.next();
            a1.next();
            if (t.keys && more && !dprobs(tile, 128u, step + 1u)) return;
            ++step;
        }
    }
}

// ---- warps 4-19: probabilities and their gradients
template <bool KEYS>
__device__ __forceinline__ bool bwd_probabilities(const BwdParams& p, const BwdItem& t, const float* stat0, const float* stat1, BwdBars& bar,
                                                  RingAt<BwdRings::kB0>& b0, RingAt<BwdRings::kB1>& b1, uint32_t& step,
                                                  uint32_t t_s, int r, int quarter, int lane) {
    const AttnShape& s = p.s;
    const f32x2 sc2 = pk2(s.scale_log2, s.scale_log2);
    f32x2 row_lse = 0, row_d = 0;
    int limit = 0;                                             // queries: keys the row sees
    if (!KEYS) {
        const float* stats = p.stats + (int64_t(t.n * s.heads + t.head) * p.q_tiles + t.tile) * (2 * kAttnTile) + (r - t.row0);
        const float l = ld_dependent(stats), d = ld_dependent(stats + kAttnTile);
        row_lse = pk2(l, l);
        row_d = pk2(d, d);
        limit = r < t.sm.q_hi ? attn_key_limit(s, t.sm, r) : 0;
        if (limit == 1) limit = 0;                             // a weight of 1, whatever its score: no gradient
    }
    int tile = t.first + t.begin % (t.last - t.first);
    for (int i = 0; i < t.total; ++i) {
        const int c0 = tile * kAttnTile + quarter * 32;        // the first column's query or key
        if (++tile == t.last) tile = t.first;
        if (!mbar_wait_warp(&bar.s, step & 1u, p.dev_status, kStatusBwdWait)) return false;
        if (KEYS && !mbar_wait_warp(&bar.b0_full[b0.slot], b0.phase, p.dev_status, kStatusBwdTma)) return false;
        tc_fence_after();
        uint32_t sr[32], w[16];
        tmem_ld_32x32(t_s, sr);
        tmem_ld_wait_32(sr);
        if (!KEYS) {
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.p);
        }
        const float* nl = stat0 + b0.slot * kAttnTile + quarter * 32;
        f32x2 pr[16];
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            f32x2 l0 = row_lse, l1 = row_lse;
            if (KEYS) {
                const ulonglong2 l = *reinterpret_cast<const ulonglong2*>(nl + 2 * e);
                l0 = l.x; l1 = l.y;
            }
            float z[4];
            upk2(fma2(pk2(__uint_as_float(sr[2 * e]), __uint_as_float(sr[2 * e + 1])), sc2, l0), z[0], z[1]);
            upk2(fma2(pk2(__uint_as_float(sr[2 * e + 2]), __uint_as_float(sr[2 * e + 3])), sc2, l1), z[2], z[3]);
            pr[e] = pk2(ex2(z[0]), ex2(z[1]));
            pr[e + 1] = pk2(ex2(z[2]), ex2(z[3]));
        }
        if (KEYS) {
            // queries in front of the first that sees the row's key
            const int from = s.causal ? r - t.sm.shift - c0 : 0;
            if (__any_sync(0xffffffffu, from > 0)) {
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float a, b;
                    upk2(pr[e], a, b);
                    pr[e] = pk2(2 * e < from ? 0.f : a, 2 * e + 1 < from ? 0.f : b);
                }
            }
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                float a, b;
                upk2(pr[e], a, b);
                w[e] = pack_bf16(a, b);
            }
            tmem_st_32x16(t_s, w);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.p);
        }
        if (!mbar_wait_warp(&bar.dp[step & 1u], (step >> 1) & 1u, p.dev_status, kStatusBwdWait)) return false;
        if (KEYS && !mbar_wait_warp(&bar.b1_full[b1.slot], b1.phase, p.dev_status, kStatusBwdTma)) return false;
        tc_fence_after();
        const uint32_t t_dp = t_s + (KEYS || !(i & 1) ? 128u : 256u);
        const float* nd = stat1 + b1.slot * kAttnTile + quarter * 32;
        tmem_ld_32x32(t_dp, sr);
        tmem_ld_wait_32(sr);
#pragma unroll
        for (int e = 0; e < 16; e += 2) {
            f32x2 d0 = row_d, d1 = row_d;
            if (KEYS) {
                const ulonglong2 d = *reinterpret_cast<const ulonglong2*>(nd + 2 * e);
                d0 = d.x; d1 = d.y;
            }
            float a, b;
            upk2(mul2(pr[e], add2(pk2(__uint_as_float(sr[2 * e]), __uint_as_float(sr[2 * e + 1])), d0)), a, b);
            w[e] = pack_bf16(a, b);
            upk2(mul2(pr[e + 1], add2(pk2(__uint_as_float(sr[2 * e + 2]), __uint_as_float(sr[2 * e + 3])), d1)), a, b);
            w[e + 1] = pack_bf16(a, b);
        }
        if (KEYS) {
            if (t.sm.kl == 1) {                                // every query sees one key only
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = 0u;
            }
            // causal, as many queries as keys or more: the first that sees a key sees this one only, a weight of 1 whatever its score
            const int one = r == 0 ? -t.sm.shift - c0 : -1;
            if (s.causal && __any_sync(0xffffffffu, unsigned(one) < 32u)) {
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] &= one == 2 * e ? 0xFFFF0000u : one == 2 * e + 1 ? 0xFFFFu : 0xFFFFFFFFu;
            }
        } else {
            const int valid = limit - c0;                      // what lies behind may be anything
            if (__any_sync(0xffffffffu, valid < 32)) {
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] &= 2 * e + 1 < valid ? 0xFFFFFFFFu : 2 * e < valid ? 0xFFFFu : 0u;
            }
        }
        tmem_st_32x16(t_dp, w);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar.ds[step & 1u]);
        b0.next();
        b1.next();
        ++step;
    }
    return true;
}

// 32 columns of a share's sums (which: 0 dk, 1 dv) as they are: 16 bytes of a row, rows side by side.
__device__ __forceinline__ void store_share(const BwdParams& p, const BwdItem& t, uint32_t taddr, int which, int row, int c0, int parts64) {
    if (c0 >= p.s.dh) return;
    uint32_t r[32];
    tmem_ld_32x32(taddr, r);
    tmem_ld_wait_32(r);
    float4* to = reinterpret_cast<float4*>(p.partial) +
                 ((int64_t(t.part) * p.key_items + t.base) * 2 + which) * (parts64 * 16 * kAttnTile) + (c0 / 4) * kAttnTile + row;
#pragma unroll
    for (int c = 0; c < 8; ++c)
        to[c * kAttnTile] = make_float4(__uint_as_float(r[4 * c]), __uint_as_float(r[4 * c + 1]), __uint_as_float(r[4 * c + 2]), __uint_as_float(r[4 * c + 3]));
}
// dk and dv of a tile of keys from its shares, in their order: blockIdx.x the tile, blockIdx.y dk or dv, blockIdx.z 16 channels.
__global__ void __launch_bounds__(256) attention_bwd_join_kernel(const BwdParams p, int parts64, int block_rows) {
    const AttnShape& s = p.s;
    const int which = blockIdx.y, c = blockIdx.z * 2 + (threadIdx.x >> 7), row = threadIdx.x & 127;
    griddep_wait();
    if (c >= s.dh / 8) return;
    const BwdItem t = bwd_item(p, blockIdx.x * unsigned(p.parts), block_rows);
    const int64_t tile = int64_t(parts64) * 16 * kAttnTile, step = int64_t(p.key_items) * 2 * tile;
    const float4* from = reinterpret_cast<const float4*>(p.partial) + (int64_t(t.base) * 2 + which) * tile + 2 * c * kAttnTile + row;
    float a[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    auto add = [&](int x) {
        const float4 u = ld_dependent_cg(from + x * step), v = ld_dependent_cg(from + x * step + kAttnTile);
        a[0] += u.x; a[1] += u.y; a[2] += u.z; a[3] += u.w; a[4] += v.x; a[5] += v.y; a[6] += v.z; a[7] += v.w;
    };
    if (t.row0 + row < t.sm.kl) {
        if (t.whole >= p.parts) {
#pragma unroll 4
            for (int x = 0; x < p.parts; ++x) add(x);
        } else {                                               // shares without steps have written nothing
            for (int x = 0; x < p.parts; ++x)
                if (int64_t(t.whole) * x / p.parts != int64_t(t.whole) * (x + 1) / p.parts) add(x);
        }
    }
    if (t.row0 + row < s.Lk) {
        const int64_t ld = which == 0 ? p.lddk : p.lddv;
        const float mul = which == 0 ? s.scale : 1.0f;
        *reinterpret_cast<uint4*>((which == 0 ? p.dk : p.dv) + (int64_t(t.n) * s.Lk + t.row0 + row) * ld + t.head * s.dh + c * 8) =
            make_uint4(pack_bf16(a[0] * mul, a[1] * mul), pack_bf16(a[2] * mul, a[3] * mul), pack_bf16(a[4] * mul, a[5] * mul),
                       pack_bf16(a[6] * mul, a[7] * mul));
    }
}

__global__ void __launch_bounds__(kBwdThreads, 1) attention_bwd_kernel(const __grid_constant__ BwdMaps m, const BwdParams p) {
    using R = BwdRings;
    extern __shared__ __align__(1024) unsigned char smem[];
    float *stat0 = reinterpret_cast<float*>(smem + R::kTiles), *stat1 = stat0 + R::kB0 * kAttnTile;
    BwdBars& bar = *reinterpret_cast<BwdBars*>(smem + R::kTiles + R::kStats);
    const AttnShape& s = p.s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((smem_u32(smem) & 1023u) != 0) {                       // the tiles' swizzle needs it; dynamic shared memory begins there
        if (threadIdx.x == 0 && p.dev_status != nullptr) atomicExch(p.dev_status, kStatusBwdSmem);
        return;
    }
    if (threadIdx.x == 0) {
        mbar_init(&bar.keep_full, 1); mbar_init(&bar.keep_empty, 1); mbar_init(&bar.staged, kBwdWarps);
        for (int i = 0; i < R::kB0; ++i) { mbar_init(&bar.b0_full[i], 1); mbar_init(&bar.b0_empty[i], 1); }
        for (int i = 0; i < R::kB1; ++i) { mbar_init(&bar.b1_full[i], 1); mbar_init(&bar.b1_empty[i], 1); }
        mbar_init(&bar.s, 1); mbar_init(&bar.p, kBwdWarps); mbar_init(&bar.acc, 1); mbar_init(&bar.drain, 1);
        for (int i = 0; i < 2; ++i) { mbar_init(&bar.dp[i], 1); mbar_init(&bar.ds[i], kBwdWarps); }
        for (int i = 0; i < 2; ++i) { mbar_init(&bar.item_full[i], 1); mbar_init(&bar.item_empty[i], kBwdWarps + 2); }
        fence_barrier_init();
    }
    if (warp == 1 && lane < 7) tma_prefetch_desc(&m.q + lane);
    if (warp == 0) { __syncwarp(); tmem_alloc(&bar.tmem_slot, 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = bar.tmem_slot;
    griddep_wait();                                // the statistics; the call's operands were complete before that kernel began

    if (warp == 1) {
        if (elect_one()) bwd_load(m, p, smem, stat0, stat1, bar);
        __syncwarp();
    } else if (warp == 0) {
        bwd_issue(p, smem, bar, tmem_base, lane);
        __syncwarp();
        if (elect_one()) mma_drain(&bar.drain);                // the lane that issued
        __syncwarp();
    } else if (warp == 2) {
        RingAt<2> told;
        uint32_t keep = 0;
        for (;;) {
            const unsigned index = bwd_next(p, bar, told, lane);
            if (index >= p.items) break;
            const BwdItem t = bwd_item(p, index);
            if (t.total == 0) continue;
            if (!mbar_wait_warp(&bar.staged, keep, p.dev_status, kStatusBwdWait)) break;
            if (elect_one()) {
                if (!t.keys || p.parts == 1) {                 // the shares' sums went to memory as they are
#pragma unroll
                    for (int h = 0; h < R::kParts; ++h) tma_store_4d(t.keys ? &m.dk : &m.dq, smem + h * kAttnPart, 64 * h, t.head, t.row0, t.n);
                    if (t.keys) {
#pragma unroll
                        for (int h = 0; h < R::kParts; ++h) tma_store_4d(&m.dv, smem + R::kTile + h * kAttnPart, 64 * h, t.head, t.row0, t.n);
                    }
                    bulk_commit_group();
                    bulk_wait_read_all();
                }
                mbar_arrive(&bar.keep_empty);
            }
            __syncwarp();
            keep ^= 1u;
        }
    } else if (warp >= kBwdFirst) {
        const int quarter = (warp - kBwdFirst) >> 2, row = (warp & 3) * 32 + lane;
        const uint32_t t_lane = tmem_base + (uint32_t((warp & 3) * 32) << 16), t_s = t_lane + uint32_t(quarter * 32);
        RingAt<2> told;
        uint32_t keep = 0;
        RingAt<R::kB0> b0;
        RingAt<R::kB1> b1;
        uint32_t step = 0, item_par = 0;
        for (;;) {
            const unsigned index = bwd_next(p, bar, told, lane);
            if (index >= p.items) break;
            const BwdItem t = bwd_item(p, index);
            if (t.total == 0) {                                // nothing seen: the gradient is zero
                if (t.keys && p.parts > 1) continue;
                if (t.keys) {
                    const int rows = min(kAttnTile, s.Lk - t.row0);
                    const int64_t at = int64_t(t.n) * s.Lk + t.row0;
                    zero_rows(p.dk + at * p.lddk + t.head * s.dh, p.lddk, rows, s.dh, int(threadIdx.x) - kBwdFirst * 32, kBwdWarps * 32);
                    zero_rows(p.dv + at * p.lddv + t.head * s.dh, p.lddv, rows, s.dh, int(threadIdx.x) - kBwdFirst * 32, kBwdWarps * 32);
                } else {
                    zero_rows(p.dq + (int64_t(t.n) * s.Lq + t.row0) * p.lddq + t.head * s.dh, p.lddq, min(kAttnTile, s.Lq - t.row0), s.dh, int(threadIdx.x) - kBwdFirst * 32, kBwdWarps * 32);
                }
                continue;
            }
            const int r = t.row0 + row;
            const bool done = t.keys ? bwd_probabilities<true>(p, t, stat0, stat1, bar, b0, b1, step, t_s, r, quarter, lane)
                                     : bwd_probabilities<false>(p, t, stat0, stat1, bar, b0, b1, step, t_s, r, quarter, lane);
            if (!done || !mbar_wait_warp(&bar.acc, item_par, p.dev_status, kStatusBwdWait)) break;
            tc_fence_after();
            if (t.keys && p.parts > 1) {
                store_share(p, t, t_s + 384u, 0, row, quarter * 32, R::kParts);
                store_share(p, t, t_s + 256u, 1, row, quarter * 32, R::kParts);
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar.staged);
                keep ^= 1u;
                item_par ^= 1u;
                continue;
            }
            const bool kept = t.keys ? r < t.sm.kl : r >= t.sm.q_lo && r < t.sm.q_hi;
            stage_rows<BwdRings::kParts>(t_s + 384u, smem, row, quarter, s.dh, kept, s.scale);
            if (t.keys) stage_rows<BwdRings::kParts>(t_s + 256u, smem + R::kTile, row, quarter, s.dh, kept, 1.0f);
            tc_fence_before();
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.staged);
            keep ^= 1u;
            item_par ^= 1u;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem_base, 512);
}

// ---- up to 64 channels: small CTAs, two an SM, one tile each.  The other side comes in blocks of 64, so that S, dP and the sums of a
// CTA fit 256 columns of tensor memory; what one CTA waits for, the other's work covers.  Warps 0-7: thread = lane, four warps per half
// of the 64 columns; one lane of warp 8 issues, warp 9 loads and clears rows outside the lengths.
constexpr int kSmallBlock = 64, kSmallStages = 3, kSmallThreads = 320, kSmallPart = kSmallBlock * 128;
constexpr size_t kSmallSmem = size_t(2) * kAttnPart + size_t(kSmallStages) * (2 * kSmallPart + 2 * kSmallBlock * 4) + 1024;

struct SmallBars { uint64_t drain, keep, full[kSmallStages], ready[kSmallStages], empty[kSmallStages], s, dp[2], read, ds[2], acc; };

// KEYS: A0 = K, A1 = V, B0 = Q, B1 = dout; else A0 = Q, A1 = dout, B0 = K, B1 = V.  Columns: S at 0, dP at 64 (queries: a second
// buffer at 128), the sums at 128 (dv) and 192 (dk, dq).
template <bool KEYS>
__device__ __forceinline__ bool small_run(const BwdMaps& m, const BwdParams& p, const BwdItem& t, unsigned char* smem, SmallBars& bar, uint32_t tmem_base) {
    constexpr uint32_t kTile = kAttnPart;
    const AttnShape& s = p.s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    unsigned char* sB = smem + 2 * kTile;
    float* stat = reinterpret_cast<float*>(sB + kSmallStages * 2 * kSmallPart);              // of a stage: -lse log2(e), -D of 64 queries
    const int group = s.heads / s.kv_heads, first = t.first, last = t.last, total = t.total;
    bool ok = true;

    if (warp == 9) {
        const CUtensorMap *a0 = KEYS ? &m.k : &m.q, *a1 = KEYS ? &m.v : &m.dout, *b0 = KEYS ? &m.q : &m.k, *b1 = KEYS ? &m.dout : &m.v;
        // rows of tokens outside the lengths (zero as they come behind the last row of the matrix) are made zero where they would meet
        // zero probabilities in a sum: queries and their gradients, or keys
        const int lo = KEYS ? t.sm.q_lo : 0, hi = KEYS ? t.sm.q_hi : t.sm.kl, exist = KEYS ? s.Lq : s.Lk;
        auto make_ready = [&](int i, int block) {
            const int stage = i % kSmallStages, r0 = block * kSmallBlock;
            if (!mbar_wait_warp(&bar.full[stage], uint32_t(i / kSmallStages) & 1u, p.dev_status, kStatusBwdTma)) return false;
            if (lo > r0 || hi < min(r0 + kSmallBlock, exist)) {
                unsigned char* at = sB + stage * 2 * kSmallPart;
                for (int f = lane; f < kSmallBlock * 8; f += 32) {
                    const int r = r0 + (f >> 3);
                    if (r < lo || r >= hi) {
                        *reinterpret_cast<uint4*>(at + f * 16) = make_uint4(0u, 0u, 0u, 0u);
                        if (KEYS) *reinterpret_cast<uint4*>(at + kSmallPart + f * 16) = make_uint4(0u, 0u, 0u, 0u);
                    }
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.ready[stage]);
            return true;
        };
        if (elect_one()) {
            mbar_expect_tx(&bar.keep, 2 * kTile);
            for (int x = 0; x < 2; ++x) {          // boxes of 64 rows
                tma_load_4d(smem + x * kSmallPart, a0, &bar.keep, 0, t.head, t.row0 + x * kSmallBlock, t.n);
                tma_load_4d(smem + kTile + x * kSmallPart, a1, &bar.keep, 0, t.head, t.row0 + x * kSmallBlock, t.n);
            }
        }
        __syncwarp();
        int head = KEYS ? t.head * group + t.begin / (last - first) : t.head / group, block = first + t.begin % (last - first), before = block, i = 0;
        for (; i < total; ++i) {
            const int stage = i % kSmallStages, use = i / kSmallStages;
            if (use > 0) ok = mbar_wait_warp(&bar.empty[stage], uint32_t(use - 1) & 1u, p.dev_status, kStatusBwdWait);
            if (!ok) break;
            if (elect_one()) {
                unsigned char* to = sB + stage * 2 * kSmallPart;
                mbar_expect_tx(&bar.full[stage], 2 * kSmallPart + (KEYS ? 2 * kSmallBlock * 4 : 0));
                tma_load_4d(to, b0, &bar.full[stage], 0, head, block * kSmallBlock, t.n);
                tma_load_4d(to + kSmallPart, b1, &bar.full[stage], 0, head, block * kSmallBlock, t.n);
                if (KEYS) {
                    const float* from = p.stats + (int64_t(t.n * s.heads + head) * p.q_tiles + (block >> 1)) * (2 * kAttnTile) + (block & 1) * kSmallBlock;
                    bulk_load(stat + stage * 2 * kSmallBlock, from, kSmallBlock * 4, &bar.full[stage]);
                    bulk_load(stat + stage * 2 * kSmallBlock + kSmallBlock, from + kAttnTile, kSmallBlock * 4, &bar.full[stage]);
                }
            }
            __syncwarp();
            if (p.ragged && i > 0) {               // one step behind the loads
                ok = make_ready(i - 1, before);
                if (!ok) { ++i; break; }
                if (++before == last) before = first;
            }
            if (++block == last) { block = first; ++head; }
        }
        if (ok && p.ragged) ok = make_ready(total - 1, before);
        // what was requested lands before the CTA's shared memory is given up, on every way out
        mbar_wait_warp(&bar.keep, 0, nullptr, 0);
        for (int x = max(0, i - kSmallStages); x < i; ++x) mbar_wait_warp(&bar.full[x % kSmallStages], uint32_t(x / kSmallStages) & 1u, nullptr, 0);
    } else if (warp == 8) {
        if (elect_one()) {
            const uint32_t idesc_s = make_idesc_bf16(kAttnTile, kSmallBlock, false), idesc_acc = make_idesc_bf16(kAttnTile, (s.dh + 15) & ~15, true);
            const int ksteps = (s.dh + 15) / 16;
            const uint64_t dA = make_sw128_kmajor_desc(smem_u32(smem)), dB = make_sw128_kmajor_desc(smem_u32(sB)), dBt = make_sw128_mnmajor_desc(smem_u32(sB), kSmallPart);
            auto wait = [&](uint64_t* b, uint32_t parity, int32_t code) { return mbar_wait_lane(b, parity, p.dev_status, code); };
            auto landed = [&](int i) {
                const int stage = i % kSmallStages;
                return wait(p.ragged ? &bar.ready[stage] : &bar.full[stage], uint32_t(i / kSmallStages) & 1u, kStatusBwdTma);
            };
            auto score_product = [&](int i, int which, uint32_t column, uint64_t* done) {    // which: 0 scores, 1 dP
                const uint64_t a = dA + uint64_t(which) * (kTile >> 4), b = dB + uint64_t((i % kSmallStages) * 2 + which) * (kSmallPart >> 4);
                tc_fence_after();
                for (int k = 0; k < ksteps; ++k) mma_bf16(tmem_base + column, a + uint64_t(2 * k), b + uint64_t(2 * k), idesc_s, k != 0 ? 1u : 0u);
                mma_commit(done);
            };
            // bf16 operand of each half in the first half of its 32 columns
            auto acc_product = [&](int i, int which, uint32_t column, uint32_t acc) {
                const uint64_t b = dBt + uint64_t((i % kSmallStages) * 2 + which) * (kSmallPart >> 4);
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < kSmallBlock / 16; ++k)
                    mma_bf16_ts(tmem_base + acc, tmem_base + column + uint32_t((k >> 1) * 32 + (k & 1) * 8), b + uint64_t(k * 128), idesc_acc,
                                (i | k) != 0 ? 1u : 0u);
            };
            ok = wait(&bar.keep, 0, kStatusBwdTma) && landed(0);
            if (ok) {
                score_product(0, 0, 0u, &bar.s);
                score_product(0, 1, 64u, &bar.dp[0]);
            }
            // Products run in the order of their issue: one that overwrites another's operand in tensor memory is issued behind it.
            for (int i = 0; i < total && ok; ++i) {
                const uint32_t par = uint32_t(i) & 1u, next = par ^ 1u;
                const bool more = i + 1 < total;
                ok = wait(&bar.read, par, kStatusBwdWait);                     // S read (queries), P in its place (keys)
                if (!ok) break;
                if (KEYS) acc_product(i, 1, 0u, 128u);
                if (more) {
                    ok = landed(i + 1);
                    if (!ok) break;
                    score_product(i + 1, 0, 0u, &bar.s);
                    if (!KEYS) score_product(i + 1, 1, next ? 128u : 64u, &bar.dp[next]);
                }
                ok = wait(&bar.ds[par], uint32_t(i >> 1) & 1u, kStatusBwdWait);
                if (!ok) break;
                acc_product(i, 0, KEYS || !par ? 64u : 128u, 192u);
                mma_commit(&bar.empty[i % kSmallStages]);
                if (KEYS && more) score_product(i + 1, 1, 64u, &bar.dp[next]);
            }
            if (ok) mma_commit(&bar.acc);
            mma_drain(&bar.drain);
        }
        __syncwarp();
    } else {
        const int half = warp >> 2, row = (warp & 3) * 32 + lane, r = t.row0 + row;
        const uint32_t t_lane = tmem_base + (uint32_t((warp & 3) * 32) << 16), t_s = t_lane + uint32_t(half * 32);
        const f32x2 sc2 = pk2(s.scale_log2, s.scale_log2);
        f32x2 row_lse = 0, row_d = 0;
        int limit = 0;                                         // queries: keys the row sees
        if (!KEYS) {
            const float* stats = p.stats + (int64_t(t.n * s.heads + t.head) * p.q_tiles + t.tile) * (2 * kAttnTile) + row;
            const float l = ld_dependent(stats), d = ld_dependent(stats + kAttnTile);
            row_lse = pk2(l, l);
            row_d = pk2(d, d);
            limit = r < t.sm.q_hi ? attn_key_limit(s, t.sm, r) : 0;
            if (limit == 1) limit = 0;                         // a weight of 1, whatever its score: no gradient
        }
        int block = first + t.begin % (last - first);
        for (int i = 0; i < total; ++i) {
            const uint32_t par = uint32_t(i) & 1u;
            const int c0 = block * kSmallBlock + half * 32, stage = i % kSmallStages;        // the first column's query or key
            if (++block == last) block = first;
            ok = mbar_wait_warp(&bar.s, par, p.dev_status, kStatusBwdWait);
            if (KEYS) ok = ok && mbar_wait_warp(&bar.full[stage], uint32_t(i / kSmallStages) & 1u, p.dev_status, kStatusBwdTma);
            if (!ok) break;
            tc_fence_after();
            uint32_t sr[32], w[16];
            tmem_ld_32x32(t_s, sr);
            tmem_ld_wait_32(sr);
            if (!KEYS) {
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar.read);
            }
            const float* nl = stat + stage * 2 * kSmallBlock + half * 32;
            f32x2 pr[16];
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                f32x2 l0 = row_lse, l1 = row_lse;
                if (KEYS) {
                    const ulonglong2 l = *reinterpret_cast<const ulonglong2*>(nl + 2 * e);
                    l0 = l.x; l1 = l.y;
                }
                float z[4];
                upk2(fma2(pk2(__uint_as_float(sr[2 * e]), __uint_as_float(sr[2 * e + 1])), sc2, l0), z[0], z[1]);
                upk2(fma2(pk2(__uint_as_float(sr[2 * e + 2]), __uint_as_float(sr[2 * e + 3])), sc2, l1), z[2], z[3]);
                pr[e] = pk2(ex2(z[0]), ex2(z[1]));
                pr[e + 1] = pk2(ex2(z[2]), ex2(z[3]));
            }
            if (KEYS) {
                const int from = s.causal ? r - t.sm.shift - c0 : 0;           // the first query that sees the row's key
                if (__any_sync(0xffffffffu, from > 0)) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float a, b;
                        upk2(pr[e], a, b);
                        pr[e] = pk2(2 * e < from ? 0.f : a, 2 * e + 1 < from ? 0.f : b);
                    }
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float a, b;
                    upk2(pr[e], a, b);
                    w[e] = pack_bf16(a, b);
                }
                tmem_st_32x16(t_s, w);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar.read);
            }
            ok = mbar_wait_warp(&bar.dp[par], uint32_t(i >> 1) & 1u, p.dev_status, kStatusBwdWait);
            if (!ok) break;
            tc_fence_after();
            const uint32_t t_dp = t_s + (KEYS || !par ? 64u : 128u);
            tmem_ld_32x32(t_dp, sr);
            tmem_ld_wait_32(sr);
#pragma unroll
            for (int e = 0; e < 16; e += 2) {
                f32x2 d0 = row_d, d1 = row_d;
                if (KEYS) {
                    const ulonglong2 d = *reinterpret_cast<const ulonglong2*>(nl + kSmallBlock + 2 * e);
                    d0 = d.x; d1 = d.y;
                }
                float a, b;
                upk2(mul2(pr[e], add2(pk2(__uint_as_float(sr[2 * e]), __uint_as_float(sr[2 * e + 1])), d0)), a, b);
                w[e] = pack_bf16(a, b);
                upk2(mul2(pr[e + 1], add2(pk2(__uint_as_float(sr[2 * e + 2]), __uint_as_float(sr[2 * e + 3])), d1)), a, b);
                w[e + 1] = pack_bf16(a, b);
            }
            if (KEYS) {
                if (t.sm.kl == 1) {                            // every query sees one key only
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e] = 0u;
                }
                // causal, as many queries as keys or more: the first that sees a key sees this one only, a weight of 1 whatever its score
                const int one = r == 0 ? -t.sm.shift - c0 : -1;
                if (s.causal && __any_sync(0xffffffffu, unsigned(one) < 32u)) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e] &= one == 2 * e ? 0xFFFF0000u : one == 2 * e + 1 ? 0xFFFFu : 0xFFFFFFFFu;
                }
            } else {
                const int valid = limit - c0;                  // what lies behind may be anything
                if (__any_sync(0xffffffffu, valid < 32)) {
#pragma unroll
                    for (int e = 0; e < 16; ++e) w[e] &= 2 * e + 1 < valid ? 0xFFFFFFFFu : 2 * e < valid ? 0xFFFFu : 0u;
                }
            }
            tmem_st_32x16(t_dp, w);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.ds[par]);
        }
        if (ok) ok = mbar_wait_warp(&bar.acc, 0, p.dev_status, kStatusBwdWait);
        if (ok) {
            tc_fence_after();
            if (KEYS && p.parts > 1) {
                store_share(p, t, t_s + 192u, 0, row, half * 32, 1);
                store_share(p, t, t_s + 128u, 1, row, half * 32, 1);
                return true;
            }
            const bool kept = KEYS ? r < t.sm.kl : r >= t.sm.q_lo && r < t.sm.q_hi;
            stage_rows<1>(t_s + 192u, smem, row, half, s.dh, kept, s.scale);
            if (KEYS) stage_rows<1>(t_s + 128u, smem + kTile, row, half, s.dh, kept, 1.0f);
            fence_proxy_async_smem();
        }
    }
    return ok;
}

__global__ void __launch_bounds__(kSmallThreads, 2) attention_bwd_small_kernel(const __grid_constant__ BwdMaps m, const BwdParams p) {
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    __shared__ SmallBars bar;
    __shared__ uint32_t tmem_slot;
    const AttnShape& s = p.s;
    const int warp = threadIdx.x >> 5;
    const BwdItem t = bwd_item(p, blockIdx.x, kSmallBlock);
    if (t.total == 0) {                            // nothing seen: the gradient is zero
        griddep_wait();                            // no CTA ends before the kernel in front has
        if (t.keys && p.parts > 1) return;
        if (t.keys) {
            const int rows = min(kAttnTile, s.Lk - t.row0);
            const int64_t at = int64_t(t.n) * s.Lk + t.row0;
            zero_rows(p.dk + at * p.lddk + t.head * s.dh, p.lddk, rows, s.dh, int(threadIdx.x), kSmallThreads);
            zero_rows(p.dv + at * p.lddv + t.head * s.dh, p.lddv, rows, s.dh, int(threadIdx.x), kSmallThreads);
        } else {
            zero_rows(p.dq + (int64_t(t.n) * s.Lq + t.row0) * p.lddq + t.head * s.dh, p.lddq, min(kAttnTile, s.Lq - t.row0), s.dh, int(threadIdx.x), kSmallThreads);
        }
        return;
    }
    if (threadIdx.x == 0) {
        mbar_init(&bar.keep, 1); mbar_init(&bar.drain, 1);
        for (int i = 0; i < kSmallStages; ++i) { mbar_init(&bar.full[i], 1); mbar_init(&bar.ready[i], 1); mbar_init(&bar.empty[i], 1); }
        mbar_init(&bar.s, 1); mbar_init(&bar.acc, 1); mbar_init(&bar.read, 8);
        for (int i = 0; i < 2; ++i) { mbar_init(&bar.dp[i], 1); mbar_init(&bar.ds[i], 8); }
        fence_barrier_init();
    }
    if (warp == 9 && (threadIdx.x & 31) < 7) tma_prefetch_desc(&m.q + (threadIdx.x & 31));
    if (warp == 8) { __syncwarp(); tmem_alloc(&tmem_slot, 256); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = tmem_slot;
    griddep_wait();                                // the statistics; the call's operands were complete before that kernel began
    const bool ok = t.keys ? small_run<true>(m, p, t, smem, bar, tmem_base) : small_run<false>(m, p, t, smem, bar, tmem_base);
    tc_fence_before();
    const bool all = __syncthreads_and(ok);
    if (warp == 8) tmem_dealloc(tmem_base, 256);
    if (all && threadIdx.x == 0 && !(t.keys && p.parts > 1)) {
        tma_store_4d(t.keys ? &m.dk : &m.dq, smem, 0, t.head, t.row0, t.n);
        if (t.keys) tma_store_4d(&m.dv, smem + kAttnPart, 0, t.head, t.row0, t.n);
        bulk_commit_group();
        bulk_wait_read_all();
    }
}

// Per query and head: -D, D = dout . out in fp32, and -lse * log2(e), in tiles of 128 rows as the gradient kernel loads them.  Rows
// without a key, outside the lengths or behind the last get lse = +inf and D = 0: their probabilities are exp2(-inf) = 0.  A group of
// dh / 8 lanes takes a row; memory-bound, two reads.  Also clears the count of items taken.
__global__ void __launch_bounds__(256) attention_stats_kernel(const __nv_bfloat16* out, int64_t ldo, const __nv_bfloat16* dout, int64_t lddo,
                                                              const float* lse, const AttnShape s, int q_tiles, float* stats, unsigned* taken) {
    if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *taken = 0u;
    const int v = s.dh / 8, per_warp = 32 / v, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = lane / v, pos = lane - sub * v;
    const int bh = blockIdx.y, n = bh / s.heads, head = bh - n * s.heads;
    const AttnSample sm = attn_sample(s, n);
    const int rows = q_tiles * kAttnTile;
    constexpr int kAhead = 4;                      // rows of a group of lanes requested together
    const int stride = gridDim.x * 8 * per_warp;
    for (int i0 = (blockIdx.x * 8 + warp) * per_warp; i0 < rows; i0 += kAhead * stride) {
        uint4 a[kAhead], b[kAhead];
        float given[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = i0 + u * stride + sub;
            a[u] = b[u] = make_uint4(0u, 0u, 0u, 0u);
            given[u] = -INFINITY;
            if (sub < per_warp && i >= sm.q_lo && i < sm.q_hi) {
                const int64_t row = int64_t(n) * s.Lq + i;
                a[u] = __ldg(reinterpret_cast<const uint4*>(out + row * ldo + head * s.dh) + pos);
                b[u] = __ldg(reinterpret_cast<const uint4*>(dout + row * lddo + head * s.dh) + pos);
                if (pos == 0) given[u] = __ldg(lse + int64_t(bh) * s.Lq + i);
            }
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = i0 + u * stride + sub;
            const uint32_t x[4] = {a[u].x, a[u].y, a[u].z, a[u].w}, y[4] = {b[u].x, b[u].y, b[u].z, b[u].w};
            float d = 0.f;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                d = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16), d);
                d = fmaf(__uint_as_float(x[e] & 0xFFFF0000u), __uint_as_float(y[e] & 0xFFFF0000u), d);
            }
#pragma unroll
            for (int off = 8; off > 0; off >>= 1) {
                const float o = __shfl_down_sync(0xffffffffu, d, off);
                if (pos < off && pos + off < v) d += o;
            }
            if (sub < per_warp && pos == 0 && i < rows) {
                float* to = stats + (int64_t(bh) * q_tiles + i / kAttnTile) * (2 * kAttnTile) + i % kAttnTile;
                to[0] = given[u] == -INFINITY ? -INFINITY : given[u] * -1.4426950408889634f;
                to[kAttnTile] = -d;
            }
        }
    }
}

template <int NH>
hq_status launch_bwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const void* dout, int64_t lddo,
                     BwdParams p, cudaStream_t st) {
    const AttnShape& s = p.s;
    const uint32_t block = NH == 1 ? kSmallBlock : kAttnTile;  // rows of the other side's tiles; the kept ones take two boxes of 64 then
    BwdMaps m;
    if (!encode_heads_bf16(&m.q, q, s.dh, s.heads, s.Lq, s.Nb, ldq, block) || !encode_heads_bf16(&m.k, k, s.dh, s.kv_heads, s.Lk, s.Nb, ldk, block) ||
        !encode_heads_bf16(&m.v, v, s.dh, s.kv_heads, s.Lk, s.Nb, ldv, block) || !encode_heads_bf16(&m.dout, dout, s.dh, s.heads, s.Lq, s.Nb, lddo, block) ||
        !encode_heads_bf16(&m.dq, p.dq, s.dh, s.heads, s.Lq, s.Nb, p.lddq, kAttnTile) ||
        !encode_heads_bf16(&m.dk, p.dk, s.dh, s.kv_heads, s.Lk, s.Nb, p.lddk, kAttnTile) ||
        !encode_heads_bf16(&m.dv, p.dv, s.dh, s.kv_heads, s.Lk, s.Nb, p.lddv, kAttnTile))
        return HQ_ERR_CUDA;
    const unsigned sms = unsigned(sm_count());
    const int64_t slots = NH == 1 ? 2 * int64_t(sms) : int64_t(sms);
    p.key_chunk = attn_chunk(s.causal != 0, p.k_tiles, int64_t(s.Nb) * s.kv_heads, slots);
    p.chunk = attn_chunk(s.causal != 0, p.q_tiles, int64_t(s.Nb) * s.heads, slots);
    if constexpr (NH == 1) {
        if (cudaFuncSetAttribute(attention_bwd_small_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kSmallSmem)) != cudaSuccess) return HQ_ERR_CUDA;
        // the launch of few CTAs is prepared while the statistics are computed (they are placed when the last of those CTAs has ended,
        // which does not call griddep_launch): 2 x 64 tokens, 8 heads of 64 12.7 us a call otherwise, 12.3 so
        if (launch_dependent(attention_bwd_small_kernel, dim3(p.items), kSmallThreads, kSmallSmem, st, p.items <= slots, m, p) != cudaSuccess) return HQ_ERR_CUDA;
    } else {
        if (cudaFuncSetAttribute(attention_bwd_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kBwdSmem)) != cudaSuccess) return HQ_ERR_CUDA;
        if (launch_dependent(attention_bwd_kernel, dim3(p.items < sms ? p.items : sms), kBwdThreads, kBwdSmem, st, p.items <= sms, m, p) != cudaSuccess)
            return HQ_ERR_CUDA;
    }
    if (p.parts > 1) {
        const dim3 grid(p.key_items, 2, unsigned(s.dh / 8 + 1) / 2);
        if (launch_dependent(attention_bwd_join_kernel, grid, 256, 0, st, dependent_launch(int64_t(grid.x) * 2 * grid.z), p, NH, int(block)) != cudaSuccess)
            return HQ_ERR_CUDA;
    }
    return HQ_OK;
}

// Shares of a tile of keys' steps: enough that the longest item takes about half the time a slot (an SM, or half of one) has for all of
// them, where a share has eight steps at least, and only where that saves more than it costs.  Saved is what the longest item takes
// beyond a slot's average; tiles do not fill the slots evenly, so that whole items count for four tenths more than they take.  The shares'
// sums and the kernel that joins them cost twelve steps of 64 queries, and a quarter of one for each tile.  Whole / in shares: 16 x 1024
// queries on 77 keys, 8 heads of 64 53 / 67 us, 4 x 2027 causal, 4 heads of 64 61 / 79, 4 x 1575 on 300, 8 heads of 64 42 / 48, 2 x 4096, 16 / 2
// heads of 128 848 / 867, causal 513 / 478, 8 x 4096 on 77, 8 heads of 40 84 / 83, 1051 on 77, 4 heads of 64 27 / 21, 2 x 4096 on 77, 8 heads of
// 64 95 / 42, one sample of 4096, 8 / 1 heads of 64 574 / 155.
int bwd_parts(int64_t Nb, int64_t Lq, int64_t Lk, int heads, int kv_heads, int dh, bool causal) {
    const int64_t block = dh <= 64 ? kSmallBlock : kAttnTile, slots = int64_t(sm_count()) * (dh <= 64 ? 2 : 1);
    const int64_t key_steps = heads / kv_heads * ((Lq + block - 1) / block), query_steps = (Lk + block - 1) / block + 2;
    const int64_t keys = Nb * kv_heads * ((Lk + kAttnTile - 1) / kAttnTile), queries = Nb * heads * ((Lq + kAttnTile - 1) / kAttnTile);
    const int64_t work = keys * key_steps + queries * query_steps;
    int64_t parts = work > 0 ? (2 * key_steps * slots + work - 1) / work : 1;
    if (parts > key_steps / 8) parts = key_steps / 8;
    parts = parts < 1 ? 1 : parts < 16 ? parts : 16;
    const int64_t average = (causal ? work / 2 : work) / slots;
    const int64_t then = key_steps / parts > average ? key_steps / parts : average;          // the longest item, or all of them evenly
    if ((14 * key_steps / 10 - then) * block < (12 + keys / 4) * 64) parts = 1;
    // the persistent CTAs' warps wait for whole items, and waits end after a second: 2^17 steps of 2 us are a quarter of that
    const int64_t least = dh <= 64 ? 1 : (key_steps + (1 << 17) - 1) >> 17;
    return int(parts > least ? parts : least);
}

// statistics, the count of items taken, the shares' sums (room for those of the causal mask and of none: the size is asked without it)
struct BwdWorkspace { int64_t stats, taken, partial, bytes; int parts; };
BwdWorkspace bwd_workspace(int64_t Nb, int64_t Lq, int64_t Lk, int heads, int kv_heads, int dh, bool causal) {
    BwdWorkspace w;
    w.parts = bwd_parts(Nb, Lq, Lk, heads, kv_heads, dh, causal);
    const int other = bwd_parts(Nb, Lq, Lk, heads, kv_heads, dh, !causal), most = w.parts > other ? w.parts : other;
    w.stats = 0;
    w.taken = Nb * heads * ((Lq + kAttnTile - 1) / kAttnTile) * 2 * kStatBytes;
    w.partial = w.taken + 16;
    const int64_t tile = int64_t(dh <= 64 ? 64 : 128) * kAttnTile * 4, keys = Nb * kv_heads * ((Lk + kAttnTile - 1) / kAttnTile);
    w.bytes = w.partial + (most > 1 ? most * keys * 2 * tile : 0);
    return w;
}

}  // namespace
}  // namespace hq

extern "C" hq_status hq_attention_bwd_workspace_size(int64_t Nb, int64_t Lq, int64_t Lk, int heads, int kv_heads, int dh, size_t* bytes) {
    using namespace hq;
    if (bytes == nullptr) return HQ_ERR_INVALID_ARG;
    const hq_status e = attn_check(Nb, Lq, Lk, heads, kv_heads, dh, 1.0f);
    if (e != HQ_OK) return e;
    *bytes = size_t(bwd_workspace(Nb, Lq, Lk, heads, kv_heads, dh, false).bytes);
    return HQ_OK;
}

extern "C" hq_status hq_attention_bwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const void* out,
                                      int64_t ldo, const float* lse, const void* dout, int64_t lddo, int64_t Nb, int64_t Lq, int64_t Lk,
                                      int heads, int kv_heads, int dh, float scale, int causal, const int32_t* q_lens, const int32_t* k_lens,
                                      void* dq, int64_t lddq, void* dk, int64_t lddk, void* dv, int64_t lddv, void* workspace, size_t ws_bytes,
                                      int32_t* dev_status, void* stream) {
    using namespace hq;
    hq_status e = attn_check(Nb, Lq, Lk, heads, kv_heads, dh, scale);
    if (e != HQ_OK) return e;
    if (Nb == 0) return HQ_OK;
    if ((e = attn_check_matrix(q, Lq, ldq, heads, dh)) != HQ_OK || (e = attn_check_matrix(k, Lk, ldk, kv_heads, dh)) != HQ_OK ||
        (e = attn_check_matrix(v, Lk, ldv, kv_heads, dh)) != HQ_OK || (e = attn_check_matrix(out, Lq, ldo, heads, dh)) != HQ_OK ||
        (e = attn_check_matrix(dout, Lq, lddo, heads, dh)) != HQ_OK || (e = attn_check_matrix(dq, Lq, lddq, heads, dh)) != HQ_OK ||
        (e = attn_check_matrix(dk, Lk, lddk, kv_heads, dh)) != HQ_OK || (e = attn_check_matrix(dv, Lk, lddv, kv_heads, dh)) != HQ_OK)
        return e;
    if (lse == nullptr || workspace == nullptr) return HQ_ERR_INVALID_ARG;
    if (!aligned16(workspace)) return HQ_ERR_ALIGNMENT;
    const BwdWorkspace w = bwd_workspace(Nb, Lq, Lk, heads, kv_heads, dh, causal != 0);
    if (int64_t(ws_bytes) < w.bytes) return HQ_ERR_WORKSPACE;
    const int64_t q_tiles = (Lq + kAttnTile - 1) / kAttnTile, k_tiles = (Lk + kAttnTile - 1) / kAttnTile;
    const int64_t key_items = Nb * kv_heads * k_tiles, items = key_items * w.parts + Nb * heads * q_tiles;
    if (items > 0x3fffffff) return HQ_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    BwdParams p{};
    p.s = AttnShape{q_lens, k_lens, int(Nb), int(Lq), int(Lk), heads, kv_heads, dh, causal != 0, scale, float(double(scale) * 1.4426950408889634)};
    p.stats = static_cast<const float*>(workspace);
    p.taken = reinterpret_cast<unsigned*>(static_cast<unsigned char*>(workspace) + w.taken);
    p.partial = reinterpret_cast<float*>(static_cast<unsigned char*>(workspace) + w.partial);
    p.parts = w.parts;
    p.dq = static_cast<__nv_bfloat16*>(dq); p.dk = static_cast<__nv_bfloat16*>(dk); p.dv = static_cast<__nv_bfloat16*>(dv);
    p.lddq = lddq; p.lddk = lddk; p.lddv = lddv;
    p.q_tiles = int(q_tiles); p.k_tiles = int(k_tiles);
    p.key_items = unsigned(key_items); p.items = unsigned(items); p.dev_status = dev_status;
    p.ragged = q_lens != nullptr || k_lens != nullptr || (causal && Lq > Lk);
    // four rows of a group together once there are CTAs enough
    const int rows_per_cta = 8 * (32 / (dh / 8)) * (q_tiles * Nb * heads >= 2 * int64_t(sm_count()) ? 4 : 1);
    int64_t stat_ctas = (q_tiles * kAttnTile + rows_per_cta - 1) / rows_per_cta;
    if (stat_ctas > 64) stat_ctas = 64;
    attention_stats_kernel<<<dim3(unsigned(stat_ctas), unsigned(Nb * heads)), 256, 0, st>>>(
        static_cast<const __nv_bfloat16*>(out), ldo, static_cast<const __nv_bfloat16*>(dout), lddo, lse, p.s, p.q_tiles,
        static_cast<float*>(workspace), p.taken);
    if (cudaGetLastError() != cudaSuccess) return HQ_ERR_CUDA;
    return dh <= 64 ? launch_bwd<1>(q, ldq, k, ldk, v, ldv, dout, lddo, p, st) : launch_bwd<2>(q, ldq, k, ldk, v, ldv, dout, lddo, p, st);
}
