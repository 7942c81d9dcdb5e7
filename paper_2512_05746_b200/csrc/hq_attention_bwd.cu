// The gradient of attention (hq_attention_fwd.cu): the probabilities are recomputed from the scores and the row statistic.
//
//   P_ij = exp(scale q_i . k_j - lse_i),  dP = dout V^T,  D_i = dout_i . out_i,  dS = P o (dP - D)
//   dq = scale dS K,   dk = scale sum over the heads that share k of dS^T Q,   dv = sum of P^T dout
//
// Two kinds of CTA in one launch, each with the sums it owns in tensor memory for its whole life, so that nothing is added up in
// memory and the same inputs give the same bits:
//   keys     a tile of 128 keys of one (sample, key head) walks the queries of every head of its group: S^T = K Q^T, dP^T = V dout^T
//            with the keys along the lanes, P^T and dS^T as bf16 over the columns they were computed from, dv += P^T dout,
//            dk += dS^T Q;
//   queries  a tile of 128 queries of one (sample, head) walks the keys: S = Q K^T, dP = dout V^T, dq += dS K.
// The scores are computed twice (seven products a pair of tiles where five would do); what that buys is that P and dS never leave
// tensor memory (as operands of the second products they are read where they were written), no fp32 partial dq in memory and no
// order of additions that changes from run to run.
//
// Warps 0-15: thread = lane, four warps per quarter of the 128 columns; warp 16 loads, warp 17 issues.  The tile a CTA keeps (K and V,
// or Q and dout) stays in shared memory; pairs of the other side's tiles come through a ring of two.
#include "hq_attention_tile.cuh"

namespace hq {
namespace {

constexpr int32_t kStatusBwdWait = 0x710, kStatusBwdTma = 0x711;
constexpr int kBwdWarps = 16;                                  // of the probabilities
constexpr int kBwdThreads = (kBwdWarps + 2) * 32;
constexpr int kBwdStages = 2;
constexpr uint32_t kStatBytes = 2 * kAttnTile * 4;             // per query tile: lse * log2(e) of 128 rows, then D of 128 rows
template <int NH> constexpr size_t bwd_smem() { return size_t(2 + 2 * kBwdStages) * NH * kAttnPart + kBwdStages * kStatBytes + 1024; }

struct BwdParams {
    AttnShape s;
    const float* stats;                            // [Nb * heads][q_tiles][2][128]
    __nv_bfloat16 *dq, *dk, *dv;
    int64_t lddq, lddk, lddv;
    int q_tiles;
    unsigned key_ctas;
    int32_t* dev_status;
};

struct BwdBars { uint64_t keep, full[kBwdStages], empty[kBwdStages], s, dp, read, p, ds, acc; };

// KEYS: the CTA keeps a tile of keys and values (A0 = K, A1 = V; B0 = Q, B1 = dout), else one of queries (A0 = Q, A1 = dout; B0 = K,
// B1 = V).  Tensor memory: S at columns 0, dP at 128; KEYS: dv at 256, dk at 384; else dP's second buffer at 256, dq at 384.
template <int NH, bool KEYS>
__device__ __forceinline__ void bwd_run(const CUtensorMap* tmA0, const CUtensorMap* tmA1, const CUtensorMap* tmB0, const CUtensorMap* tmB1,
                                        const BwdParams& p, unsigned char* smem, BwdBars& bar, uint32_t tmem_base, int n, int head, int tile,
                                        const AttnSample& sm) {
    constexpr int kTile = NH * kAttnPart;
    const AttnShape& s = p.s;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    unsigned char* sA = smem;
    unsigned char* sB = smem + 2 * kTile;
    float* sStat = reinterpret_cast<float*>(sB + kBwdStages * 2 * kTile);
    const int row0 = tile * kAttnTile;
    const int group = s.heads / s.kv_heads;
    // the other side's tiles [first, last) of each head
    int first, last;
    if (KEYS) {
        first = max(sm.q_lo, s.causal ? row0 - sm.shift : 0) / kAttnTile;
        last = row0 < sm.kl ? (sm.q_hi + kAttnTile - 1) / kAttnTile : 0;
    } else {
        const int end = min(row0 + kAttnTile, sm.q_hi) - 1;
        first = 0;
        last = row0 > end || end < sm.q_lo ? 0 : (attn_key_limit(s, sm, end) + kAttnTile - 1) / kAttnTile;
    }
    const int per_head = max(0, last - first);
    const int total = KEYS ? per_head * group : per_head;
    if (total == 0) {                              // nothing seen: the gradient is zero
        if (KEYS) {
            const int rows = min(kAttnTile, s.Lk - row0);
            const int64_t r = int64_t(n) * s.Lk + row0;
            zero_rows(p.dk + r * p.lddk + head * s.dh, p.lddk, rows, s.dh);
            zero_rows(p.dv + r * p.lddv + head * s.dh, p.lddv, rows, s.dh);
        } else {
            zero_rows(p.dq + (int64_t(n) * s.Lq + row0) * p.lddq + head * s.dh, p.lddq, min(kAttnTile, s.Lq - row0), s.dh);
        }
        return;
    }

    if (warp == kBwdWarps) {
        if (elect_one()) {
            bool ok = true;
            int loads = 0;
            mbar_expect_tx(&bar.keep, 2 * kTile + (KEYS ? 0 : kStatBytes));
            load_tile<NH>(sA, tmA0, &bar.keep, head, row0, n);
            load_tile<NH>(sA + kTile, tmA1, &bar.keep, head, row0, n);
            if (!KEYS) bulk_load(sStat, p.stats + (int64_t(n * s.heads + head) * p.q_tiles + tile) * (2 * kAttnTile), kStatBytes, &bar.keep);
            int b_head = KEYS ? head * group : head / group, b_tile = first;
            for (int i = 0; i < total && ok; ++i) {
                const int stage = i % kBwdStages, use = i / kBwdStages;
                if (use > 0) ok = mbar_wait(&bar.empty[stage], uint32_t(use - 1) & 1u, p.dev_status, kStatusBwdWait);
                if (!ok) break;
                unsigned char* to = sB + stage * 2 * kTile;
                mbar_expect_tx(&bar.full[stage], 2 * kTile + (KEYS ? kStatBytes : 0));
                load_tile<NH>(to, tmB0, &bar.full[stage], b_head, b_tile * kAttnTile, n);
                load_tile<NH>(to + kTile, tmB1, &bar.full[stage], b_head, b_tile * kAttnTile, n);
                if (KEYS)
                    bulk_load(sStat + stage * 2 * kAttnTile, p.stats + (int64_t(n * s.heads + b_head) * p.q_tiles + b_tile) * (2 * kAttnTile),
                              kStatBytes, &bar.full[stage]);
                ++loads;
                if (++b_tile == last) { b_tile = first; ++b_head; }
            }
            // what was requested lands before the CTA's shared memory is given up, on every way out
            mbar_wait(&bar.keep, 0, nullptr, 0);
            for (int i = max(0, loads - kBwdStages); i < loads; ++i) mbar_wait(&bar.full[i % kBwdStages], uint32_t(i / kBwdStages) & 1u, nullptr, 0);
        }
        __syncwarp();
    } else if (warp == kBwdWarps + 1) {
        const uint32_t idesc_s = make_idesc_bf16(kAttnTile, kAttnTile, false);
        const uint32_t idesc_acc = make_idesc_bf16(kAttnTile, (s.dh + 15) & ~15, true);
        const int ksteps = (s.dh + 15) / 16;
        const uint64_t dA = make_sw128_kmajor_desc(smem_u32(sA));
        auto stage_of = [&](int i) { return sB + (i % kBwdStages) * 2 * kTile; };
        // the stage's tiles have landed, and rows of tokens outside the lengths are zero
        int b_tile = first;
        auto landed = [&](int i) {
            if (!__all_sync(0xffffffffu, mbar_wait(&bar.full[i % kBwdStages], uint32_t(i / kBwdStages) & 1u, p.dev_status, kStatusBwdTma))) return false;
            const int r0 = b_tile * kAttnTile;
            const int lo = KEYS ? sm.q_lo - r0 : 0, hi = (KEYS ? sm.q_hi : sm.kl) - r0;
            const int exist = (KEYS ? s.Lq : s.Lk) - r0;       // rows behind these are zero as they come
            if (lo > 0 || hi < min(kAttnTile, exist)) {
                clear_rows<NH>(stage_of(i), lo, hi, lane);
                if (KEYS) clear_rows<NH>(stage_of(i) + kTile, lo, hi, lane);
                fence_proxy_async_smem();
                __syncwarp();
            }
            if (++b_tile == last) b_tile = first;
            return true;
        };
        auto score_product = [&](int i, int which, uint32_t column, uint64_t* done) {          // which: 0 scores, 1 dP
            const uint64_t da = dA + uint64_t(which * (kTile >> 4));
            const uint64_t db = make_sw128_kmajor_desc(smem_u32(stage_of(i) + which * kTile));
            for (int k = 0; k < ksteps; ++k) {
                const uint64_t step = uint64_t((k >> 2) * (kAttnPart >> 4) + 2 * (k & 3));
                mma_bf16(tmem_base + column, da + step, db + step, idesc_s, k != 0 ? 1u : 0u);
            }
            mma_commit(done);
        };
        // bf16 elements of each quarter in the first half of its 32 columns
        auto acc_product = [&](int i, int which, uint32_t column, uint32_t acc) {
            const uint64_t db = make_sw128_mnmajor_desc(smem_u32(stage_of(i) + which * kTile), kAttnPart);
#pragma unroll
            for (int k = 0; k < kAttnTile / 16; ++k)
                mma_bf16_ts(tmem_base + acc, tmem_base + column + uint32_t((k >> 1) * 32 + (k & 1) * 8), db + uint64_t(k * 128), idesc_acc,
                            (i | k) != 0 ? 1u : 0u);
        };
        auto wait = [&](uint64_t* b, int i) { return __all_sync(0xffffffffu, mbar_wait(b, uint32_t(i) & 1u, p.dev_status, kStatusBwdWait)); };
        bool ok = __all_sync(0xffffffffu, mbar_wait(&bar.keep, 0, p.dev_status, kStatusBwdTma)) && landed(0);
        if (ok) {
            if (elect_one()) {
                tc_fence_after();
                score_product(0, 0, 0u, &bar.s);
                score_product(0, 1, 128u, &bar.dp);
            }
            __syncwarp();
        }
        // Products run in the order of their issue: one that overwrites another's operand in tensor memory is issued behind it.
        for (int i = 0; i < total && ok; ++i) {
            if (KEYS) {
                ok = wait(&bar.p, i);
                if (!ok) break;
                if (elect_one()) { tc_fence_after(); acc_product(i, 1, 0u, 256u); }
                __syncwarp();
                if (i + 1 < total) {
                    ok = landed(i + 1);
                    if (!ok) break;
                    if (elect_one()) { tc_fence_after(); score_product(i + 1, 0, 0u, &bar.s); }
                    __syncwarp();
                }
                ok = wait(&bar.ds, i);
                if (!ok) break;
                if (elect_one()) {
                    tc_fence_after();
                    acc_product(i, 0, 128u, 384u);
                    mma_commit(&bar.empty[i % kBwdStages]);
                    if (i + 1 < total) score_product(i + 1, 1, 128u, &bar.dp);
                }
                __syncwarp();
            } else {
                if (i + 1 < total) {
                    ok = landed(i + 1) && wait(&bar.read, i);
                    if (!ok) break;
                    if (elect_one()) {
                        tc_fence_after();
                        score_product(i + 1, 0, 0u, &bar.s);
                        score_product(i + 1, 1, 128u + 128u * uint32_t((i + 1) & 1), &bar.dp);
                    }
                    __syncwarp();
                }
                ok = wait(&bar.ds, i);
                if (!ok) break;
                if (elect_one()) {
                    tc_fence_after();
                    acc_product(i, 0, 128u + 128u * uint32_t(i & 1), 384u);
                    mma_commit(&bar.empty[i % kBwdStages]);
                }
                __syncwarp();
            }
        }
        if (ok) {
            if (elect_one()) mma_commit(&bar.acc);
            __syncwarp();
        }
    } else {
        const int quarter = warp >> 2;                         // columns quarter * 32 ..
        const int lane_row = (warp & 3) * 32 + lane, r = row0 + lane_row;
        const uint32_t t_lane = tmem_base + (uint32_t((warp & 3) * 32) << 16);
        const uint32_t t_s = t_lane + uint32_t(quarter * 32);
        const float sc = s.scale_log2;
        bool ok = true;
        int b_tile = first;
        float row_lse = 0.f, row_d = 0.f;
        int limit = 0;                                         // queries: keys the row sees
        if (!KEYS) {
            ok = __all_sync(0xffffffffu, mbar_wait(&bar.keep, 0, p.dev_status, kStatusBwdTma));
            row_lse = sStat[lane_row];
            row_d = sStat[kAttnTile + lane_row];
            limit = r < sm.q_hi ? attn_key_limit(s, sm, r) : 0;
        }
        for (int i = 0; i < total && ok; ++i) {
            const uint32_t par = uint32_t(i) & 1u;
            const int c0 = b_tile * kAttnTile + quarter * 32;  // the first column's query or key
            if (++b_tile == last) b_tile = first;
            const float* stat = sStat + (i % kBwdStages) * 2 * kAttnTile + quarter * 32;
            if (KEYS) ok = mbar_wait(&bar.full[i % kBwdStages], uint32_t(i / kBwdStages) & 1u, p.dev_status, kStatusBwdTma);
            ok = __all_sync(0xffffffffu, ok && mbar_wait(&bar.s, par, p.dev_status, kStatusBwdWait));
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
            float pr[32];
            const f32x2 sc2 = pk2(sc, sc);
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
                float4 l = make_float4(row_lse, row_lse, row_lse, row_lse);
                if (KEYS) l = *reinterpret_cast<const float4*>(stat + e);
                float z[4];
                upk2(fma2(pk2(__uint_as_float(sr[e]), __uint_as_float(sr[e + 1])), sc2, pk2(-l.x, -l.y)), z[0], z[1]);
                upk2(fma2(pk2(__uint_as_float(sr[e + 2]), __uint_as_float(sr[e + 3])), sc2, pk2(-l.z, -l.w)), z[2], z[3]);
#pragma unroll
                for (int c = 0; c < 4; ++c) pr[e + c] = ex2(z[c]);
            }
            // what the row does not see: keys behind its limit, or queries in front of the first that sees it
            if (KEYS) {
                const int from = s.causal ? r - sm.shift - c0 : 0;
                if (__any_sync(0xffffffffu, from > 0)) {
#pragma unroll
                    for (int e = 0; e < 32; ++e)
                        if (e < from) pr[e] = 0.f;
                }
#pragma unroll
                for (int e = 0; e < 16; ++e) w[e] = pack_bf16(pr[2 * e], pr[2 * e + 1]);
                tmem_st_32x16(t_s, w);
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar.p);
            }
            const int valid = KEYS ? 32 : limit - c0;
            const bool cut = !KEYS && __any_sync(0xffffffffu, valid < 32);
            ok = __all_sync(0xffffffffu, mbar_wait(&bar.dp, par, p.dev_status, kStatusBwdWait));
            if (!ok) break;
            tc_fence_after();
            const uint32_t t_dp = t_s + (KEYS ? 128u : 128u + 128u * par);
            uint32_t dp[32];
            tmem_ld_32x32(t_dp, dp);
            tmem_ld_wait_32(dp);
#pragma unroll
            for (int e = 0; e < 32; e += 4) {
                float4 d = make_float4(row_d, row_d, row_d, row_d);
                if (KEYS) d = *reinterpret_cast<const float4*>(stat + kAttnTile + e);
                float g[4];
                upk2(mul2(pk2(pr[e], pr[e + 1]), sub2(pk2(__uint_as_float(dp[e]), __uint_as_float(dp[e + 1])), pk2(d.x, d.y))), g[0], g[1]);
                upk2(mul2(pk2(pr[e + 2], pr[e + 3]), sub2(pk2(__uint_as_float(dp[e + 2]), __uint_as_float(dp[e + 3])), pk2(d.z, d.w))), g[2], g[3]);
                if (cut) {
#pragma unroll
                    for (int x = 0; x < 4; ++x)
                        if (e + x >= valid) g[x] = 0.f;
                }
                w[e / 2] = pack_bf16(g[0], g[1]);
                w[e / 2 + 1] = pack_bf16(g[2], g[3]);
            }
            tmem_st_32x16(t_dp, w);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.ds);
        }
        if (ok) ok = __all_sync(0xffffffffu, mbar_wait(&bar.acc, 0, p.dev_status, kStatusBwdWait));
        if (ok) {
            tc_fence_after();
            const uint32_t c = uint32_t(quarter * 32);
            if (KEYS) {
                const bool row_ok = r < s.Lk, keep = r < sm.kl;
                const int64_t at = int64_t(n) * s.Lk + (row_ok ? r : 0);
                store_rows(t_lane + 256u + c, p.dv + at * p.lddv + head * s.dh, int(c), s.dh, row_ok, keep, 1.0f);
                store_rows(t_lane + 384u + c, p.dk + at * p.lddk + head * s.dh, int(c), s.dh, row_ok, keep, s.scale);
            } else {
                const bool row_ok = r < s.Lq, keep = limit > 0;
                const int64_t at = int64_t(n) * s.Lq + (row_ok ? r : 0);
                store_rows(t_lane + 384u + c, p.dq + at * p.lddq + head * s.dh, int(c), s.dh, row_ok, keep, s.scale);
            }
        }
    }
}

template <int NH>
__global__ void __launch_bounds__(kBwdThreads, 1)
attention_bwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                     const __grid_constant__ CUtensorMap tmDo, const BwdParams p) {
    extern __shared__ __align__(1024) unsigned char smem_bwd[];
    __shared__ BwdBars bar;
    __shared__ uint32_t tmem_slot;
    unsigned char* smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_bwd) + 1023) & ~uintptr_t(1023));
    const AttnShape& s = p.s;
    const int warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) {
        mbar_init(&bar.keep, 1);
        for (int i = 0; i < kBwdStages; ++i) { mbar_init(&bar.full[i], 1); mbar_init(&bar.empty[i], 1); }
        mbar_init(&bar.s, 1); mbar_init(&bar.dp, 1); mbar_init(&bar.acc, 1);
        mbar_init(&bar.read, kBwdWarps); mbar_init(&bar.p, kBwdWarps); mbar_init(&bar.ds, kBwdWarps);
        fence_barrier_init();
    }
    if (warp == kBwdWarps + 1) { __syncwarp(); tmem_alloc(&tmem_slot, 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = tmem_slot;
    // tiles of keys first (they walk every head of their group), then tiles of queries; under the causal mask the first keys and
    // the last queries walk the most
    if (blockIdx.x < p.key_ctas) {
        const unsigned per = unsigned(s.Nb) * unsigned(s.kv_heads), tile = blockIdx.x / per, bh = blockIdx.x - tile * per;
        const int n = int(bh / s.kv_heads);
        bwd_run<NH, true>(&tmK, &tmV, &tmQ, &tmDo, p, smem, bar, tmem_base, n, int(bh) - n * s.kv_heads, int(tile), attn_sample(s, n));
    } else {
        const unsigned b = blockIdx.x - p.key_ctas, per = unsigned(s.Nb) * unsigned(s.heads), block = b / per, bh = b - block * per;
        const int n = int(bh / s.heads), tile = s.causal ? p.q_tiles - 1 - int(block) : int(block);
        bwd_run<NH, false>(&tmQ, &tmDo, &tmK, &tmV, p, smem, bar, tmem_base, n, int(bh) - n * s.heads, tile, attn_sample(s, n));
    }
    tc_fence_before();
    __syncthreads();
    if (warp == kBwdWarps + 1) tmem_dealloc(tmem_base, 512);
}

// Per query and head: D = dout . out in fp32, and lse * log2(e), in tiles of 128 rows as the gradient kernel loads them.  Rows without
// a key, outside the lengths or behind the last get lse = +inf and D = 0: their probabilities are exp2(-inf) = 0.  A group of
// dh / 8 lanes takes a row; memory-bound, two reads.
__global__ void __launch_bounds__(256) attention_stats_kernel(const __nv_bfloat16* out, int64_t ldo, const __nv_bfloat16* dout, int64_t lddo,
                                                              const float* lse, const AttnShape s, int q_tiles, float* stats) {
    const int v = s.dh / 8, per_warp = 32 / v, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int sub = lane / v, pos = lane - sub * v;
    const int bh = blockIdx.y, n = bh / s.heads, head = bh - n * s.heads;
    const AttnSample sm = attn_sample(s, n);
    const int rows = q_tiles * kAttnTile;
    for (int i0 = (blockIdx.x * 8 + warp) * per_warp; i0 < rows; i0 += gridDim.x * 8 * per_warp) {
        const int i = i0 + sub;
        const bool mine = sub < per_warp && i < rows, live = mine && i >= sm.q_lo && i < sm.q_hi;
        float d = 0.f;
        if (live) {
            const int64_t row = int64_t(n) * s.Lq + i;
            const uint4 a = __ldg(reinterpret_cast<const uint4*>(out + row * ldo + head * s.dh) + pos);
            const uint4 b = __ldg(reinterpret_cast<const uint4*>(dout + row * lddo + head * s.dh) + pos);
            const uint32_t x[4] = {a.x, a.y, a.z, a.w}, y[4] = {b.x, b.y, b.z, b.w};
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                d = fmaf(__uint_as_float(x[e] << 16), __uint_as_float(y[e] << 16), d);
                d = fmaf(__uint_as_float(x[e] & 0xFFFF0000u), __uint_as_float(y[e] & 0xFFFF0000u), d);
            }
        }
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) {
            const float o = __shfl_down_sync(0xffffffffu, d, off);
            if (pos < off && pos + off < v) d += o;
        }
        if (mine && pos == 0) {
            float* to = stats + (int64_t(bh) * q_tiles + i / kAttnTile) * (2 * kAttnTile) + i % kAttnTile;
            float l = INFINITY;
            if (live) {
                const float given = __ldg(lse + int64_t(bh) * s.Lq + i);
                if (given != -INFINITY) l = given * 1.4426950408889634f;
            }
            to[0] = l;
            to[kAttnTile] = d;
        }
    }
}

template <int NH>
hq_status launch_bwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const void* dout, int64_t lddo,
                     const BwdParams& p, unsigned grid, cudaStream_t st) {
    const AttnShape& s = p.s;
    CUtensorMap tmQ, tmK, tmV, tmDo;
    if (!encode_heads_bf16(&tmQ, q, s.dh, s.heads, s.Lq, s.Nb, ldq, kAttnTile) ||
        !encode_heads_bf16(&tmK, k, s.dh, s.kv_heads, s.Lk, s.Nb, ldk, kAttnTile) ||
        !encode_heads_bf16(&tmV, v, s.dh, s.kv_heads, s.Lk, s.Nb, ldv, kAttnTile) ||
        !encode_heads_bf16(&tmDo, dout, s.dh, s.heads, s.Lq, s.Nb, lddo, kAttnTile))
        return HQ_ERR_CUDA;
    if (cudaFuncSetAttribute(attention_bwd_kernel<NH>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(bwd_smem<NH>())) != cudaSuccess)
        return HQ_ERR_CUDA;
    attention_bwd_kernel<NH><<<grid, kBwdThreads, bwd_smem<NH>(), st>>>(tmQ, tmK, tmV, tmDo, p);
    return cudaGetLastError() == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}

int64_t stats_bytes(int64_t Nb, int64_t Lq, int heads) { return Nb * heads * ((Lq + kAttnTile - 1) / kAttnTile) * kStatBytes; }

}  // namespace
}  // namespace hq

extern "C" hq_status hq_attention_bwd_workspace_size(int64_t Nb, int64_t Lq, int64_t Lk, int heads, int kv_heads, int dh, size_t* bytes) {
    using namespace hq;
    if (bytes == nullptr) return HQ_ERR_INVALID_ARG;
    const hq_status e = attn_check(Nb, Lq, Lk, heads, kv_heads, dh, 1.0f);
    if (e != HQ_OK) return e;
    *bytes = size_t(stats_bytes(Nb, Lq, heads));
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
    if (int64_t(ws_bytes) < stats_bytes(Nb, Lq, heads)) return HQ_ERR_WORKSPACE;
    const int64_t q_tiles = (Lq + kAttnTile - 1) / kAttnTile, k_tiles = (Lk + kAttnTile - 1) / kAttnTile;
    const int64_t key_ctas = Nb * kv_heads * k_tiles, grid = key_ctas + Nb * heads * q_tiles;
    if (grid > 0x7fffffff) return HQ_ERR_UNSUPPORTED;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    BwdParams p{};
    p.s = AttnShape{q_lens, k_lens, int(Nb), int(Lq), int(Lk), heads, kv_heads, dh, causal != 0, scale, float(double(scale) * 1.4426950408889634)};
    p.stats = static_cast<const float*>(workspace);
    p.dq = static_cast<__nv_bfloat16*>(dq); p.dk = static_cast<__nv_bfloat16*>(dk); p.dv = static_cast<__nv_bfloat16*>(dv);
    p.lddq = lddq; p.lddk = lddk; p.lddv = lddv;
    p.q_tiles = int(q_tiles); p.key_ctas = unsigned(key_ctas); p.dev_status = dev_status;
    const int rows_per_cta = 8 * (32 / (dh / 8));
    int64_t stat_ctas = (q_tiles * kAttnTile + rows_per_cta - 1) / rows_per_cta;
    if (stat_ctas > 64) stat_ctas = 64;
    attention_stats_kernel<<<dim3(unsigned(stat_ctas), unsigned(Nb * heads)), 256, 0, st>>>(
        static_cast<const __nv_bfloat16*>(out), ldo, static_cast<const __nv_bfloat16*>(dout), lddo, lse, p.s, p.q_tiles, static_cast<float*>(workspace));
    if (cudaGetLastError() != cudaSuccess) return HQ_ERR_CUDA;
    return dh <= 64 ? launch_bwd<1>(q, ldq, k, ldk, v, ldv, dout, lddo, p, unsigned(grid), st)
                    : launch_bwd<2>(q, ldq, k, ldk, v, ldv, dout, lddo, p, unsigned(grid), st);
}
