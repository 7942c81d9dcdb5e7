// Attention with the statistic its gradient needs: per sample, head and query, out = sum_j softmax_j(scale q . k_j) v_j over the keys
// the query sees, lse = log sum_j exp(scale q . k_j).  Queries, keys and values are matrices of their own (pitches, lengths, heads that
// share keys and values).
//
// Persistent CTAs: an item is two tiles of 128 queries of one (sample, head), which walk the keys in blocks of 128:
//   S = Q K^T        both operands from shared memory (128-byte swizzle), fp32 in 128 columns of tensor memory
//   P = exp2(c S - c m) as bf16 in tensor memory
//   O += P V         P from tensor memory, V from shared memory, read along its keys without a transpose
// Warp 0 issues, warp 1 takes items and loads, warp 2 stores, warp 3 clears rows outside the lengths; warps 4-11 do the softmax of the first
// tile and warps 12-19 that of the second: thread = query row, 64 of the block's 128 keys; the two halves of a row tell each other their
// maximum.  Up to 64 channels P has columns of its own, and the next block's S is computed under this one's exponentials; above, P
// stands over S, whose next block comes behind the product that reads P, and the other tile's exponentials cover that time.
// The running maximum moves only when a block's maximum exceeds it by more than 2^8 in the exponent: the weights stay below 2^8, the
// division by the row sum at the end is the same, and O is read and rescaled in tensor memory almost never.  P is rounded to bf16
// (the products' type), the row sum runs over the unrounded weights in fp32.
#include "hq_attention_tile.cuh"

namespace hq {
namespace {

constexpr int32_t kStatusFwdWait = 0x700, kStatusFwdTma = 0x701, kStatusFwdSmem = 0x702;
constexpr int kFwdWarps = 16, kFwdFirst = 4;       // of the softmax; in front of them the others
constexpr int kFwdThreads = (kFwdFirst + kFwdWarps) * 32;

template <int NH> struct FwdRings {
    static constexpr int kQ = NH == 1 ? 2 : 1;     // pairs of query tiles: the next item's loads begin under this one's last steps
    static constexpr int kK = NH == 1 ? 4 : 2, kV = NH == 1 ? 4 : 2;
    static constexpr int kTile = NH * kAttnPart;
    static constexpr int kTiles = (2 * kQ + kK + kV) * kTile;
};
// Columns of tensor memory: S of the tiles at 0 and 128, then
template <int NH> struct FwdTmem {
    static __device__ __forceinline__ uint32_t o(int t) { return 256u + uint32_t(t) * (NH == 1 ? 64u : 128u); }
    // bf16 weights of keys 64 h ..: over the scores of the half where there are no columns left
    static __device__ __forceinline__ uint32_t p(int t, int h) { return NH == 1 ? 384u + uint32_t(t * 64 + h * 32) : uint32_t(t * 128 + h * 64); }
};

struct FwdParams {
    AttnShape s;
    __nv_bfloat16* out;
    int64_t ldo;
    float* lse;                                    // [Nb][heads][Lq]
    int q_blocks, ragged;                          // pairs of query tiles; rows outside the lengths may lie in a tile
    unsigned items;
    unsigned* taken;                               // items taken beyond the first of every CTA, or NULL: every grid-th
    int32_t* dev_status;
};
struct FwdMaps { CUtensorMap q, k, v, out; };
template <int NH> struct FwdBars {
    using R = FwdRings<NH>;
    uint64_t q_full[R::kQ], q_empty[R::kQ], k_full[R::kK], k_empty[R::kK], v_full[R::kV], v_ready[R::kV], v_empty[R::kV];
    uint64_t s[2], read[2], p[2], o[2], staged[R::kQ], item_full[2], item_empty[2];
    uint64_t turn[2][8], pair[8];                  // a warp of the first tile has done its exponentials / one of the second; halves of a row
    float most[2][2][2][kAttnTile];                // [exchange & 1][tile][half][row]: a half row's maximum, at the end its sum
    uint32_t item[2], tmem_slot;
};
template <int NH> constexpr size_t fwd_smem() { return size_t(FwdRings<NH>::kTiles) + sizeof(FwdBars<NH>); }

struct FwdItem {
    int n, head, q0, nb[2], blocks;                // key blocks of each tile: as far as its last query sees
    AttnSample sm;
};
__device__ __forceinline__ FwdItem fwd_item(const FwdParams& p, unsigned index) {
    const AttnShape& s = p.s;
    FwdItem t;
    const unsigned per = unsigned(s.Nb) * unsigned(s.heads), block = index / per, bh = index - block * per;
    t.n = int(bh / unsigned(s.heads));
    t.head = int(bh) - t.n * s.heads;
    // causal: the blocks with the most keys first
    t.q0 = (s.causal ? p.q_blocks - 1 - int(block) : int(block)) * 2 * kAttnTile;
    t.sm = attn_sample(s, t.n);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int first = t.q0 + i * kAttnTile, last = min(first + kAttnTile, t.sm.q_hi) - 1;
        t.nb[i] = first > last || last < t.sm.q_lo ? 0 : (attn_key_limit(s, t.sm, last) + kAttnTile - 1) / kAttnTile;
    }
    t.blocks = max(t.nb[0], t.nb[1]);
    return t;
}

// ---- warp 1, one lane: takes items, tells the others, loads their tiles
template <int NH>
__device__ __forceinline__ void fwd_load(const FwdMaps& m, const FwdParams& p, unsigned char* smem, FwdBars<NH>& bar) {
    using R = FwdRings<NH>;
    unsigned char *sK = smem + 2 * R::kQ * R::kTile, *sV = sK + R::kK * R::kTile;
    const int group = p.s.heads / p.s.kv_heads;
    RingAt<R::kQ> q;
    RingAt<R::kK> k;
    RingAt<R::kV> v;
    RingAt<2> told;
    int nq = 0, nk = 0;                            // begun so far
    int nv = 0;
    bool ok = true;
    unsigned index = blockIdx.x;
    while (ok) {
        ok = mbar_wait_lane(&bar.item_empty[told.slot], told.phase ^ 1u, p.dev_status, kStatusFwdWait);
        if (!ok) break;
        bar.item[told.slot] = index;
        mbar_arrive(&bar.item_full[told.slot]);
        told.next();
        if (index >= p.items) break;
        const FwdItem t = fwd_item(p, index);
        index = p.taken != nullptr ? gridDim.x + atomicAdd(p.taken, 1u) : index + gridDim.x;
        if (t.blocks == 0) continue;
        ok = mbar_wait_lane(&bar.q_empty[q.slot], q.phase ^ 1u, p.dev_status, kStatusFwdWait);
        if (!ok) break;
        unsigned char* to = smem + 2 * q.slot * R::kTile;
        mbar_expect_tx(&bar.q_full[q.slot], 2 * R::kTile);
        load_tile<NH>(to, &m.q, &bar.q_full[q.slot], t.head, t.q0, t.n);
        load_tile<NH>(to + R::kTile, &m.q, &bar.q_full[q.slot], t.head, t.q0 + kAttnTile, t.n);
        q.next();
        ++nq;
        for (int j = 0; j < t.blocks; ++j) {
            ok = mbar_wait_lane(&bar.k_empty[k.slot], k.phase ^ 1u, p.dev_status, kStatusFwdWait);
            if (!ok) break;
            mbar_expect_tx(&bar.k_full[k.slot], R::kTile);
            load_tile<NH>(sK + k.slot * R::kTile, &m.k, &bar.k_full[k.slot], t.head / group, j * kAttnTile, t.n);
            k.next();
            ++nk;
            ok = mbar_wait_lane(&bar.v_empty[v.slot], v.phase ^ 1u, p.dev_status, kStatusFwdWait);
            if (!ok) break;
            mbar_expect_tx(&bar.v_full[v.slot], R::kTile);
            load_tile<NH>(sV + v.slot * R::kTile, &m.v, &bar.v_full[v.slot], t.head / group, j * kAttnTile, t.n);
            v.next();
            ++nv;
        }
    }
    // what was requested lands before the CTA's shared memory is given up, on every way out
    for (int i = max(0, nq - R::kQ); i < nq; ++i) mbar_wait_lane(&bar.q_full[i % R::kQ], uint32_t(i / R::kQ) & 1u, nullptr, 0);
    for (int i = max(0, nk - R::kK); i < nk; ++i) mbar_wait_lane(&bar.k_full[i % R::kK], uint32_t(i / R::kK) & 1u, nullptr, 0);
    for (int i = max(0, nv - R::kV); i < nv; ++i) mbar_wait_lane(&bar.v_full[i % R::kV], uint32_t(i / R::kV) & 1u, nullptr, 0);
}

// The next item's number (p.items and beyond: none, or a wait ran out), the same in every lane.
template <int NH>
__device__ __forceinline__ unsigned fwd_next(const FwdParams& p, FwdBars<NH>& bar, RingAt<2>& told, int lane) {
    if (!mbar_wait_warp(&bar.item_full[told.slot], told.phase, p.dev_status, kStatusFwdWait)) return 0xffffffffu;
    const unsigned index = *const_cast<volatile uint32_t*>(&bar.item[told.slot]);
    __syncwarp();
    if (lane == 0) mbar_arrive(&bar.item_empty[told.slot]);
    told.next();
    return index;
}

// ---- warp 3: values of tokens behind a sample's last are made zero: they would meet zero weights
template <int NH>
__device__ __forceinline__ void fwd_clear(const FwdParams& p, unsigned char* smem, FwdBars<NH>& bar, int lane) {
    using R = FwdRings<NH>;
    unsigned char* sV = smem + (2 * R::kQ + R::kK) * R::kTile;
    RingAt<R::kV> v;
    RingAt<2> told;
    for (;;) {
        const unsigned index = fwd_next<NH>(p, bar, told, lane);
        if (index >= p.items) return;
        const FwdItem t = fwd_item(p, index);
        for (int j = 0; j < t.blocks; ++j) {
            if (!mbar_wait_warp(&bar.v_full[v.slot], v.phase, p.dev_status, kStatusFwdTma)) return;
            if (t.sm.kl < min(p.s.Lk, (j + 1) * kAttnTile)) clear_rows<NH>(sV + v.slot * R::kTile, 0, t.sm.kl - j * kAttnTile, lane);
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.v_ready[v.slot]);
            v.next();
        }
    }
}

// ---- warp 0, one lane: products.  They run in the order of their issue.
template <int NH>
__device__ __forceinline__ void fwd_issue(const FwdParams& p, unsigned char* smem, FwdBars<NH>& bar, uint32_t tmem_base) {
    using R = FwdRings<NH>;
    using T = FwdTmem<NH>;
    const AttnShape& s = p.s;
    unsigned char *sK = smem + 2 * R::kQ * R::kTile, *sV = sK + R::kK * R::kTile;
    const uint32_t idesc_s = make_idesc_bf16(kAttnTile, kAttnTile, false);
    const uint32_t idesc_o = make_idesc_bf16(kAttnTile, (s.dh + 15) & ~15, true);
    const int ksteps = (s.dh + 15) / 16;
    constexpr uint64_t kTileUnits = R::kTile >> 4;
    const uint64_t dQ = make_sw128_kmajor_desc(smem_u32(smem)), dK = make_sw128_kmajor_desc(smem_u32(sK));
    const uint64_t dV = make_sw128_mnmajor_desc(smem_u32(sV), kAttnPart);
    auto wait = [&](uint64_t* b, uint32_t parity, int32_t code) { return mbar_wait_lane(b, parity, p.dev_status, code); };
    RingAt<R::kQ> q;
    RingAt<R::kK> k;
    RingAt<R::kV> v;
    RingAt<2> told;
    uint32_t n_p[2] = {0, 0};                      // blocks of each tile over all items
    for (;;) {
        if (!wait(&bar.item_full[told.slot], told.phase, kStatusFwdWait)) return;
        const unsigned index = *const_cast<volatile uint32_t*>(&bar.item[told.slot]);
        mbar_arrive(&bar.item_empty[told.slot]);
        told.next();
        if (index >= p.items) return;
        const FwdItem t = fwd_item(p, index);
        if (t.blocks == 0) continue;
        const uint64_t a = dQ + uint64_t(q.slot) * (2 * kTileUnits);
        if (!wait(&bar.q_full[q.slot], q.phase, kStatusFwdTma)) return;
        q.next();
        auto scores = [&](int tile) {
            const uint64_t da = a + uint64_t(tile) * kTileUnits, db = dK + uint64_t(k.slot) * kTileUnits;
            tc_fence_after();
            for (int x = 0; x < ksteps; ++x) {
                const uint64_t step = uint64_t((x >> 2) * (kAttnPart >> 4) + 2 * (x & 3));
                mma_bf16(tmem_base + uint32_t(tile * 128), da + step, db + step, idesc_s, x != 0 ? 1u : 0u);
            }
            mma_commit(&bar.s[tile]);
        };
        auto values = [&](int tile, int j) {
            const uint64_t db = dV + uint64_t(v.slot) * kTileUnits;
            tc_fence_after();
#pragma unroll
            for (int x = 0; x < kAttnTile / 16; ++x)
                mma_bf16_ts(tmem_base + T::o(tile), tmem_base + T::p(tile, x >> 2) + uint32_t(8 * (x & 3)), db + uint64_t(x * 128), idesc_o,
                            (j | x) != 0 ? 1u : 0u);
            mma_commit(&bar.o[tile]);
        };
        if (!wait(&bar.k_full[k.slot], k.phase, kStatusFwdTma)) return;
#pragma unroll
        for (int x = 0; x < 2; ++x)
            if (t.nb[x] > 0) scores(x);
        mma_commit(&bar.k_empty[k.slot]);
        k.next();
        for (int j = 0; j < t.blocks; ++j) {
            const bool more = j + 1 < t.blocks;
            if (more && !wait(&bar.k_full[k.slot], k.phase, kStatusFwdTma)) return;
            if (NH == 1 && more) {                 // the next S as soon as this one has been read
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    if (j + 1 < t.nb[x]) {
                        if (!wait(&bar.read[x], n_p[x] & 1u, kStatusFwdWait)) return;
                        scores(x);
                    }
                mma_commit(&bar.k_empty[k.slot]);
                k.next();
            }
            if (!wait(p.ragged ? &bar.v_ready[v.slot] : &bar.v_full[v.slot], v.phase, kStatusFwdTma)) return;
#pragma unroll
            for (int x = 0; x < 2; ++x)
                if (j < t.nb[x]) {
                    if (!wait(&bar.p[x], n_p[x] & 1u, kStatusFwdWait)) return;
                    values(x, j);
                    ++n_p[x];
                    if (NH == 2 && j + 1 < t.nb[x]) scores(x);
                }
            mma_commit(&bar.v_empty[v.slot]);
            v.next();
            if (NH == 2 && more) {
                mma_commit(&bar.k_empty[k.slot]);
                k.next();
            }
        }
    }
}

template <int NH>
__global__ void __launch_bounds__(kFwdThreads, 1) attention_fwd_kernel(const __grid_constant__ FwdMaps m, const FwdParams p) {
    using R = FwdRings<NH>;
    using T = FwdTmem<NH>;
    extern __shared__ __align__(1024) unsigned char smem[];
    FwdBars<NH>& bar = *reinterpret_cast<FwdBars<NH>*>(smem + R::kTiles);
    const AttnShape& s = p.s;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    if ((smem_u32(smem) & 1023u) != 0) {           // the tiles' swizzle needs it; dynamic shared memory begins there
        if (threadIdx.x == 0 && p.dev_status != nullptr) atomicExch(p.dev_status, kStatusFwdSmem);
        return;
    }
    if (threadIdx.x == 0) {
        for (int i = 0; i < R::kQ; ++i) { mbar_init(&bar.q_full[i], 1); mbar_init(&bar.q_empty[i], 1); mbar_init(&bar.staged[i], kFwdWarps); }
        for (int i = 0; i < R::kK; ++i) { mbar_init(&bar.k_full[i], 1); mbar_init(&bar.k_empty[i], 1); }
        for (int i = 0; i < R::kV; ++i) { mbar_init(&bar.v_full[i], 1); mbar_init(&bar.v_ready[i], 1); mbar_init(&bar.v_empty[i], 1); }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bar.s[i], 1); mbar_init(&bar.o[i], 1);
            for (int w = 0; w < 8; ++w) mbar_init(&bar.turn[i][w], 1);
            mbar_init(&bar.read[i], kFwdWarps / 2); mbar_init(&bar.p[i], kFwdWarps / 2);
            mbar_init(&bar.item_full[i], 1); mbar_init(&bar.item_empty[i], kFwdWarps + 2 + (p.ragged ? 1 : 0));
        }
        for (int i = 0; i < 8; ++i) mbar_init(&bar.pair[i], 2);
        fence_barrier_init();
    }
    if (warp == 1 && lane < 4) tma_prefetch_desc(&m.q + lane);
    if (warp == 0) { __syncwarp(); tmem_alloc(&bar.tmem_slot, 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = bar.tmem_slot;

    if (warp == 0) {
        if (elect_one()) fwd_issue<NH>(p, smem, bar, tmem_base);
        __syncwarp();
    } else if (warp == 1) {
        if (elect_one()) fwd_load<NH>(m, p, smem, bar);
        __syncwarp();
    } else if (warp == 2) {
        RingAt<2> told;
        RingAt<R::kQ> q;
        for (;;) {
            const unsigned index = fwd_next<NH>(p, bar, told, lane);
            if (index >= p.items) break;
            const FwdItem t = fwd_item(p, index);
            if (t.blocks == 0) continue;
            if (!mbar_wait_warp(&bar.staged[q.slot], q.phase, p.dev_status, kStatusFwdWait)) break;
            if (elect_one()) {
                const unsigned char* from = smem + 2 * q.slot * R::kTile;
                for (int x = 0; x < 2; ++x)
                    if (t.q0 + x * kAttnTile < s.Lq) {
#pragma unroll
                        for (int h = 0; h < NH; ++h)
                            tma_store_4d(&m.out, from + x * R::kTile + h * kAttnPart, 64 * h, t.head, t.q0 + x * kAttnTile, t.n);
                    }
                bulk_commit_group();
                bulk_wait_read_all();
                mbar_arrive(&bar.q_empty[q.slot]);
            }
            __syncwarp();
            q.next();
        }
    } else if (warp == 3) {
        if (p.ragged) fwd_clear<NH>(p, smem, bar, lane);
    } else {
        const int tile = (warp - kFwdFirst) >> 3, half = ((warp - kFwdFirst) >> 2) & 1, row = (warp & 3) * 32 + lane;
        const uint32_t t_lane = tmem_base + (uint32_t((warp & 3) * 32) << 16);
        const uint32_t t_s = t_lane + uint32_t(tile * 128 + half * 64), t_p = t_lane + T::p(tile, half), t_o = t_lane + T::o(tile);
        const float sc = s.scale_log2;
        RingAt<2> told;
        RingAt<R::kQ> q;
        uint64_t* pair = &bar.pair[tile * 4 + (warp & 3)];
        const int lot = half * 4 + (warp & 3);
        uint32_t n = 0, turns = 0, told_pair = 0;  // blocks over all items; of these where both tiles take turns; exchanges
        // gives the row's other half a value, returns the other's
        auto exchange = [&](float mine, float& other) {
            bar.most[told_pair & 1u][tile][half][row] = mine;
            __syncwarp();
            if (lane == 0) mbar_arrive(pair);
            const bool told_ok = mbar_wait_warp(pair, told_pair & 1u, p.dev_status, kStatusFwdWait);
            other = *const_cast<volatile float*>(&bar.most[told_pair & 1u][tile][half ^ 1][row]);
            ++told_pair;
            return told_ok;
        };
        for (;;) {
            const unsigned index = fwd_next<NH>(p, bar, told, lane);
            if (index >= p.items) break;
            const FwdItem t = fwd_item(p, index);
            const int i = t.q0 + tile * kAttnTile + row;
            float* lse = p.lse + (int64_t(t.n) * s.heads + t.head) * s.Lq + i;
            if (t.blocks == 0) {                   // no query of the two tiles sees a key
                const int first = t.q0 + tile * kAttnTile;
                zero_rows(p.out + (int64_t(t.n) * s.Lq + first) * p.ldo + t.head * s.dh, p.ldo, min(kAttnTile, s.Lq - first), s.dh,
                          (int(threadIdx.x) - kFwdFirst * 32) & 255, 256);
                if (half == 0 && i < s.Lq) *lse = -INFINITY;
                continue;
            }
            const int blocks = t.nb[tile], both = min(t.nb[0], t.nb[1]);
            const int limit = i < t.sm.q_hi ? attn_key_limit(s, t.sm, i) : 0;
            float m_run = -INFINITY, l_run = 0.f;
            bool ok = true;
            for (int j = 0; j < blocks; ++j) {
                ok = mbar_wait_warp(&bar.s[tile], n & 1u, p.dev_status, kStatusFwdWait);
                if (!ok) break;
                tc_fence_after();
                uint32_t sreg[64];
#pragma unroll
                for (int c = 0; c < 2; ++c) tmem_ld_32x32(t_s + uint32_t(c * 32), *reinterpret_cast<uint32_t (*)[32]>(&sreg[32 * c]));
#pragma unroll
                for (int c = 0; c < 2; ++c) tmem_ld_wait_32(*reinterpret_cast<uint32_t (*)[32]>(&sreg[32 * c]));
                if (NH == 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&bar.read[tile]);
                }
                const int valid = limit - j * kAttnTile - half * 64;
                if (__any_sync(0xffffffffu, valid < 64)) {
#pragma unroll
                    for (int e = 0; e < 64; ++e)
                        if (e >= valid) sreg[e] = 0xFF800000u;
                }
                float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int e = 0; e < 64; e += 8) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) m4[c] = max3(m4[c], __uint_as_float(sreg[e + 2 * c]), __uint_as_float(sreg[e + 2 * c + 1]));
                }
                float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3])), other;
                ok = exchange(mx, other);
                if (!ok) break;
                mx = fmaxf(mx, other);
                // first block with a key: the difference is infinite; none yet: -inf - -inf compares false and -inf stays
                const bool moved = (mx - m_run) * sc > 8.0f;
                const float m_new = moved ? mx : m_run;
                const float mc = m_new == -INFINITY ? 0.f : m_new * sc;
                // exactly 1 where the maximum stays: of a contracted m sc - m sc the rounding would be left
                const float alpha = moved ? ex2(m_run * sc - mc) : 1.0f;
                if (j > 0) {                       // the product before has read P, and O may be rescaled
                    ok = mbar_wait_warp(&bar.o[tile], (n - 1u) & 1u, p.dev_status, kStatusFwdWait);
                    if (!ok) break;
                    if (__any_sync(0xffffffffu, moved)) {
                        tc_fence_after();
                        for (int c = half * 32; c < s.dh; c += (c & 31) == 16 ? 48 : 16) {        // its 32 columns of each 64
                            uint32_t r[16];
                            tmem_ld_32x16(t_o + uint32_t(c), r);
                            tmem_ld_wait_16(r);
#pragma unroll
                            for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * alpha);
                            tmem_st_32x16(t_o + uint32_t(c), r);
                        }
                    }
                }
                // The two warps of a scheduler take turns at the exponentials (16 a clock in an SM): side by side both would be at them, then
                // both at the rest.  Only the order of work hangs on this.
                if (j < both) {
                    if (tile == 1) ok = mbar_wait_warp(&bar.turn[0][lot], turns & 1u, p.dev_status, kStatusFwdWait);
                    else if (turns > 0) ok = mbar_wait_warp(&bar.turn[1][lot], (turns - 1u) & 1u, p.dev_status, kStatusFwdWait);
                    if (!ok) break;
                }
                const f32x2 sc2 = pk2(sc, sc), nmc2 = pk2(-mc, -mc);
                f32x2 sum2[2] = {pk2(0.f, 0.f), pk2(0.f, 0.f)};
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    uint32_t w[16];
#pragma unroll
                    for (int e = 0; e < 16; ++e) {
                        float z0, z1;
                        upk2(fma2(pk2(__uint_as_float(sreg[32 * c + 2 * e]), __uint_as_float(sreg[32 * c + 2 * e + 1])), sc2, nmc2), z0, z1);
                        const float p0 = ex2(z0), p1 = ex2(z1);
                        sum2[e & 1] = add2(sum2[e & 1], pk2(p0, p1));
                        w[e] = pack_bf16(p0, p1);
                    }
                    tmem_st_32x16(t_p + uint32_t(c * 16), w);
                }
                if (j < both) {
                    if (lane == 0) mbar_arrive(&bar.turn[tile][lot]);
                    ++turns;
                }
                float s0, s1;
                upk2(add2(sum2[0], sum2[1]), s0, s1);
                l_run = fmaf(l_run, alpha, s0 + s1);
                m_run = m_new;
                tmem_st_wait();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bar.p[tile]);
                ++n;
            }
            float other = 0.f;
            ok = ok && exchange(l_run, other);
            l_run += other;
            if (ok && blocks > 0) ok = mbar_wait_warp(&bar.o[tile], (n - 1u) & 1u, p.dev_status, kStatusFwdWait);
            else if (ok) ok = mbar_wait_warp(&bar.q_full[q.slot], q.phase, p.dev_status, kStatusFwdTma);     // zeros are staged behind the tile's load
            if (!ok) break;
            tc_fence_after();
            const bool keep = limit > 0 && blocks > 0;
            const float inv = keep ? 1.0f / l_run : 0.f;
            unsigned char* stage = smem + (2 * q.slot + tile) * R::kTile;
#pragma unroll
            for (int h = 0; h < NH; ++h) stage_rows<NH>(t_o + uint32_t(h * 64 + half * 32), stage, row, h * 2 + half, s.dh, keep, inv);
            if (half == 0 && i < s.Lq) *lse = keep ? m_run * s.scale + logf(l_run) : -INFINITY;
            tc_fence_before();
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar.staged[q.slot]);
            q.next();
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 0) tmem_dealloc(tmem_base, 512);
}

template <int NH>
hq_status launch_fwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, const FwdParams& p, cudaStream_t st) {
    const AttnShape& s = p.s;
    FwdMaps m;
    if (!encode_heads_bf16(&m.q, q, s.dh, s.heads, s.Lq, s.Nb, ldq, kAttnTile) ||
        !encode_heads_bf16(&m.k, k, s.dh, s.kv_heads, s.Lk, s.Nb, ldk, kAttnTile) ||
        !encode_heads_bf16(&m.v, v, s.dh, s.kv_heads, s.Lk, s.Nb, ldv, kAttnTile) ||
        !encode_heads_bf16(&m.out, p.out, s.dh, s.heads, s.Lq, s.Nb, p.ldo, kAttnTile))
        return HQ_ERR_CUDA;
    if (cudaFuncSetAttribute(attention_fwd_kernel<NH>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(fwd_smem<NH>())) != cudaSuccess)
        return HQ_ERR_CUDA;
    const unsigned sms = unsigned(sm_count()), grid = p.items < sms ? p.items : sms;
    attention_fwd_kernel<NH><<<grid, kFwdThreads, fwd_smem<NH>(), st>>>(m, p);
    return cudaGetLastError() == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}

}  // namespace
}  // namespace hq

extern "C" hq_status hq_attention_fwd_workspace_size(int64_t Nb, int64_t Lq, int64_t Lk, int heads, int kv_heads, int dh, size_t* bytes) {
    using namespace hq;
    if (bytes == nullptr) return HQ_ERR_INVALID_ARG;
    const hq_status e = attn_check(Nb, Lq, Lk, heads, kv_heads, dh, 1.0f);
    if (e != HQ_OK) return e;
    *bytes = 0;
    return HQ_OK;
}

extern "C" hq_status hq_attention_fwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, int64_t Nb,
                                      int64_t Lq, int64_t Lk, int heads, int kv_heads, int dh, float scale, int causal,
                                      const int32_t* q_lens, const int32_t* k_lens, void* out, int64_t ldo, float* lse, void* workspace,
                                      size_t ws_bytes, int32_t* dev_status, void* stream) {
    using namespace hq;
    hq_status e = attn_check(Nb, Lq, Lk, heads, kv_heads, dh, scale);
    if (e != HQ_OK) return e;
    if (Nb == 0) return HQ_OK;
    if ((e = attn_check_matrix(q, Lq, ldq, heads, dh)) != HQ_OK || (e = attn_check_matrix(k, Lk, ldk, kv_heads, dh)) != HQ_OK ||
        (e = attn_check_matrix(v, Lk, ldv, kv_heads, dh)) != HQ_OK || (e = attn_check_matrix(out, Lq, ldo, heads, dh)) != HQ_OK)
        return e;
    if (lse == nullptr) return HQ_ERR_INVALID_ARG;
    const int64_t q_blocks = (Lq + 2 * kAttnTile - 1) / (2 * kAttnTile), items = q_blocks * Nb * heads;
    if (items > 0x3fffffff) return HQ_ERR_UNSUPPORTED;
    (void)workspace; (void)ws_bytes;
    FwdParams p{};
    p.q_blocks = int(q_blocks); p.items = unsigned(items); p.ragged = k_lens != nullptr;
    p.s = AttnShape{q_lens, k_lens, int(Nb), int(Lq), int(Lk), heads, kv_heads, dh, causal != 0, scale, float(double(scale) * 1.4426950408889634)};
    p.out = static_cast<__nv_bfloat16*>(out);
    p.ldo = ldo; p.lse = lse; p.dev_status = dev_status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dh <= 64 ? launch_fwd<1>(q, ldq, k, ldk, v, ldv, p, st) : launch_fwd<2>(q, ldq, k, ldk, v, ldv, p, st);
}
