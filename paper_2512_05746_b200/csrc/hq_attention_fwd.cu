// Attention with the statistic its gradient needs: per sample, head and query, out = sum_j softmax_j(scale q . k_j) v_j over the keys
// the query sees, lse = log sum_j exp(scale q . k_j).  Queries, keys and values are matrices of their own (pitches, lengths, heads that
// share keys and values).
//
// One CTA takes two tiles of 128 queries of one (sample, head) and walks the keys in blocks of 128.  Warps 0-3 do the softmax of
// the first tile and warps 4-7 that of the second (thread = query row = lane of tensor memory), warp 8 loads, warp 9 issues:
//   S = Q K^T        both operands from shared memory (128-byte swizzle), fp32 in 128 columns of tensor memory
//   P = exp2(c S - c m) as bf16 over the columns of S that the row's thread has read
//   O += P V         P from tensor memory, V from shared memory, read along its keys without a transpose
// While one tile's exponentials run, the tensor core has the other tile's two products.  The running maximum moves only when a
// block's maximum exceeds it by more than 2^8 in the exponent: the weights stay below 2^8, the division by the row sum at the end
// is the same, and O is read and rescaled in tensor memory almost never.  P is rounded to bf16 (the products' type), the row sum
// runs over the unrounded weights in fp32.
#include "hq_attention_tile.cuh"

namespace hq {
namespace {

constexpr int32_t kStatusFwdWait = 0x700, kStatusFwdTma = 0x701;
constexpr int kFwdThreads = 320;
constexpr int kFwdSlots = 4;                       // K and V tiles in flight, in the order K0 V0 K1 V1 ...
template <int NH> constexpr size_t fwd_smem() { return size_t(2 + kFwdSlots) * NH * kAttnPart + 1024; }

struct FwdParams {
    AttnShape s;
    __nv_bfloat16* out;
    int64_t ldo;
    float* lse;                                    // [Nb][heads][Lq]
    int q_blocks;                                  // CTAs along the queries
    int32_t* dev_status;
};

template <int NH>
__global__ void __launch_bounds__(kFwdThreads, 1)
attention_fwd_kernel(const __grid_constant__ CUtensorMap tmQ, const __grid_constant__ CUtensorMap tmK,
                     const __grid_constant__ CUtensorMap tmV, const FwdParams p) {
    extern __shared__ __align__(1024) unsigned char smem_fwd[];
    constexpr int kTile = NH * kAttnPart;
    unsigned char* sQ = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_fwd) + 1023) & ~uintptr_t(1023));
    unsigned char* sKV = sQ + 2 * kTile;
    __shared__ uint64_t bar_q, bar_full[kFwdSlots], bar_empty[kFwdSlots], bar_s[2], bar_p[2], bar_o[2];
    __shared__ uint32_t tmem_slot;

    const AttnShape& s = p.s;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int bh = blockIdx.x % (s.Nb * s.heads), block = blockIdx.x / (s.Nb * s.heads);
    const int n = bh / s.heads, head = bh - n * s.heads;
    // causal: the blocks with the most keys first
    const int q0 = (s.causal ? p.q_blocks - 1 - block : block) * 2 * kAttnTile;
    const AttnSample sm = attn_sample(s, n);
    // key blocks of each tile: as far as its last query sees
    int nb[2];
#pragma unroll
    for (int t = 0; t < 2; ++t) {
        const int first = q0 + t * kAttnTile, last = min(first + kAttnTile, sm.q_hi) - 1;
        nb[t] = first > last || last < sm.q_lo ? 0 : (attn_key_limit(s, sm, last) + kAttnTile - 1) / kAttnTile;
    }
    const int nblocks = max(nb[0], nb[1]);

    if (tid == 0) {
        mbar_init(&bar_q, 1);
        for (int i = 0; i < kFwdSlots; ++i) { mbar_init(&bar_full[i], 1); mbar_init(&bar_empty[i], 1); }
        for (int t = 0; t < 2; ++t) { mbar_init(&bar_s[t], 1); mbar_init(&bar_p[t], 4); mbar_init(&bar_o[t], 1); }
        fence_barrier_init();
    }
    if (warp == 9) { __syncwarp(); tmem_alloc(&tmem_slot, 512); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = tmem_slot;          // S of the tiles at columns 0 and 128, O at 256 and 384

    if (warp == 8) {
        if (nblocks > 0 && elect_one()) {
            bool ok = true;
            const int group_head = head / (s.heads / s.kv_heads);
            int loads = 0;
            mbar_expect_tx(&bar_q, 2 * kTile);
            load_tile<NH>(sQ, &tmQ, &bar_q, head, q0, n);
            load_tile<NH>(sQ + kTile, &tmQ, &bar_q, head, q0 + kAttnTile, n);
            for (int i = 0; i < 2 * nblocks && ok; ++i) {
                const int slot = i % kFwdSlots, use = i / kFwdSlots;
                if (use > 0) ok = mbar_wait(&bar_empty[slot], uint32_t(use - 1) & 1u, p.dev_status, kStatusFwdWait);
                if (!ok) break;
                mbar_expect_tx(&bar_full[slot], kTile);
                load_tile<NH>(sKV + slot * kTile, (i & 1) ? &tmV : &tmK, &bar_full[slot], group_head, (i >> 1) * kAttnTile, n);
                ++loads;
            }
            // what was requested lands before the CTA's shared memory is given up, on every way out
            mbar_wait(&bar_q, 0, nullptr, 0);
            for (int i = max(0, loads - kFwdSlots); i < loads; ++i) mbar_wait(&bar_full[i % kFwdSlots], uint32_t(i / kFwdSlots) & 1u, nullptr, 0);
        }
        __syncwarp();
    } else if (warp == 9) {
        if (nblocks > 0) {
            const uint32_t idesc_s = make_idesc_bf16(kAttnTile, kAttnTile, false);
            const uint32_t idesc_o = make_idesc_bf16(kAttnTile, (s.dh + 15) & ~15, true);
            const int ksteps = (s.dh + 15) / 16;
            const uint64_t dq = make_sw128_kmajor_desc(smem_u32(sQ));
            bool ok = mbar_wait(&bar_q, 0, p.dev_status, kStatusFwdTma);
            auto slot_of = [&](int i) { return sKV + (i % kFwdSlots) * kTile; };
            auto landed = [&](int i) { return mbar_wait(&bar_full[i % kFwdSlots], uint32_t(i / kFwdSlots) & 1u, p.dev_status, kStatusFwdTma); };
            auto s_product = [&](int t, int j) {
                const uint64_t dk = make_sw128_kmajor_desc(smem_u32(slot_of(2 * j))), da = dq + uint64_t(t * (kTile >> 4));
                for (int k = 0; k < ksteps; ++k) {
                    const uint64_t step = uint64_t((k >> 2) * (kAttnPart >> 4) + 2 * (k & 3));
                    mma_bf16(tmem_base + uint32_t(t * 128), da + step, dk + step, idesc_s, k != 0 ? 1u : 0u);
                }
                mma_commit(&bar_s[t]);
            };
            // K of block j + 1 is free once both tiles have their S of it (or do not want it), V of block j after both products
            ok = __all_sync(0xffffffffu, ok && landed(0));
            if (ok) {
                if (elect_one()) {
                    tc_fence_after();
                    for (int t = 0; t < 2; ++t)
                        if (nb[t] > 0) s_product(t, 0);
                    mma_commit(&bar_empty[0]);
                }
                __syncwarp();
            }
            for (int j = 0; j < nblocks && ok; ++j) {
                ok = __all_sync(0xffffffffu, landed(2 * j + 1) && (j + 1 >= nblocks || landed(2 * j + 2)));
                if (!ok) break;
                if (sm.kl < min(s.Lk, (j + 1) * kAttnTile)) {  // tokens behind the sample's last: their values must not meet the zero weights
                    clear_rows<NH>(slot_of(2 * j + 1), 0, sm.kl - j * kAttnTile, lane);
                    fence_proxy_async_smem();
                    __syncwarp();
                }
                for (int t = 0; t < 2 && ok; ++t) {
                    if (j < nb[t]) ok = __all_sync(0xffffffffu, mbar_wait(&bar_p[t], uint32_t(j) & 1u, p.dev_status, kStatusFwdWait));
                    if (!ok) break;
                    if (elect_one()) {
                        tc_fence_after();
                        if (j < nb[t]) {
                            const uint64_t dv = make_sw128_mnmajor_desc(smem_u32(slot_of(2 * j + 1)), kAttnPart);
#pragma unroll
                            for (int k = 0; k < kAttnTile / 16; ++k)
                                mma_bf16_ts(tmem_base + uint32_t(256 + t * 128), tmem_base + uint32_t(t * 128 + 8 * k), dv + uint64_t(k * 128),
                                            idesc_o, (j | k) != 0 ? 1u : 0u);
                            mma_commit(&bar_o[t]);
                        }
                        if (t == 1) mma_commit(&bar_empty[(2 * j + 1) % kFwdSlots]);
                        // products run in the order of their issue: the next S overwrites P behind the product that reads it
                        if (j + 1 < nb[t]) s_product(t, j + 1);
                        if (t == 1 && j + 1 < nblocks) mma_commit(&bar_empty[(2 * j + 2) % kFwdSlots]);
                    }
                    __syncwarp();
                }
            }
        }
    } else {
        const int t = warp >> 2;
        const int row = (warp & 3) * 32 + lane, i = q0 + t * kAttnTile + row;
        const uint32_t t_s = tmem_base + (uint32_t((warp & 3) * 32) << 16) + uint32_t(t * 128);
        const uint32_t t_o = t_s + 256u;
        const int blocks = nb[t];
        const int limit = i < sm.q_hi ? attn_key_limit(s, sm, i) : 0;
        const float sc = s.scale_log2;
        float m_run = -INFINITY, l_run = 0.f;
        bool ok = true;
        for (int j = 0; j < blocks; ++j) {
            const uint32_t par = uint32_t(j) & 1u;
            ok = __all_sync(0xffffffffu, mbar_wait(&bar_s[t], par, p.dev_status, kStatusFwdWait));
            if (!ok) break;
            tc_fence_after();
            uint32_t sreg[128];
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld_32x32(t_s + uint32_t(c * 32), *reinterpret_cast<uint32_t (*)[32]>(&sreg[32 * c]));
#pragma unroll
            for (int c = 0; c < 4; ++c) tmem_ld_wait_32(*reinterpret_cast<uint32_t (*)[32]>(&sreg[32 * c]));
            const int valid = limit - j * kAttnTile;
            if (__any_sync(0xffffffffu, valid < kAttnTile)) {
#pragma unroll
                for (int e = 0; e < 128; ++e)
                    if (e >= valid) sreg[e] = 0xFF800000u;
            }
            float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int e = 0; e < 128; e += 8) {
#pragma unroll
                for (int c = 0; c < 4; ++c) m4[c] = max3(m4[c], __uint_as_float(sreg[e + 2 * c]), __uint_as_float(sreg[e + 2 * c + 1]));
            }
            const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
            // first block with a key: the difference is infinite; none yet: -inf - -inf compares false and -inf stays
            const float m_new = (mx - m_run) * sc > 8.0f ? mx : m_run;
            const float mc = m_new == -INFINITY ? 0.f : m_new * sc;
            const float alpha = ex2(m_run * sc - mc);
            const f32x2 sc2 = pk2(sc, sc), nmc2 = pk2(-mc, -mc);
            f32x2 sum2[2] = {pk2(0.f, 0.f), pk2(0.f, 0.f)};
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                uint32_t w[16];
#pragma unroll
                for (int e = 0; e < 16; ++e) {
                    float z0, z1;
                    upk2(fma2(pk2(__uint_as_float(sreg[32 * c + 2 * e]), __uint_as_float(sreg[32 * c + 2 * e + 1])), sc2, nmc2), z0, z1);
                    const float p0 = ex2(z0), p1 = ex2(z1);
                    sum2[e & 1] = add2(sum2[e & 1], pk2(p0, p1));
                    w[e] = pack_bf16(p0, p1);
                }
                tmem_st_32x16(t_s + uint32_t(c * 16), w);
            }
            float s0, s1;
            upk2(add2(sum2[0], sum2[1]), s0, s1);
            l_run = fmaf(l_run, alpha, s0 + s1);
            m_run = m_new;
            if (j > 0 && __any_sync(0xffffffffu, alpha != 1.0f)) {
                ok = __all_sync(0xffffffffu, mbar_wait(&bar_o[t], par ^ 1u, p.dev_status, kStatusFwdWait));
                if (!ok) break;
                tc_fence_after();
                for (int c = 0; c < s.dh; c += 16) {
                    uint32_t r[16];
                    tmem_ld_32x16(t_o + uint32_t(c), r);
                    tmem_ld_wait_16(r);
#pragma unroll
                    for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * alpha);
                    tmem_st_32x16(t_o + uint32_t(c), r);
                }
            }
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar_p[t]);
        }
        if (ok && blocks > 0) {
            ok = __all_sync(0xffffffffu, mbar_wait(&bar_o[t], uint32_t(blocks - 1) & 1u, p.dev_status, kStatusFwdWait));
            tc_fence_after();
        }
        if (ok) {
            const bool row_ok = i < s.Lq, keep = limit > 0 && blocks > 0;
            __nv_bfloat16* dst = p.out + (int64_t(n) * s.Lq + (row_ok ? i : 0)) * p.ldo + head * s.dh;
            const float inv = keep ? 1.0f / l_run : 0.f;
            for (int c = 0; c < s.dh; c += 32) store_rows(t_o + uint32_t(c), dst, c, s.dh, row_ok, keep, inv);
            if (row_ok) p.lse[(int64_t(n) * s.heads + head) * s.Lq + i] = keep ? m_run * s.scale + logf(l_run) : -INFINITY;
        }
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 9) tmem_dealloc(tmem_base, 512);
}

template <int NH>
hq_status launch_fwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, FwdParams p, cudaStream_t st) {
    const AttnShape& s = p.s;
    CUtensorMap tmQ, tmK, tmV;
    if (!encode_heads_bf16(&tmQ, q, s.dh, s.heads, s.Lq, s.Nb, ldq, kAttnTile) ||
        !encode_heads_bf16(&tmK, k, s.dh, s.kv_heads, s.Lk, s.Nb, ldk, kAttnTile) ||
        !encode_heads_bf16(&tmV, v, s.dh, s.kv_heads, s.Lk, s.Nb, ldv, kAttnTile))
        return HQ_ERR_CUDA;
    if (cudaFuncSetAttribute(attention_fwd_kernel<NH>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(fwd_smem<NH>())) != cudaSuccess)
        return HQ_ERR_CUDA;
    p.q_blocks = (s.Lq + 2 * kAttnTile - 1) / (2 * kAttnTile);
    const unsigned grid = unsigned(p.q_blocks) * unsigned(s.Nb) * unsigned(s.heads);
    attention_fwd_kernel<NH><<<grid, kFwdThreads, fwd_smem<NH>(), st>>>(tmQ, tmK, tmV, p);
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
    if (((Lq + 255) / 256) * Nb * heads > 0x7fffffff) return HQ_ERR_UNSUPPORTED;
    (void)workspace; (void)ws_bytes;
    FwdParams p{};
    p.s = AttnShape{q_lens, k_lens, int(Nb), int(Lq), int(Lk), heads, kv_heads, dh, causal != 0, scale, float(double(scale) * 1.4426950408889634)};
    p.out = static_cast<__nv_bfloat16*>(out);
    p.ldo = ldo; p.lse = lse; p.dev_status = dev_status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dh <= 64 ? launch_fwd<1>(q, ldq, k, ldk, v, ldv, p, st) : launch_fwd<2>(q, ldq, k, ldk, v, ldv, p, st);
}
