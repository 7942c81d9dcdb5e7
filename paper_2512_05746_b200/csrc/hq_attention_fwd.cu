// Attention with the statistic its gradient needs: per sample, head and query, out = sum_j softmax_j(scale q . k_j) v_j over the keys
// the query sees, lse = log sum_j exp(scale q . k_j).  Queries, keys and values are matrices of their own (pitches, lengths, heads that
// share keys and values).
//
// One CTA takes a tile of 128 queries of one (sample, head) and walks the keys in blocks of 64; four CTAs share an SM (two above 64
// channels).  Warps 0-3: thread = query row = lane of tensor memory; one lane of warp 4 loads and issues:
//   S = Q K^T        both operands from shared memory (128-byte swizzle), fp32 in 64 columns of tensor memory
//   P = exp2(c S - c m) as bf16 through shared memory, so that S of the next block is computed during this one's softmax
//   O += P V         V read along its keys without a transpose, O in dh columns
// What a CTA waits for, the others' exponentials cover: persistent CTAs of two tiles with blocks of 128 keys, P in tensor memory and 8 or
// 16 softmax warps came to 245-265 us at 64 x 1024 tokens, 8 heads of 64 (201 so) and 174 at 2 x 4096 causal, 16 / 2 heads of 128 (144), both
// timed on a cool GPU; in a run of calls this form takes 219 and 166 us.  Unmasked, 2 x 4096 with 16 heads of 128, those took 290-305
// where this takes 337.
// The running maximum moves only when a block's maximum exceeds it by more than 2^8 in the exponent: the weights stay below 2^8, the
// division by the row sum at the end is the same, and O is read and rescaled in tensor memory almost never.  P is rounded to bf16
// (the products' type), the row sum runs over the unrounded weights in fp32.
// Bound by the exponentials (16 a clock in an SM: 119 us of the 219) and the waits between a block's steps.
#include "hq_attention_tile.cuh"

namespace hq {
namespace {

constexpr int32_t kStatusFwdWait = 0x700, kStatusFwdTma = 0x701;

struct FwdParams {
    AttnShape s;
    __nv_bfloat16* out;
    int64_t ldo;
    float* lse;                                    // [Nb][heads][Lq]
    unsigned chunk;                                // order of the tiles (attn_order)
    int32_t* dev_status;
};
struct FwdMaps { CUtensorMap q, k, v, out; };

constexpr int kFwdBlock = 64, kFwdThreads = 160;
template <int NH> constexpr int fwd_ctas() { return NH == 1 ? 4 : 2; }
template <int NH> constexpr size_t fwd_smem() { return size_t(NH) * (kAttnPart + 2 * kFwdBlock * 128) + kAttnTile * kFwdBlock * 2 + 1024; }

template <int NH>
__global__ void __launch_bounds__(kFwdThreads, fwd_ctas<NH>())
attention_fwd_kernel(const __grid_constant__ FwdMaps m, const FwdParams p) {
    constexpr int KB = kFwdBlock, kPart = KB * 128, kTmemCols = NH == 1 ? 128 : 256;
    extern __shared__ __align__(1024) unsigned char smem_raw[];
    unsigned char* sQ = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
    unsigned char *sK = sQ + NH * kAttnPart, *sV = sK + NH * kPart, *sP = sV + NH * kPart;     // P: unswizzled core matrices
    __shared__ uint64_t bar_q, bar_k, bar_v, bar_s, bar_o, bar_read, bar_p, bar_drain;
    __shared__ uint32_t tmem_slot;
    constexpr uint32_t kPGroup = (KB / 8) * 128;

    const AttnShape& s = p.s;
    const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
    const int q_tiles = (s.Lq + kAttnTile - 1) / kAttnTile;
    unsigned block, bh;
    attn_order(blockIdx.x, unsigned(q_tiles), unsigned(s.Nb) * unsigned(s.heads), p.chunk, block, bh);
    const int n = int(bh / unsigned(s.heads)), head = int(bh) - n * s.heads;
    const int q0 = (s.causal ? q_tiles - 1 - int(block) : int(block)) * kAttnTile;
    const AttnSample sm = attn_sample(s, n);
    const int end = min(q0 + kAttnTile, sm.q_hi) - 1;
    const int blocks = q0 > end || end < sm.q_lo ? 0 : (attn_key_limit(s, sm, end) + KB - 1) / KB;
    if (blocks == 0) {                             // no query of the tile sees a key
        const int rows = min(kAttnTile, s.Lq - q0);
        zero_rows(p.out + (int64_t(n) * s.Lq + q0) * p.ldo + head * s.dh, p.ldo, rows, s.dh, tid, kFwdThreads);
        if (tid < rows) p.lse[(int64_t(n) * s.heads + head) * s.Lq + q0 + tid] = -INFINITY;
        return;
    }
    if (tid == 0) {
        mbar_init(&bar_q, 1); mbar_init(&bar_k, 1); mbar_init(&bar_v, 1);
        mbar_init(&bar_s, 1); mbar_init(&bar_o, 1); mbar_init(&bar_read, 4); mbar_init(&bar_p, 4); mbar_init(&bar_drain, 1);
        fence_barrier_init();
    }
    if (warp == 4 && lane < 4) tma_prefetch_desc(&m.q + lane);
    if (warp == 1) { __syncwarp(); tmem_alloc(&tmem_slot, kTmemCols); tmem_relinquish(); }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem_base = tmem_slot;
    bool ok = true;

    if (warp == 4) {
        if (elect_one()) {
            const uint32_t idesc_s = make_idesc_bf16(kAttnTile, KB, false), idesc_o = make_idesc_bf16(kAttnTile, (s.dh + 15) & ~15, true);
            const int ksteps = (s.dh + 15) / 16, group_head = head / (s.heads / s.kv_heads);
            const uint64_t dq = make_sw128_kmajor_desc(smem_u32(sQ)), dk = make_sw128_kmajor_desc(smem_u32(sK));
            const uint64_t dp = make_desc_noswizzle(smem_u32(sP), 128, kPGroup), dv = make_sw128_mnmajor_desc(smem_u32(sV), kPart);
            auto wait = [&](uint64_t* b, uint32_t parity, int32_t code) { return mbar_wait_lane(b, parity, p.dev_status, code); };
            auto load = [&](unsigned char* to, const CUtensorMap* tm, uint64_t* bar, int j) {
                mbar_expect_tx(bar, NH * kPart);
#pragma unroll
                for (int h = 0; h < NH; ++h) tma_load_4d(to + h * kPart, tm, bar, 64 * h, group_head, j * KB, n);
            };
            auto scores = [&]() {
                for (int k = 0; k < ksteps; ++k)
                    mma_bf16(tmem_base, dq + uint64_t((k >> 2) * (kAttnPart >> 4) + 2 * (k & 3)), dk + uint64_t((k >> 2) * (kPart >> 4) + 2 * (k & 3)),
                             idesc_s, k != 0 ? 1u : 0u);
                mma_commit(&bar_s);
            };
            mbar_expect_tx(&bar_q, NH * kAttnPart);
            load_tile<NH>(sQ, &m.q, &bar_q, head, q0, n);
            load(sK, &m.k, &bar_k, 0);
            load(sV, &m.v, &bar_v, 0);
            int k_loads = 1, v_loads = 1;          // begun so far
            ok = wait(&bar_q, 0, kStatusFwdTma) && wait(&bar_k, 0, kStatusFwdTma);
            if (ok) { tc_fence_after(); scores(); }
            for (int j = 0; j < blocks && ok; ++j) {
                const uint32_t par = uint32_t(j) & 1u;
                const bool more = j + 1 < blocks;
                if (more) {
                    ok = wait(&bar_s, par, kStatusFwdWait);                    // the K buffer has been read
                    if (!ok) break;
                    load(sK, &m.k, &bar_k, j + 1);
                    ++k_loads;
                }
                if (j > 0) {
                    ok = wait(&bar_o, par ^ 1u, kStatusFwdWait);               // ... and the V buffer
                    if (!ok) break;
                    load(sV, &m.v, &bar_v, j);
                    ++v_loads;
                }
                if (more) {
                    ok = wait(&bar_read, par, kStatusFwdWait) && wait(&bar_k, par ^ 1u, kStatusFwdTma);
                    if (!ok) break;
                    tc_fence_after();
                    scores();
                }
                ok = wait(&bar_v, par, kStatusFwdTma) && wait(&bar_p, par, kStatusFwdWait);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int k = 0; k < KB / 16; ++k)  // 16 keys on: two core-matrix columns of P, 16 rows of V
                    mma_bf16(tmem_base + uint32_t(KB), dp + uint64_t(k * 16), dv + uint64_t(k * 128), idesc_o, (j | k) != 0 ? 1u : 0u);
                mma_commit(&bar_o);
            }
            // what was requested lands before the CTA's shared memory is given up, on every way out
            mma_drain(&bar_drain);
            mbar_wait_lane(&bar_q, 0, nullptr, 0);
            mbar_wait_lane(&bar_k, uint32_t(k_loads - 1) & 1u, nullptr, 0);
            mbar_wait_lane(&bar_v, uint32_t(v_loads - 1) & 1u, nullptr, 0);
        }
        __syncwarp();
    } else {
        const int i = q0 + tid, limit = i < sm.q_hi ? attn_key_limit(s, sm, i) : 0;
        const uint32_t t_s = tmem_base + (uint32_t(warp * 32) << 16), t_o = t_s + uint32_t(KB);
        const float sc = s.scale_log2;
        float m_run = -INFINITY, l_run = 0.f;
        for (int j = 0; j < blocks; ++j) {
            const uint32_t par = uint32_t(j) & 1u;
            ok = mbar_wait_warp(&bar_s, par, p.dev_status, kStatusFwdWait);
            if (!ok) break;
            tc_fence_after();
            uint32_t sreg[KB];
#pragma unroll
            for (int c = 0; c < KB / 32; ++c) tmem_ld_32x32(t_s + uint32_t(c * 32), *reinterpret_cast<uint32_t (*)[32]>(&sreg[32 * c]));
#pragma unroll
            for (int c = 0; c < KB / 32; ++c) tmem_ld_wait_32(*reinterpret_cast<uint32_t (*)[32]>(&sreg[32 * c]));
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar_read);
            const int valid = limit - j * KB;
            if (__any_sync(0xffffffffu, valid < KB)) {
#pragma unroll
                for (int e = 0; e < KB; ++e)
                    if (e >= valid) sreg[e] = 0xFF800000u;
            }
            float m4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int e = 0; e < KB; e += 8) {
#pragma unroll
                for (int c = 0; c < 4; ++c) m4[c] = max3(m4[c], __uint_as_float(sreg[e + 2 * c]), __uint_as_float(sreg[e + 2 * c + 1]));
            }
            const float mx = fmaxf(fmaxf(m4[0], m4[1]), fmaxf(m4[2], m4[3]));
            // first block with a key: the difference is infinite; none yet: -inf - -inf compares false and -inf stays
            const bool moved = (mx - m_run) * sc > 8.0f;
            const float m_new = moved ? mx : m_run;
            const float mc = m_new == -INFINITY ? 0.f : m_new * sc;
            const float alpha = moved ? ex2(m_run * sc - mc) : 1.0f;
            const f32x2 sc2 = pk2(sc, sc), nmc2 = pk2(-mc, -mc);
            f32x2 sum2[2] = {pk2(0.f, 0.f), pk2(0.f, 0.f)};
            unsigned char* prow = sP + (tid >> 3) * kPGroup + (tid & 7) * 16;
            if (j > 0) {                           // the product before has read P, and O may be rescaled
                ok = mbar_wait_warp(&bar_o, par ^ 1u, p.dev_status, kStatusFwdWait);
                if (!ok) break;
            }
#pragma unroll
            for (int g = 0; g < KB / 8; ++g) {
                uint32_t w[4];
#pragma unroll
                for (int h = 0; h < 4; ++h) {
                    float z0, z1;
                    upk2(fma2(pk2(__uint_as_float(sreg[8 * g + 2 * h]), __uint_as_float(sreg[8 * g + 2 * h + 1])), sc2, nmc2), z0, z1);
                    const float p0 = ex2(z0), p1 = ex2(z1);
                    sum2[h & 1] = add2(sum2[h & 1], pk2(p0, p1));
                    w[h] = pack_bf16(p0, p1);
                }
                *reinterpret_cast<uint4*>(prow + g * 128) = make_uint4(w[0], w[1], w[2], w[3]);
            }
            float s0, s1;
            upk2(add2(sum2[0], sum2[1]), s0, s1);
            l_run = fmaf(l_run, alpha, s0 + s1);
            m_run = m_new;
            if (j > 0 && __any_sync(0xffffffffu, moved)) {
                tc_fence_after();
                for (int c = 0; c < s.dh; c += 16) {
                    uint32_t r[16];
                    tmem_ld_32x16(t_o + uint32_t(c), r);
                    tmem_ld_wait_16(r);
#pragma unroll
                    for (int e = 0; e < 16; ++e) r[e] = __float_as_uint(__uint_as_float(r[e]) * alpha);
                    tmem_st_32x16(t_o + uint32_t(c), r);
                }
                tmem_st_wait();
            }
            if (sm.kl < min(s.Lk, (j + 1) * KB)) { // values of tokens behind the sample's last: they would meet zero weights
                ok = mbar_wait_warp(&bar_v, par, p.dev_status, kStatusFwdTma);
                if (!ok) break;
                const int first = sm.kl - j * KB;
                for (int f = first * 8 * NH + tid; f < KB * 8 * NH; f += 128) {
                    const int r = f / (8 * NH), c = f - r * 8 * NH;
                    *reinterpret_cast<uint4*>(sV + (c >> 3) * kPart + r * 128 + (c & 7) * 16) = make_uint4(0u, 0u, 0u, 0u);
                }
            }
            fence_proxy_async_smem();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bar_p);
        }
        if (ok) ok = mbar_wait_warp(&bar_o, uint32_t(blocks - 1) & 1u, p.dev_status, kStatusFwdWait);
        if (ok) {
            tc_fence_after();
            const bool keep = limit > 0;
            const float inv = keep ? 1.0f / l_run : 0.f;
#pragma unroll
            for (int c = 0; c < 2 * NH; ++c) stage_rows<NH>(t_o + uint32_t(c * 32), sQ, tid, c, s.dh, keep, inv);
            if (i < s.Lq) p.lse[(int64_t(n) * s.heads + head) * s.Lq + i] = keep ? m_run * s.scale + logf(l_run) : -INFINITY;
            fence_proxy_async_smem();
        }
    }
    tc_fence_before();
    const bool all = __syncthreads_and(ok);
    if (warp == 1) tmem_dealloc(tmem_base, kTmemCols);
    if (all && tid == 0) {
#pragma unroll
        for (int h = 0; h < NH; ++h) tma_store_4d(&m.out, sQ + h * kAttnPart, 64 * h, head, q0, n);
        bulk_commit_group();
        bulk_wait_read_all();
    }
}

template <int NH>
hq_status launch_fwd(const void* q, int64_t ldq, const void* k, int64_t ldk, const void* v, int64_t ldv, FwdParams p, cudaStream_t st) {
    const AttnShape& s = p.s;
    FwdMaps m;
    if (!encode_heads_bf16(&m.q, q, s.dh, s.heads, s.Lq, s.Nb, ldq, kAttnTile) ||
        !encode_heads_bf16(&m.k, k, s.dh, s.kv_heads, s.Lk, s.Nb, ldk, kFwdBlock) ||
        !encode_heads_bf16(&m.v, v, s.dh, s.kv_heads, s.Lk, s.Nb, ldv, kFwdBlock) ||
        !encode_heads_bf16(&m.out, p.out, s.dh, s.heads, s.Lq, s.Nb, p.ldo, kAttnTile))
        return HQ_ERR_CUDA;
    if (cudaFuncSetAttribute(attention_fwd_kernel<NH>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(fwd_smem<NH>())) != cudaSuccess)
        return HQ_ERR_CUDA;
    const int64_t per = (s.Lq + kAttnTile - 1) / kAttnTile, pairs = int64_t(s.Nb) * s.heads;
    p.chunk = attn_chunk(s.causal, per, pairs, int64_t(fwd_ctas<NH>()) * sm_count());
    attention_fwd_kernel<NH><<<unsigned(per * pairs), kFwdThreads, fwd_smem<NH>(), st>>>(m, p);
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
    if ((Lq + kAttnTile - 1) / kAttnTile * Nb * heads > 0x3fffffff) return HQ_ERR_UNSUPPORTED;
    (void)workspace; (void)ws_bytes;
    FwdParams p{};
    p.s = AttnShape{q_lens, k_lens, int(Nb), int(Lq), int(Lk), heads, kv_heads, dh, causal != 0, scale, float(double(scale) * 1.4426950408889634)};
    p.out = static_cast<__nv_bfloat16*>(out);
    p.ldo = ldo; p.lse = lse; p.dev_status = dev_status;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    return dh <= 64 ? launch_fwd<1>(q, ldq, k, ldk, v, ldv, p, st) : launch_fwd<2>(q, ldq, k, ldk, v, ldv, p, st);
}
