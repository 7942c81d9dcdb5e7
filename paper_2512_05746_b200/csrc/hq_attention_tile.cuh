// What the attention kernels with separate queries, keys and values share (hq_attention_fwd.cu, hq_attention_bwd.cu): the view of a
// batch, which keys a query sees, tiles of 128 rows brought in by bulk tensor loads, and rows outside the lengths made zero.
#pragma once

#include "hq_common.cuh"
#include "hq_fwht.cuh"
#include "hq_mma_bf16.cuh"

namespace hq {

constexpr int kAttnTile = 128;                     // rows of a tile: tensor-memory lanes, queries or keys

struct AttnShape {
    const int32_t *q_lens, *k_lens;                // [Nb] or NULL
    int Nb, Lq, Lk, heads, kv_heads, dh;
    int causal;
    float scale, scale_log2;                       // scale and scale * log2(e)
};

// One sample: queries [q_lo, q_hi) see at least one key, query i sees keys [0, min(kl, i + shift + 1)) (causal) or [0, kl).
struct AttnSample { int q_lo, q_hi, kl, shift; };
__device__ __forceinline__ AttnSample attn_sample(const AttnShape& s, int n) {
    AttnSample r;
    int ql = s.Lq;
    r.kl = s.Lk;
    if (s.q_lens != nullptr) ql = min(max(__ldg(s.q_lens + n), 0), s.Lq);
    if (s.k_lens != nullptr) r.kl = min(max(__ldg(s.k_lens + n), 0), s.Lk);
    r.shift = r.kl - ql;
    r.q_lo = s.causal ? max(0, -r.shift) : 0;
    r.q_hi = r.kl > 0 ? ql : 0;
    if (r.q_lo > r.q_hi) r.q_lo = r.q_hi;
    return r;
}
// Keys that query i sees: [0, limit).
__device__ __forceinline__ int attn_key_limit(const AttnShape& s, const AttnSample& r, int i) {
    return s.causal ? min(r.kl, max(0, i + r.shift + 1)) : r.kl;
}

// A tile is NH parts of 128 rows x 64 channels (128-byte rows, 128-byte swizzle), parts one after the other.
constexpr int kAttnPart = kAttnTile * 128;
template <int NH>
__device__ __forceinline__ void load_tile(unsigned char* dst, const CUtensorMap* tm, uint64_t* bar, int head, int row, int sample) {
#pragma unroll
    for (int h = 0; h < NH; ++h) tma_load_4d(dst + h * kAttnPart, tm, bar, 64 * h, head, row, sample);
}
// Rows of a landed tile outside [lo, hi) become zeros (one warp): they belong to tokens outside the lengths, whose values may be
// infinite or not numbers, and would meet zero weights in a product.
template <int NH>
__device__ __forceinline__ void clear_rows(unsigned char* tile, int lo, int hi, int lane) {
    for (int h = 0; h < NH; ++h)
        for (int f = lane; f < kAttnTile * 8; f += 32) {
            const int row = f >> 3;
            if (row < lo || row >= hi) *reinterpret_cast<uint4*>(tile + h * kAttnPart + f * 16) = make_uint4(0u, 0u, 0u, 0u);
        }
}

// 32 accumulator columns of this warp's lanes as scaled bf16 into rows of global memory: `dst` is the row's first channel of the
// head, `c0` the first channel of the 32.  A row that is not kept gets zeros; one that does not exist (row_ok false) nothing.
__device__ __forceinline__ void store_rows(uint32_t taddr, __nv_bfloat16* dst, int c0, int dh, bool row_ok, bool keep, float mul) {
    for (int c = 0; c < 32 && c0 + c < dh; c += 16) {
        uint32_t r[16];
        tmem_ld_32x16(taddr + uint32_t(c), r);
        tmem_ld_wait_16(r);
        uint4 w[2];
        uint32_t* u = reinterpret_cast<uint32_t*>(w);
#pragma unroll
        for (int e = 0; e < 8; ++e)
            u[e] = keep ? pack_bf16(__uint_as_float(r[2 * e]) * mul, __uint_as_float(r[2 * e + 1]) * mul) : 0u;
        if (row_ok) {
            uint4* to = reinterpret_cast<uint4*>(dst + c0 + c);
            to[0] = w[0];
            if (c0 + c + 8 < dh) to[1] = w[1];
        }
    }
}
// Zeros for `rows` rows of one head, by `threads` threads.
__device__ __forceinline__ void zero_rows(__nv_bfloat16* base, int64_t ld, int rows, int dh, int thread, int threads) {
    const int v = dh / 8;
    for (int f = thread; f < rows * v; f += threads) {
        const int row = f / v;
        *reinterpret_cast<uint4*>(base + int64_t(row) * ld + (f - row * v) * 8) = make_uint4(0u, 0u, 0u, 0u);
    }
}

// Checks every attention call shares (host).
inline hq_status attn_check(int64_t Nb, int64_t Lq, int64_t Lk, int heads, int kv_heads, int dh, float scale) {
    if (Nb < 0 || Lq <= 0 || Lk <= 0 || heads <= 0 || kv_heads <= 0 || heads % kv_heads != 0 || dh <= 0) return HQ_ERR_SHAPE;
    if (!(scale > 0.f) || !(scale < 1e30f)) return HQ_ERR_INVALID_ARG;
    if (dh % 8 != 0 || dh > 128) return HQ_ERR_UNSUPPORTED;
    if (Nb > 65535 || heads > 65535 || Nb * heads > 65535 || Lq > (1 << 24) || Lk > (1 << 24)) return HQ_ERR_UNSUPPORTED;
    return HQ_OK;
}
// A matrix [Nb * L][ld] with `heads` heads of dh columns.
inline hq_status attn_check_matrix(const void* p, int64_t L, int64_t ld, int heads, int dh) {
    if (p == nullptr) return HQ_ERR_INVALID_ARG;
    if (ld < int64_t(heads) * dh) return HQ_ERR_SHAPE;
    if (!aligned16(p) || ld % 8 != 0) return HQ_ERR_ALIGNMENT;
    if (ld > (int64_t(1) << 31) || L * ld >= (int64_t(1) << 38)) return HQ_ERR_UNSUPPORTED;
    return HQ_OK;
}

}  // namespace hq
