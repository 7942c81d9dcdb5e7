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

// The order in which tiles of (sample, head) pairs are worked on: tiles of `chunk` pairs, tile by tile.  One pair: the CTAs at work
// share its other side's tiles in L2 (64 x 1024 tokens, 8 heads of 64, forward: 243 us with all pairs' first tiles first, 201 so).  Under
// the causal mask tiles differ in length and the longest go first among pairs enough to fill the device four times.
__host__ inline unsigned attn_chunk(bool causal, int64_t tiles, int64_t pairs, int64_t slots) {
    const int64_t c = causal ? (4 * slots + tiles - 1) / tiles : 1;
    return unsigned(c < 1 ? 1 : c < pairs ? c : pairs);
}
__device__ __forceinline__ void attn_order(unsigned index, unsigned tiles, unsigned pairs, unsigned chunk, unsigned& tile, unsigned& pair) {
    if (chunk == 1) {
        pair = index / tiles;
        tile = index - pair * tiles;
        return;
    }
    const unsigned c = index / (chunk * tiles), r = index - c * (chunk * tiles), n = min(chunk, pairs - c * chunk);
    tile = r / n;
    pair = c * chunk + (r - tile * n);
}

// A tile is NH parts of 128 rows x 64 channels (128-byte rows, 128-byte swizzle), parts one after the other.
constexpr int kAttnPart = kAttnTile * 128;
template <int NH>
__device__ __forceinline__ void load_tile(unsigned char* dst, const CUtensorMap* tm, uint64_t* bar, int head, int row, int sample) {
#pragma unroll
    for (int h = 0; h < NH; ++h) tma_load_4d(dst + h * kAttnPart, tm, bar, 64 * h, head, row, sample);
}
// 32 columns of an accumulator as scaled bf16 into the staging tile (rows of 128 bytes, 128-byte swizzle); rows not kept become zeros.
template <int NH>
__device__ __forceinline__ void stage_rows(uint32_t taddr, unsigned char* tile, int row, int quarter, int dh, bool keep, float mul) {
    if (quarter * 32 >= dh) return;
    uint32_t r[32];
    tmem_ld_32x32(taddr, r);
    tmem_ld_wait_32(r);
    unsigned char* line = tile + (quarter >> 1) * kAttnPart + row * 128;
#pragma unroll
    for (int c = 0; c < 4; ++c) {
        uint4 w;
        w.x = pack_bf16(__uint_as_float(r[8 * c]) * mul, __uint_as_float(r[8 * c + 1]) * mul);
        w.y = pack_bf16(__uint_as_float(r[8 * c + 2]) * mul, __uint_as_float(r[8 * c + 3]) * mul);
        w.z = pack_bf16(__uint_as_float(r[8 * c + 4]) * mul, __uint_as_float(r[8 * c + 5]) * mul);
        w.w = pack_bf16(__uint_as_float(r[8 * c + 6]) * mul, __uint_as_float(r[8 * c + 7]) * mul);
        if (!keep) w = make_uint4(0u, 0u, 0u, 0u);
        *reinterpret_cast<uint4*>(line + ((((quarter & 1) * 4 + c) ^ (row & 7)) * 16)) = w;
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
