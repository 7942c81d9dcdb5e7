// The norm of queries and keys for each head with the position rotation in the same pass, and its gradient: what stands between the
// QKV projection of a transformer block and its attention.
//
//   y = x / sqrt(mean(x^2) + eps) * gamma          over the dh channels of one head (gamma [dh], shared by the heads)
//   (a, b) -> (a c - b s, b c + a s)               for the pairs of the first `rot` channels; c, s: the table row of the token
//
// Gradient, with u = the rotation's transpose applied to the output's gradient, xh = x / sqrt(mean(x^2) + eps):
//   dx = (gamma u - xh mean(gamma u xh)) / sqrt(mean(x^2) + eps),     dgamma = sum over rows and heads of u xh
//
// Memory-bound: every value is read and written once, tables and gamma come from the caches.  A group of dh / 8 lanes holds one head of
// one row, 8 channels a lane (16 bytes of bf16), so that the row's sums are a few shuffles; 32 / (dh / 8) heads a warp.  Sums and
// the rotation in fp32, one rounding at the end.
//
// 65536 rows of 8 + 8 heads of 64 in bf16: 65 us, 63 % of the copy rate, the gradient 101 (61 %); in fp32 92 and 137 us (89 %).  Between
// the bounds in bf16: 20 instructions a value (24) at 66 % (49 %) of the issue slots, 46 % (48 %) of the DRAM rate and 44 % (24 %) of the
// warps, which ask for a row, wait for it, compute and store before they ask for the next.
#include "hq_common.cuh"
#include "hq_fwht.cuh"
#include "hq_vec8.cuh"

namespace hq {
namespace {

struct RopeSide { const void* x; const void* g; void* out; int64_t ldx, ldg, ldo; const float* gamma; float* dgamma; int heads; };
struct RopeParams {
    RopeSide q, k;
    int64_t rows;
    int dh, rot;
    const float *cos, *sin;                        // [npos][rot / 2]
    const int32_t* positions;                      // [rows], or NULL: row % npos
    int64_t npos;
    float eps;
    float* partial;                                // gradient of gamma: [2][blocks][dh]
};
constexpr int kRopeThreads = 256;
constexpr int kRopeMaxBlocks = 1184;               // 8 CTAs for each of 148 SMs, on every device: gamma's gradient is summed in one order

// Sum over the lanes of a group, in every lane of it.  V: their number where it is 4, 8 or 16, else 0.
template <int V>
__device__ __forceinline__ float group_sum(float x, int pos, int v, int base) {
    if constexpr (V > 0) {
#pragma unroll
        for (int off = V / 2; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
        return x;
    } else {
#pragma unroll
        for (int off = 8; off > 0; off >>= 1) {
            const float o = __shfl_down_sync(0xffffffffu, x, off);
            if (pos < off && pos + off < v) x += o;
        }
        return __shfl_sync(0xffffffffu, x, base);
    }
}

enum RopePairs { kInterleaved = 0, kHalvesByLane = 1, kHalvesAny = 2 };

// What a lane's 8 channels meet in a row's rotation: out = y c + other s, the sign of the pair's first member in s.  Interleaved pairs
// lie in the lane; halves whose distance rot / 2 is a multiple of 8 channels in another lane at the same place; other halves anywhere in
// the head.  Channels that are not rotated: 1 and 0.  VEC: every table row is 16-byte aligned.
template <int PAIRS, bool VEC>
__device__ __forceinline__ void turns(f32x2 (&c)[4], f32x2 (&s)[4], const RopeParams& p, uint32_t at, int c0) {
    const int half = p.rot >> 1;
    const float *cs = p.cos + int64_t(at) * half, *sn = p.sin + int64_t(at) * half;
    if (VEC && PAIRS == kInterleaved && c0 + 8 <= p.rot) {
        const float4 a = __ldg(reinterpret_cast<const float4*>(cs + c0 / 2)), b = __ldg(reinterpret_cast<const float4*>(sn + c0 / 2));
        c[0] = pk2(a.x, a.x); c[1] = pk2(a.y, a.y); c[2] = pk2(a.z, a.z); c[3] = pk2(a.w, a.w);
        s[0] = pk2(-b.x, b.x); s[1] = pk2(-b.y, b.y); s[2] = pk2(-b.z, b.z); s[3] = pk2(-b.w, b.w);
        return;
    }
    if (VEC && PAIRS == kHalvesByLane && c0 < p.rot) {
        const bool hi = c0 >= half;
        const int t = hi ? c0 - half : c0;
        const f32x2 sign = hi ? pk2(1.f, 1.f) : pk2(-1.f, -1.f);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
            const float4 a = __ldg(reinterpret_cast<const float4*>(cs + t) + e), b = __ldg(reinterpret_cast<const float4*>(sn + t) + e);
            c[2 * e] = pk2(a.x, a.y); c[2 * e + 1] = pk2(a.z, a.w);
            s[2 * e] = mul2(sign, pk2(b.x, b.y)); s[2 * e + 1] = mul2(sign, pk2(b.z, b.w));
        }
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float cc[2], ss[2];
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int ch = c0 + 2 * e + x;
            cc[x] = 1.f; ss[x] = 0.f;
            if (ch < p.rot) {
                const bool second = PAIRS == kInterleaved ? x == 1 : ch >= half;
                const int t = PAIRS == kInterleaved ? ch >> 1 : second ? ch - half : ch;
                cc[x] = __ldg(cs + t);
                ss[x] = second ? __ldg(sn + t) : -__ldg(sn + t);
            }
        }
        c[e] = pk2(cc[0], cc[1]); s[e] = pk2(ss[0], ss[1]);
    }
}

// The other members of the pairs of a lane's 8 channels, as they were loaded; at distances that are no multiple of 8 channels through
// `line`, the warp's 256 floats of shared memory.
template <int PAIRS, typename T>
__device__ __forceinline__ void partners(f32x2 (&o)[4], const f32x2 (&y)[4], const Vec8<T>& raw, int rot, int pos, int base, int lane, float* line) {
    const int half = rot >> 1, c0 = pos * 8;
    if (PAIRS == kInterleaved) {
#pragma unroll
        for (int e = 0; e < 4; ++e) { float a, b; upk2(y[e], a, b); o[e] = pk2(b, a); }
    } else if (PAIRS == kHalvesByLane) {
        const int step = half >> 3;
        raw.of(c0 < rot ? (c0 >= half ? lane - step : lane + step) : lane).get(o);
    } else {
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 4; ++e) { float a, b; upk2(y[e], a, b); line[lane * 8 + 2 * e] = a; line[lane * 8 + 2 * e + 1] = b; }
        __syncwarp();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float t[2];
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int ch = c0 + 2 * e + x;
                t[x] = ch < rot ? line[base * 8 + (ch >= half ? ch - half : ch + half)] : 0.f;
            }
            o[e] = pk2(t[0], t[1]);
        }
    }
}
// gamma of a lane's channels (1 without), and of their pairs' other members.
template <int PAIRS>
__device__ __forceinline__ void gammas(f32x2 (&own)[4], f32x2 (&other)[4], const float* gamma, int rot, int dh, int c0) {
    const int half = rot >> 1;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a[2] = {1.f, 1.f}, b[2] = {1.f, 1.f};
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int ch = c0 + 2 * e + x, t = ch >= rot ? ch : PAIRS == kInterleaved ? ch ^ 1 : ch >= half ? ch - half : ch + half;
            if (gamma != nullptr && ch < dh) { a[x] = __ldg(gamma + ch); b[x] = __ldg(gamma + t); }
        }
        own[e] = pk2(a[0], a[1]); other[e] = pk2(b[0], b[1]);
    }
}

// blockIdx.y: 0 queries, 1 keys.  GRAD: `g` is the output's gradient and `out` the input's.  A warp's groups of lanes take the heads of
// one row, step by step (or, where a row has fewer heads than the warp has groups, of several rows); the row's part of the tables stays in
// registers meanwhile.  Arithmetic on pairs of floats.
template <typename T, int PAIRS, bool VEC, bool GRAD, int V>
__global__ void __launch_bounds__(kRopeThreads, GRAD ? 2 : sizeof(T) == 4 ? 3 : 4) qk_rope_kernel(const RopeParams p) {
    constexpr int kAhead = 2;                                  // steps whose loads are in flight together
    __shared__ float lines[GRAD || PAIRS == kHalvesAny ? kRopeThreads * 8 : 1];
    const RopeSide& side = blockIdx.y == 0 ? p.q : p.k;
    const int v = V > 0 ? V : p.dh / 8, dh = V > 0 ? V * 8 : p.dh;
    const int per_warp = 32 / v, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, heads = side.heads;
    // lanes left over (32 no multiple of v) stand behind a head's last channel
    const int sub = lane / v, pos = sub < per_warp ? lane - sub * v : v, base = sub < per_warp ? sub * v : 0;
    const int together = heads < per_warp ? per_warp / heads : 1;                            // rows a warp takes at a time
    const int row_sub = together > 1 ? sub / heads : 0, head0 = together > 1 ? sub - row_sub * heads : sub;
    const bool group = pos < v && row_sub < together;
    float* line = lines + (PAIRS == kHalvesAny ? warp * 256 : 0);
    f32x2 gamma[4], other_gamma[4], dgamma[4];                 // without GRAD both go into the turns, where there is a gamma
    gammas<PAIRS>(gamma, other_gamma, side.gamma, p.rot, dh, pos * 8);
#pragma unroll
    for (int e = 0; e < 4; ++e) dgamma[e] = pk2(0.f, 0.f);
    const float inv_dh = 1.0f / float(dh);
    const uint32_t rows = uint32_t(p.rows), npos = uint32_t(p.npos);
    const uint32_t stride = gridDim.x * (kRopeThreads / 32) * uint32_t(together);
    uint32_t row0 = (blockIdx.x * (kRopeThreads / 32) + uint32_t(warp)) * uint32_t(together);
    const uint32_t cyc_on = stride % npos;
    uint32_t cyc = (row0 + uint32_t(row_sub)) % npos;          // the row's place in its sample
    for (; row0 < rows; row0 += stride) {
        const uint32_t row = row0 + uint32_t(row_sub);
        const bool live = group && row < rows;
        const int64_t r = live ? int64_t(row) : 0, c0 = r * side.ldx + pos * 8, g0 = GRAD ? r * side.ldg + pos * 8 : 0, o0 = r * side.ldo + pos * 8;
        Vec8<T> x_in[kAhead], g_in[kAhead];
        auto request = [&](int h0) {
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                const int head = h0 + u * per_warp + head0;
                x_in[u].clear();
                if (GRAD) g_in[u].clear();
                if (live && head < heads) {
                    x_in[u].load(side.x, c0 + head * dh);
                    if (GRAD) g_in[u].load(side.g, g0 + head * dh);
                }
            }
        };
        request(0);                                            // in front of the tables' loads
        f32x2 c[4], sn[4];
        {
            uint32_t at = 0;
            if (live) at = p.positions == nullptr ? cyc : uint32_t(min(max(__ldg(p.positions + row), 0), int(npos) - 1));
            turns<PAIRS, VEC>(c, sn, p, at, pos * 8);
            cyc += cyc_on;
            if (cyc >= npos) cyc -= npos;
            if (!GRAD) {                                       // out = (x gamma c + other gamma' s) / rms
#pragma unroll
                for (int e = 0; e < 4; ++e) { c[e] = mul2(c[e], gamma[e]); sn[e] = mul2(sn[e], other_gamma[e]); }
            }
        }
        for (int h0 = 0; h0 < heads; h0 += per_warp * kAhead) {
            if (h0 > 0) request(h0);
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
                if (u > 0 && h0 + u * per_warp >= heads) break;                              // the same in every lane
                const int head = h0 + u * per_warp + head0;
                f32x2 x[4], o[4], sq = pk2(0.f, 0.f);
                x_in[u].get(x);
#pragma unroll
                for (int e = 0; e < 4; ++e) sq = fma2(x[e], x[e], sq);
                if (!GRAD) {
                    const float inv = rsqrtf(group_sum<V>(pair_sum(sq), pos, v, base) * inv_dh + p.eps);
                    partners<PAIRS>(o, x, x_in[u], p.rot, pos, base, lane, line);
                    const f32x2 inv2 = pk2(inv, inv);
#pragma unroll
                    for (int e = 0; e < 4; ++e) x[e] = mul2(inv2, fma2(x[e], c[e], mul2(o[e], sn[e])));
                } else {
                    f32x2 w[4], dot = pk2(0.f, 0.f);
                    g_in[u].get(w);
                    partners<PAIRS>(o, w, g_in[u], p.rot, pos, base, lane, line);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        w[e] = sub2(mul2(w[e], c[e]), mul2(o[e], sn[e]));                    // u, the transpose's
                        o[e] = mul2(gamma[e], w[e]);
                        dot = fma2(o[e], x[e], dot);
                    }
                    const float inv = rsqrtf(group_sum<V>(pair_sum(sq), pos, v, base) * inv_dh + p.eps);
                    const float mean = group_sum<V>(pair_sum(dot), pos, v, base) * inv_dh * inv;             // of gamma u xh
                    const f32x2 inv2 = pk2(inv, inv), less = pk2(-mean, -mean);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const f32x2 xh = mul2(x[e], inv2);
                        // a lane without a head has no part in the sum: 1 / rms of nothing is infinite where eps is 0, and its table row nobody's
                        if (live && head < heads) dgamma[e] = fma2(w[e], xh, dgamma[e]);
                        x[e] = mul2(inv2, fma2(xh, less, o[e]));
                    }
                }
                if (live && head < heads) Vec8<T>::store(side.out, o0 + head * dh, x);
            }
        }
    }
    if (GRAD && side.dgamma != nullptr) {
        // the CTA's share: lanes of the same place in a head, in a fixed order
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float a, b;
            upk2(dgamma[e], a, b);
            lines[threadIdx.x * 8 + 2 * e] = a;
            lines[threadIdx.x * 8 + 2 * e + 1] = b;
        }
        __syncthreads();
        if (int(threadIdx.x) < dh) {
            float sum = 0.f;
            for (int w = 0; w < kRopeThreads / 32; ++w)
                for (int g = 0; g < per_warp; ++g) sum += lines[w * 256 + g * dh + threadIdx.x];
            p.partial[(int64_t(blockIdx.y) * gridDim.x + blockIdx.x) * dh + threadIdx.x] = sum;
        }
    }
}

// gamma's gradient from the CTAs' shares: blockIdx.x 8 channels, blockIdx.y queries or keys; thread = (channel, every 32nd share), the 32
// sums in order (one CTA for all channels took 15 us for the 1184 shares of a large call).
__global__ void __launch_bounds__(256) qk_rope_gamma_kernel(const RopeParams p, int blocks) {
    __shared__ float sums[256];
    const RopeSide& s = blockIdx.y == 0 ? p.q : p.k;
    griddep_wait();                                // the shares; no CTA ends before the kernel in front has
    if (s.dgamma == nullptr) return;
    const int c = blockIdx.x * 8 + (threadIdx.x & 7), way = threadIdx.x >> 3;
    const float* from = p.partial + int64_t(blockIdx.y) * blocks * p.dh + c;
    float sum = 0.f;
#pragma unroll 8
    for (int b = way; b < blocks; b += 32) sum += ld_dependent(from + int64_t(b) * p.dh);
    sums[threadIdx.x] = sum;
    __syncthreads();
    if (threadIdx.x < 8) {
        float total = 0.f;
#pragma unroll
        for (int w = 0; w < 32; ++w) total += sums[w * 8 + threadIdx.x];
        s.dgamma[c] = total;
    }
}

template <typename T, bool GRAD, int V>
hq_status launch_pairs(const RopeParams& p, int pairs, bool vec, dim3 grid, cudaStream_t st) {
    if (pairs == kInterleaved) {
        if (vec) qk_rope_kernel<T, kInterleaved, true, GRAD, V><<<grid, kRopeThreads, 0, st>>>(p);
        else qk_rope_kernel<T, kInterleaved, false, GRAD, V><<<grid, kRopeThreads, 0, st>>>(p);
    } else if (pairs == kHalvesByLane) {
        if (vec) qk_rope_kernel<T, kHalvesByLane, true, GRAD, V><<<grid, kRopeThreads, 0, st>>>(p);
        else qk_rope_kernel<T, kHalvesByLane, false, GRAD, V><<<grid, kRopeThreads, 0, st>>>(p);
    } else {
        qk_rope_kernel<T, kHalvesAny, false, GRAD, V><<<grid, kRopeThreads, 0, st>>>(p);
    }
    return cudaGetLastError() == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}
template <typename T, bool GRAD>
hq_status launch_width(const RopeParams& p, int pairs, bool vec, dim3 grid, cudaStream_t st) {
    switch (p.dh) {
        case 32: return launch_pairs<T, GRAD, 4>(p, pairs, vec, grid, st);
        case 64: return launch_pairs<T, GRAD, 8>(p, pairs, vec, grid, st);
        case 128: return launch_pairs<T, GRAD, 16>(p, pairs, vec, grid, st);
        default: return launch_pairs<T, GRAD, 0>(p, pairs, vec, grid, st);
    }
}

// A row (or several rows of few heads) for each warp, up to kRopeMaxBlocks CTAs.
int rope_blocks(int64_t rows, int heads, int kv_heads, int dh) {
    const int per_warp = 32 / (dh / 8), most = kv_heads > heads ? kv_heads : heads;
    const int64_t together = most < per_warp ? per_warp / most : 1, per_cta = (kRopeThreads / 32) * together;
    const int64_t blocks = (rows + per_cta - 1) / per_cta;
    return int(blocks < kRopeMaxBlocks ? blocks : kRopeMaxBlocks);
}

hq_status check_matrix(const void* x, int64_t ld, int heads, int dh, hq_dtype dt) {
    if (x == nullptr) return HQ_ERR_INVALID_ARG;
    if (ld < int64_t(heads) * dh) return HQ_ERR_SHAPE;
    if (!aligned16(x) || (ld * (dt == HQ_BF16 ? 2 : 4)) % 16 != 0) return HQ_ERR_ALIGNMENT;
    return HQ_OK;
}

hq_status check_call(hq_dtype dt, int64_t rows, int heads, int kv_heads, int dh, const void* cos, const void* sin, int64_t npos, int rot, float eps) {
    if (dt != HQ_F32 && dt != HQ_BF16) return HQ_ERR_INVALID_ARG;
    if (rows < 0 || heads <= 0 || kv_heads < 0 || dh <= 0 || rot < 0 || rot > dh || rot % 2 != 0) return HQ_ERR_SHAPE;
    if (dh % 8 != 0 || dh > 128 || heads > 65535 || kv_heads > 65535 || rows > 0x7fffffff) return HQ_ERR_UNSUPPORTED;
    if (rot > 0 && (cos == nullptr || sin == nullptr)) return HQ_ERR_INVALID_ARG;
    if (rot > 0 && npos <= 0) return HQ_ERR_SHAPE;
    if (!(eps >= 0.f)) return HQ_ERR_INVALID_ARG;
    return HQ_OK;
}

hq_status run(RopeParams p, hq_dtype dt, int interleaved, bool grad, cudaStream_t st) {
    if (p.rot == 0) { p.npos = 1; p.positions = nullptr; }
    if (p.npos > 0x7fffffff) p.npos = 0x7fffffff;              // rows and positions end there
    const int pairs = interleaved || p.rot == 0 ? kInterleaved : (p.rot / 2) % 8 == 0 ? kHalvesByLane : kHalvesAny;
    const int blocks = rope_blocks(p.rows, p.q.heads, p.k.heads, p.dh);
    const dim3 grid(unsigned(blocks), p.k.heads > 0 ? 2u : 1u);
    hq_status e;
    const bool vec = p.rot % 8 == 0 && aligned16(p.cos) && aligned16(p.sin);                 // every table row 16-byte aligned
    if (grad) e = dt == HQ_BF16 ? launch_width<__nv_bfloat16, true>(p, pairs, vec, grid, st) : launch_width<float, true>(p, pairs, vec, grid, st);
    else e = dt == HQ_BF16 ? launch_width<__nv_bfloat16, false>(p, pairs, vec, grid, st) : launch_width<float, false>(p, pairs, vec, grid, st);
    if (e != HQ_OK || (p.q.dgamma == nullptr && p.k.dgamma == nullptr)) return e;
    const dim3 few(unsigned(p.dh / 8), grid.y);
    return launch_dependent(qk_rope_gamma_kernel, few, 256, 0, st, dependent_launch(int64_t(few.x) * few.y), p, blocks) == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}

}  // namespace
}  // namespace hq

extern "C" hq_status hq_qk_norm_rope(const void* q, int64_t ldq, const void* k, int64_t ldk, hq_dtype xdt, int64_t rows, int heads, int kv_heads,
                                     int dh, const float* gamma_q, const float* gamma_k, float eps, const float* cos, const float* sin,
                                     int64_t npos, int rot, const int32_t* positions, int interleaved, void* q_out, int64_t ldq_out, void* k_out,
                                     int64_t ldk_out, void* stream) {
    using namespace hq;
    hq_status e = check_call(xdt, rows, heads, kv_heads, dh, cos, sin, npos, rot, eps);
    if (e != HQ_OK) return e;
    if (rows == 0) return HQ_OK;
    if ((e = check_matrix(q, ldq, heads, dh, xdt)) != HQ_OK || (e = check_matrix(q_out, ldq_out, heads, dh, xdt)) != HQ_OK) return e;
    if (kv_heads > 0 && ((e = check_matrix(k, ldk, kv_heads, dh, xdt)) != HQ_OK || (e = check_matrix(k_out, ldk_out, kv_heads, dh, xdt)) != HQ_OK)) return e;
    RopeParams p{};
    p.q = RopeSide{q, nullptr, q_out, ldq, 0, ldq_out, gamma_q, nullptr, heads};
    p.k = RopeSide{k, nullptr, k_out, ldk, 0, ldk_out, gamma_k, nullptr, kv_heads};
    p.rows = rows; p.dh = dh; p.rot = rot; p.cos = cos; p.sin = sin; p.positions = positions; p.npos = npos; p.eps = eps;
    return run(p, xdt, interleaved, false, static_cast<cudaStream_t>(stream));
}

extern "C" hq_status hq_qk_norm_rope_bwd_workspace_size(int64_t rows, int heads, int kv_heads, int dh, size_t* bytes) {
    using namespace hq;
    if (bytes == nullptr) return HQ_ERR_INVALID_ARG;
    const hq_status e = check_call(HQ_BF16, rows, heads, kv_heads, dh, nullptr, nullptr, 1, 0, 0.f);
    if (e != HQ_OK) return e;
    *bytes = size_t(2) * rope_blocks(rows, heads, kv_heads, dh) * dh * sizeof(float);
    return HQ_OK;
}

extern "C" hq_status hq_qk_norm_rope_bwd(const void* q, int64_t ldq, const void* k, int64_t ldk, hq_dtype xdt, int64_t rows, int heads,
                                         int kv_heads, int dh, const float* gamma_q, const float* gamma_k, float eps, const float* cos,
                                         const float* sin, int64_t npos, int rot, const int32_t* positions, int interleaved,
                                         const void* dq_out, int64_t lddq_out, const void* dk_out, int64_t lddk_out, void* dq, int64_t lddq,
                                         void* dk, int64_t lddk, float* dgamma_q, float* dgamma_k, void* workspace, size_t ws_bytes,
                                         void* stream) {
    using namespace hq;
    hq_status e = check_call(xdt, rows, heads, kv_heads, dh, cos, sin, npos, rot, eps);
    if (e != HQ_OK) return e;
    if (kv_heads == 0 && dgamma_k != nullptr) return HQ_ERR_INVALID_ARG;
    const bool sums = dgamma_q != nullptr || dgamma_k != nullptr;
    if (rows == 0) {
        cudaStream_t st = static_cast<cudaStream_t>(stream);
        if (dgamma_q != nullptr) HQ_CUDA_OK(cudaMemsetAsync(dgamma_q, 0, dh * sizeof(float), st));
        if (dgamma_k != nullptr) HQ_CUDA_OK(cudaMemsetAsync(dgamma_k, 0, dh * sizeof(float), st));
        return HQ_OK;
    }
    if ((e = check_matrix(q, ldq, heads, dh, xdt)) != HQ_OK || (e = check_matrix(dq_out, lddq_out, heads, dh, xdt)) != HQ_OK ||
        (e = check_matrix(dq, lddq, heads, dh, xdt)) != HQ_OK)
        return e;
    if (kv_heads > 0 && ((e = check_matrix(k, ldk, kv_heads, dh, xdt)) != HQ_OK || (e = check_matrix(dk_out, lddk_out, kv_heads, dh, xdt)) != HQ_OK ||
                         (e = check_matrix(dk, lddk, kv_heads, dh, xdt)) != HQ_OK))
        return e;
    if (sums) {
        size_t need = 0;
        if (workspace == nullptr) return HQ_ERR_INVALID_ARG;
        if ((reinterpret_cast<uintptr_t>(workspace) & 3u) != 0) return HQ_ERR_ALIGNMENT;
        hq_qk_norm_rope_bwd_workspace_size(rows, heads, kv_heads, dh, &need);
        if (ws_bytes < need) return HQ_ERR_WORKSPACE;
    }
    RopeParams p{};
    p.q = RopeSide{q, dq_out, dq, ldq, lddq_out, lddq, gamma_q, dgamma_q, heads};
    p.k = RopeSide{k, dk_out, dk, ldk, lddk_out, lddk, gamma_k, dgamma_k, kv_heads};
    p.rows = rows; p.dh = dh; p.rot = rot; p.cos = cos; p.sin = sin; p.positions = positions; p.npos = npos; p.eps = eps;
    p.partial = static_cast<float*>(workspace);
    return run(p, xdt, interleaved, true, static_cast<cudaStream_t>(stream));
}
