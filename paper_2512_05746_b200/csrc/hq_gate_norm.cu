// The gated residual of a transformer block with the norms before and after it, and its gradient: what stands between one block's last
// linear and the next one's first.
//
//   t = h, or norm(h) * post_weight               norm: LayerNorm (mean, biased variance) or RMS, over the cols values of a row
//   x' = residual * x + gate[n] * t               n = row / group: a sample's vectors
//   y = norm(x') * (plus + weight[n]) + bias[n]
//
// Gradient, with g = dy (plus + weight), xh = (x' - mean) / std, hh = (h - post mean) / post std from the forward call's statistics:
//   d = dx' + (g - mean(g) - xh mean(g xh)) / std           (mean(g): LayerNorm only)
//   dx = residual d,  dh = gate d, or (u - mean(u) - hh mean(u hh)) / post std with u = gate d post_weight
//   dgate[n] = sum d t,  dweight[n] = sum dy xh,  dbias[n] = sum dy,  dpost_weight = sum gate d hh over all rows
//
// Memory-bound: every row is read and written once, the vectors come from the caches once for a run of rows.  A team of ceil(cols / 256)
// warps, a CTA of its own, takes a run of rows, 8 columns a thread (up to 128 columns: two or four rows side by side in a warp).  Rows are copied ahead into shared memory, by each thread for itself (no barrier stands
// between the copy and its use, and no register holds what is on the way); two rows are computed together, so that their sums share the
// shuffles; sums over rows stay in the registers of the thread that owns the columns.
//
// 65536 x 1152 bf16 105 us a call (5.8 TB/s, 90 % of the copy rate), 8192 x 1152 18.4 (64 %: about 4 us of start, then instructions: 54 to 62 % of
// the issue slots at 20 warps an SM), 65536 x 512 of an fp32 stream and a bf16 branch with a norm behind it 88 (71 %: two chains of sums a batch).
#include "hq_gate_norm.cuh"

namespace hq {
namespace {

// S: type of x and x', B: of h and y.
template <typename S, typename B, bool POST, int L>
__global__ void __maxnreg__(96) gate_norm_kernel(const GateNormParams p) {
    extern __shared__ uint4 ring[];
    __shared__ float2 room[2 * 32];
    constexpr int kStages = kForwardStages;
    Team<L> t = team_of<L>(p, room);
    constexpr int kSide = Team<L>::kSide;
    const uint32_t r0 = blockIdx.x * p.chunk, r1 = min(r0 + p.chunk, p.rows);
    constexpr uint32_t batch = kPlane * kForwardPlanes<S, B>, h_at = kPlane * kRows * kPlanes<S>;
    const uint32_t base = smem_u32(ring) + uint32_t(t.warp) * kStages * batch, lane = uint32_t(t.lane) * 16u;
    const Pieces<S, L> wide(t);
    const Pieces<B, L> narrow(t);
    const bool branch = p.h.p != nullptr, normed = p.y.p != nullptr;
    const char *x = copied(p.x, wide.first), *h = copied(p.h, narrow.first);
    char *x_out = columns<S>(p.x_out, t), *y = columns<B>(p.y, t);
    typename Team<L>::Walk b, ahead;
    b.start(p, r0, r1);
    ahead = b;
    uint32_t to = base;
    auto send_next = [&]() {
        if (ahead.n > 0) {
            send(to, x, p.x.ld, ahead, t, wide);
            if (branch) send(to + h_at, h, p.h.ld, ahead, t, narrow);
            const uint32_t g = ahead.g;
            ahead.next(p, r1);
            if (ahead.g != g && ahead.n > 0) {
                ask_for_vector(p.gate, ahead.g, t);
                ask_for_vector(p.weight, ahead.g, t);
                ask_for_vector(p.bias, ahead.g, t);
            }
        }
        copies_sent();
        to = to == base + (kStages - 1) * batch ? base : to + batch;
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) send_next();
    f32x2 gate[4], weight[4], bias[4];             // gate: times post_weight
    uint32_t loaded = 0xffffffffu, at = base;
    while (b.n > 0) {
        if (b.g != loaded) {
            load_vector(gate, p.gate, b.g, t, 0.f, 1.f);
            if (POST) times_vector(gate, p.post_weight, t);
            if (normed) {
                load_vector(weight, p.weight, b.g, t, p.plus, 1.f);
                load_vector(bias, p.bias, b.g, t, 0.f, 0.f);
            }
            loaded = b.g;
        }
        copies_wait<kStages - 2>();
        if (b.live == 0) {                         // nothing but zeros to write
            put_zeros<S>(x_out, p.x_out, b, t);
            put_zeros<B>(y, p.y, b, t);
            if (p.stats != nullptr && threadIdx.x < unsigned(b.n)) reinterpret_cast<float4*>(p.stats)[b.row + threadIdx.x] = make_float4(0.f, 0.f, 0.f, 0.f);
            send_next();
            at = at == base + (kStages - 1) * batch ? base : at + batch;
            b.next(p, r1);
            continue;
        }
        f32x2 v[kRows][4];
#pragma unroll
        for (int i = 0; i < kRows; ++i) take<S>(v[i], at + lane, i);
        float mean[kRows] = {0.f, 0.f}, inv[kRows] = {1.f, 1.f}, post_mean[kRows] = {0.f, 0.f}, post_inv[kRows] = {1.f, 1.f};
        if (branch) {
            f32x2 u[kRows][4];
#pragma unroll
            for (int i = 0; i < kRows; ++i) take<B>(u[i], at + h_at + lane, i);
            if (POST) moments(t, u, p.post_layer, p.eps, post_mean, post_inv);
            const f32x2 residual = pk2(p.residual, p.residual);
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const f32x2 less = pk2(-post_mean[i], -post_mean[i]), s = pk2(post_inv[i], post_inv[i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (POST) u[i][e] = mul2(add2(u[i][e], less), s);
                    v[i][e] = fma2(residual, v[i][e], mul2(gate[e], u[i][e]));
                }
            }
        }
        send_next();                               // into the place of the batch before this one
        at = at == base + (kStages - 1) * batch ? base : at + batch;
        if (p.x_out.p != nullptr) {
            clear_dead(b, t, v);
            put<S>(x_out, p.x_out.ld, b, t, v);
        }
        if (normed) {
            moments(t, v, p.layer, p.eps, mean, inv);
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const f32x2 less = pk2(-mean[i], -mean[i]), s = pk2(inv[i], inv[i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[i][e] = fma2(mul2(add2(v[i][e], less), s), weight[e], bias[e]);
            }
            clear_dead(b, t, v);
            put<B>(y, p.y.ld, b, t, v);
        }
        if (p.stats != nullptr && t.c0 == 0) {
#pragma unroll
            for (int i = 0; i < kRows; ++i)
                if (i * kSide + t.side < b.n)
                    reinterpret_cast<float4*>(p.stats)[b.row + i * kSide + t.side] = i * kSide + t.side < b.live ? make_float4(mean[i], inv[i], post_mean[i], post_inv[i])
                                                                               : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        b.next(p, r1);
    }
}

template <typename S, typename B, int L>
cudaError_t launch_forward(const GateNormParams& p, bool post, Launch l, cudaStream_t st) {
    return launch_kernel(post ? gate_norm_kernel<S, B, true, L> : gate_norm_kernel<S, B, false, L>, p, l, kForwardPlanes<S, B>, kForwardStages, st);
}
template <typename S, typename B>
cudaError_t launch_forward(const GateNormParams& p, bool post, Launch l, cudaStream_t st) {
    switch (row_lanes(p.cols)) {
        case 8: return launch_forward<S, B, 8>(p, post, l, st);
        case 16: return launch_forward<S, B, 16>(p, post, l, st);
        default: return launch_forward<S, B, 32>(p, post, l, st);
    }
}

}  // namespace
}  // namespace hq

extern "C" hq_status hq_gate_norm(const void* x, int64_t ldx, hq_dtype xdt, const void* h, int64_t ldh, hq_dtype hdt, int64_t rows, int64_t cols,
                                  int64_t rows_per_group, const int32_t* lens, hq_norm post, const float* post_weight, const float* gate,
                                  int64_t ld_gate, float residual_scale, hq_norm norm, const float* weight, int64_t ld_weight, const float* bias,
                                  int64_t ld_bias, float weight_plus, float eps, void* x_out, int64_t ldx_out, void* y, int64_t ldy, float* stats,
                                  void* stream) {
    using namespace hq;
    int64_t group = 0;
    hq_status e = check_sizes(xdt, hdt, rows, cols, rows_per_group, lens, post, post_weight, norm, h, gate, residual_scale, &group);
    if (e != HQ_OK) return e;
    if (!(eps >= 0.f) || !(weight_plus - weight_plus == 0.f)) return HQ_ERR_INVALID_ARG;
    if ((y == nullptr) != (norm == HQ_NORM_NONE) || (y == nullptr && (weight != nullptr || bias != nullptr)) || (y == nullptr && x_out == nullptr))
        return HQ_ERR_INVALID_ARG;
    if (rows == 0) return HQ_OK;
    const int64_t groups = (rows + group - 1) / group;
    if ((e = check_matrix(x, ldx, cols, xdt)) != HQ_OK || (h != nullptr && (e = check_matrix(h, ldh, cols, hdt)) != HQ_OK) ||
        (x_out != nullptr && (e = check_matrix(x_out, ldx_out, cols, xdt)) != HQ_OK) || (y != nullptr && (e = check_matrix(y, ldy, cols, hdt)) != HQ_OK) ||
        (e = check_vectors(gate, ld_gate, groups, cols)) != HQ_OK || (e = check_vectors(weight, ld_weight, groups, cols)) != HQ_OK ||
        (e = check_vectors(bias, ld_bias, groups, cols)) != HQ_OK)
        return e;
    if (in_place_apart(x_out, ldx_out, x, ldx, rows) || in_place_apart(y, ldy, h, ldh, rows)) return HQ_ERR_SHAPE;
    if (!aligned16(stats)) return HQ_ERR_ALIGNMENT;
    GateNormParams p{};
    p.rows = uint32_t(rows); p.group = uint32_t(group); p.cols = int(cols); p.warps = team_warps(cols); p.lens = lens;
    p.layer = norm == HQ_NORM_LAYER; p.post_layer = post == HQ_NORM_LAYER; p.post_weight = post_weight;
    p.gate = Vectors{gate, ld_gate}; p.weight = Vectors{weight, ld_weight}; p.bias = Vectors{bias, ld_bias};
    p.residual = residual_scale; p.plus = weight_plus; p.eps = eps; p.stats = stats;
    p.x = matrix(x, ldx, xdt); p.h = matrix(h, ldh, hdt); p.x_out = matrix_out(x_out, ldx_out, xdt); p.y = matrix_out(y, ldy, hdt);
    // teams at a time: 96 registers leave room for 20 warps an SM, the rows on their way for as many as share 224 KB
    const int planes = kRows * ((xdt == HQ_BF16 ? 1 : 2) + (hdt == HQ_BF16 ? 1 : 2)), side = 32 / row_lanes(cols);
    const int64_t fit = int64_t(kMostShared / (size_t(planes) * kForwardStages * p.warps * 32 * 16)), by_warps = 20 / p.warps;
    const int64_t most = int64_t(sm_count()) * (fit < by_warps ? fit : by_warps);
    // runs of a dozen rows, in up to four turns of all teams: what is under way lies closer together than in one turn of long runs (one, two and
    // four turns, LayerNorm in front alone: 65536 rows of 1152 bf16 115, 107 and 111 us, 131072 of 256 57, 52 and 49, 300000 of 128 fp32 109, 106
    // and 97; RMS on both sides, 65536 of 512 fp32 97, 90 and 89).  One turn where both norms take means: a run is bound by its instructions, and
    // each run's start is felt (29491 x 1280 bf16 64, 68 and 74, 16384 x 2304 72, 73 and 76; not narrow rows: 300000 x 128 68, 62 and 63).
    // The rule is a coarse one: a LayerNorm beside an RMS norm in bf16 would be better off with one turn from 512 columns on, too (29491 x 1280
    // 60, 64 and 68; 65536 x 512 54, 59 and 59).
    const int64_t one = (rows + most - 1) / most, turns = one / (12 * side), limit = norm == HQ_NORM_LAYER && post == HQ_NORM_LAYER ? 1 : 4;
    const int64_t teams = most * (turns < 1 ? 1 : turns > limit ? limit : turns), chunk = (rows + teams - 1) / teams;
    p.chunk = uint32_t(chunk < kRows * side ? kRows * side : chunk);
    const Launch l{unsigned((rows + p.chunk - 1) / p.chunk), unsigned(p.warps * 32)};
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool after = post != HQ_NORM_NONE;
    cudaError_t c;
    if (xdt == HQ_BF16) c = hdt == HQ_BF16 ? launch_forward<__nv_bfloat16, __nv_bfloat16>(p, after, l, st) : launch_forward<__nv_bfloat16, float>(p, after, l, st);
    else c = hdt == HQ_BF16 ? launch_forward<float, __nv_bfloat16>(p, after, l, st) : launch_forward<float, float>(p, after, l, st);
    return c == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}
