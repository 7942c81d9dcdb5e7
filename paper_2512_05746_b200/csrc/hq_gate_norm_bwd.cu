// The gradient of the gated residual with its norms; its formulas stand in hq_gate_norm.cu.
//
// One pass over x', h and the gradients of both outputs, 12 bytes an element of bf16; sums over rows in registers, a part for each team that
// took rows of a group, joined by a second kernel in a fixed order.
//
// 65536 x 1152 bf16 152 to 165 us a call (5.5 to 6.0 TB/s, 86 to 93 % of the copy rate), 8192 x 1152 28 (62 %: 24 here at 15 warps an SM and 55 % of the issue slots, the
// rest the join of 14 parts a group).
#include "hq_gate_norm.cuh"

namespace hq {
namespace {

// Where a group ends (and behind a team's last row) its sums leave: to the gradient itself where the whole group was this team's, else to the
// team's part (the first of its two for the group of its first row, else the second), which gate_norm_sums_kernel joins.
template <typename S, typename B, bool POST, int L, int kStages>
__global__ void __maxnreg__(128) gate_norm_grad_kernel(const GateNormParams p) {
    extern __shared__ uint4 ring[];
    __shared__ float2 room[2 * 32];
    __shared__ float4 moments_in[kStages][kMaxWarps][Team<L>::kBatch];         // the statistics on their way: each warp copies its own
    Team<L> t = team_of<L>(p, room);
    constexpr int kSide = Team<L>::kSide;
    const uint32_t team = blockIdx.x, r0 = team * p.chunk, r1 = min(r0 + p.chunk, p.rows);
    griddep_launch();                              // all teams are at work at once: the joining kernel takes no place of theirs
    constexpr uint32_t batch = kPlane * kGradPlanes<S, B>, s_size = kPlane * kRows * kPlanes<S>, b_size = kPlane * kRows * kPlanes<B>;
    constexpr uint32_t y_at = s_size, d_at = s_size + b_size, h_at = 2 * s_size + b_size;
    const uint32_t base = smem_u32(ring) + uint32_t(t.warp) * kStages * batch, lane = uint32_t(t.lane) * 16u;
    const Pieces<S, L> wide(t);
    const Pieces<B, L> narrow(t);
    const bool normed = p.dy.p != nullptr, gated = p.dgate.p != nullptr, later = p.dx_out.p != nullptr, branch = POST || gated;       // h itself is read
    const char *x = copied(p.x, wide.first), *dy = copied(p.dy, narrow.first), *dx_out = copied(p.dx_out, wide.first), *h = copied(p.h, narrow.first);
    char *dx = columns<S>(p.dx, t), *dh = columns<B>(p.dh, t);
    typename Team<L>::Walk b, ahead;
    b.start(p, r0, r1);
    ahead = b;
    uint32_t to = base, at = base;
    int slot = 0, now = 0;                         // of the statistics: to send to, to take from
    auto send_next = [&]() {
        if (ahead.n > 0) {
            if (normed) { send(to, x, p.x.ld, ahead, t, wide); send(to + y_at, dy, p.dy.ld, ahead, t, narrow); }
            if (later) send(to + d_at, dx_out, p.dx_out.ld, ahead, t, wide);
            if (branch) send(to + h_at, h, p.h.ld, ahead, t, narrow);
            if ((normed || POST) && t.lane < Team<L>::kBatch)
                copy_bytes(smem_u32(&moments_in[slot][t.warp][t.lane]), p.stats + 4 * (int64_t(ahead.row) + (t.lane < ahead.live ? t.lane : 0)), t.lane < ahead.live ? 16u : 0u);
            const uint32_t g = ahead.g;
            ahead.next(p, r1);
            if (ahead.g != g && ahead.n > 0) {
                ask_for_vector(p.gate, ahead.g, t);
                ask_for_vector(p.weight, ahead.g, t);
            }
        }
        slot = slot == kStages - 1 ? 0 : slot + 1;
        copies_sent();
        to = to == base + (kStages - 1) * batch ? base : to + batch;
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) send_next();
    f32x2 dpost[4], gate[4], weight[4], dweight[4], dbias[4], dgate[4];
    fill(dpost, 0.f);
    bool fresh = true, begun = b.g * p.group == r0;            // begun: the group's first row is this team's
    bool lived = false;                            // the group has rows here: the vectors of one without any may hold anything
    while (b.n > 0) {
        if (fresh) {
            load_vector(gate, p.gate, b.g, t, 0.f, 1.f);       // with a norm behind the block: times post_weight
            if (POST) times_vector(gate, p.post_weight, t);
            load_vector(weight, p.weight, b.g, t, p.plus, 1.f);
            fill(dweight, 0.f); fill(dbias, 0.f); fill(dgate, 0.f);
            fresh = false;
        }
        __syncwarp();                              // no lane of the warp still reads the batch before this one
        send_next();                               // into its place
        copies_wait<kStages - 1>();
        float4 stats[kRows];                       // zeros for rows that are not there
#pragma unroll
        for (int i = 0; i < kRows; ++i) stats[i] = normed || POST ? moments_in[now][t.warp][i * kSide + t.side] : make_float4(0.f, 0.f, 0.f, 0.f);
        now = now == kStages - 1 ? 0 : now + 1;
        if (b.live == 0) {                         // nothing but zeros to write
            put_zeros<S>(dx, p.dx, b, t);
            put_zeros<B>(dh, p.dh, b, t);
        } else {
            lived = true;
            f32x2 d[kRows][4];
            if (normed) {
                f32x2 xh[kRows][4];
                float2 s[kRows];
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    const f32x2 less = pk2(-stats[i].x, -stats[i].x), inv = pk2(stats[i].y, stats[i].y);
                    f32x2 a = pk2(0.f, 0.f), c = pk2(0.f, 0.f);
                    take<S>(xh[i], at + lane, i);
                    take<B>(d[i], at + y_at + lane, i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        xh[i][e] = mul2(add2(xh[i][e], less), inv);
                        dbias[e] = add2(dbias[e], d[i][e]);
                        dweight[e] = fma2(d[i][e], xh[i][e], dweight[e]);
                        d[i][e] = mul2(d[i][e], weight[e]);
                        a = add2(a, d[i][e]);
                        c = fma2(d[i][e], xh[i][e], c);
                    }
                    s[i] = t.col ? make_float2(pair_sum(a), pair_sum(c)) : make_float2(0.f, 0.f);
                }
                team_sums(t, s[0], s[1]);
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    const float mg = p.layer ? -s[i].x * t.per_row : 0.f, mx = -s[i].y * t.per_row;
                    const f32x2 inv = pk2(stats[i].y, stats[i].y), g2 = pk2(mg, mg), x2 = pk2(mx, mx);
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[i][e] = mul2(inv, fma2(xh[i][e], x2, add2(d[i][e], g2)));
                }
            } else {
#pragma unroll
                for (int i = 0; i < kRows; ++i) fill(d[i], 0.f);
            }
            if (later) {
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    f32x2 o[4];
                    take<S>(o, at + d_at + lane, i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[i][e] = add2(d[i][e], o[e]);
                }
            }
            if (p.dx.p != nullptr) {
                const f32x2 residual = pk2(p.residual, p.residual);
                f32x2 o[kRows][4];
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[i][e] = mul2(residual, d[i][e]);
                }
                clear_dead(b, t, o);
                put<S>(dx, p.dx.ld, b, t, o);
            }
            if (POST) {
                f32x2 hh[kRows][4];
                float2 s[kRows];
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    const f32x2 less = pk2(-stats[i].z, -stats[i].z), inv = pk2(stats[i].w, stats[i].w);
                    f32x2 a = pk2(0.f, 0.f), c = pk2(0.f, 0.f);
                    take<B>(hh[i], at + h_at + lane, i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        hh[i][e] = mul2(add2(hh[i][e], less), inv);
                        dgate[e] = fma2(d[i][e], hh[i][e], dgate[e]);              // both sums' part: dgate is post_weight times it, dpost gate times it
                        d[i][e] = mul2(d[i][e], gate[e]);
                        a = add2(a, d[i][e]);
                        c = fma2(d[i][e], hh[i][e], c);
                    }
                    s[i] = t.col ? make_float2(pair_sum(a), pair_sum(c)) : make_float2(0.f, 0.f);
                }
                if (p.dh.p != nullptr) {
                    team_sums(t, s[0], s[1]);
#pragma unroll
                    for (int i = 0; i < kRows; ++i) {
                        const float mg = p.post_layer ? -s[i].x * t.per_row : 0.f, mx = -s[i].y * t.per_row;
                        const f32x2 inv = pk2(stats[i].w, stats[i].w), g2 = pk2(mg, mg), x2 = pk2(mx, mx);
#pragma unroll
                        for (int e = 0; e < 4; ++e) d[i][e] = mul2(inv, fma2(hh[i][e], x2, add2(d[i][e], g2)));
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    f32x2 o[4];
                    if (gated) take<B>(o, at + h_at + lane, i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (gated) dgate[e] = fma2(d[i][e], o[e], dgate[e]);
                        d[i][e] = mul2(d[i][e], gate[e]);
                    }
                }
            }
            if (p.dh.p != nullptr) {
                clear_dead(b, t, d);
                put<B>(dh, p.dh.ld, b, t, d);
            }
        }
        at = at == base + (kStages - 1) * batch ? base : at + batch;
        const uint32_t g = b.g, done = b.row + uint32_t(b.n);
        const bool over = b.left == b.n;           // the group's last row
        b.next(p, r1);
        if (!over && done < r1) continue;
        fresh = true;                              // the group's sums leave
        const bool whole = begun && over, first = g * p.group <= r0;
        begun = true;
        const bool counts = lived;
        lived = false;
        if constexpr (L < 32) {                    // of the rows side by side
            side_sums<L>(dweight);
            side_sums<L>(dbias);
            side_sums<L>(dgate);
        }
        if (!t.col || t.side > 0) continue;
        if (POST && counts) {
            load_vector(gate, p.gate, g, t, 0.f, 1.f);
#pragma unroll
            for (int e = 0; e < 4; ++e) dpost[e] = fma2(gate[e], dgate[e], dpost[e]);
        }
        if (whole) {
            if (POST && gated) times_vector(dgate, p.post_weight, t);
            if (p.dweight.p != nullptr) Vec8<float>::store_wide(p.dweight.p, int64_t(g) * p.dweight.ld + t.c0, dweight);
            if (p.dbias.p != nullptr) Vec8<float>::store_wide(p.dbias.p, int64_t(g) * p.dbias.ld + t.c0, dbias);
            if (gated) Vec8<float>::store_wide(p.dgate.p, int64_t(g) * p.dgate.ld + t.c0, dgate);
        } else if (p.parts != nullptr) {
            const int64_t part = (int64_t(team) * 2 + (first ? 0 : 1)) * 3 * p.cols + t.c0;
            if (p.dweight.p != nullptr) Vec8<float>::store_wide(p.parts, part, dweight);
            if (p.dbias.p != nullptr) Vec8<float>::store_wide(p.parts, part + p.cols, dbias);
            if (gated) Vec8<float>::store_wide(p.parts, part + 2 * p.cols, dgate);
        }
    }
    if (POST && p.dpost != nullptr && t.col && t.side == 0) Vec8<float>::store_wide(p.post_parts, int64_t(team) * p.cols + t.c0, dpost);
}

// The parts of groups that several teams took, joined in order, and dpost_weight's.  blockIdx.x: heads x `wide` columns of a group (head: the
// group itself, or, where there are more groups than teams, the group at a border of two teams' rows, which the first border inside it takes),
// then the columns of dpost_weight.  Thread = (4 columns, every 1024 / wide'th part).
struct Joins { uint32_t teams, heads, group_ctas, post_ctas; int wide, post_wide, by_group; };         // CTAs: of a head, of dpost_weight
// One value of each of four parts in one statement: as loads of their own the compiler puts each sum behind its load.
__device__ __forceinline__ void ld_four(float4 (&x)[4], const float4* const (&from)[4]) {
#define HQ_OUT4(u) "=f"(x[u].x), "=f"(x[u].y), "=f"(x[u].z), "=f"(x[u].w)
    asm volatile("ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%16];\n\tld.global.cg.v4.f32 {%4, %5, %6, %7}, [%17];\n\t"
                 "ld.global.cg.v4.f32 {%8, %9, %10, %11}, [%18];\n\tld.global.cg.v4.f32 {%12, %13, %14, %15}, [%19];"
                 : HQ_OUT4(0), HQ_OUT4(1), HQ_OUT4(2), HQ_OUT4(3) : "l"(from[0]), "l"(from[1]), "l"(from[2]), "l"(from[3]) : "memory");
#undef HQ_OUT4
}
__device__ __forceinline__ float4 plus(float4 a, float4 b) { return make_float4(a.x + b.x, a.y + b.y, a.z + b.z, a.w + b.w); }
__global__ void __launch_bounds__(256) gate_norm_sums_kernel(const GateNormParams p, const Joins j) {
    __shared__ float4 sums[3][256];
    const uint32_t head = blockIdx.x / j.group_ctas;
    const bool post = head >= j.heads;
    const int wide = post ? j.post_wide : j.wide, lanes = wide / 4, ways = 256 / lanes, way = int(threadIdx.x) / lanes, mine = int(threadIdx.x) - way * lanes;
    const int c = int(blockIdx.x - (post ? j.heads : head) * j.group_ctas) * wide + mine * 4;
    uint32_t g = 0, from = 0, to = j.teams - 1;
    bool second = false;
    if (!post) {
        g = j.by_group ? head : (head + 1) * p.chunk / p.group;
        const uint32_t first = g * p.group, last = (p.rows - first > p.group ? first + p.group : p.rows) - 1;
        from = first / p.chunk;
        to = last / p.chunk;
        if (from == to || (!j.by_group && from != head)) return;
        second = first != from * p.chunk;          // the group is not the one of that team's first row
    }
    const bool want0 = post || p.dweight.p != nullptr, want1 = !post && p.dbias.p != nullptr, want2 = !post && p.dgate.p != nullptr;
    float4 sum0 = make_float4(0.f, 0.f, 0.f, 0.f), sum1 = sum0, sum2 = sum0;
    griddep_wait();                                // the parts; no CTA that writes ends before the kernel in front has
    if (c < p.cols) {
        const float* parts = post ? p.post_parts + c : p.parts + c;
        const int64_t step = post ? p.cols : int64_t(6) * p.cols;
        if (post) {                                // many parts: four at a time; of one behind the last the last one is read and not added
            for (uint32_t i = from + way; i <= to; i += 4 * ways) {
                const float4* part[4];
                float4 x[4];
#pragma unroll
                for (int u = 0; u < 4; ++u) part[u] = reinterpret_cast<const float4*>(parts + min(i + u * ways, to) * step);
                ld_four(x, part);
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    if (i + u * ways <= to) sum0 = plus(sum0, x[u]);
            }
        } else {
#pragma unroll 2
            for (uint32_t i = from + way; i <= to; i += ways) {
                const float4* part = reinterpret_cast<const float4*>(parts + i * step + (second && i == from ? 3 * p.cols : 0));
                if (want0) sum0 = plus(sum0, ld_dependent_cg(part));
                if (want1) sum1 = plus(sum1, ld_dependent_cg(part + p.cols / 4));
                if (want2) sum2 = plus(sum2, ld_dependent_cg(part + p.cols / 2));
            }
        }
    }
    sums[0][threadIdx.x] = sum0; sums[1][threadIdx.x] = sum1; sums[2][threadIdx.x] = sum2;
    __syncthreads();
    for (int k = way; k < 3; k += ways) {          // thread = (4 columns, sum): the ways in order
        if (c >= p.cols || !(k == 0 ? want0 : k == 1 ? want1 : want2)) continue;
        float4 s = sums[k][mine];
        for (int w = 1; w < ways; ++w) s = plus(s, sums[k][w * lanes + mine]);
        if (k == 2 && p.post_weight != nullptr) {
            const float4 v = *reinterpret_cast<const float4*>(p.post_weight + c);
            s = make_float4(s.x * v.x, s.y * v.y, s.z * v.z, s.w * v.w);
        }
        float* out = post ? p.dpost : k == 0 ? p.dweight.p + g * p.dweight.ld : k == 1 ? p.dbias.p + g * p.dbias.ld : p.dgate.p + g * p.dgate.ld;
        *reinterpret_cast<float4*>(out + c) = s;
    }
}

constexpr int kGradWarps = 148 * 15;               // warps at a time, on every device: gradients are summed in one order
int64_t least_chunk(int64_t cols) { return 2 * kRows * (32 / row_lanes(cols)); }
int64_t grad_chunk(int64_t rows, int64_t cols) {
    const int64_t teams = kGradWarps / team_warps(cols), chunk = (rows + teams - 1) / teams, least = least_chunk(cols);
    return chunk < least ? least : chunk;
}
// Teams of a call of at most so many rows: fewer rows may make more teams, as a chunk is a whole number of rows (of 1152 columns 8192 rows make
// 432, 7992 rows 444).
int64_t most_teams(int64_t rows, int64_t cols) {
    const int64_t teams = kGradWarps / team_warps(cols), least = least_chunk(cols), few = (rows + least - 1) / least;
    return few < teams ? few : teams;
}
size_t parts_bytes(int64_t teams, int64_t cols) { return size_t(teams) * 7 * size_t(cols) * sizeof(float); }
template <typename S, typename B, int L>
cudaError_t launch_grad(const GateNormParams& p, bool post, Launch l, cudaStream_t st) {
    if constexpr (sizeof(S) + sizeof(B) == 8 && L == 32) {     // the widest rows of fp32 on both sides: 256 KB in two stages
        if (size_t(kGradPlanes<S, B>) * kGradStages * l.threads * 16 > kMostShared)
            return launch_kernel(post ? gate_norm_grad_kernel<S, B, true, L, 1> : gate_norm_grad_kernel<S, B, false, L, 1>, p, l, kGradPlanes<S, B>, 1, st);
    }
    return launch_kernel(post ? gate_norm_grad_kernel<S, B, true, L, kGradStages> : gate_norm_grad_kernel<S, B, false, L, kGradStages>, p, l, kGradPlanes<S, B>,
                         kGradStages, st);
}
template <typename S, typename B>
cudaError_t launch_grad(const GateNormParams& p, bool post, Launch l, cudaStream_t st) {
    switch (row_lanes(p.cols)) {
        case 8: return launch_grad<S, B, 8>(p, post, l, st);
        case 16: return launch_grad<S, B, 16>(p, post, l, st);
        default: return launch_grad<S, B, 32>(p, post, l, st);
    }
}

}  // namespace
}  // namespace hq

extern "C" hq_status hq_gate_norm_bwd_workspace_size(int64_t rows, int64_t cols, int64_t rows_per_group, size_t* bytes) {
    using namespace hq;
    if (bytes == nullptr) return HQ_ERR_INVALID_ARG;
    int64_t group = 0;
    const hq_status e = check_sizes(HQ_BF16, HQ_BF16, rows, cols, rows_per_group, nullptr, HQ_NORM_NONE, nullptr, HQ_NORM_NONE, nullptr, nullptr, 1.f, &group);
    if (e != HQ_OK) return e;
    *bytes = parts_bytes(most_teams(rows, cols), cols);
    return HQ_OK;
}

extern "C" hq_status hq_gate_norm_bwd(const void* x_out, int64_t ldx_out, hq_dtype xdt, const void* h, int64_t ldh, hq_dtype hdt, const float* stats,
                                      int64_t rows, int64_t cols, int64_t rows_per_group, const int32_t* lens, hq_norm post,
                                      const float* post_weight, const float* gate, int64_t ld_gate, float residual_scale, hq_norm norm,
                                      const float* weight, int64_t ld_weight, float weight_plus, const void* dx_out, int64_t lddx_out, const void* dy,
                                      int64_t lddy, void* dx, int64_t lddx, void* dh, int64_t lddh, float* dpost_weight, float* dgate,
                                      int64_t ld_dgate, float* dweight, int64_t ld_dweight, float* dbias, int64_t ld_dbias, void* workspace,
                                      size_t ws_bytes, void* stream) {
    using namespace hq;
    int64_t group = 0;
    hq_status e = check_sizes(xdt, hdt, rows, cols, rows_per_group, lens, post, post_weight, norm, h, gate, residual_scale, &group);
    if (e != HQ_OK) return e;
    if (!(weight_plus - weight_plus == 0.f)) return HQ_ERR_INVALID_ARG;
    const bool normed = norm != HQ_NORM_NONE, after = post != HQ_NORM_NONE;
    if (normed != (dy != nullptr) || (!normed && (weight != nullptr || dweight != nullptr || dbias != nullptr)) || (dy == nullptr && dx_out == nullptr && rows > 0))
        return HQ_ERR_INVALID_ARG;
    if (h == nullptr && (dgate != nullptr || dh != nullptr)) return HQ_ERR_INVALID_ARG;
    if (!after && dpost_weight != nullptr) return HQ_ERR_INVALID_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0) {                               // no groups but the one vector of all rows
        for (float* v : {rows_per_group == 0 ? dgate : nullptr, rows_per_group == 0 ? dweight : nullptr, rows_per_group == 0 ? dbias : nullptr, dpost_weight})
            if (v != nullptr) HQ_CUDA_OK(cudaMemsetAsync(v, 0, size_t(cols) * sizeof(float), st));
        return HQ_OK;
    }
    const int64_t groups = (rows + group - 1) / group;
    if ((normed && ((e = check_matrix(x_out, ldx_out, cols, xdt)) != HQ_OK || (e = check_matrix(dy, lddy, cols, hdt)) != HQ_OK)) ||
        (h != nullptr && (e = check_matrix(h, ldh, cols, hdt)) != HQ_OK) || (dx_out != nullptr && (e = check_matrix(dx_out, lddx_out, cols, xdt)) != HQ_OK) ||
        (dx != nullptr && (e = check_matrix(dx, lddx, cols, xdt)) != HQ_OK) || (dh != nullptr && (e = check_matrix(dh, lddh, cols, hdt)) != HQ_OK) ||
        (e = check_vectors(gate, ld_gate, groups, cols)) != HQ_OK || (e = check_vectors(weight, ld_weight, groups, cols)) != HQ_OK ||
        (e = check_vectors(dgate, ld_dgate, groups, cols)) != HQ_OK || (e = check_vectors(dweight, ld_dweight, groups, cols)) != HQ_OK ||
        (e = check_vectors(dbias, ld_dbias, groups, cols)) != HQ_OK)
        return e;
    if (in_place_apart(dx, lddx, dx_out, lddx_out, rows) || in_place_apart(dh, lddh, dy, lddy, rows) || in_place_apart(dh, lddh, h, ldh, rows)) return HQ_ERR_SHAPE;
    if ((normed || after) && stats == nullptr) return HQ_ERR_INVALID_ARG;
    if (!aligned16(stats) || !aligned16(dpost_weight)) return HQ_ERR_ALIGNMENT;
    GateNormParams p{};
    p.rows = uint32_t(rows); p.group = uint32_t(group); p.cols = int(cols); p.warps = team_warps(cols); p.lens = lens;
    p.chunk = uint32_t(grad_chunk(rows, cols));
    const int64_t teams = (rows + p.chunk - 1) / p.chunk;
    const bool sums = dgate != nullptr || dweight != nullptr || dbias != nullptr;
    // parts are for groups that several teams took; without a sum over rows, or where every group is one team's, there are none
    const bool split = sums && p.chunk % p.group != 0 && teams > 1;
    if (split || dpost_weight != nullptr) {
        if (workspace == nullptr) return HQ_ERR_INVALID_ARG;
        if (!aligned16(workspace)) return HQ_ERR_ALIGNMENT;
        if (ws_bytes < parts_bytes(teams, cols)) return HQ_ERR_WORKSPACE;
    }
    p.layer = norm == HQ_NORM_LAYER; p.post_layer = post == HQ_NORM_LAYER; p.post_weight = post_weight;
    p.gate = Vectors{gate, ld_gate}; p.weight = Vectors{weight, ld_weight};
    p.residual = residual_scale; p.plus = weight_plus; p.stats = const_cast<float*>(stats);
    p.x = matrix(x_out, ldx_out, xdt); p.h = matrix(h, ldh, hdt); p.dx_out = matrix(dx_out, lddx_out, xdt); p.dy = matrix(dy, lddy, hdt);
    p.dx = matrix_out(dx, lddx, xdt); p.dh = matrix_out(dh, lddh, hdt);
    p.dgate = VectorsOut{dgate, ld_dgate}; p.dweight = VectorsOut{dweight, ld_dweight}; p.dbias = VectorsOut{dbias, ld_dbias};
    p.dpost = dpost_weight;
    p.parts = split ? static_cast<float*>(workspace) : nullptr;
    p.post_parts = static_cast<float*>(workspace) + size_t(teams) * 6 * cols;
    const Launch l{unsigned(teams), unsigned(p.warps * 32)};
    cudaError_t c;
    if (xdt == HQ_BF16) c = hdt == HQ_BF16 ? launch_grad<__nv_bfloat16, __nv_bfloat16>(p, after, l, st) : launch_grad<__nv_bfloat16, float>(p, after, l, st);
    else c = hdt == HQ_BF16 ? launch_grad<float, __nv_bfloat16>(p, after, l, st) : launch_grad<float, float>(p, after, l, st);
    if (c != cudaSuccess) return HQ_ERR_CUDA;
    if (!split && dpost_weight == nullptr) return HQ_OK;
    Joins j{};
    j.teams = uint32_t(teams);
    j.by_group = groups < teams;
    j.heads = !split ? 0u : uint32_t(j.by_group ? groups : teams - 1);
    // columns a CTA: as many as leave a thread two parts or more (one group of all rows, dpost_weight: 64 threads a column's parts)
    auto wide_for = [](int64_t parts) { int wide = 1024; while (wide > 16 && parts > 1024 / wide * 2) wide /= 2; return wide; };
    j.wide = wide_for(p.group / p.chunk + 2);
    j.post_wide = wide_for(teams);
    j.group_ctas = uint32_t((cols + j.wide - 1) / j.wide);
    j.post_ctas = dpost_weight != nullptr ? uint32_t((cols + j.post_wide - 1) / j.post_wide) : 0u;
    return launch_dependent(gate_norm_sums_kernel, dim3(j.heads * j.group_ctas + j.post_ctas), 256, 0, st, true, p, j) == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}
