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
// warps holds a row, 8 values a thread, so that the rows' sums are shuffles and one exchange through shared memory, and the sums over rows
// stay in the registers of the thread that owns the columns.
#include "hq_common.cuh"
#include "hq_vec8.cuh"

namespace hq {
namespace {

constexpr int kMaxCols = 4096;
constexpr int kMaxWarps = 16;
constexpr int kRows = 2;                           // rows of a team's batch

struct Matrix { const void* p; int64_t ld; };
struct MatrixOut { void* p; int64_t ld; };
struct Vectors { const float* p; int64_t ld; };    // [groups][cols]
struct VectorsOut { float* p; int64_t ld; };

struct GateNormParams {
    int64_t rows, group;                           // group: rows that share their vectors
    int64_t chunk;                                 // rows of a team (forward), of a CTA (gradient)
    int cols, warps;                               // warps of a team
    int layer, post_layer;                         // the norms' kind: 1 with a mean
    const int32_t* lens;                           // [groups] rows that are there, or NULL
    const float* post_weight;
    Vectors gate, weight, bias;
    float residual, plus, eps;
    float* stats;                                  // [rows][4]
    Matrix x, h;                                   // gradient: x is the forward call's x'
    MatrixOut x_out, y;
    Matrix dx_out, dy;
    MatrixOut dx, dh;
    VectorsOut dgate, dweight, dbias;
    float *dpost, *parts, *post_parts;             // parts: [CTAs][first, last segment][weight, bias, gate][cols]; post_parts: [CTAs][cols]
};

// Rows [row, row + n) of one group, the first `live` of them within its length.
struct Batch { int64_t row, g; int n, live; };
__device__ __forceinline__ Batch batch_at(const GateNormParams& p, int64_t row, int64_t g, int64_t end) {
    const int64_t first = g * p.group, last = min(first + p.group, end);
    Batch b{row, g, 0, 0};
    if (row < last) {
        b.n = int(min(int64_t(kRows), last - row));
        b.live = b.n;
        if (p.lens != nullptr) b.live = int(min(max(first + p.lens[g] - row, int64_t(0)), int64_t(b.n)));
    }
    return b;
}

__device__ __forceinline__ void fill(f32x2 (&v)[4], float x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pk2(x, x);
}
// A group's values for this thread's columns, plus `add`; `none` without a vector.
__device__ __forceinline__ void load_vector(f32x2 (&v)[4], const Vectors& from, int64_t g, int c0, bool col, float add, float none) {
    if (from.p == nullptr || !col) { fill(v, none); return; }
    const float4* q = reinterpret_cast<const float4*>(from.p + g * from.ld + c0);
    const float4 a = q[0], b = q[1];
    v[0] = pk2(a.x + add, a.y + add); v[1] = pk2(a.z + add, a.w + add); v[2] = pk2(b.x + add, b.y + add); v[3] = pk2(b.z + add, b.w + add);
}
__device__ __forceinline__ void store_vector(float* to, const f32x2 (&v)[4]) {
    float4 a, b;
    upk2(v[0], a.x, a.y); upk2(v[1], a.z, a.w); upk2(v[2], b.x, b.y); upk2(v[3], b.z, b.w);
    reinterpret_cast<float4*>(to)[0] = a;
    reinterpret_cast<float4*>(to)[1] = b;
}

// A thread's place: lane, warp of its team, its 8 columns; and the team's exchange of sums, two buffers in turn, so that one barrier
// stands between the writes and the reads of an exchange and none behind it.
struct Team {
    int lane, warp, warps, id, c0, cols;
    bool col;
    float2* room;                                  // [2][kRows][kMaxWarps], this team's warps first
    int turn;
    __device__ __forceinline__ void sync() const {
        if (warps > 1) asm volatile("bar.sync %0, %1;" ::"r"(id + 1), "r"(warps * 32) : "memory");
        else __syncwarp();
    }
};
__device__ __forceinline__ Team team_of(const GateNormParams& p, float2* room) {
    Team t;
    const int warp = int(threadIdx.x >> 5);
    t.lane = int(threadIdx.x & 31);
    t.warps = p.warps;
    t.id = warp / p.warps;
    t.warp = warp - t.id * p.warps;
    t.c0 = (t.warp * 32 + t.lane) * 8;
    t.cols = p.cols;
    t.col = t.c0 < p.cols;
    t.room = room + t.id * p.warps;
    t.turn = 0;
    return t;
}
__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) x += __shfl_xor_sync(0xffffffffu, x, off);
    return x;
}
__device__ __forceinline__ float sum8(const f32x2 (&v)[4]) { return pair_sum(add2(add2(v[0], v[1]), add2(v[2], v[3]))); }

// Two sums of every row over the team.
__device__ __forceinline__ void team_sums(Team& t, float2 (&s)[kRows]) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) s[i] = make_float2(warp_sum(s[i].x), warp_sum(s[i].y));
    if (t.warps == 1) return;
    float2* room = t.room + t.turn * kRows * kMaxWarps;
    t.turn ^= 1;
    if (t.lane == 0) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) room[i * kMaxWarps + t.warp] = s[i];
    }
    t.sync();
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        float2 a = make_float2(0.f, 0.f);
        for (int w = 0; w < t.warps; ++w) {
            const float2 o = room[i * kMaxWarps + w];
            a.x += o.x; a.y += o.y;
        }
        s[i] = a;
    }
}

// Mean (0 unless `layer`) and 1 / standard deviation of every row.  A warp takes the mean of its own values first and its squares about
// that, and the warps' parts are joined about the row's mean: no difference of large sums, and one exchange.
__device__ __forceinline__ void moments(Team& t, const f32x2 (&v)[kRows][4], int layer, float eps, float (&mean)[kRows], float (&inv)[kRows]) {
    const float mine = float(min(256, t.cols - t.warp * 256)), all = float(t.cols);
    float q[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) mean[i] = layer ? warp_sum(t.col ? sum8(v[i]) : 0.f) / mine : 0.f;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const f32x2 m = pk2(-mean[i], -mean[i]);
        f32x2 sq = pk2(0.f, 0.f);
#pragma unroll
        for (int e = 0; e < 4; ++e) { const f32x2 d = add2(v[i][e], m); sq = fma2(d, d, sq); }
        q[i] = warp_sum(t.col ? pair_sum(sq) : 0.f);
    }
    if (t.warps > 1) {
        float2* room = t.room + t.turn * kRows * kMaxWarps;
        t.turn ^= 1;
        if (t.lane == 0) {
#pragma unroll
            for (int i = 0; i < kRows; ++i) room[i * kMaxWarps + t.warp] = make_float2(mean[i], q[i]);
        }
        t.sync();
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            float sum = 0.f, m2 = 0.f;
            for (int w = 0; w < t.warps; ++w) sum += room[i * kMaxWarps + w].x * float(min(256, t.cols - w * 256));
            const float m = sum / all;
            for (int w = 0; w < t.warps; ++w) {
                const float2 o = room[i * kMaxWarps + w];
                m2 += o.y + float(min(256, t.cols - w * 256)) * ((o.x - m) * (o.x - m));
            }
            mean[i] = m;
            q[i] = m2;
        }
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) inv[i] = rsqrtf(q[i] / all + eps);
}

template <typename T>
__device__ __forceinline__ void request(Vec8<T> (&v)[kRows], const Matrix& m, const Batch& b, const Team& t) {
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        v[i].clear();
        if (i < b.live && t.col) v[i].load(m.p, (b.row + i) * m.ld + t.c0);
    }
}

// S: type of x and x', B: of h and y.
template <typename S, typename B, bool POST>
__global__ void __launch_bounds__(kMaxWarps * 32) gate_norm_kernel(const GateNormParams p) {
    __shared__ float2 room[2 * kRows * kMaxWarps];
    Team t = team_of(p, room);
    const int teams = int(blockDim.x >> 5) / p.warps;
    const int64_t r0 = (int64_t(blockIdx.x) * teams + t.id) * p.chunk, r1 = min(r0 + p.chunk, p.rows);
    if (r0 >= r1) return;
    Batch b = batch_at(p, r0, r0 / p.group, r1);
    f32x2 gate[4], weight[4], bias[4], post_weight[4];
    if (POST) load_vector(post_weight, Vectors{p.post_weight, 0}, 0, t.c0, t.col, 0.f, 1.f);
    int64_t loaded = -1;
    Vec8<S> x_in[kRows];
    Vec8<B> h_in[kRows];
    request(x_in, p.x, b, t);
    if (p.h.p != nullptr) request(h_in, p.h, b, t);
    while (b.n > 0) {
        if (b.g != loaded) {
            load_vector(gate, p.gate, b.g, t.c0, t.col, 0.f, 1.f);
            if (p.y.p != nullptr) {
                load_vector(weight, p.weight, b.g, t.c0, t.col, p.plus, 1.f);
                load_vector(bias, p.bias, b.g, t.c0, t.col, 0.f, 0.f);
            }
            loaded = b.g;
        }
        const int64_t next_row = b.row + b.n;
        const Batch next = batch_at(p, next_row, b.g + (next_row == (b.g + 1) * p.group), r1);
        f32x2 v[kRows][4], u[kRows][4];
#pragma unroll
        for (int i = 0; i < kRows; ++i) x_in[i].get(v[i]);
        request(x_in, p.x, next, t);                           // in flight while this batch is computed
        float mean[kRows], inv[kRows], post_mean[kRows], post_inv[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) { mean[i] = 0.f; inv[i] = 1.f; post_mean[i] = 0.f; post_inv[i] = 1.f; }
        if (p.h.p != nullptr) {
#pragma unroll
            for (int i = 0; i < kRows; ++i) h_in[i].get(u[i]);
            request(h_in, p.h, next, t);
            if (POST) moments(t, u, p.post_layer, p.eps, post_mean, post_inv);
            const f32x2 residual = pk2(p.residual, p.residual);
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const f32x2 m = pk2(-post_mean[i], -post_mean[i]), s = pk2(post_inv[i], post_inv[i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (POST) u[i][e] = mul2(mul2(add2(u[i][e], m), s), post_weight[e]);
                    v[i][e] = fma2(residual, v[i][e], mul2(gate[e], u[i][e]));
                }
            }
        }
        if (p.x_out.p != nullptr) {
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                if (i >= b.live) fill(v[i], 0.f);
                if (i < b.n && t.col) Vec8<S>::store(p.x_out.p, (b.row + i) * p.x_out.ld + t.c0, v[i]);
            }
        }
        if (p.y.p != nullptr) {
            moments(t, v, p.layer, p.eps, mean, inv);
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const f32x2 m = pk2(-mean[i], -mean[i]), s = pk2(inv[i], inv[i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[i][e] = fma2(mul2(add2(v[i][e], m), s), weight[e], bias[e]);
                if (i >= b.live) fill(v[i], 0.f);
                if (i < b.n && t.col) Vec8<B>::store(p.y.p, (b.row + i) * p.y.ld + t.c0, v[i]);
            }
        }
        if (p.stats != nullptr && t.warp == 0 && t.lane == 0) {
#pragma unroll
            for (int i = 0; i < kRows; ++i)
                if (i < b.n)
                    reinterpret_cast<float4*>(p.stats)[b.row + i] = i < b.live ? make_float4(mean[i], inv[i], post_mean[i], post_inv[i])
                                                                               : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        b = next;
    }
}

// A CTA takes `chunk` rows, its teams their batches in turn.  Where a group ends (and behind the last row) the teams' sums over the group's
// rows are joined in order and leave: to the gradient itself where the whole group lay in this CTA, else to the CTA's part (the first of its
// two for the group that its first row belongs to, else the second), which gate_norm_sums_kernel joins.
template <typename S, typename B, bool POST>
__global__ void __launch_bounds__(kMaxWarps * 32) gate_norm_grad_kernel(const GateNormParams p) {
    __shared__ float2 room[2 * kRows * kMaxWarps];
    __shared__ float lines[8 * 256];               // sums of several teams: at most 8 warps of 256 columns
    Team t = team_of(p, room);
    const int teams = int(blockDim.x >> 5) / p.warps;
    const int64_t r0 = int64_t(blockIdx.x) * p.chunk, r1 = min(r0 + p.chunk, p.rows);
    const bool normed = p.dy.p != nullptr, gated = p.dgate.p != nullptr, later = p.dx_out.p != nullptr;
    const bool branch = POST || gated;             // h itself is read
    f32x2 post_weight[4], dpost[4];
    fill(dpost, 0.f);
    if (POST) load_vector(post_weight, Vectors{p.post_weight, 0}, 0, t.c0, t.col, 0.f, 1.f);
    const float per = 1.f / float(p.cols);
    for (int64_t g = r0 / p.group; g * p.group < r1; ++g) {
        const int64_t first = max(g * p.group, r0), last = min((g + 1) * p.group, r1);
        f32x2 gate[4], weight[4], dweight[4], dbias[4], dgate[4];
        fill(dweight, 0.f); fill(dbias, 0.f); fill(dgate, 0.f);
        load_vector(gate, p.gate, g, t.c0, t.col, 0.f, 1.f);
        load_vector(weight, p.weight, g, t.c0, t.col, p.plus, 1.f);
        for (int64_t row = first + t.id * kRows; row < last; row += teams * kRows) {
            const Batch b = batch_at(p, row, g, last);
            Vec8<S> x_in[kRows], d_in[kRows];
            Vec8<B> y_in[kRows], h_in[kRows];
            float4 stats[kRows];
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                stats[i] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (i < b.live && (normed || POST)) stats[i] = reinterpret_cast<const float4*>(p.stats)[b.row + i];
            }
            if (normed) { request(x_in, p.x, b, t); request(y_in, p.dy, b, t); }
            if (later) request(d_in, p.dx_out, b, t);
            if (branch) request(h_in, p.h, b, t);
            f32x2 d[kRows][4];
            if (normed) {
                f32x2 xh[kRows][4];
                float2 s[kRows];
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    const f32x2 m = pk2(-stats[i].x, -stats[i].x), inv = pk2(stats[i].y, stats[i].y);
                    f32x2 a = pk2(0.f, 0.f), c = pk2(0.f, 0.f);
                    x_in[i].get(xh[i]);
                    y_in[i].get(d[i]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        xh[i][e] = mul2(add2(xh[i][e], m), inv);
                        dbias[e] = add2(dbias[e], d[i][e]);
                        dweight[e] = fma2(d[i][e], xh[i][e], dweight[e]);
                        d[i][e] = mul2(d[i][e], weight[e]);
                        a = add2(a, d[i][e]);
                        c = fma2(d[i][e], xh[i][e], c);
                    }
                    s[i] = t.col ? make_float2(pair_sum(a), pair_sum(c)) : make_float2(0.f, 0.f);
                }
                team_sums(t, s);
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    const float mg = p.layer ? -s[i].x * per : 0.f, mx = -s[i].y * per;
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
                    d_in[i].get(o);
#pragma unroll
                    for (int e = 0; e < 4; ++e) d[i][e] = add2(d[i][e], o[e]);
                }
            }
            if (p.dx.p != nullptr) {
                const f32x2 residual = pk2(p.residual, p.residual);
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    f32x2 o[4];
#pragma unroll
                    for (int e = 0; e < 4; ++e) o[e] = mul2(residual, d[i][e]);
                    if (i >= b.live) fill(o, 0.f);
                    if (i < b.n && t.col) Vec8<S>::store(p.dx.p, (b.row + i) * p.dx.ld + t.c0, o);
                }
            }
            if (POST) {
                f32x2 hh[kRows][4];
                float2 s[kRows];
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    const f32x2 m = pk2(-stats[i].z, -stats[i].z), inv = pk2(stats[i].w, stats[i].w);
                    f32x2 a = pk2(0.f, 0.f), c = pk2(0.f, 0.f);
                    h_in[i].get(hh[i]);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        hh[i][e] = mul2(add2(hh[i][e], m), inv);
                        dgate[e] = fma2(d[i][e], hh[i][e], dgate[e]);          // both sums' part: dgate = post_weight times it, dpost gate times it
                        d[i][e] = mul2(mul2(d[i][e], gate[e]), post_weight[e]);
                        a = add2(a, d[i][e]);
                        c = fma2(d[i][e], hh[i][e], c);
                    }
                    s[i] = t.col ? make_float2(pair_sum(a), pair_sum(c)) : make_float2(0.f, 0.f);
                }
                if (p.dh.p != nullptr) {
                    team_sums(t, s);
#pragma unroll
                    for (int i = 0; i < kRows; ++i) {
                        const float mg = p.post_layer ? -s[i].x * per : 0.f, mx = -s[i].y * per;
                        const f32x2 inv = pk2(stats[i].w, stats[i].w), g2 = pk2(mg, mg), x2 = pk2(mx, mx);
#pragma unroll
                        for (int e = 0; e < 4; ++e) d[i][e] = mul2(inv, fma2(hh[i][e], x2, add2(d[i][e], g2)));
                    }
                }
            } else {
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    f32x2 o[4];
                    if (gated) h_in[i].get(o);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (gated) dgate[e] = fma2(d[i][e], o[e], dgate[e]);
                        d[i][e] = mul2(d[i][e], gate[e]);
                    }
                }
            }
            if (p.dh.p != nullptr) {
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    if (i >= b.live) fill(d[i], 0.f);
                    if (i < b.n && t.col) Vec8<B>::store(p.dh.p, (b.row + i) * p.dh.ld + t.c0, d[i]);
                }
            }
        }
        if (teams > 1) {                           // the other teams' sums, in order
            float* line = lines + t.id * t.warps * 256 + t.c0;
            f32x2* sums[3] = {dweight, dbias, dgate};
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                __syncthreads();
                if (t.id > 0) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) { float a, c; upk2(sums[k][e], a, c); line[2 * e] = a; line[2 * e + 1] = c; }
                }
                __syncthreads();
                if (t.id == 0) {
                    for (int o = 1; o < teams; ++o) {
                        const float* other = line + o * t.warps * 256;
#pragma unroll
                        for (int e = 0; e < 4; ++e) sums[k][e] = add2(sums[k][e], pk2(other[2 * e], other[2 * e + 1]));
                    }
                }
            }
        }
        if (t.id == 0 && t.col) {
            if (POST) {
#pragma unroll
                for (int e = 0; e < 4; ++e) dpost[e] = fma2(gate[e], dgate[e], dpost[e]);
            }
            const int64_t whole_end = min((g + 1) * p.group, p.rows);
            if (first == g * p.group && last == whole_end) {
                if (POST && gated) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) dgate[e] = mul2(dgate[e], post_weight[e]);
                }
                if (p.dweight.p != nullptr) store_vector(p.dweight.p + g * p.dweight.ld + t.c0, dweight);
                if (p.dbias.p != nullptr) store_vector(p.dbias.p + g * p.dbias.ld + t.c0, dbias);
                if (gated) store_vector(p.dgate.p + g * p.dgate.ld + t.c0, dgate);
            } else if (p.parts != nullptr) {
                float* to = p.parts + (int64_t(blockIdx.x) * 2 + (first == r0 ? 0 : 1)) * 3 * p.cols + t.c0;
                if (p.dweight.p != nullptr) store_vector(to, dweight);
                if (p.dbias.p != nullptr) store_vector(to + p.cols, dbias);
                if (gated) store_vector(to + 2 * p.cols, dgate);
            }
        }
    }
    if (POST && p.dpost != nullptr && t.id == 0 && t.col) store_vector(p.post_parts + int64_t(blockIdx.x) * p.cols + t.c0, dpost);
}

// The parts of groups that lie in several CTAs, and of dpost_weight, joined in order.  blockIdx.x: `wide` columns; y: a group, or, where
// there are more groups than CTAs, the group at a border of two CTAs' rows, which the first border inside it takes; z: the sum (0 weight,
// 1 bias, 2 gate, 3 post_weight).  Thread = (column, every 256 / wide'th part).
__global__ void __launch_bounds__(256) gate_norm_sums_kernel(const GateNormParams p, int ctas, int wide, int by_group) {
    __shared__ float sums[256];
    const int z = int(blockIdx.z), ways = 256 / wide, c = int(blockIdx.x) * wide + int(threadIdx.x) % wide, way = int(threadIdx.x) / wide;
    const VectorsOut out = z == 0 ? p.dweight : z == 1 ? p.dbias : z == 2 ? p.dgate : VectorsOut{p.dpost, 0};
    griddep_wait();                                // the parts; no CTA ends before the kernel in front has
    if (out.p == nullptr || (z < 3 ? p.parts == nullptr : blockIdx.y > 0)) return;
    int64_t g = 0, from = 0, to = ctas - 1;
    bool second = false;
    if (z < 3) {
        g = by_group ? int64_t(blockIdx.y) : (int64_t(blockIdx.y) + 1) * p.chunk / p.group;
        const int64_t first = g * p.group, last = min(first + p.group, p.rows) - 1;
        from = first / p.chunk;
        to = last / p.chunk;
        if (from == to || (!by_group && from != int64_t(blockIdx.y))) return;
        second = first != from * p.chunk;          // the group is not the one of that CTA's first row
    }
    float sum = 0.f;
    if (c < p.cols) {
        const float* parts = z < 3 ? p.parts + z * p.cols + c : p.post_parts + c;
        const int64_t step = z < 3 ? int64_t(6) * p.cols : p.cols;
#pragma unroll 8
        for (int64_t i = from + way; i <= to; i += ways) sum += ld_dependent(parts + i * step + (second && i == from ? 3 * p.cols : 0));
    }
    sums[threadIdx.x] = sum;
    __syncthreads();
    if (way == 0 && c < p.cols) {
        for (int w = 1; w < ways; ++w) sum += sums[w * wide + threadIdx.x];
        if (z == 2 && p.post_weight != nullptr) sum *= p.post_weight[c];
        out.p[g * out.ld + c] = sum;
    }
}

// ------------------------------------------------------------------------------------------------------------- host

int team_warps(int64_t cols) { return int((cols + 255) / 256); }
// Teams of a CTA: up to 8 warps, and no more than a group's rows keep busy.
int team_count(int64_t cols, int64_t group) {
    const int64_t most = 8 / team_warps(cols), busy = (group + kRows - 1) / kRows;
    return int(most < 1 ? 1 : most < busy ? most : busy);
}
constexpr int kGradWarps = 148 * 15;               // warps at a time, on every device: gradients are summed in one order
int64_t grad_chunk(int64_t rows, int64_t cols, int64_t group) {
    const int teams = team_count(cols, group), warps = teams * team_warps(cols);
    const int64_t ctas = kGradWarps / warps, least = int64_t(teams) * kRows * 2;
    const int64_t chunk = (rows + ctas - 1) / ctas;
    return chunk < least ? least : chunk;
}

hq_status check_matrix(const void* x, int64_t ld, int64_t cols, hq_dtype dt) {
    if (x == nullptr) return HQ_ERR_INVALID_ARG;
    if (ld < cols) return HQ_ERR_SHAPE;
    if (!aligned16(x) || (ld * (dt == HQ_BF16 ? 2 : 4)) % 16 != 0) return HQ_ERR_ALIGNMENT;
    return HQ_OK;
}
hq_status check_vectors(const float* v, int64_t ld, int64_t groups, int64_t cols) {
    if (v == nullptr) return HQ_OK;
    if (groups > 1 && ld < cols) return HQ_ERR_SHAPE;
    return aligned16(v) && (groups <= 1 || ld % 4 == 0) ? HQ_OK : HQ_ERR_ALIGNMENT;
}
bool type_ok(hq_dtype t) { return t == HQ_F32 || t == HQ_BF16; }
bool norm_ok(hq_norm n) { return n == HQ_NORM_LAYER || n == HQ_NORM_RMS || n == HQ_NORM_NONE; }
// What both calls check of their sizes; *group: rows of a group.
hq_status check_sizes(hq_dtype xdt, hq_dtype hdt, int64_t rows, int64_t cols, int64_t rows_per_group, const int32_t* lens, hq_norm post,
                      const float* post_weight, hq_norm norm, const void* h, const void* gate, float residual, int64_t* group) {
    if (!type_ok(xdt) || !type_ok(hdt) || !norm_ok(post) || !norm_ok(norm)) return HQ_ERR_INVALID_ARG;
    if (rows < 0 || cols <= 0 || rows_per_group < 0) return HQ_ERR_SHAPE;
    if (cols % 8 != 0 || cols > kMaxCols || rows > 0x7fffffff) return HQ_ERR_UNSUPPORTED;
    if (lens != nullptr && rows_per_group == 0) return HQ_ERR_INVALID_ARG;
    if (post == HQ_NORM_NONE && post_weight != nullptr) return HQ_ERR_INVALID_ARG;
    if (!aligned16(post_weight)) return HQ_ERR_ALIGNMENT;
    if (!(residual - residual == 0.f)) return HQ_ERR_INVALID_ARG;
    if (h == nullptr && (post != HQ_NORM_NONE || gate != nullptr || residual != 1.f)) return HQ_ERR_INVALID_ARG;
    *group = rows_per_group > 0 ? rows_per_group : rows > 0 ? rows : 1;
    return HQ_OK;
}

template <typename S, typename B>
cudaError_t launch_forward(const GateNormParams& p, bool post, unsigned grid, unsigned threads, cudaStream_t st) {
    if (post) gate_norm_kernel<S, B, true><<<grid, threads, 0, st>>>(p);
    else gate_norm_kernel<S, B, false><<<grid, threads, 0, st>>>(p);
    return cudaGetLastError();
}
template <typename S, typename B>
cudaError_t launch_grad(const GateNormParams& p, bool post, unsigned grid, unsigned threads, cudaStream_t st) {
    if (post) gate_norm_grad_kernel<S, B, true><<<grid, threads, 0, st>>>(p);
    else gate_norm_grad_kernel<S, B, false><<<grid, threads, 0, st>>>(p);
    return cudaGetLastError();
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
    if (!aligned16(stats)) return HQ_ERR_ALIGNMENT;
    GateNormParams p{};
    p.rows = rows; p.group = group; p.cols = int(cols); p.warps = team_warps(cols); p.lens = lens;
    p.layer = norm == HQ_NORM_LAYER; p.post_layer = post == HQ_NORM_LAYER; p.post_weight = post_weight;
    p.gate = Vectors{gate, ld_gate}; p.weight = Vectors{weight, ld_weight}; p.bias = Vectors{bias, ld_bias};
    p.residual = residual_scale; p.plus = weight_plus; p.eps = eps; p.stats = stats;
    p.x = Matrix{x, ldx}; p.h = Matrix{h, ldh}; p.x_out = MatrixOut{x_out, ldx_out}; p.y = MatrixOut{y, ldy};
    const int teams = p.warps > 8 ? 1 : 8 / p.warps;
    const int64_t most = int64_t(sm_count()) * (24 / p.warps);             // teams at a time
    p.chunk = (rows + most - 1) / most;
    if (p.chunk < kRows) p.chunk = kRows;
    const int64_t used = (rows + p.chunk - 1) / p.chunk;
    const unsigned grid = unsigned((used + teams - 1) / teams), threads = unsigned(teams * p.warps * 32);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool after = post != HQ_NORM_NONE;
    cudaError_t c;
    if (xdt == HQ_BF16) c = hdt == HQ_BF16 ? launch_forward<__nv_bfloat16, __nv_bfloat16>(p, after, grid, threads, st) : launch_forward<__nv_bfloat16, float>(p, after, grid, threads, st);
    else c = hdt == HQ_BF16 ? launch_forward<float, __nv_bfloat16>(p, after, grid, threads, st) : launch_forward<float, float>(p, after, grid, threads, st);
    return c == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}

extern "C" hq_status hq_gate_norm_bwd_workspace_size(int64_t rows, int64_t cols, int64_t rows_per_group, size_t* bytes) {
    using namespace hq;
    if (bytes == nullptr) return HQ_ERR_INVALID_ARG;
    int64_t group = 0;
    const hq_status e = check_sizes(HQ_BF16, HQ_BF16, rows, cols, rows_per_group, nullptr, HQ_NORM_NONE, nullptr, HQ_NORM_NONE, nullptr, nullptr, 1.f, &group);
    if (e != HQ_OK) return e;
    const int64_t chunk = grad_chunk(rows, cols, group), ctas = (rows + chunk - 1) / chunk;
    *bytes = size_t(ctas) * 7 * size_t(cols) * sizeof(float);
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
    if ((normed || after) && stats == nullptr) return HQ_ERR_INVALID_ARG;
    if (!aligned16(stats) || !aligned16(dpost_weight)) return HQ_ERR_ALIGNMENT;
    GateNormParams p{};
    p.rows = rows; p.group = group; p.cols = int(cols); p.warps = team_warps(cols); p.lens = lens;
    p.chunk = grad_chunk(rows, cols, group);
    const int64_t ctas = (rows + p.chunk - 1) / p.chunk;
    const bool sums = dgate != nullptr || dweight != nullptr || dbias != nullptr;
    // a part for a group that lies in several CTAs; without a sum over rows, or where every group lies in one CTA, none is written
    const bool split = sums && (p.chunk % group != 0) && ctas > 1;
    if (split || dpost_weight != nullptr) {
        size_t need = 0;
        if (workspace == nullptr) return HQ_ERR_INVALID_ARG;
        if (!aligned16(workspace)) return HQ_ERR_ALIGNMENT;
        hq_gate_norm_bwd_workspace_size(rows, cols, rows_per_group, &need);
        if (ws_bytes < need) return HQ_ERR_WORKSPACE;
    }
    p.layer = norm == HQ_NORM_LAYER; p.post_layer = post == HQ_NORM_LAYER; p.post_weight = post_weight;
    p.gate = Vectors{gate, ld_gate}; p.weight = Vectors{weight, ld_weight};
    p.residual = residual_scale; p.plus = weight_plus; p.stats = const_cast<float*>(stats);
    p.x = Matrix{x_out, ldx_out}; p.h = Matrix{h, ldh}; p.dx_out = Matrix{dx_out, lddx_out}; p.dy = Matrix{dy, lddy};
    p.dx = MatrixOut{dx, lddx}; p.dh = MatrixOut{dh, lddh};
    p.dgate = VectorsOut{dgate, ld_dgate}; p.dweight = VectorsOut{dweight, ld_dweight}; p.dbias = VectorsOut{dbias, ld_dbias};
    p.dpost = dpost_weight;
    p.parts = split ? static_cast<float*>(workspace) : nullptr;
    p.post_parts = static_cast<float*>(workspace) + size_t(ctas) * 6 * cols;
    const int teams = team_count(cols, group);
    const unsigned grid = unsigned(ctas), threads = unsigned(teams * p.warps * 32);
    cudaError_t c;
    if (xdt == HQ_BF16) c = hdt == HQ_BF16 ? launch_grad<__nv_bfloat16, __nv_bfloat16>(p, after, grid, threads, st) : launch_grad<__nv_bfloat16, float>(p, after, grid, threads, st);
    else c = hdt == HQ_BF16 ? launch_grad<float, __nv_bfloat16>(p, after, grid, threads, st) : launch_grad<float, float>(p, after, grid, threads, st);
    if (c != cudaSuccess) return HQ_ERR_CUDA;
    if (!split && dpost_weight == nullptr) return HQ_OK;
    const int by_group = groups <= ctas - 1;
    const int64_t heads = !split ? 1 : by_group ? groups : ctas - 1;
    int wide = 8;                                  // columns a CTA: as few as keep the number of CTAs in the thousands
    while (wide < 128 && (cols + wide - 1) / wide * heads > 2048) wide *= 2;
    const dim3 few(unsigned((cols + wide - 1) / wide), unsigned(heads), dpost_weight != nullptr ? 4u : 3u);
    return launch_dependent(gate_norm_sums_kernel, few, 256, 0, st, dependent_launch(int64_t(few.x) * few.y * few.z), p, int(ctas), wide, by_group) == cudaSuccess
               ? HQ_OK : HQ_ERR_CUDA;
}
