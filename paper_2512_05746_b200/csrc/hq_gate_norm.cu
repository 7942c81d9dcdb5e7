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
// warps, a CTA of its own, takes a run of rows, 8 columns a thread.  Rows are copied ahead into shared memory, by each thread for itself (no barrier stands
// between the copy and its use, and no register holds what is on the way); two rows are computed together, so that their sums share the
// shuffles; sums over rows stay in the registers of the thread that owns the columns.
#include "hq_common.cuh"
#include "hq_vec8.cuh"

namespace hq {
namespace {

constexpr int kMaxCols = 4096;
constexpr int kMaxWarps = 16;
constexpr int kRows = 2;                           // rows of a team's batch

struct Matrix { const void* p; uint32_t ld; };     // pitch in bytes
struct MatrixOut { void* p; uint32_t ld; };
struct Vectors { const float* p; int64_t ld; };    // [groups][cols]
struct VectorsOut { float* p; int64_t ld; };

struct GateNormParams {
    uint32_t rows, group, chunk;                   // group: rows that share their vectors; chunk: rows of a team
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
    float *dpost, *parts, *post_parts;             // parts: [teams][first, last group][weight, bias, gate][cols]; post_parts: [teams][cols]
};

// ---- a team's walk over its rows ----

// Rows [row, row + n) of group g, the first `live` of them within its length; left, alive: rows of the group from `row` on, and within its length.
struct Walk {
    uint32_t row, g;
    int left, alive, n, live;
    __device__ __forceinline__ void enter(const GateNormParams& p, uint32_t behind) {        // behind: rows of the group in front of `row`
        left = int(min(p.group - behind, p.rows - row));
        alive = p.lens != nullptr && left > 0 ? min(p.lens[g] - int(behind), left) : left;
    }
    __device__ __forceinline__ void count(uint32_t end) {
        n = min(min(kRows, left), int(end - row));
        live = max(0, min(n, alive));
    }
    __device__ __forceinline__ void start(const GateNormParams& p, uint32_t at, uint32_t end) {
        row = at;
        g = at / p.group;
        enter(p, at - g * p.group);
        count(end);
    }
    __device__ __forceinline__ void next(const GateNormParams& p, uint32_t end) {
        row += uint32_t(n);
        left -= n;
        alive -= n;
        if (left == 0) { ++g; enter(p, 0); }
        count(end);
    }
};

// ---- a team, and its exchange of sums: two buffers in turn, so that one barrier stands between the writes and the reads of an exchange and
// none behind it. ----
struct Team {
    int lane, warp, warps, c0, cols;
    bool col;                                      // the thread has columns
    float share, per_warp, per_row;                // columns of warp (lane & 15); 1 / columns of this warp, of the row
    float2* room;                                  // [2][32]
    int turn;
};
__device__ __forceinline__ Team team_of(const GateNormParams& p, float2* room) {
    Team t;
    t.lane = int(threadIdx.x & 31);
    t.warps = p.warps;
    t.warp = int(threadIdx.x >> 5);
    t.c0 = (t.warp * 32 + t.lane) * 8;
    t.cols = p.cols;
    t.col = t.c0 < p.cols;
    t.share = float(max(0, min(256, p.cols - (t.lane & 15) * 256)));
    t.per_warp = 1.f / float(min(256, p.cols - t.warp * 256));
    t.per_row = 1.f / float(p.cols);
    t.room = room;
    t.turn = 0;
    return t;
}
__device__ __forceinline__ float sum8(const f32x2 (&v)[4]) { return pair_sum(add2(add2(v[0], v[1]), add2(v[2], v[3]))); }
__device__ __forceinline__ float xor_add(float x, int off) { return x + __shfl_xor_sync(0xffffffffu, x, off); }
__device__ __forceinline__ float from_lane(float x, int lane) { return __shfl_sync(0xffffffffu, x, lane); }
// Two values' sums over the warp: lanes 0 .. 15 have the first's, lanes 16 .. 31 the second's.
__device__ __forceinline__ float sum_of_two(float a, float b, int lane) {
    const bool low = lane < 16;
    float s = (low ? a : b) + __shfl_xor_sync(0xffffffffu, low ? b : a, 16);
    s = xor_add(s, 8); s = xor_add(s, 4); s = xor_add(s, 2);
    return xor_add(s, 1);
}

// The sums of a pair of values of each of two rows over the team.
__device__ __forceinline__ void team_sums(Team& t, float2& a, float2& b) {
    const bool low = t.lane < 16, left = (t.lane & 8) == 0;
    const float2 mine = low ? a : b, other = low ? b : a;
    const float x = mine.x + __shfl_xor_sync(0xffffffffu, other.x, 16), y = mine.y + __shfl_xor_sync(0xffffffffu, other.y, 16);
    float s = (left ? x : y) + __shfl_xor_sync(0xffffffffu, left ? y : x, 8);                // eight lanes a value: a.x, a.y, b.x, b.y
    s = xor_add(s, 4); s = xor_add(s, 2); s = xor_add(s, 1);
    if (t.warps > 1) {
        float* room = reinterpret_cast<float*>(t.room + t.turn * 32);                        // [4][kMaxWarps]
        t.turn ^= 1;
        if ((t.lane & 7) == 0) room[(t.lane >> 3) * kMaxWarps + t.warp] = s;
        __syncthreads();
        const int w = t.lane & 7, from = (t.lane >> 3) * kMaxWarps + w;
        s = w < t.warps ? room[from] : 0.f;
        if (w + 8 < t.warps) s += room[from + 8];
        s = xor_add(s, 4); s = xor_add(s, 2); s = xor_add(s, 1);
    }
    a = make_float2(from_lane(s, 0), from_lane(s, 8));
    b = make_float2(from_lane(s, 16), from_lane(s, 24));
}

// Mean (0 unless `layer`) and 1 / standard deviation of both rows.  A warp takes the mean of its own values first and its squares about
// that, and the warps' parts are joined about the row's mean: no difference of large sums, and one exchange.
__device__ __forceinline__ void moments(Team& t, const f32x2 (&v)[kRows][4], int layer, float eps, float (&mean)[kRows], float (&inv)[kRows]) {
    float m = 0.f;                                 // of row lane / 16
    mean[0] = mean[1] = 0.f;
    if (layer) {
        m = sum_of_two(t.col ? sum8(v[0]) : 0.f, t.col ? sum8(v[1]) : 0.f, t.lane) * t.per_warp;
        mean[0] = from_lane(m, 0);
        mean[1] = from_lane(m, 16);
    }
    float q[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const f32x2 less = pk2(-mean[i], -mean[i]);
        f32x2 sq = pk2(0.f, 0.f);
#pragma unroll
        for (int e = 0; e < 4; ++e) { const f32x2 d = add2(v[i][e], less); sq = fma2(d, d, sq); }
        q[i] = t.col ? pair_sum(sq) : 0.f;
    }
    float m2 = sum_of_two(q[0], q[1], t.lane);
    if (t.warps > 1) {
        float2* room = t.room + t.turn * 32;       // [kRows][kMaxWarps]
        t.turn ^= 1;
        if ((t.lane & 15) == 0) room[t.lane + t.warp] = make_float2(m, m2);
        __syncthreads();
        const float2 o = (t.lane & 15) < t.warps ? room[t.lane] : make_float2(0.f, 0.f);
        m = 0.f;
        if (layer) {
            m = t.share * o.x;
            m = xor_add(m, 8); m = xor_add(m, 4); m = xor_add(m, 2);
            m = xor_add(m, 1) * t.per_row;
            mean[0] = from_lane(m, 0);
            mean[1] = from_lane(m, 16);
        }
        m2 = o.y + t.share * ((o.x - m) * (o.x - m));
        m2 = xor_add(m2, 8); m2 = xor_add(m2, 4); m2 = xor_add(m2, 2);
        m2 = xor_add(m2, 1);
    }
    m2 = rsqrtf(m2 * t.per_row + eps);
    inv[0] = from_lane(m2, 0);
    inv[1] = from_lane(m2, 16);
}

// ---- vectors of a thread's columns ----
__device__ __forceinline__ void fill(f32x2 (&v)[4], float x) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = pk2(x, x);
}
// A group's values for this thread's columns, plus `add`; `none` without a vector.
__device__ __forceinline__ void load_vector(f32x2 (&v)[4], const Vectors& from, uint32_t g, const Team& t, float add, float none) {
    if (from.p == nullptr || !t.col) { fill(v, none); return; }
    const float4* q = reinterpret_cast<const float4*>(from.p + int64_t(g) * from.ld + t.c0);
    const float4 a = q[0], b = q[1];
    v[0] = pk2(a.x + add, a.y + add); v[1] = pk2(a.z + add, a.w + add); v[2] = pk2(b.x + add, b.y + add); v[3] = pk2(b.z + add, b.w + add);
}

// ---- rows on their way through shared memory: a thread's 16 or 32 bytes of a row, in planes of 16 bytes a thread.  Neighbouring lanes copy
// neighbouring 16 bytes; of fp32 they are another lane's of the warp (copied by their own lane, half of every sector would be asked for twice) ----
template <typename T> constexpr int kPlanes = int(sizeof(T)) * 8 / 16;
__device__ __forceinline__ void copy_ahead(uint32_t to, const void* from, bool there) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_sent() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
    __syncwarp();
}
__device__ __forceinline__ uint64_t row_at(uint32_t row, uint32_t ld) { return uint64_t(row) * ld; }
// Where this thread's copies of a row begin, and its own columns' place in an output.
template <typename T> __device__ __forceinline__ const char* copied(const Matrix& m, const Team& t) {
    return static_cast<const char*>(m.p) + (sizeof(T) == 2 ? t.c0 * 2 : (t.warp * 256 + t.lane * 4) * 4);
}
template <typename T> __device__ __forceinline__ char* columns(const MatrixOut& m, const Team& t) { return static_cast<char*>(m.p) + t.c0 * int(sizeof(T)); }
// `at`: the batch's first plane; zeros for rows that are not there.
template <typename T>
__device__ __forceinline__ void send(uint32_t at, const char* from, uint32_t ld, const Walk& b, const Team& t) {
    const uint32_t plane = blockDim.x * 16u;
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const bool live = i < b.live;
        const char* row = from + row_at(b.row, ld) + (live ? uint32_t(i) * uint64_t(ld) : 0u);
        if constexpr (sizeof(T) == 2) {
            copy_ahead(at + uint32_t(i) * plane + threadIdx.x * 16u, t.col ? row : row - t.c0 * 2, live && t.col);
        } else {
#pragma unroll
            for (int k = 0; k < 2; ++k) {          // piece k * 32 + lane of the warp's 64: of lane piece / 2, plane piece % 2
                const int c = t.warp * 256 + (k * 32 + t.lane) * 4;
                const bool col = c < t.cols;
                copy_ahead(at + (uint32_t(i) * 2u + (t.lane & 1u)) * plane + ((threadIdx.x & ~31u) + uint32_t(k * 16 + t.lane / 2)) * 16u,
                           col ? row + k * 512 : row - (t.warp * 256 + t.lane * 4) * 4, live && col);
            }
        }
    }
}
__device__ __forceinline__ uint4 plane_at(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
// This thread's columns of row i of the batch whose first plane is `at`.
template <typename T>
__device__ __forceinline__ void take(f32x2 (&v)[4], uint32_t at, int i) {
    const uint32_t plane = blockDim.x * 16u, mine = at + threadIdx.x * 16u;
    Vec8<T> raw;
    if constexpr (sizeof(T) == 2) {
        raw.w = plane_at(mine + uint32_t(i) * plane);
    } else {
        const uint4 a = plane_at(mine + uint32_t(2 * i) * plane), b = plane_at(mine + uint32_t(2 * i + 1) * plane);
        raw.a = make_float4(__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w));
        raw.b = make_float4(__uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w));
    }
    raw.get(v);
}
// Rows that are not there leave as zeros.
__device__ __forceinline__ void clear_dead(const Walk& b, f32x2 (&v)[kRows][4]) {
    if (b.live == b.n) return;
#pragma unroll
    for (int i = 0; i < kRows; ++i)
        if (i >= b.live) fill(v[i], 0.f);
}
template <typename T>
__device__ __forceinline__ void put(char* to, uint32_t ld, const Walk& b, const Team& t, const f32x2 (&v)[kRows][4]) {
    char* row = to + row_at(b.row, ld);            // a batch has a row
    if (t.col) Vec8<T>::store_wide(row, 0, v[0]);
    if (t.col && b.n > 1) Vec8<T>::store_wide(row + ld, 0, v[1]);
}

template <typename T>
__device__ __forceinline__ void put_zeros(char* to, const MatrixOut& m, const Walk& b, const Team& t) {
    if (m.p == nullptr) return;
    f32x2 v[kRows][4];
#pragma unroll
    for (int i = 0; i < kRows; ++i) fill(v[i], 0.f);
    put<T>(to, m.ld, b, t, v);
}

// Batches on their way: what keeps about 40 KB an SM in flight at 15 warps and more.
template <typename S, typename B> constexpr int kForwardPlanes = kRows * (kPlanes<S> + kPlanes<B>);
template <typename S, typename B> constexpr int kGradPlanes = 2 * kForwardPlanes<S, B>;
constexpr int kForwardStages = 3, kGradStages = 2;
constexpr size_t kMostShared = 224 * 1024;

// S: type of x and x', B: of h and y.
template <typename S, typename B, bool POST>
__global__ void __maxnreg__(96) gate_norm_kernel(const GateNormParams p) {
    extern __shared__ uint4 ring[];
    __shared__ float2 room[2 * 32];
    constexpr int kStages = kForwardStages;
    Team t = team_of(p, room);
    const uint32_t r0 = blockIdx.x * p.chunk, r1 = min(r0 + p.chunk, p.rows);
    const uint32_t plane = blockDim.x * 16u, batch = plane * kForwardPlanes<S, B>, h_at = plane * kRows * kPlanes<S>;
    const uint32_t base = smem_u32(ring);
    const bool branch = p.h.p != nullptr, normed = p.y.p != nullptr;
    const char *x = copied<S>(p.x, t), *h = copied<B>(p.h, t);
    char *x_out = columns<S>(p.x_out, t), *y = columns<B>(p.y, t);
    Walk b, ahead;
    b.start(p, r0, r1);
    ahead = b;
    uint32_t to = base;
    auto send_next = [&]() {
        if (ahead.n > 0) {
            send<S>(to, x, p.x.ld, ahead, t);
            if (branch) send<B>(to + h_at, h, p.h.ld, ahead, t);
            ahead.next(p, r1);
        }
        copies_sent();
        to = to == base + (kStages - 1) * batch ? base : to + batch;
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) send_next();
    f32x2 gate[4], weight[4], bias[4], post_weight[4];
    if (POST) load_vector(post_weight, Vectors{p.post_weight, 0}, 0, t, 0.f, 1.f);
    uint32_t loaded = 0xffffffffu, at = base;
    while (b.n > 0) {
        if (b.g != loaded) {
            load_vector(gate, p.gate, b.g, t, 0.f, 1.f);
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
        for (int i = 0; i < kRows; ++i) take<S>(v[i], at, i);
        float mean[kRows] = {0.f, 0.f}, inv[kRows] = {1.f, 1.f}, post_mean[kRows] = {0.f, 0.f}, post_inv[kRows] = {1.f, 1.f};
        if (branch) {
            f32x2 u[kRows][4];
#pragma unroll
            for (int i = 0; i < kRows; ++i) take<B>(u[i], at + h_at, i);
            if (POST) moments(t, u, p.post_layer, p.eps, post_mean, post_inv);
            const f32x2 residual = pk2(p.residual, p.residual);
#pragma unroll
            for (int i = 0; i < kRows; ++i) {
                const f32x2 less = pk2(-post_mean[i], -post_mean[i]), s = pk2(post_inv[i], post_inv[i]);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    if (POST) u[i][e] = mul2(mul2(add2(u[i][e], less), s), post_weight[e]);
                    v[i][e] = fma2(residual, v[i][e], mul2(gate[e], u[i][e]));
                }
            }
        }
        send_next();                               // into the place of the batch before this one
        at = at == base + (kStages - 1) * batch ? base : at + batch;
        if (p.x_out.p != nullptr) {
            clear_dead(b, v);
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
            clear_dead(b, v);
            put<B>(y, p.y.ld, b, t, v);
        }
        if (p.stats != nullptr && t.c0 == 0) {
#pragma unroll
            for (int i = 0; i < kRows; ++i)
                if (i < b.n)
                    reinterpret_cast<float4*>(p.stats)[b.row + i] = i < b.live ? make_float4(mean[i], inv[i], post_mean[i], post_inv[i])
                                                                               : make_float4(0.f, 0.f, 0.f, 0.f);
        }
        b.next(p, r1);
    }
}

// Where a group ends (and behind a team's last row) its sums leave: to the gradient itself where the whole group was this team's, else to the
// team's part (the first of its two for the group of its first row, else the second), which gate_norm_sums_kernel joins.
template <typename S, typename B, bool POST, int kStages>
__global__ void __maxnreg__(128) gate_norm_grad_kernel(const GateNormParams p) {
    extern __shared__ uint4 ring[];
    __shared__ float2 room[2 * 32];
    Team t = team_of(p, room);
    const uint32_t team = blockIdx.x, r0 = team * p.chunk, r1 = min(r0 + p.chunk, p.rows);
    griddep_launch();                              // all teams are at work at once: the joining kernel takes no place of theirs
    const uint32_t plane = blockDim.x * 16u, batch = plane * kGradPlanes<S, B>, s_size = plane * kRows * kPlanes<S>, b_size = plane * kRows * kPlanes<B>;
    const uint32_t base = smem_u32(ring), y_at = s_size, d_at = s_size + b_size, h_at = 2 * s_size + b_size;
    const bool normed = p.dy.p != nullptr, gated = p.dgate.p != nullptr, later = p.dx_out.p != nullptr, branch = POST || gated;       // h itself is read
    const char *x = copied<S>(p.x, t), *dy = copied<B>(p.dy, t), *dx_out = copied<S>(p.dx_out, t), *h = copied<B>(p.h, t);
    char *dx = columns<S>(p.dx, t), *dh = columns<B>(p.dh, t);
    Walk b, ahead;
    b.start(p, r0, r1);
    ahead = b;
    uint32_t to = base, at = base;
    auto send_next = [&]() {
        if (ahead.n > 0) {
            if (normed) { send<S>(to, x, p.x.ld, ahead, t); send<B>(to + y_at, dy, p.dy.ld, ahead, t); }
            if (later) send<S>(to + d_at, dx_out, p.dx_out.ld, ahead, t);
            if (branch) send<B>(to + h_at, h, p.h.ld, ahead, t);
            ahead.next(p, r1);
        }
        copies_sent();
        to = to == base + (kStages - 1) * batch ? base : to + batch;
    };
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) send_next();
    f32x2 post_weight[4], dpost[4], gate[4], weight[4], dweight[4], dbias[4], dgate[4];
    fill(dpost, 0.f);
    if (POST) load_vector(post_weight, Vectors{p.post_weight, 0}, 0, t, 0.f, 1.f);
    bool fresh = true, begun = b.g * p.group == r0;            // begun: the group's first row is this team's
    while (b.n > 0) {
        if (fresh) {
            load_vector(gate, p.gate, b.g, t, 0.f, 1.f);
            load_vector(weight, p.weight, b.g, t, p.plus, 1.f);
            fill(dweight, 0.f); fill(dbias, 0.f); fill(dgate, 0.f);
            fresh = false;
        }
        float4 stats[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            stats[i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (i < b.live && (normed || POST)) stats[i] = reinterpret_cast<const float4*>(p.stats)[b.row + i];
        }
        __syncwarp();                              // no lane of the warp still reads the batch before this one
        send_next();                               // into its place
        copies_wait<kStages - 1>();
        if (b.live == 0) {                         // nothing but zeros to write
            put_zeros<S>(dx, p.dx, b, t);
            put_zeros<B>(dh, p.dh, b, t);
        } else {
            f32x2 d[kRows][4];
            if (normed) {
                f32x2 xh[kRows][4];
                float2 s[kRows];
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    const f32x2 less = pk2(-stats[i].x, -stats[i].x), inv = pk2(stats[i].y, stats[i].y);
                    f32x2 a = pk2(0.f, 0.f), c = pk2(0.f, 0.f);
                    take<S>(xh[i], at, i);
                    take<B>(d[i], at + y_at, i);
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
                    take<S>(o, at + d_at, i);
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
                clear_dead(b, o);
                put<S>(dx, p.dx.ld, b, t, o);
            }
            if (POST) {
                f32x2 hh[kRows][4];
                float2 s[kRows];
#pragma unroll
                for (int i = 0; i < kRows; ++i) {
                    const f32x2 less = pk2(-stats[i].z, -stats[i].z), inv = pk2(stats[i].w, stats[i].w);
                    f32x2 a = pk2(0.f, 0.f), c = pk2(0.f, 0.f);
                    take<B>(hh[i], at + h_at, i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        hh[i][e] = mul2(add2(hh[i][e], less), inv);
                        dgate[e] = fma2(d[i][e], hh[i][e], dgate[e]);              // both sums' part: dgate is post_weight times it, dpost gate times it
                        d[i][e] = mul2(mul2(d[i][e], gate[e]), post_weight[e]);
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
                    if (gated) take<B>(o, at + h_at, i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        if (gated) dgate[e] = fma2(d[i][e], o[e], dgate[e]);
                        d[i][e] = mul2(d[i][e], gate[e]);
                    }
                }
            }
            if (p.dh.p != nullptr) {
                clear_dead(b, d);
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
        if (!t.col) continue;
        if (POST) {
#pragma unroll
            for (int e = 0; e < 4; ++e) dpost[e] = fma2(gate[e], dgate[e], dpost[e]);
        }
        if (whole) {
            if (POST && gated) {
#pragma unroll
                for (int e = 0; e < 4; ++e) dgate[e] = mul2(dgate[e], post_weight[e]);
            }
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
    if (POST && p.dpost != nullptr && t.col) Vec8<float>::store_wide(p.post_parts, int64_t(team) * p.cols + t.c0, dpost);
}

// The parts of groups that several teams took, joined in order, and dpost_weight's.  blockIdx.x: heads x `wide` columns of a group (head: the
// group itself, or, where there are more groups than teams, the group at a border of two teams' rows, which the first border inside it takes),
// then the columns of dpost_weight.  Thread = (4 columns, every 1024 / wide'th part).
struct Joins { uint32_t teams, heads, group_ctas, post_ctas; int wide, post_wide, by_group; };         // CTAs: of a head, of dpost_weight
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
#pragma unroll 4
        for (uint32_t i = from + way; i <= to; i += ways) {
            const float4* part = reinterpret_cast<const float4*>(parts + i * step + (second && i == from ? 3 * p.cols : 0));
            if (want0) sum0 = plus(sum0, ld_dependent_cg(part));
            if (want1) sum1 = plus(sum1, ld_dependent_cg(part + p.cols / 4));
            if (want2) sum2 = plus(sum2, ld_dependent_cg(part + p.cols / 2));
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

// ------------------------------------------------------------------------------------------------------------- host

int team_warps(int64_t cols) { return int((cols + 255) / 256); }
constexpr int kGradWarps = 148 * 15;               // warps at a time, on every device: gradients are summed in one order
int64_t grad_chunk(int64_t rows, int64_t cols) {
    const int64_t teams = kGradWarps / team_warps(cols), chunk = (rows + teams - 1) / teams;
    return chunk < 2 * kRows ? 2 * kRows : chunk;
}
hq_status check_matrix(const void* x, int64_t ld, int64_t cols, hq_dtype dt) {
    if (x == nullptr) return HQ_ERR_INVALID_ARG;
    if (ld < cols) return HQ_ERR_SHAPE;
    if (!aligned16(x) || (ld * (dt == HQ_BF16 ? 2 : 4)) % 16 != 0) return HQ_ERR_ALIGNMENT;
    return ld < int64_t(1) << 30 ? HQ_OK : HQ_ERR_UNSUPPORTED;             // a pitch in bytes has 32 bits
}
Matrix matrix(const void* p, int64_t ld, hq_dtype dt) { return Matrix{p, p != nullptr ? uint32_t(ld) * (dt == HQ_BF16 ? 2u : 4u) : 0u}; }
MatrixOut matrix_out(void* p, int64_t ld, hq_dtype dt) { return MatrixOut{p, p != nullptr ? uint32_t(ld) * (dt == HQ_BF16 ? 2u : 4u) : 0u}; }
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

struct Launch { unsigned grid, threads; };
cudaError_t launch_kernel(void (*kern)(GateNormParams), const GateNormParams& p, Launch l, int planes, int stages, cudaStream_t st) {
    const size_t smem = size_t(planes) * stages * l.threads * 16;
    const cudaError_t e = smem <= 40 * 1024 ? cudaSuccess : cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(smem));
    if (e != cudaSuccess) { (void)cudaGetLastError(); return e; }
    kern<<<l.grid, l.threads, smem, st>>>(p);
    return cudaGetLastError();
}
template <typename S, typename B>
cudaError_t launch_forward(const GateNormParams& p, bool post, Launch l, cudaStream_t st) {
    return launch_kernel(post ? gate_norm_kernel<S, B, true> : gate_norm_kernel<S, B, false>, p, l, kForwardPlanes<S, B>, kForwardStages, st);
}
template <typename S, typename B>
cudaError_t launch_grad(const GateNormParams& p, bool post, Launch l, cudaStream_t st) {
    if constexpr (sizeof(S) + sizeof(B) == 8) {    // the widest rows of fp32 on both sides: 256 KB in two stages
        if (size_t(kGradPlanes<S, B>) * kGradStages * l.threads * 16 > kMostShared)
            return launch_kernel(post ? gate_norm_grad_kernel<S, B, true, 1> : gate_norm_grad_kernel<S, B, false, 1>, p, l, kGradPlanes<S, B>, 1, st);
    }
    return launch_kernel(post ? gate_norm_grad_kernel<S, B, true, kGradStages> : gate_norm_grad_kernel<S, B, false, kGradStages>, p, l, kGradPlanes<S, B>,
                         kGradStages, st);
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
    p.rows = uint32_t(rows); p.group = uint32_t(group < rows ? group : rows); p.cols = int(cols); p.warps = team_warps(cols); p.lens = lens;
    p.layer = norm == HQ_NORM_LAYER; p.post_layer = post == HQ_NORM_LAYER; p.post_weight = post_weight;
    p.gate = Vectors{gate, ld_gate}; p.weight = Vectors{weight, ld_weight}; p.bias = Vectors{bias, ld_bias};
    p.residual = residual_scale; p.plus = weight_plus; p.eps = eps; p.stats = stats;
    p.x = matrix(x, ldx, xdt); p.h = matrix(h, ldh, hdt); p.x_out = matrix_out(x_out, ldx_out, xdt); p.y = matrix_out(y, ldy, hdt);
    // teams at a time: 96 registers leave room for 20 warps an SM, the rows on their way for as many as share 224 KB
    const int planes = kRows * ((xdt == HQ_BF16 ? 1 : 2) + (hdt == HQ_BF16 ? 1 : 2));
    const int64_t fit = int64_t(kMostShared / (size_t(planes) * kForwardStages * p.warps * 32 * 16)), by_warps = 20 / p.warps;
    const int64_t most = int64_t(sm_count()) * (fit < by_warps ? fit : by_warps), chunk = (rows + most - 1) / most;
    p.chunk = uint32_t(chunk < kRows ? kRows : chunk);
    const Launch l{unsigned((rows + p.chunk - 1) / p.chunk), unsigned(p.warps * 32)};
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const bool after = post != HQ_NORM_NONE;
    cudaError_t c;
    if (xdt == HQ_BF16) c = hdt == HQ_BF16 ? launch_forward<__nv_bfloat16, __nv_bfloat16>(p, after, l, st) : launch_forward<__nv_bfloat16, float>(p, after, l, st);
    else c = hdt == HQ_BF16 ? launch_forward<float, __nv_bfloat16>(p, after, l, st) : launch_forward<float, float>(p, after, l, st);
    return c == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}

extern "C" hq_status hq_gate_norm_bwd_workspace_size(int64_t rows, int64_t cols, int64_t rows_per_group, size_t* bytes) {
    using namespace hq;
    if (bytes == nullptr) return HQ_ERR_INVALID_ARG;
    int64_t group = 0;
    const hq_status e = check_sizes(HQ_BF16, HQ_BF16, rows, cols, rows_per_group, nullptr, HQ_NORM_NONE, nullptr, HQ_NORM_NONE, nullptr, nullptr, 1.f, &group);
    if (e != HQ_OK) return e;
    const int64_t chunk = grad_chunk(rows, cols), teams = (rows + chunk - 1) / chunk;
    *bytes = size_t(teams) * 7 * size_t(cols) * sizeof(float);
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
    p.rows = uint32_t(rows); p.group = uint32_t(group < rows ? group : rows); p.cols = int(cols); p.warps = team_warps(cols); p.lens = lens;
    p.chunk = uint32_t(grad_chunk(rows, cols));
    const int64_t teams = (rows + p.chunk - 1) / p.chunk;
    const bool sums = dgate != nullptr || dweight != nullptr || dbias != nullptr;
    // parts are for groups that several teams took; without a sum over rows, or where every group is one team's, there are none
    const bool split = sums && p.chunk % p.group != 0 && teams > 1;
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
    // columns a CTA: as many as leave a thread two parts or more
    auto wide_for = [](int64_t parts) { int wide = 1024; while (wide > 32 && parts > 1024 / wide * 2) wide /= 2; return wide; };
    j.wide = wide_for(p.group / p.chunk + 2);
    j.post_wide = wide_for(teams);
    j.group_ctas = uint32_t((cols + j.wide - 1) / j.wide);
    j.post_ctas = dpost_weight != nullptr ? uint32_t((cols + j.post_wide - 1) / j.post_wide) : 0u;
    return launch_dependent(gate_norm_sums_kernel, dim3(j.heads * j.group_ctas + j.post_ctas), 256, 0, st, true, p, j) == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}
