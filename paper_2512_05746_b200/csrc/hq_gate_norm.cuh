// What the gated residual with its norms (hq_gate_norm.cu) and its gradient (hq_gate_norm_bwd.cu) have in common: a team's walk over its rows, its
// sums, the rows on their way through shared memory, and the checks of the calls.
#pragma once

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
// BATCH: rows of a batch, kRows for each row that stands side by side in a warp.
template <int BATCH> struct Walk {
    uint32_t row, g;
    int left, alive, n, live;
    __device__ __forceinline__ void enter(const GateNormParams& p, uint32_t behind) {        // behind: rows of the group in front of `row`
        left = int(min(p.group - behind, p.rows - row));
        alive = p.lens != nullptr && left > 0 ? min(max(p.lens[g], 0) - int(behind), left) : left;       // below zero by a group's rows at most
    }
    __device__ __forceinline__ void count(uint32_t end) {
        n = min(min(BATCH, left), int(end - row));
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
template <int L> struct Team {                     // L lanes a row; fewer than 32: one warp, 32 / L rows side by side
    static constexpr int kSide = 32 / L, kBatch = kRows * kSide;
    using Walk = hq::Walk<kBatch>;
    int lane, place, side, warp, warps, c0, cols;  // place: the lane's in its row; side: its row's number
    bool col;                                      // the thread has columns
    float share, per_warp, per_row;                // columns of warp (lane & 15); 1 / columns of this warp, of the row
    float2* room;                                  // [2][32]
    int turn;
};
template <int L> __device__ __forceinline__ Team<L> team_of(const GateNormParams& p, float2* room) {
    Team<L> t;
    t.lane = int(threadIdx.x & 31);
    t.place = L == 32 ? t.lane : t.lane % L;
    t.side = L == 32 ? 0 : t.lane / L;
    t.warps = p.warps;
    t.warp = int(threadIdx.x >> 5);
    t.c0 = L == 32 ? (t.warp * 32 + t.lane) * 8 : t.place * 8;
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

// Over the L lanes of a row, in every one of them.
template <int L> __device__ __forceinline__ float row_sum(float x) {
#pragma unroll
    for (int off = L / 2; off > 0; off >>= 1) x = xor_add(x, off);
    return x;
}

// The sums of a pair of values of each of two rows over the team.
template <int L> __device__ __forceinline__ void team_sums(Team<L>& t, float2& a, float2& b) {
    if constexpr (L < 32) {
        a = make_float2(row_sum<L>(a.x), row_sum<L>(a.y));
        b = make_float2(row_sum<L>(b.x), row_sum<L>(b.y));
        return;
    }
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
template <int L>
__device__ __forceinline__ void moments(Team<L>& t, const f32x2 (&v)[kRows][4], int layer, float eps, float (&mean)[kRows], float (&inv)[kRows]) {
    float m = 0.f;                                 // of row lane / 16
    mean[0] = mean[1] = 0.f;
    if (L < 32 && layer) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) mean[i] = row_sum<L>(t.col ? sum8(v[i]) : 0.f) * t.per_row;
    } else if (layer) {
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
    if constexpr (L < 32) {
#pragma unroll
        for (int i = 0; i < kRows; ++i) inv[i] = rsqrtf(row_sum<L>(q[i]) * t.per_row + eps);
        return;
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
template <int L>
__device__ __forceinline__ void load_vector(f32x2 (&v)[4], const Vectors& from, uint32_t g, const Team<L>& t, float add, float none) {
    if (from.p == nullptr || !t.col) { fill(v, none); return; }
    const float4* q = reinterpret_cast<const float4*>(from.p + int64_t(g) * from.ld + t.c0);
    const float4 a = q[0], b = q[1];
    v[0] = pk2(a.x + add, a.y + add); v[1] = pk2(a.z + add, a.w + add); v[2] = pk2(b.x + add, b.y + add); v[3] = pk2(b.z + add, b.w + add);
}

// The same asked for ahead of its use: rows with vectors of their own wait for them one by one (32768 x 1152 bf16, a vector triple a row, 193 -> 154 us,
// gradient 268 -> 221).
template <int L>
__device__ __forceinline__ void ask_for_vector(const Vectors& from, uint32_t g, const Team<L>& t) {
    if (from.p != nullptr && t.col) asm volatile("prefetch.global.L2 [%0];" ::"l"(from.p + int64_t(g) * from.ld + t.c0));
}
template <int L>
__device__ __forceinline__ void times_vector(f32x2 (&v)[4], const float* by, const Team<L>& t) {
    f32x2 w[4];
    load_vector(w, Vectors{by, 0}, 0, t, 0.f, 1.f);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = mul2(v[e], w[e]);
}

// ---- rows on their way through shared memory: a thread's 16 or 32 bytes of a row, in planes of 16 bytes a lane, 512 bytes a plane; each warp
// copies its own.  Neighbouring lanes copy neighbouring 16 bytes; of fp32 they are another lane's of the warp (copied by their own lane, half of
// every sector would be asked for twice) ----
template <typename T> constexpr int kPlanes = int(sizeof(T)) * 8 / 16;
constexpr uint32_t kPlane = 512;
__device__ __forceinline__ void copy_bytes(uint32_t to, const void* from, uint32_t bytes) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(bytes) : "memory");
}
__device__ __forceinline__ void copies_sent() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
    __syncwarp();
}
__device__ __forceinline__ uint64_t row_at(uint32_t row, uint32_t ld) { return uint64_t(row) * ld; }

// What a thread copies of a row of T: pieces of 16 bytes (two of fp32: number k * L + place of the row's 2 L in this warp, that of lane piece / 2,
// plane piece % 2), with their bytes (0 behind the last column) and places.
template <typename T, int L> struct Pieces {
    uint32_t to, bytes[kPlanes<T>], apart;         // apart: from the first to the second in the row (0 where that has no columns)
    int first;                                     // bytes from the row's beginning (0 behind the last column)
    __device__ __forceinline__ explicit Pieces(const Team<L>& t) {
        if constexpr (sizeof(T) == 2) {
            to = uint32_t(t.lane) * 16u;
            bytes[0] = t.col ? 16u : 0u;
            first = t.col ? t.c0 * 2 : 0;
            apart = 0;
        } else {
            const int c = t.warp * 256 + t.place * 4;
            to = uint32_t(t.lane & 1) * kPlane + uint32_t((t.lane & ~(L - 1)) + t.place / 2) * 16u;
            bytes[0] = c < t.cols ? 16u : 0u;
            bytes[1] = c + L * 4 < t.cols ? 16u : 0u;
            first = c < t.cols ? c * 4 : 0;
            apart = c + L * 4 < t.cols ? uint32_t(L) * 16u : 0u;
        }
    }
};
// `at`: the warp's first plane of the matrix; from: the matrix's first row, at this thread's first piece; zeros for rows that are not there.
template <typename T, int L>
__device__ __forceinline__ void send(uint32_t at, const char* from, uint32_t ld, const typename Team<L>::Walk& b, const Team<L>& t, const Pieces<T, L>& mine) {
    const char* base = from + row_at(b.row, ld);
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
        const uint32_t r = uint32_t(i * Team<L>::kSide + t.side);
        const bool live = int(r) < b.live;
        const char* row = L == 32 && i == 0 ? base : base + (live ? r * uint64_t(ld) : 0u);
        copy_bytes(at + mine.to + uint32_t(i * kPlanes<T>) * kPlane, row, live ? mine.bytes[0] : 0u);
        if constexpr (sizeof(T) == 4)
            copy_bytes(at + mine.to + uint32_t(i * 2) * kPlane + uint32_t(L) * 8u, row + mine.apart, live ? mine.bytes[1] : 0u);
    }
}
__device__ __forceinline__ uint4 plane_at(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
    return v;
}
// This lane's columns of row i; `at`: the lane's place in the matrix's first plane.
template <typename T>
__device__ __forceinline__ void take(f32x2 (&v)[4], uint32_t at, int i) {
    Vec8<T> raw;
    if constexpr (sizeof(T) == 2) {
        raw.w = plane_at(at + uint32_t(i) * kPlane);
    } else {
        const uint4 a = plane_at(at + uint32_t(2 * i) * kPlane), b = plane_at(at + uint32_t(2 * i + 1) * kPlane);
        raw.a = make_float4(__uint_as_float(a.x), __uint_as_float(a.y), __uint_as_float(a.z), __uint_as_float(a.w));
        raw.b = make_float4(__uint_as_float(b.x), __uint_as_float(b.y), __uint_as_float(b.z), __uint_as_float(b.w));
    }
    raw.get(v);
}
template <typename T, int L> __device__ __forceinline__ char* columns(const MatrixOut& m, const Team<L>& t) { return static_cast<char*>(m.p) + t.c0 * int(sizeof(T)); }
__device__ __forceinline__ const char* copied(const Matrix& m, int first) { return static_cast<const char*>(m.p) + first; }

// Rows that are not there leave as zeros.
template <int L>
__device__ __forceinline__ void clear_dead(const typename Team<L>::Walk& b, const Team<L>& t, f32x2 (&v)[kRows][4]) {
    if (b.live == b.n) return;
#pragma unroll
    for (int i = 0; i < kRows; ++i)
        if (i * Team<L>::kSide + t.side >= b.live) fill(v[i], 0.f);
}
template <typename T, int L>
__device__ __forceinline__ void put(char* to, uint32_t ld, const typename Team<L>::Walk& b, const Team<L>& t, const f32x2 (&v)[kRows][4]) {
    char* row = to + row_at(b.row, ld) + (L == 32 ? 0u : uint32_t(t.side) * uint64_t(ld));
    if (t.col && (L == 32 || t.side < b.n)) Vec8<T>::store_wide(row, 0, v[0]);                 // a batch has a row
    if (t.col && Team<L>::kSide + t.side < b.n) Vec8<T>::store_wide(row + Team<L>::kSide * uint64_t(ld), 0, v[1]);
}
template <typename T, int L>
__device__ __forceinline__ void put_zeros(char* to, const MatrixOut& m, const typename Team<L>::Walk& b, const Team<L>& t) {
    if (m.p == nullptr) return;
    f32x2 v[kRows][4];
#pragma unroll
    for (int i = 0; i < kRows; ++i) fill(v[i], 0.f);
    put<T>(to, m.ld, b, t, v);
}

// A sum over the rows that stand side by side, in every lane of the column.
template <int L> __device__ __forceinline__ void side_sums(f32x2 (&v)[4]) {
#pragma unroll
    for (int off = L; off < 32; off *= 2) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = add2(v[e], __shfl_xor_sync(0xffffffffu, v[e], off));
    }
}

// Batches in shared memory: one is computed, the others are on their way (40 KB an SM keep the copy rate; 80 KB of bf16 in the forward, 60 in
// the gradient).
template <typename S, typename B> constexpr int kForwardPlanes = kRows * (kPlanes<S> + kPlanes<B>);
template <typename S, typename B> constexpr int kGradPlanes = 2 * kForwardPlanes<S, B>;
constexpr int kForwardStages = 3, kGradStages = 2;
constexpr size_t kMostShared = 224 * 1024;

// ------------------------------------------------------------------------------------------------------------- host

inline int team_warps(int64_t cols) { return int((cols + 255) / 256); }
inline hq_status check_matrix(const void* x, int64_t ld, int64_t cols, hq_dtype dt) {
    if (x == nullptr) return HQ_ERR_INVALID_ARG;
    if (ld < cols) return HQ_ERR_SHAPE;
    if (!aligned16(x) || (ld * (dt == HQ_BF16 ? 2 : 4)) % 16 != 0) return HQ_ERR_ALIGNMENT;
    return ld < int64_t(1) << 30 ? HQ_OK : HQ_ERR_UNSUPPORTED;             // a pitch in bytes has 32 bits
}
// In place: rows at other places than the input's are rows that are still to be read.
inline bool in_place_apart(const void* out, int64_t ld_out, const void* in, int64_t ld_in, int64_t rows) {
    return out != nullptr && out == in && ld_out != ld_in && rows > 1;
}
inline Matrix matrix(const void* p, int64_t ld, hq_dtype dt) { return Matrix{p, p != nullptr ? uint32_t(ld) * (dt == HQ_BF16 ? 2u : 4u) : 0u}; }
inline MatrixOut matrix_out(void* p, int64_t ld, hq_dtype dt) { return MatrixOut{p, p != nullptr ? uint32_t(ld) * (dt == HQ_BF16 ? 2u : 4u) : 0u}; }
inline hq_status check_vectors(const float* v, int64_t ld, int64_t groups, int64_t cols) {
    if (v == nullptr) return HQ_OK;
    if (groups > 1 && ld < cols) return HQ_ERR_SHAPE;
    return aligned16(v) && (groups <= 1 || ld % 4 == 0) ? HQ_OK : HQ_ERR_ALIGNMENT;
}
inline bool type_ok(hq_dtype t) { return t == HQ_F32 || t == HQ_BF16; }
inline bool norm_ok(hq_norm n) { return n == HQ_NORM_LAYER || n == HQ_NORM_RMS || n == HQ_NORM_NONE; }
// What both calls check of their sizes; *group: rows of a group.
inline hq_status check_sizes(hq_dtype xdt, hq_dtype hdt, int64_t rows, int64_t cols, int64_t rows_per_group, const int32_t* lens, hq_norm post,
                      const float* post_weight, hq_norm norm, const void* h, const void* gate, float residual, int64_t* group) {
    if (!type_ok(xdt) || !type_ok(hdt) || !norm_ok(post) || !norm_ok(norm)) return HQ_ERR_INVALID_ARG;
    if (rows < 0 || cols <= 0 || rows_per_group < 0) return HQ_ERR_SHAPE;
    if (cols % 8 != 0 || cols > kMaxCols || rows > 0x7fffffff) return HQ_ERR_UNSUPPORTED;
    if (lens != nullptr && rows_per_group == 0) return HQ_ERR_INVALID_ARG;
    if (post == HQ_NORM_NONE && post_weight != nullptr) return HQ_ERR_INVALID_ARG;
    if (!aligned16(post_weight)) return HQ_ERR_ALIGNMENT;
    if (!(residual - residual == 0.f)) return HQ_ERR_INVALID_ARG;
    if (h == nullptr && (post != HQ_NORM_NONE || gate != nullptr || residual != 1.f)) return HQ_ERR_INVALID_ARG;
    *group = rows_per_group > 0 && rows_per_group < rows ? rows_per_group : rows > 0 ? rows : 1;        // one group: at most all rows
    return HQ_OK;
}

// Lanes of a row: fewer than a warp's for narrow ones.
inline int row_lanes(int64_t cols) { return cols <= 64 ? 8 : cols <= 128 ? 16 : 32; }
struct Launch { unsigned grid, threads; };
inline cudaError_t launch_kernel(void (*kern)(GateNormParams), const GateNormParams& p, Launch l, int planes, int stages, cudaStream_t st) {
    const size_t smem = size_t(planes) * stages * l.threads * 16;
    // one value whatever the call needs: another host thread's call of the same kernel may set it between these two
    const cudaError_t e = smem <= 40 * 1024 ? cudaSuccess : cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kMostShared));
    if (e != cudaSuccess) { (void)cudaGetLastError(); return e; }
    kern<<<l.grid, l.threads, smem, st>>>(p);
    return cudaGetLastError();
}

}  // namespace
}  // namespace hq
