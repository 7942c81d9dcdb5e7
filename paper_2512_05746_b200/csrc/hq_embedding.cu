// Embedding lookup with scaling, and the gradient of its table by sorted tokens.
//
//   out[t] = scale table[id[t]]                    a row of zeros for an id outside the table
//   dtable[v] = base[v] + scale sum of dout[t] over the tokens t of id v, in ascending order, in fp32
//
// Memory-bound: the lookup reads ids and rows and writes rows; the gradient reads every token's row once and writes every row of the table once.
//
// The gradient has three kernels.  (1) order: CTA b owns a slice of the ids, reads all ids once, keeps the tokens of its slice in their order
// and counts those of smaller ids (where its part of the sorted order begins), then sorts its tokens by id with one stable counting sort:
// no atomics, so the order is the same on every run.  (2) sums: the sorted tokens are cut into spans of equal length, whatever ids they
// hold (most tokens may be of one id); a team of threads adds up a span's rows with several rows in flight and writes a row of the table
// whenever the id changes.  The first and the last sum of a span go to the workspace where their id goes on in the spans beside it; CTAs
// behind the spans fill the rows without tokens.  (3) join: ids that lie in several spans, the parts in order.
#include <climits>

#include "hq_common.cuh"
#include "hq_vec8.cuh"

namespace hq {
namespace {

// ---------------------------------------------------------------------------------------------------------- lookup

template <typename I> __device__ __forceinline__ int64_t id_at(const void* ids, int64_t t) { return int64_t(__ldg(static_cast<const I*>(ids) + t)); }

struct LookupParams { const void *ids, *table; void* out; int64_t tokens, classes, ld_table, ld_out; int vectors; float scale; };

// A thread takes 8 channels of kTogether tokens at a time (ids first, then the rows, then the stores).
template <typename I, typename T, typename U>
__global__ void __launch_bounds__(256) embedding_kernel(const LookupParams p) {
    constexpr int kTogether = 4;
    const uint32_t lane_token = threadIdx.x / uint32_t(p.vectors), slots = 256u / uint32_t(p.vectors);       // tokens of a CTA's step
    const f32x2 s = pk2(p.scale, p.scale);
    // wide rows (more vectors than threads): a CTA a token, its threads over the row
    if (slots == 0) {
        for (int64_t t = blockIdx.x; t < p.tokens; t += gridDim.x) {
            const int64_t id = id_at<I>(p.ids, t);
            const bool there = id >= 0 && id < p.classes;
            for (int v = int(threadIdx.x); v < p.vectors; v += 256) {
                Vec8<T> x;
                x.clear();
                if (there) x.load(p.table, id * p.ld_table + v * 8);
                f32x2 f[4];
                x.get(f);
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = mul2(f[e], s);
                if (!there) f[0] = f[1] = f[2] = f[3] = pk2(0.f, 0.f);
                Vec8<U>::store(p.out, t * p.ld_out + v * 8, f);
            }
        }
        return;
    }
    if (lane_token >= slots) return;
    const int c0 = int(threadIdx.x - lane_token * uint32_t(p.vectors)) * 8;
    const int64_t step = int64_t(gridDim.x) * slots;
    for (int64_t t0 = int64_t(blockIdx.x) * slots + lane_token; t0 < p.tokens; t0 += step * kTogether) {
        int64_t id[kTogether];
        Vec8<T> x[kTogether];
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int64_t t = t0 + u * step;
            id[u] = t < p.tokens ? id_at<I>(p.ids, t) : -1;
        }
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            x[u].clear();
            if (id[u] >= 0 && id[u] < p.classes) x[u].load(p.table, id[u] * p.ld_table + c0);
        }
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int64_t t = t0 + u * step;
            if (t >= p.tokens) break;
            f32x2 f[4];
            x[u].get(f);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = mul2(f[e], s);
            Vec8<U>::store(p.out, t * p.ld_out + c0, f);
        }
    }
}

// -------------------------------------------------------------------------------------------------------- gradient

constexpr int kOrderThreads = 1024;
constexpr int kOrderWarps = kOrderThreads / 32;
constexpr int kSlice = kOrderThreads;              // ids a CTA of the order at most: a thread each in the scan, 128 KB of counters

struct GradParams {
    const void* ids;
    const void *dout, *base;
    void* dtable;
    int64_t ld_dout, ld_base, ld_dtable, classes;
    uint32_t tokens, slice;                        // slice: ids of an order CTA
    uint32_t span, longest, spans, span_ctas;      // positions of a span; tokens of the longest id that one span takes whole
    int vectors;
    float scale;
    uint2 *found, *sorted;                         // [tokens] (id in the slice, token) as found; (id, token) by id
    uint32_t* start;                               // [classes + 1] first position of each id
    float* parts;                                  // [spans][first, last][dim]
};

__device__ __forceinline__ uint32_t lanes_below() { uint32_t m; asm("mov.u32 %0, %%lanemask_lt;" : "=r"(m)); return m; }

// Exclusive sum of x over the CTA's threads; *total is the whole.  One barrier in front of its use of `room` and one behind.
__device__ __forceinline__ uint32_t exclusive_sum(uint32_t x, uint32_t* room, uint32_t* total) {
    const int lane = int(threadIdx.x & 31), warp = int(threadIdx.x >> 5);
    uint32_t sum = x;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const uint32_t o = __shfl_up_sync(0xffffffffu, sum, off);
        if (lane >= off) sum += o;
    }
    __syncthreads();
    if (lane == 31) room[warp] = sum;
    __syncthreads();
    uint32_t before = lane < warp ? room[lane] : 0u, all = room[lane];
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) {
        before += __shfl_xor_sync(0xffffffffu, before, off);
        all += __shfl_xor_sync(0xffffffffu, all, off);
    }
    *total = all;
    return before + sum - x;
}

template <typename I>
__global__ void __launch_bounds__(kOrderThreads) embedding_order_kernel(const GradParams p) {
    extern __shared__ uint32_t counts[];           // [warp][id of the slice]
    __shared__ uint32_t room[kOrderWarps], offset[kSlice];
    constexpr int kAhead = 8;
    const int lane = int(threadIdx.x & 31), warp = int(threadIdx.x >> 5);
    const int64_t v0 = int64_t(blockIdx.x) * p.slice, v1 = min(v0 + int64_t(p.slice), p.classes);
    const uint32_t size = uint32_t(v1 - v0);
    // a warp's run of ids, read twice: how many are of the slice and how many smaller; then where they go
    const uint32_t run = (p.tokens + kOrderThreads - 1) / kOrderThreads * 32, from = min(uint32_t(warp) * run, p.tokens), to = min(from + run, p.tokens);
    uint32_t mine = 0, less = 0;
    for (uint32_t t0 = from + lane; t0 < to; t0 += 32 * kAhead) {
        int64_t id[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) id[u] = t0 + 32 * u < to ? id_at<I>(p.ids, t0 + 32 * u) : -1;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            less += id[u] >= 0 && id[u] < v0;
            mine += id[u] >= v0 && id[u] < v1;
        }
    }
    uint32_t n, first;
    (void)exclusive_sum(less, room, &first);       // the slice's first position
    const uint32_t at = exclusive_sum(mine, room, &n);
    uint32_t to_here = __shfl_sync(0xffffffffu, at, 0);        // the warp's
    for (uint32_t t0 = from; t0 < to; t0 += 32 * kAhead) {
        int64_t id[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) id[u] = t0 + 32 * u + lane < to ? id_at<I>(p.ids, t0 + 32 * u + lane) : -1;
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const bool here = id[u] >= v0 && id[u] < v1;
            const uint32_t who = __ballot_sync(0xffffffffu, here);
            if (here) p.found[first + to_here + __popc(who & lanes_below())] = make_uint2(uint32_t(id[u] - v0), t0 + 32 * u + lane);
            to_here += __popc(who);
        }
    }
    for (uint32_t i = threadIdx.x; i < uint32_t(kOrderWarps) * size; i += kOrderThreads) counts[i] = 0;
    __syncthreads();
    // the slice's tokens, a run for each warp: counted by id, then placed
    const uint2* list = p.found + first;
    const uint32_t part = (n + kOrderThreads - 1) / kOrderThreads * 32, begin = min(uint32_t(warp) * part, n), end = min(begin + part, n);
    uint32_t* count = counts + uint32_t(warp) * size;
    constexpr int kBatch = 4;
    for (uint32_t j0 = begin; j0 < end; j0 += 32 * kBatch) {
        uint32_t key[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) key[u] = j0 + 32 * u + lane < end ? list[j0 + 32 * u + lane].x : 0xffffffffu;
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const uint32_t same = __match_any_sync(0xffffffffu, key[u]);
            if (key[u] != 0xffffffffu && (same & lanes_below()) == 0) count[key[u]] += __popc(same);
            __syncwarp();
        }
    }
    __syncthreads();
    uint32_t sum = 0;
    if (threadIdx.x < size) {
        for (int w = 0; w < kOrderWarps; ++w) {
            const uint32_t c = counts[uint32_t(w) * size + threadIdx.x];
            counts[uint32_t(w) * size + threadIdx.x] = sum;
            sum += c;
        }
    }
    uint32_t all;
    const uint32_t begins = exclusive_sum(sum, room, &all);
    if (threadIdx.x < size) {
        offset[threadIdx.x] = begins;
        p.start[v0 + threadIdx.x] = first + begins;
    }
    if (v1 == p.classes && threadIdx.x == 0) p.start[p.classes] = first + n;
    __syncthreads();
    for (uint32_t j0 = begin; j0 < end; j0 += 32 * kBatch) {
        uint2 e[kBatch];
#pragma unroll
        for (int u = 0; u < kBatch; ++u) e[u] = j0 + 32 * u + lane < end ? list[j0 + 32 * u + lane] : make_uint2(0xffffffffu, 0u);
#pragma unroll
        for (int u = 0; u < kBatch; ++u) {
            const uint32_t same = __match_any_sync(0xffffffffu, e[u].x), rank = __popc(same & lanes_below());
            if (e[u].x != 0xffffffffu) {
                p.sorted[first + offset[e[u].x] + count[e[u].x] + rank] = make_uint2(uint32_t(v0) + e[u].x, e[u].y);
            }
            __syncwarp();
            if (e[u].x != 0xffffffffu && rank == 0) count[e[u].x] += __popc(same);
            __syncwarp();
        }
    }
}

__device__ __forceinline__ uint32_t ld_dependent_u32(const uint32_t* p) {
    uint32_t v;
    asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

// Row v of the table from the sum of its tokens' rows.
template <typename U>
__device__ __forceinline__ void write_row(const GradParams& p, uint32_t v, int c0, const f32x2 (&sum)[4]) {
    const f32x2 s = pk2(p.scale, p.scale);
    f32x2 f[4];
    if (p.base != nullptr) {
        Vec8<U> b;
        b.load(p.base, int64_t(v) * p.ld_base + c0);
        b.get(f);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = fma2(sum[e], s, f[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = mul2(sum[e], s);
    }
    Vec8<U>::store(p.dtable, int64_t(v) * p.ld_dtable + c0, f);
}

// blockIdx.x: spans, then the rows without tokens; y: 256 vectors of 8 channels.
template <typename T, typename U>
__global__ void __launch_bounds__(256) embedding_sums_kernel(const GradParams p) {
    constexpr int kAhead = 8;
    const int across = min(p.vectors - int(blockIdx.y) * 256, 256), slots = 256 / across, slot = int(threadIdx.x) / across;
    if (slot >= slots) return;
    const int c0 = (int(blockIdx.y) * 256 + int(threadIdx.x) - slot * across) * 8;
    griddep_wait();
    if (blockIdx.x >= p.span_ctas) {               // rows without tokens
        constexpr int kTogether = 4;
        const int64_t step = int64_t(gridDim.x - p.span_ctas) * slots;
        for (int64_t r0 = int64_t(blockIdx.x - p.span_ctas) * slots + slot; r0 < p.classes; r0 += step * kTogether) {
            bool empty[kTogether];
            Vec8<U> b[kTogether];
#pragma unroll
            for (int u = 0; u < kTogether; ++u) {
                const int64_t v = r0 + u * step;
                empty[u] = v < p.classes && ld_dependent_u32(p.start + v) == ld_dependent_u32(p.start + v + 1);
            }
#pragma unroll
            for (int u = 0; u < kTogether; ++u) {
                b[u].clear();
                if (empty[u] && p.base != nullptr) b[u].load(p.base, (r0 + u * step) * p.ld_base + c0);
            }
#pragma unroll
            for (int u = 0; u < kTogether; ++u) {
                if (!empty[u]) continue;
                f32x2 f[4];
                b[u].get(f);
                Vec8<U>::store(p.dtable, (r0 + u * step) * p.ld_dtable + c0, f);
            }
        }
        return;
    }
    const uint32_t s = blockIdx.x * uint32_t(slots) + uint32_t(slot), n = ld_dependent_u32(p.start + p.classes);
    uint32_t a = s * p.span, b = min(a + p.span, n);
    if (s >= p.spans || a >= b) return;
    // an id of at most `longest` tokens belongs to the span of its first one, whole; a longer one to every span that it lies in
    bool open_left = false, open_right = false;
    {
        const uint32_t id0 = ld_dependent_cg(p.sorted + a).x, id1 = ld_dependent_cg(p.sorted + b - 1).x;
        const uint32_t begin0 = ld_dependent_u32(p.start + id0), end0 = ld_dependent_u32(p.start + id0 + 1);
        const uint32_t begin1 = ld_dependent_u32(p.start + id1), end1 = ld_dependent_u32(p.start + id1 + 1);
        if (begin0 < a) {
            if (end0 - begin0 <= p.longest) a = end0;
            else open_left = true;
        }
        if (a >= b) return;
        if (end1 > b) {
            if (end1 - begin1 <= p.longest) b = end1;
            else open_right = true;
        }
    }
    f32x2 sum[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) sum[e] = pk2(0.f, 0.f);
    uint32_t now = 0xffffffffu;
    auto leave = [&](bool left, bool right) {
        if (!left && !right) { write_row<U>(p, now, c0, sum); return; }
        float* to = p.parts + (int64_t(s) * 2 + (left ? 0 : 1)) * p.vectors * 8 + c0;
        Vec8<float>::store(to, 0, sum);
    };
    for (uint32_t j = a; j < b; j += kAhead) {
        uint2 e[kAhead];
        Vec8<T> x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) e[u] = j + u < b ? ld_dependent_cg(p.sorted + j + u) : make_uint2(0u, 0u);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            x[u].clear();
            if (j + u < b) x[u].load(p.dout, int64_t(e[u].y) * p.ld_dout + c0);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (j + u >= b) break;
            if (e[u].x != now) {
                if (now != 0xffffffffu) { leave(open_left, false); open_left = false; }
                now = e[u].x;
#pragma unroll
                for (int k = 0; k < 4; ++k) sum[k] = pk2(0.f, 0.f);
            }
            f32x2 f[4];
            x[u].get(f);
#pragma unroll
            for (int k = 0; k < 4; ++k) sum[k] = add2(sum[k], f[k]);
        }
    }
    leave(open_left, open_right);
}

// Ids that lie in several spans.  blockIdx.x: kJoinSpans spans, of which those whose last id begins there and goes on are looked at; y: 32
// channels.  Thread = (4 channels, every 32nd part).
constexpr int kJoinSpans = 16;
template <typename U>
__global__ void __launch_bounds__(256) embedding_join_kernel(const GradParams p) {
    __shared__ uint32_t whose[kJoinSpans];
    __shared__ f32x2 sums[256][2];
    griddep_wait();
    const uint32_t n = ld_dependent_u32(p.start + p.classes), s0 = blockIdx.x * kJoinSpans;
    if (threadIdx.x < kJoinSpans) {
        const uint32_t s = s0 + threadIdx.x, a = s * p.span, b = a + p.span;
        uint32_t id = 0xffffffffu;
        if (s < p.spans && b < n) {
            id = ld_dependent_cg(p.sorted + b - 1).x;
            const uint32_t begin = ld_dependent_u32(p.start + id), end = ld_dependent_u32(p.start + id + 1);
            if (begin < a || end <= b || end - begin <= p.longest) id = 0xffffffffu;
        }
        whose[threadIdx.x] = id;
    }
    __syncthreads();
    const int group = int(threadIdx.x & 7), way = int(threadIdx.x >> 3), c = int(blockIdx.y) * 32 + group * 4, dim = p.vectors * 8;
    for (int k = 0; k < kJoinSpans; ++k) {
        const uint32_t id = whose[k];
        if (id == 0xffffffffu) continue;
        const uint32_t s = s0 + k, last = (ld_dependent_u32(p.start + id + 1) - 1) / p.span;
        f32x2 sum[2] = {pk2(0.f, 0.f), pk2(0.f, 0.f)};
        if (c < dim) {
#pragma unroll 4
            for (uint32_t i = s + way; i <= last; i += 32) {
                const float4 x = ld_dependent_cg(reinterpret_cast<const float4*>(p.parts + (int64_t(i) * 2 + (i == s ? 1 : 0)) * dim + c));
                sum[0] = add2(sum[0], pk2(x.x, x.y));
                sum[1] = add2(sum[1], pk2(x.z, x.w));
            }
        }
        sums[threadIdx.x][0] = sum[0];
        sums[threadIdx.x][1] = sum[1];
        __syncthreads();
        if (way == 0 && c < dim && (group & 1) == 0) {         // 8 channels: this thread's and its neighbour's
            f32x2 f[4] = {sums[threadIdx.x][0], sums[threadIdx.x][1], sums[threadIdx.x + 1][0], sums[threadIdx.x + 1][1]};
            for (int w = 1; w < 32; ++w) {
#pragma unroll
                for (int e = 0; e < 4; ++e) f[e] = add2(f[e], sums[w * 8 + group + (e >> 1)][e & 1]);
            }
            write_row<U>(p, id, c, f);
        }
        __syncthreads();
    }
}

// ------------------------------------------------------------------------------------------------------------- host

bool type_ok(hq_dtype t) { return t == HQ_F32 || t == HQ_BF16; }
hq_status check_rows(const void* x, int64_t ld, int64_t dim, hq_dtype dt) {
    if (x == nullptr) return HQ_ERR_INVALID_ARG;
    if (ld < dim) return HQ_ERR_SHAPE;
    return aligned16(x) && (ld * (dt == HQ_BF16 ? 2 : 4)) % 16 == 0 ? HQ_OK : HQ_ERR_ALIGNMENT;
}
hq_status check_call(int id_bytes, int64_t tokens, int64_t classes, int64_t dim, hq_dtype a, hq_dtype b, float scale) {
    if ((id_bytes != 4 && id_bytes != 8) || !type_ok(a) || !type_ok(b) || !(scale - scale == 0.f)) return HQ_ERR_INVALID_ARG;
    if (tokens < 0 || classes <= 0 || dim <= 0) return HQ_ERR_SHAPE;
    if (dim % 8 != 0 || dim > (1 << 16) || tokens > 0x7fffffff || classes > 0x7fffffff) return HQ_ERR_UNSUPPORTED;
    return HQ_OK;
}

struct Plan { uint32_t slice, slices, span, spans; size_t found, sorted, start, parts, bytes; };
Plan plan_of(int64_t tokens, int64_t classes, int64_t dim) {
    Plan a{};
    const int64_t slice = (classes + 147) / 148;
    a.slice = uint32_t(slice < kSlice ? slice : kSlice);
    a.slices = uint32_t((classes + a.slice - 1) / a.slice);
    // spans that keep a thousand threads an SM busy, of 8 to 64 tokens
    int64_t span = 8;
    while (span < 64 && tokens * (dim / 8) > span * 148 * 1024) span *= 2;
    a.span = uint32_t(span);
    a.spans = uint32_t((tokens + span - 1) / span);
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    a.found = 0;
    a.sorted = up(size_t(tokens) * sizeof(uint2));
    a.start = a.sorted + up(size_t(tokens) * sizeof(uint2));
    a.parts = a.start + up((size_t(classes) + 1) * sizeof(uint32_t));
    a.bytes = a.parts + size_t(a.spans) * 2 * size_t(dim) * sizeof(float);
    return a;
}

template <typename T, typename U>
cudaError_t launch_lookup(const LookupParams& p, int id_bytes, unsigned grid, cudaStream_t st) {
    if (id_bytes == 4) embedding_kernel<int32_t, T, U><<<grid, 256, 0, st>>>(p);
    else embedding_kernel<int64_t, T, U><<<grid, 256, 0, st>>>(p);
    return cudaGetLastError();
}
template <typename T, typename U>
cudaError_t launch_sums(const GradParams& p, dim3 grid, cudaStream_t st) {
    return launch_dependent(embedding_sums_kernel<T, U>, grid, 256, 0, st, dependent_launch(int64_t(grid.x) * grid.y), p);
}

}  // namespace
}  // namespace hq

extern "C" hq_status hq_embedding(const void* ids, int id_bytes, int64_t tokens, const void* table, hq_dtype tdt, int64_t classes, int64_t dim,
                                  int64_t ld_table, float scale, void* out, hq_dtype odt, int64_t ld_out, void* stream) {
    using namespace hq;
    hq_status e = check_call(id_bytes, tokens, classes, dim, tdt, odt, scale);
    if (e != HQ_OK) return e;
    if (tokens == 0) return HQ_OK;
    if (ids == nullptr) return HQ_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(ids) % uintptr_t(id_bytes) != 0) return HQ_ERR_ALIGNMENT;
    if ((e = check_rows(table, ld_table, dim, tdt)) != HQ_OK || (e = check_rows(out, ld_out, dim, odt)) != HQ_OK) return e;
    const LookupParams p{ids, table, out, tokens, classes, ld_table, ld_out, int(dim / 8), scale};
    const int64_t slots = p.vectors > 256 ? 1 : 256 / p.vectors, ctas = (tokens + slots - 1) / slots, most = int64_t(sm_count()) * 8;
    const unsigned grid = unsigned(ctas < most ? ctas : most);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t c;
    if (tdt == HQ_BF16) c = odt == HQ_BF16 ? launch_lookup<__nv_bfloat16, __nv_bfloat16>(p, id_bytes, grid, st) : launch_lookup<__nv_bfloat16, float>(p, id_bytes, grid, st);
    else c = odt == HQ_BF16 ? launch_lookup<float, __nv_bfloat16>(p, id_bytes, grid, st) : launch_lookup<float, float>(p, id_bytes, grid, st);
    return c == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}

extern "C" hq_status hq_embedding_bwd_workspace_size(int64_t tokens, int64_t classes, int64_t dim, size_t* bytes) {
    using namespace hq;
    if (bytes == nullptr) return HQ_ERR_INVALID_ARG;
    const hq_status e = check_call(4, tokens, classes, dim, HQ_F32, HQ_F32, 1.f);
    if (e != HQ_OK) return e;
    *bytes = plan_of(tokens, classes, dim).bytes;
    return HQ_OK;
}

extern "C" hq_status hq_embedding_bwd(const void* ids, int id_bytes, int64_t tokens, const void* dout, hq_dtype ddt, int64_t ld_dout, int64_t classes,
                                      int64_t dim, float scale, const void* base, int64_t ld_base, void* dtable, hq_dtype gdt, int64_t ld_dtable,
                                      void* workspace, size_t ws_bytes, void* stream) {
    using namespace hq;
    hq_status e = check_call(id_bytes, tokens, classes, dim, ddt, gdt, scale);
    if (e != HQ_OK) return e;
    if ((tokens > 0 && ids == nullptr) || workspace == nullptr) return HQ_ERR_INVALID_ARG;
    if (reinterpret_cast<uintptr_t>(ids) % uintptr_t(id_bytes) != 0 || !aligned16(workspace)) return HQ_ERR_ALIGNMENT;
    if ((tokens > 0 && (e = check_rows(dout, ld_dout, dim, ddt)) != HQ_OK) || (e = check_rows(dtable, ld_dtable, dim, gdt)) != HQ_OK ||
        (base != nullptr && (e = check_rows(base, ld_base, dim, gdt)) != HQ_OK))
        return e;
    if (base == dtable && ld_base != ld_dtable) return HQ_ERR_SHAPE;
    const Plan a = plan_of(tokens, classes, dim);
    if (ws_bytes < a.bytes) return HQ_ERR_WORKSPACE;
    char* ws = static_cast<char*>(workspace);
    GradParams p{};
    p.ids = ids; p.dout = dout; p.base = base; p.dtable = dtable; p.ld_dout = ld_dout; p.ld_base = ld_base; p.ld_dtable = ld_dtable; p.classes = classes;
    p.tokens = uint32_t(tokens); p.slice = a.slice; p.span = a.span; p.longest = a.span * 4; p.spans = a.spans; p.vectors = int(dim / 8); p.scale = scale;
    p.found = reinterpret_cast<uint2*>(ws + a.found); p.sorted = reinterpret_cast<uint2*>(ws + a.sorted);
    p.start = reinterpret_cast<uint32_t*>(ws + a.start); p.parts = reinterpret_cast<float*>(ws + a.parts);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    const size_t smem = size_t(kOrderWarps) * a.slice * sizeof(uint32_t);
    if (id_bytes == 4) {
        HQ_CUDA_OK(cudaFuncSetAttribute(embedding_order_kernel<int32_t>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kOrderWarps * kSlice * sizeof(uint32_t))));
        embedding_order_kernel<int32_t><<<a.slices, kOrderThreads, smem, st>>>(p);
    } else {
        HQ_CUDA_OK(cudaFuncSetAttribute(embedding_order_kernel<int64_t>, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kOrderWarps * kSlice * sizeof(uint32_t))));
        embedding_order_kernel<int64_t><<<a.slices, kOrderThreads, smem, st>>>(p);
    }
    if (cudaGetLastError() != cudaSuccess) return HQ_ERR_CUDA;
    const int slots = p.vectors > 256 ? 1 : 256 / p.vectors;
    p.span_ctas = (a.spans + slots - 1) / slots;
    int64_t fill = base != nullptr && base == dtable ? 0 : (classes + slots * 4 - 1) / (slots * 4);
    if (fill > int64_t(148) * 16) fill = int64_t(148) * 16;
    const dim3 grid(p.span_ctas + unsigned(fill), unsigned((p.vectors + 255) / 256));
    if (grid.x == 0) return HQ_OK;
    cudaError_t c;
    if (ddt == HQ_BF16) c = gdt == HQ_BF16 ? launch_sums<__nv_bfloat16, __nv_bfloat16>(p, grid, st) : launch_sums<__nv_bfloat16, float>(p, grid, st);
    else c = gdt == HQ_BF16 ? launch_sums<float, __nv_bfloat16>(p, grid, st) : launch_sums<float, float>(p, grid, st);
    if (c != cudaSuccess) return HQ_ERR_CUDA;
    if (tokens <= int64_t(p.longest)) return HQ_OK;            // no id has more tokens than one span takes
    const dim3 join((a.spans + kJoinSpans - 1) / kJoinSpans, unsigned((dim + 31) / 32));
    c = gdt == HQ_BF16 ? launch_dependent(embedding_join_kernel<__nv_bfloat16>, join, 256, 0, st, dependent_launch(int64_t(join.x) * join.y), p)
                       : launch_dependent(embedding_join_kernel<float>, join, 256, 0, st, dependent_launch(int64_t(join.x) * join.y), p);
    return c == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}
