// Embedding lookup with scaling, and the gradient of its table by sorted tokens.
//
//   out[t] = scale table[id[t]]                    a row of zeros for an id outside the table
//   dtable[v] = base[v] + scale sum of dout[t] over the tokens t of id v, in ascending order, in fp32
//
// Memory-bound: the lookup reads ids and rows and writes rows; the gradient reads every token's row once and writes every row of the table once.
//
// The gradient has three kernels.  (1) order: CTA b owns a slice of the ids, reads all ids once, keeps the tokens of its slice in their order
// and counts those of smaller ids (where its part of the sorted order begins), then sorts its tokens by id with one stable counting sort, a
// warp's run of tokens after the other's: no atomics, so the order is the same on every run.  It writes its slice's rows of the table that have no tokens, too: all of them in front of
// the rest, while the memory is idle, where the tokens are fewer than the ids (or an fp32 base is added to).  (2) sums: the sorted tokens are cut into spans of equal length,
// whatever ids they hold (most tokens may be of one id); a team of threads adds up a span's rows with several rows in flight and writes a row of
// the table whenever the id changes.  An id of up to `longest` tokens belongs to the span of its first one; the sums of a longer one go to the
// workspace, one for each span, and (3) join adds them up in order.  Up to 128 tokens are added up by the first kernel alone.
//
// 19712 tokens of 768 bf16 (32768 ids): lookup 10.2 us a call (4.1 TB/s), gradient 36 where more than half of the tokens are of one id: order 16, of
// which 8 would do for its 50 MB of zeros, sums 13, join 9; each kernel's start and two or three loads that wait for one another are half of it.
#include "hq_common.cuh"
#include "hq_vec8.cuh"

namespace hq {
namespace {

// ---------------------------------------------------------------------------------------------------------- lookup

// 32 bits of an id are enough to tell whether it is in the table where its upper ones are zero: one outside becomes 2^32 - 1.
template <typename I> __device__ __forceinline__ uint32_t id_at(const void* ids, uint32_t t) {
    if constexpr (sizeof(I) == 4) return uint32_t(__ldg(static_cast<const int32_t*>(ids) + t));
    else {
        const uint64_t id = uint64_t(__ldg(static_cast<const long long*>(ids) + t));
        return id >> 32 == 0 ? uint32_t(id) : 0xffffffffu;
    }
}

// A CTA's threads over rows of `vectors` times 8 channels: `across` threads a row (blockIdx.y: 256 of them), as many rows as fit 256 threads.
struct Spread { int threads, slots; unsigned slices; };
inline Spread spread(int vectors) {
    const int across = vectors < 256 ? vectors : 256, slots = 256 / across;
    return Spread{(across * slots + 31) / 32 * 32, slots, unsigned((vectors + 255) / 256)};
}
struct Place { int slots, slot, c0; };             // slot >= slots: a thread without columns
__device__ __forceinline__ Place place_of(int vectors) {
    const int across = min(vectors - int(blockIdx.y) * 256, 256), slots = 256 / min(vectors, 256), slot = int(threadIdx.x) / across;
    return Place{slots, slot, (int(blockIdx.y) * 256 + int(threadIdx.x) - slot * across) * 8};
}

struct LookupParams { const void *ids, *table; void* out; uint32_t ld_table, ld_out, classes, tokens; int vectors; float scale; };       // pitches in bytes

// A thread takes 8 channels of kTogether tokens: the ids, then the rows, then the stores.  bf16, three to eight at a time: 19712 tokens of 768 12 us
// with any, 30000 of 1152 16, 15 (four), 16 (six) and 16 (eight), 262144 of 64 10, 10, 11 and 15; one 16, 25 and 14.  fp32, two, four and eight:
// 21 with any, 25, 27 and 31, 14, 16 and 19.
template <typename T> constexpr int kTogether = sizeof(T) == 2 ? 6 : 4;
template <typename I, typename T, typename U>
__global__ void __launch_bounds__(256) embedding_kernel(const LookupParams p) {
    constexpr int kN = kTogether<T>;
    const Place at = place_of(p.vectors);
    if (at.slot >= at.slots) return;
    const char* table = static_cast<const char*>(p.table) + at.c0 * int(sizeof(T));
    char* out = static_cast<char*>(p.out) + at.c0 * int(sizeof(U));
    const uint32_t t0 = blockIdx.x * uint32_t(at.slots * kN) + uint32_t(at.slot);
    uint32_t id[kN];
    Vec8<T> x[kN];
#pragma unroll
    for (int u = 0; u < kN; ++u) id[u] = t0 + u * at.slots < p.tokens ? id_at<I>(p.ids, t0 + u * at.slots) : 0xffffffffu;
#pragma unroll
    for (int u = 0; u < kN; ++u) {
        x[u].clear();
        if (id[u] < p.classes) x[u].load_wide(table + uint64_t(id[u]) * p.ld_table, 0);
    }
    const f32x2 s = pk2(p.scale, p.scale);
#pragma unroll
    for (int u = 0; u < kN; ++u) {
        const uint32_t t = t0 + u * at.slots;
        if (t >= p.tokens) break;
        f32x2 f[4];
        x[u].get(f);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = mul2(f[e], s);
        Vec8<U>::store_wide(out + uint64_t(t) * p.ld_out, 0, f);
    }
}

// -------------------------------------------------------------------------------------------------------- gradient

constexpr int kOrderThreads = 1024;
constexpr int kOrderWarps = kOrderThreads / 32;
constexpr int kSlice = kOrderThreads;              // ids a CTA of the order at most: a thread each in the scan, 128 KB of counters
constexpr size_t kOrderShared = 208 * 1024;        // counters and kept tokens of an order CTA at most, beside the kernel's own 9 KB
constexpr int kKept = 768;                         // tokens of its slice that a warp keeps in shared memory at most (16 bits of id, 32 of token)

struct GradParams {
    const void* ids;
    const void *dout, *base;
    void* dtable;
    uint32_t ld_dout, ld_base, ld_dtable;          // pitches in bytes
    uint32_t classes, tokens, slice, kept;         // slice: ids of an order CTA; kept: tokens that each of its warps has room for
    uint32_t span, longest, spans;                 // positions of a span; tokens of the longest id that one span takes whole
    int vectors, half;                             // half: dtable is bf16
    bool in_place, fill_first;
    float scale;
    uint2* sorted;                                 // [tokens] (id, token) by id
    uint32_t* start;                               // [classes + 1] first position of each id
    uint4* longs;                                  // (id, first position, end) of ids of more than `longest` tokens: slice s has
    uint32_t* long_count;                          // long_count[s] from its first position / longest + s on
    float* parts;                                  // [spans][first, last][dim]
};

__device__ __forceinline__ uint32_t lanes_below() { uint32_t m; asm("mov.u32 %0, %%lanemask_lt;" : "=r"(m)); return m; }

// Exclusive sum of x over the CTA's threads; *total is the whole.  One barrier in front of its use of `room` and one before it is read.
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

// Rows [0, size) of a slice that begins at row v0: base's, or zeros; `counts` (per row) not zero: left to its tokens' sum.  A warp a row.
__device__ __forceinline__ void fill_rows(const GradParams& p, uint32_t v0, uint32_t size, const uint32_t* counts) {
    const int lane = int(threadIdx.x & 31), pieces = p.half ? p.vectors : 2 * p.vectors;         // of 16 bytes
    for (uint32_t r = threadIdx.x >> 5; r < size; r += kOrderWarps) {
        if (counts != nullptr && counts[r] != 0) continue;
        uint4* to = reinterpret_cast<uint4*>(static_cast<char*>(p.dtable) + uint64_t(v0 + r) * p.ld_dtable);
        if (p.base == nullptr) {
#pragma unroll 4
            for (int v = lane; v < pieces; v += 32) to[v] = make_uint4(0u, 0u, 0u, 0u);
        } else {
            const uint4* from = reinterpret_cast<const uint4*>(static_cast<const char*>(p.base) + uint64_t(v0 + r) * p.ld_base);
            constexpr int kAhead = 5;
            for (int v = lane; v < pieces; v += 32 * kAhead) {
                uint4 x[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) x[u] = v + 32 * u < pieces ? from[v + 32 * u] : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
                for (int u = 0; u < kAhead; ++u)
                    if (v + 32 * u < pieces) to[v + 32 * u] = x[u];
            }
        }
    }
}

// Four ids from token t on, of a run that ends at `end`; `wide`: 16-byte loads.
template <typename I>
__device__ __forceinline__ void four_ids(uint32_t (&id)[4], const void* ids, uint32_t t, uint32_t end, bool wide) {
    if (sizeof(I) == 4 && wide && t + 4 <= end) {
        const int4 v = __ldg(reinterpret_cast<const int4*>(static_cast<const int32_t*>(ids) + t));
        id[0] = uint32_t(v.x); id[1] = uint32_t(v.y); id[2] = uint32_t(v.z); id[3] = uint32_t(v.w);
    } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) id[k] = t + k < end ? id_at<I>(ids, t + k) : 0xffffffffu;
    }
}

// The same with zeros for every row, by bulk copies of the zeros in shared memory, beside what the warps do (as stores they stand in the way of
// the ids' loads: 32768 x 768 rows of bf16 6 us).  The issuing lanes wait for them before the CTA ends.
constexpr uint32_t kZeros = 4096;                  // bytes
__device__ __forceinline__ void zero_rows(const GradParams& p, uint32_t v0, uint32_t size, const uint4* zeros) {
    const uint32_t row_bytes = uint32_t(p.vectors) * (p.half ? 16u : 32u);
    char* first = static_cast<char*>(p.dtable) + uint64_t(v0) * p.ld_dtable;
    // rows without gaps are one line
    const uint64_t line = p.ld_dtable == row_bytes ? uint64_t(size) * row_bytes : row_bytes;
    const uint32_t lines = p.ld_dtable == row_bytes ? 1u : size, pieces = uint32_t((line + kZeros - 1) / kZeros);
    for (uint32_t i = threadIdx.x & 31; i < lines * pieces; i += 32) {
        const uint32_t r = i / pieces;
        const uint64_t at = uint64_t(i - r * pieces) * kZeros;
        asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;"
                     ::"l"(first + uint64_t(r) * p.ld_dtable + at), "r"(smem_u32(zeros)), "r"(uint32_t(min(line - at, uint64_t(kZeros)))) : "memory");
    }
    bulk_commit_group();
}

__device__ __forceinline__ uint32_t ld_dependent_u32(const uint32_t* p) {
    uint32_t v;
    asm volatile("ld.global.u32 %0, [%1];" : "=r"(v) : "l"(p) : "memory");
    return v;
}

// HELD: an fp32 row with a base holds it already (in place, or copied by the order kernel): each value is added to once, without a wait for it.
__device__ __forceinline__ void add_to(float* to, float4 x) {
    asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(to), "f"(x.x), "f"(x.y), "f"(x.z), "f"(x.w) : "memory");
}

// Row v of the table from the sum of its tokens' rows.
template <typename U, bool HELD = true>
__device__ __forceinline__ void write_row(const GradParams& p, uint32_t v, int c0, const f32x2 (&sum)[4]) {
    const f32x2 s = pk2(p.scale, p.scale);
    f32x2 f[4];
    if (HELD && sizeof(U) == 4 && p.base != nullptr) {
        float* to = reinterpret_cast<float*>(static_cast<char*>(p.dtable) + uint64_t(v) * p.ld_dtable) + c0;
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
            float4 x;
            upk2(mul2(sum[e], s), x.x, x.y);
            upk2(mul2(sum[e + 1], s), x.z, x.w);
            add_to(to + 2 * e, x);
        }
        return;
    }
    if (p.base != nullptr) {
        Vec8<U> b;
        b.load_wide(static_cast<const char*>(p.base) + uint64_t(v) * p.ld_base, c0);
        b.get(f);
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = fma2(sum[e], s, f[e]);
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = mul2(sum[e], s);
    }
    Vec8<U>::store_wide(static_cast<char*>(p.dtable) + uint64_t(v) * p.ld_dtable, c0, f);
}

// 16 bytes of a row that a thread adds up (8 channels of bf16, 4 of fp32), and rows on their way to each thread: 64 KB a CTA.
template <typename T> constexpr int kPiece = 16 / int(sizeof(T));
constexpr int kFlight = 16;
constexpr int kEntries = 2048;                     // sorted tokens of a CTA's spans

// Row v of the table, N channels from c0 on, from the sum of its tokens' rows.
template <typename U, int N, bool HELD = true>
__device__ __forceinline__ void write_channels(const GradParams& p, uint32_t v, int c0, const f32x2 (&sum)[N / 2]) {
    if constexpr (N == 8) {
        write_row<U, HELD>(p, v, c0, sum);
    } else {
        const U* base = reinterpret_cast<const U*>(static_cast<const char*>(p.base) + uint64_t(v) * p.ld_base) + c0;
        U* to = reinterpret_cast<U*>(static_cast<char*>(p.dtable) + uint64_t(v) * p.ld_dtable) + c0;
        float f[4];
#pragma unroll
        for (int e = 0; e < 2; ++e) upk2(sum[e], f[2 * e], f[2 * e + 1]);
        if constexpr (sizeof(U) == 4) {
            const float4 x = make_float4(f[0] * p.scale, f[1] * p.scale, f[2] * p.scale, f[3] * p.scale);
            if (p.base == nullptr) {
                *reinterpret_cast<float4*>(to) = x;
            } else if (HELD) {
                add_to(to, x);
            } else {
                const float4 o = *reinterpret_cast<const float4*>(base);
                *reinterpret_cast<float4*>(to) = make_float4(o.x + x.x, o.y + x.y, o.z + x.z, o.w + x.w);
            }
        } else {
            uint2 o = make_uint2(0u, 0u);
            if (p.base != nullptr) o = *reinterpret_cast<const uint2*>(base);
            const __nv_bfloat162 lo = __floats2bfloat162_rn(fmaf(f[0], p.scale, __uint_as_float(o.x << 16)), fmaf(f[1], p.scale, __uint_as_float(o.x & 0xFFFF0000u)));
            const __nv_bfloat162 hi = __floats2bfloat162_rn(fmaf(f[2], p.scale, __uint_as_float(o.y << 16)), fmaf(f[3], p.scale, __uint_as_float(o.y & 0xFFFF0000u)));
            *reinterpret_cast<uint2*>(to) = make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
        }
    }
}

// A thread's piece added to its sums.
template <int N> __device__ __forceinline__ void add_piece(f32x2 (&sum)[N / 2], const uint4& x) {
    const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
    for (int k = 0; k < N / 2; ++k) {
        if constexpr (N == 8) sum[k] = add2(sum[k], pk2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xFFFF0000u)));
        else sum[k] = add2(sum[k], pk2(__uint_as_float(w[2 * k]), __uint_as_float(w[2 * k + 1])));
    }
}

// The rows of a slice whose tokens are few: places[r] .. places[r + 1] of `tokens` are row r's (n behind the last).  As many threads as a row has
// pieces take a row.
template <typename T, typename U>
__device__ __forceinline__ void sum_rows(const GradParams& p, uint32_t v0, uint32_t size, uint32_t n, const uint32_t* places, const uint32_t* tokens) {
    constexpr int kAhead = 8, kN = kPiece<T>;
    const int pieces = p.vectors * 8 / kN, across = min(pieces, kOrderThreads), teams = kOrderThreads / across, team = int(threadIdx.x) / across;
    if (team >= teams) return;
    const char* dout = static_cast<const char*>(p.dout);
    for (uint32_t r = uint32_t(team); r < size; r += uint32_t(teams)) {
        const uint32_t begin = places[r], end = r + 1 < size ? places[r + 1] : n;
        if (begin == end) continue;
        for (int v = int(threadIdx.x) - team * across; v < pieces; v += across) {
            f32x2 sum[kN / 2];
#pragma unroll
            for (int k = 0; k < kN / 2; ++k) sum[k] = pk2(0.f, 0.f);
            for (uint32_t j = begin; j < end; j += kAhead) {
                uint4 x[kAhead];
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    x[u] = make_uint4(0u, 0u, 0u, 0u);
                    if (j + u < end) x[u] = *reinterpret_cast<const uint4*>(dout + uint64_t(tokens[j + u]) * p.ld_dout + v * 16);
                }
#pragma unroll
                for (int u = 0; u < kAhead; ++u) {
                    if (j + u >= end) break;
                    add_piece<kN>(sum, x[u]);
                }
            }
            write_channels<U, kN, false>(p, v0 + r, v * kN, sum);
        }
    }
}

// HERE: at most kHere tokens, whose rows are added up here as well (64 labels into 1001 x 1152: the kernel of the sums and its start took 4 of 10 us).
constexpr int kHere = 128;
template <typename I, typename T, typename U, bool HERE>
__global__ void __launch_bounds__(kOrderThreads) embedding_order_kernel(const GradParams p) {
    extern __shared__ uint32_t counts[];           // [warp][id of the slice], then [warp][kept] tokens and [warp][kept] ids in the slice
    __shared__ uint32_t room[kOrderWarps], offset[kSlice];
    __shared__ __align__(128) uint4 zeros[kZeros / 16];
    __shared__ uint32_t chosen[HERE ? kHere : 1];  // the slice's tokens by id
    const int lane = int(threadIdx.x & 31), warp = int(threadIdx.x >> 5);
    const uint32_t v0 = blockIdx.x * p.slice, v1 = min(v0 + p.slice, p.classes), size = v1 - v0;
    uint32_t* count = counts + uint32_t(warp) * size;
    uint32_t* kept = counts + kOrderWarps * p.slice + uint32_t(warp) * p.kept;
    uint16_t* kept_id = reinterpret_cast<uint16_t*>(counts + kOrderWarps * (p.slice + p.kept)) + uint32_t(warp) * p.kept;
    if (!HERE) griddep_launch();                   // the sums' CTAs find room as these end
    const bool zeroing = p.base == nullptr && p.fill_first;
    if (zeroing) {
        if (threadIdx.x < kZeros / 16) zeros[threadIdx.x] = make_uint4(0u, 0u, 0u, 0u);
        fence_proxy_async_smem();
        __syncthreads();
        if (warp == 0) zero_rows(p, v0, size, zeros);
    } else if (!p.in_place && p.fill_first) {
        fill_rows(p, v0, size, nullptr);
    }
    for (uint32_t i = lane; i < size; i += 32) count[i] = 0;
    // a warp's run of ids: how many are smaller than the slice's, how many are of it, and which, as far as there is room
    const uint32_t run = (p.tokens + 32 * 128 - 1) / (32 * 128) * 128, from = min(uint32_t(warp) * run, p.tokens), to = min(from + run, p.tokens);
    const bool wide = (reinterpret_cast<uintptr_t>(p.ids) & 15u) == 0;
    uint32_t less = 0, mine = 0;                   // mine: the warp's, the same in every lane
    constexpr int kAhead = 4;
    for (uint32_t t0 = from + lane * 4; t0 < to + lane * 4; t0 += 128 * kAhead) {              // the same number of steps in every lane
        uint32_t id[kAhead][4];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) four_ids<I>(id[u], p.ids, t0 + 128 * u, to, wide);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            bool here[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                less += id[u][k] < v0;
                here[k] = id[u][k] - v0 < size;
            }
            if (!__any_sync(0xffffffffu, here[0] || here[1] || here[2] || here[3])) continue;
            uint32_t at = mine, of_all = 0;        // tokens in front of this lane's first, of the step
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const uint32_t who = __ballot_sync(0xffffffffu, here[k]);
                at += __popc(who & lanes_below());
                of_all += __popc(who);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (here[k] && at < p.kept) { kept[at] = t0 + 128 * u + k; kept_id[at] = uint16_t(id[u][k] - v0); }
                at += here[k];
            }
            mine += of_all;
        }
    }
    __syncwarp();
    // the warp's tokens of the slice, 32 at a time: f(id in the slice or 2^32 - 1, token, lanes of the same id).  Where they were too many, from
    // the ids again.
    auto each = [&](auto f) {
        constexpr int kBatch = 4;
        const bool again = mine > p.kept;
        const uint32_t begin = again ? from : 0u, end = again ? to : mine;
        for (uint32_t j0 = begin + lane; j0 < end + lane; j0 += 32 * kBatch) {
            uint32_t key[kBatch], token[kBatch], same[kBatch];
#pragma unroll
            for (int u = 0; u < kBatch; ++u) {
                const uint32_t j = j0 + 32 * u;
                key[u] = 0xffffffffu;
                token[u] = j;
                if (j < end) {
                    if (again) {
                        const uint32_t id = id_at<I>(p.ids, j) - v0;
                        if (id < size) key[u] = id;
                    } else {
                        key[u] = kept_id[j];
                        token[u] = kept[j];
                    }
                }
            }
#pragma unroll
            for (int u = 0; u < kBatch; ++u) same[u] = __match_any_sync(0xffffffffu, key[u]);
#pragma unroll
            for (int u = 0; u < kBatch; ++u) f(key[u], token[u], same[u]);
        }
    };
    each([&](uint32_t key, uint32_t, uint32_t same) {
        if (key != 0xffffffffu && (same & lanes_below()) == 0) count[key] += __popc(same);
        __syncwarp();
    });
    uint32_t first, n, longs;
    (void)exclusive_sum(less, room, &first);       // the slice's first position; the warps' counts are complete behind its barriers
    uint32_t sum = 0;
    if (threadIdx.x < size) {
#pragma unroll 8
        for (int w = 0; w < kOrderWarps; ++w) {
            const uint32_t c = counts[uint32_t(w) * size + threadIdx.x];
            counts[uint32_t(w) * size + threadIdx.x] = sum;
            sum += c;
        }
    }
    const uint32_t begins = first + exclusive_sum(sum, room, &n);
    if (threadIdx.x < size) {
        offset[threadIdx.x] = begins;
        p.start[v0 + threadIdx.x] = begins;
    }
    if (v1 == p.classes && threadIdx.x == 0) p.start[p.classes] = first + n;
    const bool is_long = sum > p.longest;
    const uint32_t nth = exclusive_sum(is_long ? 1u : 0u, room, &longs);       // (its barriers stand in front of the use of `offset`, too)
    if (is_long) p.longs[first / p.longest + blockIdx.x + nth] = make_uint4(v0 + threadIdx.x, begins, begins + sum, 0u);
    if (threadIdx.x == 0) p.long_count[blockIdx.x] = longs;
    each([&](uint32_t key, uint32_t token, uint32_t same) {
        const uint32_t rank = __popc(same & lanes_below());
        const bool there = key != 0xffffffffu;
        if (there) {
            const uint32_t at = offset[key] + count[key] + rank;
            if (HERE) chosen[at - first] = token;
            else p.sorted[at] = make_uint2(v0 + key, token);
        }
        __syncwarp();
        if (there && rank == 0) count[key] += __popc(same);
        __syncwarp();
    });
    if constexpr (HERE) {
        if (zeroing && warp == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");        // behind the zeros
        __syncthreads();                           // every warp has placed its tokens
        if (threadIdx.x < size) offset[threadIdx.x] -= first;
        __syncthreads();
        sum_rows<T, U>(p, v0, size, n, offset, chosen);
    }
    if (!p.in_place && !p.fill_first) {
        __syncthreads();
        if (threadIdx.x < size) offset[threadIdx.x] = sum;
        __syncthreads();
        fill_rows(p, v0, size, offset);
    }
    if (zeroing && warp == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");
}

// Span blockIdx.x * slots + slot of blockDim.x / slots threads.  The CTA's sorted tokens are in shared memory; each thread copies its piece of
// kFlight rows ahead there, for itself, so that few teams keep the memory busy and the spans may be long.  BASED: a bf16 base, whose rows are
// asked for as far ahead.
template <typename T, typename U, bool BASED>
__global__ void __launch_bounds__(256) embedding_sums_kernel(const GradParams p) {
    extern __shared__ uint4 rows[];                // [kFlight][threads]
    __shared__ uint2 entries[kEntries];
    constexpr int kN = kPiece<T>;
    const int pieces = p.vectors * 8 / kN;
    const Place at = place_of(pieces);
    const int c0 = at.c0 / 8 * kN;
    griddep_wait();
    griddep_launch();                              // the joining kernel's CTAs find room as these end
    const uint32_t n = ld_dependent_u32(p.start + p.classes), from = blockIdx.x * uint32_t(at.slots) * p.span;
    if (from >= n) return;
    const uint32_t known = min(n - from, uint32_t(at.slots) * p.span + p.longest);
    for (uint32_t i = threadIdx.x; i < known; i += blockDim.x) entries[i] = ld_dependent_cg(p.sorted + from + i);
    __syncthreads();
    const uint32_t s = blockIdx.x * uint32_t(at.slots) + uint32_t(at.slot);
    uint32_t a = uint32_t(at.slot) * p.span, b = min(a + p.span, n - from);    // places in `entries`
    if (at.slot >= at.slots || a >= b) return;
    // an id of at most `longest` tokens belongs to the span of its first one, whole; a longer one to every span that it lies in
    bool open_left = false, open_right = false;
    {
        const uint32_t id0 = entries[a].x, id1 = entries[b - 1].x;
        const uint32_t begin0 = ld_dependent_u32(p.start + id0), end0 = ld_dependent_u32(p.start + id0 + 1);
        const uint32_t begin1 = ld_dependent_u32(p.start + id1), end1 = ld_dependent_u32(p.start + id1 + 1);
        if (begin0 < from + a) {
            if (end0 - begin0 <= p.longest) a = end0 - from;
            else open_left = true;
        }
        if (a >= b) return;
        if (end1 - begin1 > p.longest) open_right = end1 > from + b;
        else b = end1 - from;
    }
    const char* dout = static_cast<const char*>(p.dout) + c0 * int(sizeof(T));
    const uint32_t ring = smem_u32(rows) + threadIdx.x * 16u, step = blockDim.x * 16u;
    auto send = [&](uint32_t j) {
        if (j < b) {
            if (BASED && (j == a || entries[j].x != entries[j - 1].x))
                asm volatile("prefetch.global.L2 [%0];" ::"l"(static_cast<const char*>(p.base) + uint64_t(entries[j].x) * p.ld_base + c0 * 2));
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16;"
                         ::"r"(ring + (j % kFlight) * step), "l"(dout + uint64_t(entries[j].y) * p.ld_dout) : "memory");
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    f32x2 sum[kN / 2];
#pragma unroll
    for (int k = 0; k < kN / 2; ++k) sum[k] = pk2(0.f, 0.f);
    uint32_t now = entries[a].x;
    auto leave = [&](bool left, bool right) {
        if (!left && !right) { write_channels<U, kN>(p, now, c0, sum); return; }
        float* part = p.parts + (int64_t(s) * 2 + (left ? 0 : 1)) * p.vectors * 8 + c0;
#pragma unroll
        for (int k = 0; k < kN / 2; k += 2) {
            float4 v;
            upk2(sum[k], v.x, v.y);
            upk2(sum[k + 1], v.z, v.w);
            *reinterpret_cast<float4*>(part + 2 * k) = v;
        }
    };
#pragma unroll 1
    for (uint32_t k = 0; k < kFlight - 1; ++k) send(a + k);
#pragma unroll 2
    for (uint32_t j = a; j < b; ++j) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kFlight - 2) : "memory");
        uint4 x;
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "r"(ring + (j % kFlight) * step) : "memory");
        send(j + kFlight - 1);                     // into the place of the row before this one
        const uint32_t id = entries[j].x;
        if (id != now) {
            leave(open_left, false);
            open_left = false;
            now = id;
#pragma unroll
            for (int k = 0; k < kN / 2; ++k) sum[k] = pk2(0.f, 0.f);
        }
        add_piece<kN>(sum, x);
    }
    leave(open_left, open_right);
}

// 8 values of each of four parts in one statement: as loads of their own the compiler put each part's sum behind its load, and an id of 690
// parts, 22 a thread, took 10 us of waits.
__device__ __forceinline__ void ld_four_parts(float (&x)[4][8], const float* const (&from)[4]) {
#define HQ_OUT8(u) "=f"(x[u][0]), "=f"(x[u][1]), "=f"(x[u][2]), "=f"(x[u][3]), "=f"(x[u][4]), "=f"(x[u][5]), "=f"(x[u][6]), "=f"(x[u][7])
    asm volatile(
        "ld.global.cg.v4.f32 {%0, %1, %2, %3}, [%32];\n\tld.global.cg.v4.f32 {%4, %5, %6, %7}, [%32 + 16];\n\t"
        "ld.global.cg.v4.f32 {%8, %9, %10, %11}, [%33];\n\tld.global.cg.v4.f32 {%12, %13, %14, %15}, [%33 + 16];\n\t"
        "ld.global.cg.v4.f32 {%16, %17, %18, %19}, [%34];\n\tld.global.cg.v4.f32 {%20, %21, %22, %23}, [%34 + 16];\n\t"
        "ld.global.cg.v4.f32 {%24, %25, %26, %27}, [%35];\n\tld.global.cg.v4.f32 {%28, %29, %30, %31}, [%35 + 16];"
        : HQ_OUT8(0), HQ_OUT8(1), HQ_OUT8(2), HQ_OUT8(3) : "l"(from[0]), "l"(from[1]), "l"(from[2]), "l"(from[3]) : "memory");
#undef HQ_OUT8
}

// Ids that lie in several spans.  blockIdx.x: a slice of the order, whose long ids are taken one after the other; y: 64 channels.
// Thread = (8 channels, every 32nd part).
template <typename U>
__global__ void __launch_bounds__(256) embedding_join_kernel(const GradParams p) {
    __shared__ f32x2 sums[8][8][4];
    const int lane = int(threadIdx.x & 31), warp = int(threadIdx.x >> 5), group = lane & 7, way = int(threadIdx.x >> 3);
    const int c0 = int(blockIdx.y) * 64 + group * 8, dim = p.vectors * 8;
    griddep_wait();
    const uint32_t count = ld_dependent_u32(p.long_count + blockIdx.x), slice_at = ld_dependent_u32(p.start + blockIdx.x * p.slice);
    if (count == 0) return;
    for (uint32_t k = 0; k < count; ++k) {
        const uint4 entry = ld_dependent_cg(p.longs + slice_at / p.longest + blockIdx.x + k);
        const uint32_t id = entry.x, first = entry.y / p.span, last = (entry.z - 1) / p.span;
        f32x2 sum[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = pk2(0.f, 0.f);
        if (c0 < dim) {
            for (uint32_t i0 = first + way; i0 <= last; i0 += 32 * 4) {
                const float* part[4];              // of a part behind the last: the last one's, which is not added
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    const uint32_t i = min(i0 + 32 * u, last);
                    part[u] = p.parts + (int64_t(i) * 2 + (i == first ? 1 : 0)) * dim + c0;
                }
                float x[4][8];
                ld_four_parts(x, part);
#pragma unroll
                for (int u = 0; u < 4; ++u) {
                    if (i0 + 32 * u > last) break;
#pragma unroll
                    for (int e = 0; e < 4; ++e) sum[e] = add2(sum[e], pk2(x[u][2 * e], x[u][2 * e + 1]));
                }
            }
        }
        // four ways of a warp, then the warps in order
#pragma unroll
        for (int off = 8; off <= 16; off *= 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sum[e] = add2(sum[e], __shfl_xor_sync(0xffffffffu, sum[e], off));
        }
        __syncthreads();                           // the sums of the id before this one are read
        if (lane < 8) {
#pragma unroll
            for (int e = 0; e < 4; ++e) sums[warp][group][e] = sum[e];
        }
        __syncthreads();
        if (warp == 0 && lane < 8 && c0 < dim) {
            for (int w = 1; w < 8; ++w) {
#pragma unroll
                for (int e = 0; e < 4; ++e) sum[e] = add2(sum[e], sums[w][group][e]);
            }
            write_row<U>(p, id, c0, sum);
        }
    }
}

// ------------------------------------------------------------------------------------------------------------- host

bool type_ok(hq_dtype t) { return t == HQ_F32 || t == HQ_BF16; }
hq_status check_rows(const void* x, int64_t ld, int64_t dim, hq_dtype dt) {
    if (x == nullptr) return HQ_ERR_INVALID_ARG;
    if (ld < dim) return HQ_ERR_SHAPE;
    if (!aligned16(x) || (ld * (dt == HQ_BF16 ? 2 : 4)) % 16 != 0) return HQ_ERR_ALIGNMENT;
    return ld < int64_t(1) << 30 ? HQ_OK : HQ_ERR_UNSUPPORTED;             // a pitch in bytes has 32 bits
}
uint32_t pitch_of(int64_t ld, hq_dtype dt) { return uint32_t(ld) * (dt == HQ_BF16 ? 2u : 4u); }
hq_status check_call(int id_bytes, int64_t tokens, int64_t classes, int64_t dim, hq_dtype a, hq_dtype b, float scale) {
    if ((id_bytes != 4 && id_bytes != 8) || !type_ok(a) || !type_ok(b) || !(scale - scale == 0.f)) return HQ_ERR_INVALID_ARG;
    if (tokens < 0 || classes <= 0 || dim <= 0) return HQ_ERR_SHAPE;
    if (dim % 8 != 0 || dim > (1 << 16) || tokens > 0x7fffffff || classes > 0x7fffffff) return HQ_ERR_UNSUPPORTED;
    return HQ_OK;
}

struct Plan { uint32_t slice, slices, span, spans, longest; size_t start, longs, long_count, parts, bytes; };
constexpr int64_t kLongestSpan = 64, kSumsThreads = 148 * 2 * 256;         // threads: of two CTAs an SM
// Tokens of which a span of `span` (or fewer) is enough: spans for two CTAs an SM, and where an id may lie in many of them no shorter than
// sqrt(tokens) / 6: adding up their sums takes as long as a span's rows then (3691 tokens of 64 channels, half of them of one id: spans of one
// token 29 us a call).
int64_t tokens_of_span(int64_t span, int64_t pieces) {
    const int64_t resident = span * kSumsThreads / pieces, joined = 36 * span * span;
    return resident < joined ? resident : joined;
}
Plan plan_of(int64_t tokens, int64_t classes, int64_t dim, int piece) {
    Plan a{};
    const int64_t slice = (classes + 147) / 148;
    a.slice = uint32_t(slice < kSlice ? slice : kSlice);
    a.slices = uint32_t((classes + a.slice - 1) / a.slice);
    const int64_t pieces = dim / piece, slots = 256 / (pieces < 256 ? pieces : 256);
    a.longest = kLongestSpan;
    int64_t span = 1;
    while (span < kLongestSpan && tokens > tokens_of_span(span, pieces)) span *= 2;
    while (span > 1 && slots * span + a.longest > kEntries) span /= 2;         // no more tokens in a CTA than its room for entries
    a.span = uint32_t(span);
    a.spans = uint32_t((tokens + span - 1) / span);
    auto up = [](size_t x) { return (x + 255) / 256 * 256; };
    a.start = up(size_t(tokens) * sizeof(uint2));  // behind the sorted tokens
    a.longs = a.start + up((size_t(classes) + 1) * sizeof(uint32_t));
    a.long_count = a.longs + up((size_t(tokens) / a.longest + a.slices + 1) * sizeof(uint4));
    a.parts = a.long_count + up(size_t(a.slices) * sizeof(uint32_t));
    a.bytes = a.parts + size_t(a.spans) * 2 * size_t(dim) * sizeof(float);
    return a;
}
// Bytes for at most so many tokens: the spans get longer with the tokens, and there are most of them where they are about to.
size_t most_bytes(int64_t tokens, int64_t classes, int64_t dim, int piece) {
    const Plan a = plan_of(tokens, classes, dim, piece);
    int64_t spans = a.spans;
    for (int64_t span = 1; span < a.span; span *= 2) {
        const int64_t most = tokens_of_span(span, dim / piece), n = ((most < tokens ? most : tokens) + span - 1) / span;
        if (n > spans) spans = n;
    }
    return a.parts + size_t(spans) * 2 * size_t(dim) * sizeof(float);
}

template <typename T, typename U>
cudaError_t launch_lookup(const LookupParams& p, int id_bytes, cudaStream_t st) {
    const Spread s = spread(p.vectors);
    const uint32_t per = uint32_t(s.slots * kTogether<T>);
    const dim3 grid((p.tokens + per - 1) / per, s.slices);
    if (id_bytes == 4) embedding_kernel<int32_t, T, U><<<grid, s.threads, 0, st>>>(p);
    else embedding_kernel<int64_t, T, U><<<grid, s.threads, 0, st>>>(p);
    return cudaGetLastError();
}
template <typename I> auto order_here(hq_dtype ddt, hq_dtype gdt) -> void (*)(GradParams) {
    if (ddt == HQ_BF16) return gdt == HQ_BF16 ? embedding_order_kernel<I, __nv_bfloat16, __nv_bfloat16, true> : embedding_order_kernel<I, __nv_bfloat16, float, true>;
    return gdt == HQ_BF16 ? embedding_order_kernel<I, float, __nv_bfloat16, true> : embedding_order_kernel<I, float, float, true>;
}
template <typename T, typename U>
cudaError_t launch_sums(const GradParams& p, cudaStream_t st) {
    const Spread s = spread(p.vectors * 8 / kPiece<T>);
    const size_t smem = size_t(kFlight) * s.threads * 16;
    void (*kern)(GradParams) = embedding_sums_kernel<T, U, false>;
    if constexpr (sizeof(U) == 2)
        if (p.base != nullptr) kern = embedding_sums_kernel<T, U, true>;
    if (smem > 24 * 1024) {                        // 48 KB without asking, less the entries' 16; one value for every call, as another host thread's may come between
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kFlight * 256 * 16);
        if (e != cudaSuccess) { (void)cudaGetLastError(); return e; }
    }
    return launch_dependent(kern, dim3((p.spans + s.slots - 1) / s.slots, s.slices), s.threads, smem, st, true, p);
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
    const LookupParams p{ids, table, out, pitch_of(ld_table, tdt), pitch_of(ld_out, odt), uint32_t(classes), uint32_t(tokens), int(dim / 8), scale};
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    cudaError_t c;
    if (tdt == HQ_BF16) c = odt == HQ_BF16 ? launch_lookup<__nv_bfloat16, __nv_bfloat16>(p, id_bytes, st) : launch_lookup<__nv_bfloat16, float>(p, id_bytes, st);
    else c = odt == HQ_BF16 ? launch_lookup<float, __nv_bfloat16>(p, id_bytes, st) : launch_lookup<float, float>(p, id_bytes, st);
    return c == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}

extern "C" hq_status hq_embedding_bwd_workspace_size(int64_t tokens, int64_t classes, int64_t dim, size_t* bytes) {
    using namespace hq;
    if (bytes == nullptr) return HQ_ERR_INVALID_ARG;
    const hq_status e = check_call(4, tokens, classes, dim, HQ_F32, HQ_F32, 1.f);
    if (e != HQ_OK) return e;
    const size_t half = most_bytes(tokens, classes, dim, kPiece<__nv_bfloat16>), full = most_bytes(tokens, classes, dim, kPiece<float>);
    *bytes = half > full ? half : full;            // of either type of dout
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
    const Plan a = plan_of(tokens, classes, dim, ddt == HQ_BF16 ? kPiece<__nv_bfloat16> : kPiece<float>);
    if (ws_bytes < a.bytes) return HQ_ERR_WORKSPACE;
    char* ws = static_cast<char*>(workspace);
    auto words = [&](size_t at) { return reinterpret_cast<uint32_t*>(ws + at); };
    GradParams p{};
    p.ids = ids; p.dout = dout; p.base = base; p.dtable = dtable; p.classes = uint32_t(classes);
    p.ld_dout = tokens > 0 ? pitch_of(ld_dout, ddt) : 0; p.ld_base = base != nullptr ? pitch_of(ld_base, gdt) : 0; p.ld_dtable = pitch_of(ld_dtable, gdt);
    p.tokens = uint32_t(tokens); p.slice = a.slice; p.span = a.span; p.longest = a.longest; p.spans = a.spans; p.vectors = int(dim / 8); p.half = gdt == HQ_BF16;
    p.in_place = base == dtable; p.fill_first = tokens < classes || (base != nullptr && gdt == HQ_F32); p.scale = scale;
    p.sorted = reinterpret_cast<uint2*>(ws);
    p.start = words(a.start); p.longs = reinterpret_cast<uint4*>(ws + a.longs); p.long_count = words(a.long_count); p.parts = reinterpret_cast<float*>(ws + a.parts);
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    // room for every token of a warp's run, as far as shared memory goes
    const size_t counters = size_t(kOrderWarps) * a.slice * sizeof(uint32_t), each = kOrderWarps * (sizeof(uint32_t) + sizeof(uint16_t));
    const size_t run = size_t(tokens + 32 * 128 - 1) / (32 * 128) * 128, fit = (kOrderShared - counters) / each / 2 * 2;
    p.kept = uint32_t(run < fit ? run : fit);
    if (p.kept > kKept) p.kept = kKept;
    const size_t smem = counters + p.kept * each;
    const bool here = tokens <= kHere;
    if (here) p.fill_first = tokens < classes;     // behind the fill and a barrier the sums are written as they are
    void (*order)(GradParams) = !here ? (id_bytes == 4 ? embedding_order_kernel<int32_t, float, float, false> : embedding_order_kernel<int64_t, float, float, false>)
                                : id_bytes == 4 ? order_here<int32_t>(ddt, gdt) : order_here<int64_t>(ddt, gdt);
    // 48 KB without asking, less the kernel's own 9; one value for every call, as another host thread's may come between
    if (smem > 32 * 1024) HQ_CUDA_OK(cudaFuncSetAttribute(order, cudaFuncAttributeMaxDynamicSharedMemorySize, int(kOrderShared)));
    order<<<a.slices, kOrderThreads, smem, st>>>(p);
    if (cudaGetLastError() != cudaSuccess) return HQ_ERR_CUDA;
    if (here) return HQ_OK;
    cudaError_t c;
    if (ddt == HQ_BF16) c = gdt == HQ_BF16 ? launch_sums<__nv_bfloat16, __nv_bfloat16>(p, st) : launch_sums<__nv_bfloat16, float>(p, st);
    else c = gdt == HQ_BF16 ? launch_sums<float, __nv_bfloat16>(p, st) : launch_sums<float, float>(p, st);
    if (c != cudaSuccess) return HQ_ERR_CUDA;
    const dim3 join(a.slices, unsigned((dim + 63) / 64));
    c = gdt == HQ_BF16 ? launch_dependent(embedding_join_kernel<__nv_bfloat16>, join, 256, 0, st, true, p) : launch_dependent(embedding_join_kernel<float>, join, 256, 0, st, true, p);
    return c == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}
