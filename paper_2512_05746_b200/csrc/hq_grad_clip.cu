// The norm of all gradients of a training step, and clipping by it.
//
//   norm = sqrt(sum over tensors and elements of g^2),   c = min(1, max_norm / (norm + eps)),   out = c g
//
// Memory-bound: one pass that reads every gradient, one that reads and writes it.  The tensors are one line of chunks of equal size, laid
// out in the kernel's parameters (address, count and first chunk of each, and each CTA's first tensor), so that a call of hundreds of tensors is
// two launches without a table in memory.  Few chunks: a CTA takes a run of them.  Many: the CTAs' chunks lie side by side, so that all that is
// under way lies in one moving window.  The second pass takes the chunks
// from the last one down: what the first pass read last is still in L2.
//
// A thread's squares are summed in fp32 over 8 elements at a time and these in fp64; a group of 8 whose squares leave fp32's range is
// squared in fp64 instead.  Threads, warps and CTAs are joined in a fixed order: the same gradients give the same bits.
//
// 642 M gradients of bf16 in 287 tensors, clipped to fp32: norm 212 us (6.0 TB/s, 94 % of the copy rate), outputs 677 (5.7 TB/s; runs of chunks a CTA 710).
// 280 tensors of 4.1 M fp32 together: 14 us a call, 12 of them on the host.
#include <climits>

#include "hq_common.cuh"
#include "hq_vec8.cuh"

namespace hq {
namespace {

constexpr int kThreads = 256;
constexpr int kNormBlocks = 148 * 6, kScaleBlocks = 148 * 4;                       // resident at once; on every device: one order of the sums
constexpr int64_t kUnit = kThreads * 8;            // elements a CTA takes at a time
constexpr int kMost = 1088;                        // tensors of a launch: 28 bytes each of 32 KB of parameters, 2 for each CTA
constexpr int kParts = 4096;                       // sums of CTAs of all launches of a call

// N tensors; first[n] is the first chunk behind them.
template <int N> struct Tensors {
    const void* in[N];
    void* out[N];
    int64_t count[N];                              // elements, and the two types in bits 62 (in) and 61 (out): 1 bf16
    uint32_t first[N + 1];
    uint16_t at[kNormBlocks];                      // the tensor of the chunk a CTA begins with
    bool side_by_side;
    int n;
    int64_t chunk;                                 // elements, a multiple of kUnit
    double* parts;                                 // a sum of each CTA of the norm's launches: this launch's, for the second pass all
    int parts_n;                                   // their number
    float *norm, *coef;
    float max_norm, eps;
    bool clip, write_norm;
};
constexpr int64_t kInBf16 = int64_t(1) << 62, kOutBf16 = int64_t(1) << 61, kCount = kOutBf16 - 1;

template <typename T> __device__ __forceinline__ float element(const void* p, int64_t i);
template <> __device__ __forceinline__ float element<float>(const void* p, int64_t i) { return static_cast<const float*>(p)[i]; }
template <> __device__ __forceinline__ float element<__nv_bfloat16>(const void* p, int64_t i) { return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]); }

// Squares of 8 values.  A square below fp32's range is off by 2^-150 at most: a sum above 2^-120 by 2^-27 of itself for all 8, less than a
// rounding.  Smaller sums, and those near or behind the range's other end, are taken in fp64; NaN stays NaN.  (32 values to one fp64 addition
// hold 24 registers more: 100 M of bf16 42 us, not 29.)
__device__ __forceinline__ double squares(const f32x2 (&f)[4]) {
    f32x2 s = mul2(f[0], f[0]);
#pragma unroll
    for (int e = 1; e < 4; ++e) s = fma2(f[e], f[e], s);
    const float q = pair_sum(s);
    if (q >= 0x1p-120f && q <= 0x1p120f) return double(q);
    double d = 0.0;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        float a, b;
        upk2(f[e], a, b);
        if (a != 0.f) d += double(a) * double(a);              // most often all 8 are zero
        if (b != 0.f) d += double(b) * double(b);
    }
    return d;
}

// Elements [from, to) of a tensor, all of a CTA's threads; `shift` elements lie between the border in front of the tensor (of 8 elements: 16
// bytes of bf16, 32 of fp32) and its first one, and vectors begin at multiples of 8 elements from that border.
template <typename T>
__device__ __forceinline__ double sum_squares(const void* in, int64_t from, int64_t to, int shift) {
    constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;
    const int64_t v0 = (from + shift) / 8 * 8 - shift;         // the vector that holds `from`
    double sum = 0.0;
    for (int64_t base = v0 + int64_t(threadIdx.x) * 8; base < to; base += kUnit * kAhead) {
        Vec8<T> v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t i = base + u * kUnit;
            v[u].clear();
            if (i >= from && i + 8 <= to) v[u].load_wide(in, i);
        }
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t i = base + u * kUnit;
            if (i >= to) break;
            f32x2 f[4];
            v[u].get(f);
            if (i < from || i + 8 > to) {                      // the ends
                float e[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) e[k] = i + k >= from && i + k < to ? element<T>(in, i + k) : 0.f;
#pragma unroll
                for (int k = 0; k < 4; ++k) f[k] = pk2(e[2 * k], e[2 * k + 1]);
            }
            sum += squares(f);
        }
    }
    return sum;
}

// A CTA's chunks: a run of equal length.
__device__ __forceinline__ void my_chunks(uint32_t all, uint32_t& from, uint32_t& to) {
    const uint32_t per = (all + gridDim.x - 1) / gridDim.x;
    from = min(blockIdx.x * per, all);
    to = min(from + per, all);
}
template <typename T> __device__ __forceinline__ int shift_of(const void* p) { return int((reinterpret_cast<uintptr_t>(p) / sizeof(T)) & 7u); }

template <int N>
__global__ void __launch_bounds__(kThreads) grad_norm_kernel(const __grid_constant__ Tensors<N> p) {
    __shared__ double sums[kThreads / 32];
    griddep_launch();                              // the second pass finds room as CTAs end, and waits for all of them
    double sum = 0.0;
    auto take = [&](int k, uint32_t c, uint32_t end) {         // chunks [c, end) of tensor k
        const int64_t count = p.count[k] & kCount, from = int64_t(c - p.first[k]) * p.chunk, to = min(int64_t(end - p.first[k]) * p.chunk, count);
        if (p.count[k] & kInBf16) sum += sum_squares<__nv_bfloat16>(p.in[k], from, to, shift_of<__nv_bfloat16>(p.in[k]));
        else sum += sum_squares<float>(p.in[k], from, to, shift_of<float>(p.in[k]));
    };
    const uint32_t all = p.first[p.n];
    int k = p.at[blockIdx.x];
    if (p.side_by_side) {
        for (uint32_t c = blockIdx.x; c < all; c += gridDim.x) {
            while (p.first[k + 1] <= c) ++k;
            take(k, c, c + 1);
        }
    } else {
        uint32_t c, end;
        for (my_chunks(all, c, end); c < end; ++k) {           // this CTA's part of each tensor
            const uint32_t stop = min(end, p.first[k + 1]);
            take(k, c, stop);
            c = stop;
        }
    }
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = sum;
    __syncthreads();
    if (threadIdx.x == 0) {
#pragma unroll
        for (int w = 1; w < kThreads / 32; ++w) sum += sums[w];
        p.parts[blockIdx.x] = sum;
    }
}

__device__ __forceinline__ double ld_dependent_f64(const double* p) {
    double v;
    asm volatile("ld.global.f64 %0, [%1];" : "=d"(v) : "l"(p) : "memory");
    return v;
}
// The parts' sum, in every thread.
__device__ __forceinline__ double all_parts(const double* parts, int n, double* room) {
    double sum = 0.0;
    for (int i = int(threadIdx.x); i < n; i += kThreads) sum += ld_dependent_f64(parts + i);
#pragma unroll
    for (int off = 16; off > 0; off >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, off);
    if ((threadIdx.x & 31) == 0) room[threadIdx.x >> 5] = sum;
    __syncthreads();
    sum = 0.0;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) sum += room[w];
    return sum;
}

// 8 values that nothing reads from L2 again, and 8 that are written once: they give way to what is still to be read.
template <typename T> __device__ __forceinline__ void load_last(Vec8<T>& v, const void* base, int64_t at) {
    if constexpr (sizeof(T) == 2) {
        asm volatile("ld.global.cs.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(v.w.x), "=r"(v.w.y), "=r"(v.w.z), "=r"(v.w.w) : "l"(static_cast<const T*>(base) + at));
    } else {
        asm volatile("ld.global.L1::no_allocate.L2::evict_first.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=f"(v.a.x), "=f"(v.a.y), "=f"(v.a.z), "=f"(v.a.w), "=f"(v.b.x), "=f"(v.b.y), "=f"(v.b.z), "=f"(v.b.w) : "l"(static_cast<const T*>(base) + at));
    }
}
template <typename U> __device__ __forceinline__ void store_once(void* base, int64_t at, const f32x2 (&f)[4]) {
    U* p = static_cast<U*>(base) + at;
    float x[8];
#pragma unroll
    for (int e = 0; e < 4; ++e) upk2(f[e], x[2 * e], x[2 * e + 1]);
    if constexpr (sizeof(U) == 2) {
        uint32_t u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * e], x[2 * e + 1]);
            u[e] = *reinterpret_cast<const uint32_t*>(&h);
        }
        asm volatile("st.global.cs.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(u[0]), "r"(u[1]), "r"(u[2]), "r"(u[3]) : "memory");
    } else if ((reinterpret_cast<uintptr_t>(p) & 31u) == 0) {
        asm volatile("st.global.L1::no_allocate.L2::evict_first.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                     ::"l"(p), "f"(x[0]), "f"(x[1]), "f"(x[2]), "f"(x[3]), "f"(x[4]), "f"(x[5]), "f"(x[6]), "f"(x[7]) : "memory");
    } else {
        Vec8<U>::store(base, at, f);
    }
}

// out = c in, elements [from, to).
template <typename T, typename U>
__device__ __forceinline__ void scale(const void* in, void* out, int64_t from, int64_t to, int shift, bool wide_out, float c) {
    constexpr int kAhead = sizeof(T) == 2 ? 4 : 2;
    const f32x2 c2 = pk2(c, c);
    auto request = [&](Vec8<T> (&v)[kAhead], int64_t base) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t i = base + u * kUnit;
            v[u].clear();
            if (i >= from && i + 8 <= to) load_last(v[u], in, i);
        }
    };
    auto write = [&](const Vec8<T> (&v)[kAhead], int64_t base) {
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int64_t i = base + u * kUnit;
            if (i >= to) break;
            const bool whole = i >= from && i + 8 <= to;
            f32x2 f[4];
            v[u].get(f);
#pragma unroll
            for (int e = 0; e < 4; ++e) f[e] = mul2(f[e], c2);
            if (whole && wide_out) { store_once<U>(out, i, f); continue; }
            float e[8];
#pragma unroll
            for (int k = 0; k < 4; ++k) upk2(f[k], e[2 * k], e[2 * k + 1]);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                if (i + k < from || i + k >= to) continue;
                const float x = whole ? e[k] : element<T>(in, i + k) * c;
                if constexpr (sizeof(U) == 2) static_cast<__nv_bfloat16*>(out)[i + k] = __float2bfloat16_rn(x);
                else static_cast<float*>(out)[i + k] = x;
            }
        }
    };
    // two groups of vectors in turn: loads are on their way while the other group is written
    constexpr int64_t kStep = kUnit * kAhead;
    Vec8<T> a[kAhead], b[kAhead];
    int64_t base = (from + shift) / 8 * 8 - shift + int64_t(threadIdx.x) * 8;
    request(a, base);
    while (base < to) {
        request(b, base + kStep);
        write(a, base);
        base += kStep;
        if (base >= to) break;
        request(a, base + kStep);
        write(b, base);
        base += kStep;
    }
}

template <int N>
__global__ void __launch_bounds__(kThreads) grad_scale_kernel(const __grid_constant__ Tensors<N> p) {
    __shared__ double room[kThreads / 32];
    griddep_wait();                                // the parts; no CTA ends before the kernel in front has
    const double norm = sqrt(all_parts(p.parts, p.parts_n, room));
    const double ratio = double(p.max_norm) / (norm + double(p.eps));
    const float c = ratio < 1.0 ? float(ratio) : ratio >= 1.0 ? 1.f : float(ratio);          // NaN stays NaN
    if (p.write_norm && blockIdx.x == 0 && threadIdx.x == 0) {
        *p.norm = float(norm);
        if (p.coef != nullptr) *p.coef = c;
    }
    if (!p.clip) return;
    auto give = [&](int k, uint32_t start, uint32_t end) {     // chunks [start, end) of tensor k
        const void* in = p.in[k];
        void* out = p.out[k];
        if (in == out && c == 1.f) return;         // nothing to change
        const int64_t count = p.count[k] & kCount, from = int64_t(start - p.first[k]) * p.chunk, to = min(int64_t(end - p.first[k]) * p.chunk, count);
        const bool half_in = p.count[k] & kInBf16, half_out = p.count[k] & kOutBf16;
        const int shift = half_in ? shift_of<__nv_bfloat16>(in) : shift_of<float>(in);
        // the output's vectors begin where the input's do
        const bool wide = ((reinterpret_cast<uintptr_t>(out) - uintptr_t(shift) * (half_out ? 2 : 4)) & 15u) == 0;
        if (half_in) {
            if (half_out) scale<__nv_bfloat16, __nv_bfloat16>(in, out, from, to, shift, wide, c);
            else scale<__nv_bfloat16, float>(in, out, from, to, shift, wide, c);
        } else {
            if (half_out) scale<float, __nv_bfloat16>(in, out, from, to, shift, wide, c);
            else scale<float, float>(in, out, from, to, shift, wide, c);
        }
    };
    const uint32_t all = p.first[p.n];
    int k = p.at[blockIdx.x];
    if (p.side_by_side) {
        for (uint32_t behind = blockIdx.x; behind < all; behind += gridDim.x) {
            const uint32_t at = all - 1 - behind;
            while (p.first[k] > at) --k;
            give(k, at, at + 1);
        }
    } else {
        uint32_t from_chunk, end;
        for (my_chunks(all, from_chunk, end); end > from_chunk; --k) {
            const uint32_t start = max(from_chunk, p.first[k]);
            give(k, start, end);
            end = start;
        }
    }
}

struct Call {
    const hq_grad_tensor* t;
    int64_t n;
    bool clip;
    float max_norm, eps;
    float *norm, *coef;
    double* parts;
    int64_t chunk;
    unsigned most;                                 // CTAs of a launch of the norm
    cudaStream_t st;
};

// Tensors [from, to) laid out for both kernels; the number of their chunks.
template <int N>
uint32_t lay_out(Tensors<N>& p, const Call& c, int64_t from, int64_t to) {
    p.n = int(to - from);
    uint32_t chunks = 0;
    for (int k = 0; k < p.n; ++k) {
        const hq_grad_tensor& t = c.t[from + k];
        p.in[k] = t.grad;
        p.out[k] = t.out != nullptr ? t.out : const_cast<void*>(t.grad);
        const int32_t odt = t.out != nullptr ? t.out_dtype : t.dtype;
        p.count[k] = t.count | (t.dtype == HQ_BF16 ? kInBf16 : 0) | (odt == HQ_BF16 ? kOutBf16 : 0);
        p.first[k] = chunks;
        chunks += uint32_t((t.count + c.chunk - 1) / c.chunk);
    }
    p.first[p.n] = chunks;
    p.chunk = c.chunk;
    p.norm = c.norm; p.coef = c.coef; p.max_norm = c.max_norm; p.eps = c.eps; p.clip = c.clip;
    return chunks;
}
// The tensor each CTA begins with.
template <int N>
unsigned give_out(Tensors<N>& p, uint32_t chunks, unsigned most, bool last_first) {
    const unsigned grid = chunks < 1 ? 1u : chunks < most ? chunks : most;
    p.side_by_side = chunks / grid >= 8;
    const uint32_t per = (chunks + grid - 1) / grid;           // as in my_chunks
    int k = p.side_by_side && last_first ? p.n - 1 : 0;
    for (unsigned b = 0; b < grid; ++b) {
        const uint64_t begin = uint64_t(b) * per, end = begin + per < chunks ? begin + per : chunks;
        if (chunks == 0 || (!p.side_by_side && begin >= chunks)) { p.at[b] = 0; continue; }
        const uint64_t chunk = p.side_by_side ? (last_first ? chunks - 1 - b : b) : last_first ? end - 1 : begin;
        while (p.first[k + 1] <= chunk) ++k;
        while (p.first[k] > chunk) --k;
        p.at[b] = uint16_t(k);
    }
    return grid;
}
template <int N>
hq_status launch_norm(Tensors<N>& p, const Call& c, uint32_t chunks, int part, int* blocks) {
    const unsigned grid = give_out(p, chunks, c.most, false);
    p.parts = c.parts + part;
    *blocks = int(grid);
    grad_norm_kernel<N><<<grid, kThreads, 0, c.st>>>(p);
    return cudaGetLastError() == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}
template <int N>
hq_status launch_scale(Tensors<N>& p, const Call& c, uint32_t chunks, int parts, bool last) {
    const unsigned grid = c.clip ? give_out(p, chunks, kScaleBlocks, true) : 1u;
    p.parts = c.parts;
    p.parts_n = parts;
    p.write_norm = last;
    return launch_dependent(grad_scale_kernel<N>, grid, kThreads, 0, c.st, true, p) == cudaSuccess ? HQ_OK : HQ_ERR_CUDA;
}
// All tensors in one launch of each kernel.
template <int N>
hq_status run_once(const Call& c) {
    Tensors<N> p;
    const uint32_t chunks = lay_out(p, c, 0, c.n);
    int blocks = 0;
    const hq_status e = launch_norm(p, c, chunks, 0, &blocks);
    return e != HQ_OK ? e : launch_scale(p, c, chunks, blocks, true);
}
hq_status run_many(const Call& c) {
    Tensors<kMost> p;
    int part = 0, blocks = 0;
    for (int64_t from = 0; from < c.n; from += kMost) {        // the norms' parts of all tensors, then the outputs, the last tensors first
        const int64_t to = c.n - from > kMost ? from + kMost : c.n;
        const hq_status e = launch_norm(p, c, lay_out(p, c, from, to), part, &blocks);
        if (e != HQ_OK) return e;
        part += blocks;
    }
    for (int64_t from = (c.n - 1) / kMost * kMost, to = c.n; from >= 0; to = from, from -= kMost) {
        const hq_status e = launch_scale(p, c, lay_out(p, c, from, to), part, to == c.n);
        if (e != HQ_OK || !c.clip) return e;
    }
    return HQ_OK;
}

hq_status run(const hq_grad_tensor* t, int64_t n, bool clip, float max_norm, float eps, float* norm, float* coef, void* workspace, size_t ws_bytes,
              void* stream) {
    if (n < 0) return HQ_ERR_SHAPE;
    if ((n > 0 && t == nullptr) || norm == nullptr || workspace == nullptr) return HQ_ERR_INVALID_ARG;
    if (clip && (!(max_norm >= 0.f) || !(eps >= 0.f))) return HQ_ERR_INVALID_ARG;
    if (((reinterpret_cast<uintptr_t>(norm) | reinterpret_cast<uintptr_t>(coef)) & 3u) != 0 || (reinterpret_cast<uintptr_t>(workspace) & 7u) != 0) return HQ_ERR_ALIGNMENT;
    if (n > int64_t(kParts) * kMost) return HQ_ERR_UNSUPPORTED;
    if (ws_bytes < kParts * sizeof(double)) return HQ_ERR_WORKSPACE;
    int64_t total = 0;
    for (int64_t k = 0; k < n; ++k) {
        if (t[k].count < 0) return HQ_ERR_SHAPE;
        if (t[k].count == 0) continue;
        if (t[k].grad == nullptr || (t[k].dtype != HQ_F32 && t[k].dtype != HQ_BF16) || (t[k].out != nullptr && t[k].out_dtype != HQ_F32 && t[k].out_dtype != HQ_BF16))
            return HQ_ERR_INVALID_ARG;
        if (t[k].out == t[k].grad && t[k].out_dtype != t[k].dtype) return HQ_ERR_INVALID_ARG;
        if (reinterpret_cast<uintptr_t>(t[k].grad) % (t[k].dtype == HQ_BF16 ? 2 : 4) != 0 || reinterpret_cast<uintptr_t>(t[k].out) % (t[k].out_dtype == HQ_BF16 ? 2 : 4) != 0)
            return HQ_ERR_ALIGNMENT;
        if (t[k].count > int64_t(1) << 40) return HQ_ERR_UNSUPPORTED;
        total += t[k].count;
    }
    Call c{t, n, clip, max_norm, eps, norm, coef, static_cast<double*>(workspace), kUnit, unsigned(kNormBlocks), static_cast<cudaStream_t>(stream)};
    const int64_t launches = (n + kMost - 1) / kMost;
    if (launches * kNormBlocks > kParts) c.most = unsigned(kParts / launches);
    // chunks of one step of a CTA while these are fewer than the CTAs; larger ones keep a CTA's steps together
    while (total / c.chunk > kNormBlocks * 4 && c.chunk < kUnit * 16) c.chunk *= 2;
    while (total / c.chunk > INT_MAX / 2) c.chunk *= 2;
    // the parameters of a launch are copied three times on the host: no more of them than the tensors need
    if (n <= 32) return run_once<32>(c);
    if (n <= 128) return run_once<128>(c);
    if (n <= 384) return run_once<384>(c);
    return n <= kMost ? run_once<kMost>(c) : run_many(c);
}

}  // namespace
}  // namespace hq

extern "C" hq_status hq_grad_workspace_size(size_t* bytes) {
    if (bytes == nullptr) return HQ_ERR_INVALID_ARG;
    *bytes = hq::kParts * sizeof(double);
    return HQ_OK;
}
extern "C" hq_status hq_grad_norm(const hq_grad_tensor* tensors, int64_t n, float* norm, void* workspace, size_t ws_bytes, void* stream) {
    return hq::run(tensors, n, false, 0.f, 0.f, norm, nullptr, workspace, ws_bytes, stream);
}
extern "C" hq_status hq_grad_clip(const hq_grad_tensor* tensors, int64_t n, float max_norm, float eps, float* norm, float* coef, void* workspace,
                                  size_t ws_bytes, void* stream) {
    return hq::run(tensors, n, true, max_norm, eps, norm, coef, workspace, ws_bytes, stream);
}
