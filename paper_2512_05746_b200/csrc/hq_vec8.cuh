// 8 values of a row that a thread holds: 16 bytes of bf16 or 32 of fp32, and their fp32 form in pairs (two-wide arithmetic).
#pragma once

#include "hq_common.cuh"
#include "hq_fwht.cuh"

namespace hq {

// 8 channels of a lane, as they lie in memory and as four pairs of floats.
template <typename T> struct Vec8;
template <> struct Vec8<__nv_bfloat16> {
    uint4 w;
    __device__ __forceinline__ void clear() { w = make_uint4(0u, 0u, 0u, 0u); }
    __device__ __forceinline__ void load(const void* base, int64_t at) { w = *reinterpret_cast<const uint4*>(static_cast<const __nv_bfloat16*>(base) + at); }
    __device__ __forceinline__ Vec8 of(int lane) const {       // the other lane's
        Vec8 r;
        r.w.x = __shfl_sync(0xffffffffu, w.x, lane); r.w.y = __shfl_sync(0xffffffffu, w.y, lane);
        r.w.z = __shfl_sync(0xffffffffu, w.z, lane); r.w.w = __shfl_sync(0xffffffffu, w.w, lane);
        return r;
    }
    __device__ __forceinline__ void get(f32x2 (&f)[4]) const {
        const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int e = 0; e < 4; ++e) f[e] = pk2(__uint_as_float(u[e] << 16), __uint_as_float(u[e] & 0xFFFF0000u));
    }
    static __device__ __forceinline__ void store(void* base, int64_t at, const f32x2 (&f)[4]) {
        uint32_t u[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            float a, b;
            upk2(f[e], a, b);
            const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
            u[e] = *reinterpret_cast<const uint32_t*>(&h);
        }
        *reinterpret_cast<uint4*>(static_cast<__nv_bfloat16*>(base) + at) = make_uint4(u[0], u[1], u[2], u[3]);
    }
    __device__ __forceinline__ void load_wide(const void* base, int64_t at) { load(base, at); }
    static __device__ __forceinline__ void store_wide(void* base, int64_t at, const f32x2 (&f)[4]) { store(base, at, f); }
};
template <> struct Vec8<float> {
    float4 a, b;
    __device__ __forceinline__ void clear() { a = b = make_float4(0.f, 0.f, 0.f, 0.f); }
    __device__ __forceinline__ void load(const void* base, int64_t at) {
        const float4* p = reinterpret_cast<const float4*>(static_cast<const float*>(base) + at);
        a = p[0]; b = p[1];
    }
    __device__ __forceinline__ Vec8 of(int lane) const {
        Vec8 r;
        r.a.x = __shfl_sync(0xffffffffu, a.x, lane); r.a.y = __shfl_sync(0xffffffffu, a.y, lane);
        r.a.z = __shfl_sync(0xffffffffu, a.z, lane); r.a.w = __shfl_sync(0xffffffffu, a.w, lane);
        r.b.x = __shfl_sync(0xffffffffu, b.x, lane); r.b.y = __shfl_sync(0xffffffffu, b.y, lane);
        r.b.z = __shfl_sync(0xffffffffu, b.z, lane); r.b.w = __shfl_sync(0xffffffffu, b.w, lane);
        return r;
    }
    __device__ __forceinline__ void get(f32x2 (&f)[4]) const { f[0] = pk2(a.x, a.y); f[1] = pk2(a.z, a.w); f[2] = pk2(b.x, b.y); f[3] = pk2(b.z, b.w); }
    static __device__ __forceinline__ void store(void* base, int64_t at, const f32x2 (&f)[4]) {
        float4* p = reinterpret_cast<float4*>(static_cast<float*>(base) + at);
        float4 x, y;
        upk2(f[0], x.x, x.y); upk2(f[1], x.z, x.w); upk2(f[2], y.x, y.y); upk2(f[3], y.z, y.w);
        p[0] = x; p[1] = y;
    }
    // One access of 32 bytes where the address allows it: of two of 16, each warp's touches half of every sector of its row.
    __device__ __forceinline__ void load_wide(const void* base, int64_t at) {
        const float* p = static_cast<const float*>(base) + at;
        if ((reinterpret_cast<uintptr_t>(p) & 31u) == 0)
            asm volatile("ld.global.v8.f32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                         : "=f"(a.x), "=f"(a.y), "=f"(a.z), "=f"(a.w), "=f"(b.x), "=f"(b.y), "=f"(b.z), "=f"(b.w) : "l"(p) : "memory");
        else load(base, at);
    }
    static __device__ __forceinline__ void store_wide(void* base, int64_t at, const f32x2 (&f)[4]) {
        float* p = static_cast<float*>(base) + at;
        float4 x, y;
        upk2(f[0], x.x, x.y); upk2(f[1], x.z, x.w); upk2(f[2], y.x, y.y); upk2(f[3], y.z, y.w);
        if ((reinterpret_cast<uintptr_t>(p) & 31u) == 0)
            asm volatile("st.global.v8.f32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                         ::"l"(p), "f"(x.x), "f"(x.y), "f"(x.z), "f"(x.w), "f"(y.x), "f"(y.y), "f"(y.z), "f"(y.w) : "memory");
        else store(base, at, f);
    }
};

__device__ __forceinline__ float pair_sum(f32x2 v) { float a, b; upk2(v, a, b); return a + b; }

}  // namespace hq
