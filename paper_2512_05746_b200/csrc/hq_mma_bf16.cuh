// bf16 products on the tensor cores (tcgen05.mma kind::f16, fp32 accumulators in tensor memory): descriptors, issue, and the
// small pieces of arithmetic the attention kernels share.
#pragma once

#include <cuda.h>

#include "hq_common.cuh"

namespace hq {

// hq_gemm.cu: bf16 rows [batch][rows][pitch] whose columns h * dh .. hold head h, as (dh, head, row, sample); boxes of 64 channels
// x box_rows rows of one head in the 128-byte swizzle.  What lies beyond dh or beyond a sample's rows is filled with zeros.
bool encode_heads_bf16(CUtensorMap* tm, const void* base, uint64_t dh, uint64_t heads, uint64_t rows, uint64_t batch, uint64_t pitch,
                       uint32_t box_rows);

// Shared-memory matrix descriptor without swizzle: 8 x 16-byte core matrices; `lbo` / `sbo` are the byte distances between
// core matrices along K and along M/N for a K-major operand, and along K and along N (groups of 8) for an MN-major one.
__device__ __forceinline__ uint64_t make_desc_noswizzle(uint32_t smem_addr, uint32_t lbo, uint32_t sbo) {
    uint64_t d = 0;
    d |= uint64_t((smem_addr & 0x3FFFFu) >> 4);
    d |= uint64_t((lbo >> 4) & 0x3FFFu) << 16;
    d |= uint64_t((sbo >> 4) & 0x3FFFu) << 32;
    d |= uint64_t(1) << 46;
    return d;
}

// Instruction descriptor for kind::f16 with bf16 operands and an fp32 accumulator, tile M x N; B MN-major when asked.
__host__ __device__ constexpr uint32_t make_idesc_bf16(int M, int N, bool b_mn_major) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (b_mn_major ? (1u << 16) : 0u) | (uint32_t(N >> 3) << 17) |
           (uint32_t(M >> 4) << 24);
}

__device__ __forceinline__ void mma_bf16(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc,
                                         uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
        ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

__device__ __forceinline__ void tmem_st_32x16(uint32_t taddr, const uint32_t (&r)[16]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
        "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
          "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float ex2(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t*>(&h);
}

// The same with the A operand in tensor memory: lane r holds row r, each 32-bit column two consecutive elements of K.
__device__ __forceinline__ void mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
        : "memory");
}

// Waits of a converged warp, and of one thread, on a phase that has mostly completed when they are asked: a poll without a
// suspend-time hint and a vote take 27 cycles then (mbar_wait with a vote around it 105), and a waiting warp is told 114 cycles after
// the arrival (144 with the hint).  Bounded as mbar_wait: after about a second `code` is recorded and false returned, in every lane.
__device__ __forceinline__ bool mbar_poll(uint64_t* bar, uint32_t parity) {
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity)
        : "memory");
    return ok != 0;
}
// In line, the loop too: a call would have the live registers moved to where the callee leaves them alone, wait or not.
__device__ __forceinline__ uint32_t clock_lo() { uint32_t t; asm volatile("mov.u32 %0, %%clock;" : "=r"(t)); return t; }
__device__ __forceinline__ bool mbar_wait_warp(uint64_t* bar, uint32_t parity, int32_t* dev_status, int32_t code) {
    bool ok = __all_sync(0xffffffffu, mbar_poll(bar, parity));
    if (!ok) {
        const uint32_t t0 = clock_lo();
        do ok = __all_sync(0xffffffffu, mbar_poll(bar, parity)) != 0;
        while (!ok && __all_sync(0xffffffffu, clock_lo() - t0 < 2000000000u));
        if (!ok && dev_status) atomicExch(dev_status, code);
    }
    return ok;
}
__device__ __forceinline__ bool mbar_wait_lane(uint64_t* bar, uint32_t parity, int32_t* dev_status, int32_t code) {
    bool ok = mbar_poll(bar, parity);
    if (!ok) {
        const uint32_t t0 = clock_lo();
        do ok = mbar_poll(bar, parity);
        while (!ok && clock_lo() - t0 < 2000000000u);
        if (!ok && dev_status) atomicExch(dev_status, code);
    }
    return ok;
}

// What this thread has issued is complete before it gives up the tensor memory and the tiles (one lane; `bar`: count 1, used once): a
// CTA that a wait of another kind has ended early must not leave products running.
__device__ __forceinline__ void mma_drain(uint64_t* bar) {
    mma_commit(bar);
    mbar_wait_lane(bar, 0, nullptr, 0);
}

// 16-byte aligned bulk copy global -> shared, completion counted on an mbarrier.
__device__ __forceinline__ void bulk_load(void* smem_dst, const void* src, uint32_t bytes, uint64_t* bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(smem_dst)), "l"(src), "r"(bytes), "r"(smem_u32(bar))
                 : "memory");
}

// Descriptor of an MN-major tile of 128-byte rows (64 elements of N each) in the 128-byte swizzle.
__device__ __forceinline__ uint64_t make_sw128_mnmajor_desc(uint32_t smem_addr, uint32_t atom_stride_bytes) {
    uint64_t d = 0;
    d |= uint64_t((smem_addr & 0x3FFFFu) >> 4);
    d |= uint64_t((atom_stride_bytes >> 4) & 0x3FFFu) << 16;   // between 64-element groups along N
    d |= uint64_t(1024 >> 4) << 32;                            // between 8-row groups along K
    d |= uint64_t(1) << 46;
    d |= uint64_t(2) << 61;
    return d;
}

}  // namespace hq
