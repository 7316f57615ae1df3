// What the gfx950 kernels of all source files share: operand types, 16-byte loads and stores, exact waits, rounding to bf16 and
// copies from memory straight into LDS.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace lora {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

static __device__ __forceinline__ bf16x8 as_bf16x8(uint4 u) { return __builtin_bit_cast(bf16x8, u); }

static __device__ __forceinline__ uint4 ld16(const uint16_t *p) { return *reinterpret_cast<const uint4 *>(p); }

// 16-byte load of data that is read exactly once per launch (a decode batch's adapter weights, the
// x rows of a token-heavy shrink): marked non-temporal, so it is not kept in the caches on its way.
// A plain read of 2 GB runs at 6.2 TB/s on this chip with ordinary loads and at 7.0 TB/s with these.
static __device__ __forceinline__ uint4 ld16_stream(const uint16_t *p)
{
    typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
    const u32x4 v = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p));
    return uint4{v.x, v.y, v.z, v.w};
}

// 16-byte store of data this launch will not read again (y).
static __device__ __forceinline__ void st16_stream(uint16_t *p, uint4 v)
{
    typedef __attribute__((ext_vector_type(4))) unsigned u32x4;
    __builtin_nontemporal_store(u32x4{v.x, v.y, v.z, v.w}, reinterpret_cast<u32x4 *>(p));
}

static __device__ __forceinline__ float bf16_bits_to_f32(uint32_t b) { return __uint_as_float(b << 16); }

// The s_waitcnt immediate of the gfx9 family (gfx950 included): vmcnt in bits 3:0 and 15:14, expcnt in
// bits 6:4, lgkmcnt in bits 11:8; a field at its maximum waits for nothing.
#if defined(__HIP_DEVICE_COMPILE__) && !defined(__gfx950__)
#error "the hand-built s_waitcnt immediate below is the gfx9 encoding: this file is for gfx950"
#endif
[[maybe_unused]] constexpr unsigned kWaitcntVmcnt0 = (0u << 0) | (7u << 4) | (15u << 8) | (0u << 14);  // vmcnt(0), nothing else
static_assert(kWaitcntVmcnt0 == 0x0F70, "vmcnt(0) expcnt(7) lgkmcnt(15)");

// This wavefront's vector memory operations (its stores among them) have completed.  The two signal
// fences keep the compiler from moving memory operations across the wait in either direction.
static __device__ __forceinline__ void stores_done()
{
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    __builtin_amdgcn_s_waitcnt(kWaitcntVmcnt0);
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

// at most N of this wavefront's vector memory operations are still under way
template <int N>
static __device__ __forceinline__ void wait_vm()
{
    static_assert(N >= 0 && N < 64, "vmcnt has six bits");
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
    __atomic_signal_fence(__ATOMIC_SEQ_CST);
}

static __device__ __forceinline__ uint32_t pack_bf16_rne(float a, float b)
{
    typedef __attribute__((ext_vector_type(2))) float f32x2;
    typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
    const f32x2 f = {a, b};
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f, bf16x2));
}

// One wavefront copies 1 KB from memory into LDS without passing through registers: lane l's 16 bytes
// at gptr (per lane) land at lds_piece + 16*l (lds_piece wave-uniform).  Written as an instruction the
// compiler does not look into: for its own form of this load it waits until the copy has landed
// before the wavefront may issue anything else that touches LDS or the registers involved, which
// leaves nothing of the overlap the copy exists for.  The caller waits and synchronises the work group before anyone
// reads the destination: for all of the wavefront's memory operations (vmcnt(0)), or for all but the last N, if at least N that the compiler
// knows of are issued behind the copies on every way to the wait: a branch or a scheduling barrier between keeps them there.
static __device__ __forceinline__ void dma16_to_lds(const uint4 *gptr, const uint4 *lds_piece)
{
    const uint32_t lds_addr = __builtin_amdgcn_readfirstlane(
        (uint32_t)(uintptr_t)(const __attribute__((address_space(3))) void *)lds_piece);
    // M0 carries the LDS address of the piece; its old value is put back, so the register the
    // compiler reserves for itself is unchanged after the statement
    uint32_t saved_m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\t"
                 "s_mov_b32 m0, %0"
                 : "=&s"(saved_m0)
                 : "v"(gptr), "s"(lds_addr)
                 : "memory");
}

// Two and four such copies, to consecutive KB from LDS address `to`, for a loop in which every instruction beside its matrix
// instructions counts.  An instruction's offset is added to the address in memory and to the one in LDS, so M0 is set once:
// copy q's source is given less q KB.
static __device__ __forceinline__ void dma16x2_to_lds(const void *g0, const void *g1, uint32_t to)
{
    uint32_t saved_m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %3\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\t"
                 "global_load_lds_dwordx4 %2, off offset:1024\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved_m0)
                 : "v"(g0), "v"(g1), "s"(to)
                 : "memory");
}
static __device__ __forceinline__ void dma16x4_to_lds(const void *g0, const void *g1, const void *g2, const void *g3, uint32_t to)
{
    uint32_t saved_m0;
    asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %5\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off\n\t"
                 "global_load_lds_dwordx4 %2, off offset:1024\n\tglobal_load_lds_dwordx4 %3, off offset:2048\n\t"
                 "global_load_lds_dwordx4 %4, off offset:3072\n\ts_mov_b32 m0, %0"
                 : "=&s"(saved_m0)
                 : "v"(g0), "v"(g1), "v"(g2), "v"(g3), "s"(to)
                 : "memory");
}

}  // namespace lora
