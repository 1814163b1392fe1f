// What the MFMA kernels of attention share: fragment types, exchanges between the lanes of a row, direct loads to LDS and the waits
// that go with them.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace pa {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

__device__ __forceinline__ uint32_t pack_bf16x2(float a, float b) {
    // round to nearest even; inputs are finite probabilities or outputs
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    f32x2 v = {a, b};
    bf16x2_t r = __builtin_convertvector(v, bf16x2_t);
    return __builtin_bit_cast(uint32_t, r);
}

// The largest of a query row's values, which lie in the lanes l, l ^ 16, l ^ 32 and l ^ 48, in all of them, without going through
// LDS.  v_permlane32_swap exchanges lanes 32..63 of its first operand with lanes 0..31 of its second, v_permlane16_swap the odd
// rows of 16 lanes of the first with the even ones of the second: fed the same value twice they leave both values of a pair in
// every lane.  Written as inline assembly (the compiler builtin folded its two results into one); the s_nop pairs cover the
// wait states the instructions need after a VALU write of their operands and before a VALU read of them.
__device__ __forceinline__ float row_max(float x) {
    float a = x, b = x;
    asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
    a = b = fmaxf(a, b);
    asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
    return fmaxf(a, b);
}
// ... and their sum.
__device__ __forceinline__ float row_sum(float x) {
    float a = x, b = x;
    asm volatile("s_nop 1\n\tv_permlane32_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
    a = b = a + b;
    asm volatile("s_nop 1\n\tv_permlane16_swap_b32 %0, %1\n\ts_nop 1" : "+v"(a), "+v"(b));
    return a + b;
}

// Workgroup barrier without the memory fence of __syncthreads(): the fence would make the compiler wait
// for every outstanding global->LDS load, including the ones meant to stay in flight.  Completion of
// the loads that must be visible is awaited explicitly (wait_vm_all) before the barrier.
__device__ __forceinline__ void wg_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}
// s_waitcnt vmcnt(0) (expcnt and lgkmcnt left alone), as the builtin so that the compiler's own wait
// bookkeeping sees it and does not repeat it later.
__device__ __forceinline__ void wait_vm_all() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0x0F70);
    asm volatile("" ::: "memory");
}

// Direct global -> LDS load of 16 bytes per lane: lane l of the wave writes LDS bytes
// [lds_addr + 16 l, lds_addr + 16 l + 16) with the 16 bytes at its own global address g.  lds_addr is
// wave-uniform.  Issued as inline assembly so that the compiler does not see an LDS store in flight: it
// would otherwise wait for it before every later LDS read, and the load could not overlap the
// arithmetic on the other ring slot.  The explicit wait_vm_all() + wg_barrier() order it instead.
__device__ __forceinline__ void load_to_lds_16(const void* g, unsigned lds_addr) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(g), "s"(lds_addr) : "memory");
}
// The same with the global address given as a wave-uniform base plus a 32-bit unsigned byte offset per lane.
__device__ __forceinline__ void load_to_lds_16(const void* base, unsigned off, unsigned lds_addr) {
    asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds_addr) : "memory");
}
// One byte per lane: lane l of the wave writes the 32-bit word at lds_addr + 4 l (the byte in its low 8 bits).
__device__ __forceinline__ void load_to_lds_1(const void* g, unsigned lds_addr) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_ubyte %0, off" ::"v"(g), "s"(lds_addr) : "memory");
}
// Four bytes per lane, past the L2: lane l of the wave writes the 32-bit word at lds_addr + 4 l.
__device__ __forceinline__ void load_to_lds_4(const void* g, unsigned lds_addr) {
    asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dword %0, off sc1" ::"v"(g), "s"(lds_addr) : "memory");
}
__device__ __forceinline__ unsigned lds_address(const void* p) {
    return static_cast<unsigned>(reinterpret_cast<uintptr_t>((__attribute__((address_space(3))) const unsigned char*)(p)));
}

// The same value, of which the compiler knows nothing: what is derived from it is worked out here and not kept in registers from before a loop.
__device__ __forceinline__ unsigned worked_out_here(unsigned x) {
    asm volatile("" : "+v"(x));
    return x;
}
// Nothing is moved across this place: what is written before it is issued before it.  (Left to itself the compiler reads one fragment at a time
// from LDS, waits, and multiplies.)
__device__ __forceinline__ void in_this_order() { __builtin_amdgcn_sched_barrier(0); }
// s_waitcnt vmcnt(N): all but the newest N of the wave's loads have landed.
template <int N>
__device__ __forceinline__ void wait_vm() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt((N & 15) | ((N >> 4) << 14) | 0x0F70);
    asm volatile("" ::: "memory");
}
// The wave's LDS accesses are done, then the workgroup barrier.
__device__ __forceinline__ void lds_barrier() {
    asm volatile("" ::: "memory");
    __builtin_amdgcn_s_waitcnt(0xC07F);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
}

}  // namespace pa
