// Loads from memory straight into LDS, and the waits that go with them.
#pragma once
#include "conv_common.h"

namespace cw {

// One 16-byte-per-lane buffer load straight into LDS at byte address lds_addr (+ 16*lane).
static __device__ __forceinline__ void load_to_lds(u32x4 desc, unsigned voff, unsigned soff, unsigned lds_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
                 :
                 : "s"(lds_addr), "v"(voff), "s"(desc), "s"(soff)
                 : "memory", "m0");
}

// The same from an address of each lane's own; from an offset of its own behind one address; and a byte, zero-extended to four, to lds_addr + 4*lane.
static __device__ __forceinline__ void load_to_lds(const void *from, unsigned lds_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" : : "s"(lds_addr), "v"(from) : "memory", "m0");
}
static __device__ __forceinline__ void load_to_lds(const void *base, unsigned offset, unsigned lds_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" : : "s"(lds_addr), "v"(offset), "s"(base) : "memory", "m0");
}
static __device__ __forceinline__ void load_byte_to_lds(const void *from, unsigned lds_addr) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ubyte %1, off" : : "s"(lds_addr), "v"(from) : "memory", "m0");
}

// Waits until at most N of this thread's loads are outstanding, then the workgroup barrier.
template <int N>
static __device__ __forceinline__ void wait_loads_and_barrier() {
    static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" : : "n"(N) : "memory");
}

// The same, also waiting for this thread's own LDS accesses (reads returned, writes done).
template <int N>
static __device__ __forceinline__ void wait_lds_loads_and_barrier() {
    static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" : : "n"(N) : "memory");
}

// Waits for this thread's LDS accesses alone, then the workgroup barrier.
static __device__ __forceinline__ void wait_lds_and_barrier() { asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" : : : "memory"); }

// Raw buffer descriptor (stride 0) as four scalars, for use as an asm operand.
static __device__ __forceinline__ u32x4 make_desc(const void *p, unsigned bytes) {
    const unsigned long long v = reinterpret_cast<unsigned long long>(p);
    return u32x4{(unsigned)v, (unsigned)(v >> 32) & 0xffffu, bytes, 0x00020000u};
}

}  // namespace cw
