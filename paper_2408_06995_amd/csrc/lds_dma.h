// Loads from memory straight into LDS, and their waits: what the kernels with LDS rings share.
#pragma once
#include <hip/hip_runtime.h>

namespace fpq {

typedef int v4i __attribute__((ext_vector_type(4)));

// One wave-wide 16-byte-per-lane load from a buffer straight into LDS: lane i's bytes land at
// lds_addr + 16 i; a lane whose voff is not below the buffer's size gets zeros.  Written as inline
// assembly so that the compiler's wait-count insertion does not see an LDS write here (it would
// drain every outstanding load before each following LDS read); the waits are placed by hand in
// the main loop.  m0 carries the LDS base; nothing else in these kernels uses m0.
__device__ __forceinline__ void dma16(v4i rsrc, unsigned voff, unsigned lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(voff), "s"(rsrc)   // uniform, but may live in a VGPR
                 : "memory");
}

// The same with four bytes per lane.
__device__ __forceinline__ void dma4(v4i rsrc, unsigned voff, unsigned lds_addr)
{
    asm volatile("s_mov_b32 m0, %0\n\tbuffer_load_dword %1, %2, 0 offen lds"
                 :
                 : "s"(__builtin_amdgcn_readfirstlane(lds_addr)), "v"(voff), "s"(rsrc)
                 : "memory");
}

// Raw buffer descriptor: base address, no stride, size in bytes, 32-bit untyped data.
__device__ __forceinline__ v4i make_rsrc(const void* base, unsigned bytes)
{
    const unsigned long long b = reinterpret_cast<unsigned long long>(base);
    v4i r;
    r.x = (int)(unsigned)b;
    r.y = (int)((unsigned)(b >> 32) & 0xffffu);
    r.z = (int)bytes;
    r.w = 0x00020000;
    return r;
}

// s_waitcnt immediate that waits for vmcnt <= n only (gfx9 encoding: vmcnt in bits 3:0 and 15:14,
// expcnt 6:4 and lgkmcnt 11:8 left at their maxima).
constexpr int vmcnt_imm(int n) { return (n & 15) | (7 << 4) | (15 << 8) | ((n >> 4) << 14); }

__device__ __forceinline__ unsigned lds_address(const void* p)
{
    return (unsigned)(size_t)(const __attribute__((address_space(3))) void*)p;
}

// This wavefront's loads have landed and its reads of LDS are done, and so are those of all wavefronts of the workgroup.
__device__ __forceinline__ void dma_barrier() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

}  // namespace fpq
