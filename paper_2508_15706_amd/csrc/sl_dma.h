// Loads from memory into LDS past the registers, and the waits that belong to them.
#pragma once
#include "sl_device.h"

// 16 bytes per lane from memory to LDS at `lds` + 16 * lane, past the registers.  The instruction is
// written out because the compiler, which cannot tell the stages apart, would wait for all of them before every read
// of LDS; it has no result in a register, and the waits for it are written out too.  (m0 is the compiler's own, which warns that it will not
// be kept: that is what the list of clobbers is to say.)
#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
SL_DEV void dma16(const unsigned char *base, unsigned lane_off, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(lane_off), "s"(base) : "m0", "memory");
}
// The same with 4 bytes per lane, each from an address of its own, to `lds` + 4 * lane.
SL_DEV void dma4(const void *from, unsigned lds)
{
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(from) : "m0", "memory");
}
#pragma clang diagnostic pop
template <int N>
SL_DEV void wait_dma() { asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory"); }
// All waves' reads of LDS are done and have arrived.
SL_DEV void stage_barrier()
{
    asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
}
