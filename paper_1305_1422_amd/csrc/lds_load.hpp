// Loads straight into LDS: lane l's bytes go to LDS byte address lds_base + (bytes a lane) l; lds_base, wavefront-uniform, is passed in M0.
//
// Written as inline assembly on purpose: the compiler would otherwise make every later LDS read wait for these loads, although they fill
// a buffer that is NOT being read; the ordering that matters is enforced by hand (a wait for vector memory before the barrier that
// publishes the buffer).  M0 is a reserved register that the compiler reloads before each use of its own, so overwriting it is safe.
// A load takes M0 as it was a wait state earlier: the s_nop (the compiler keeps such distances for its own instructions only).
#pragma once

#include <hip/hip_runtime.h>

namespace som {

#pragma clang diagnostic push
#pragma clang diagnostic ignored "-Winline-asm"
// 16 bytes per lane from a full 64-bit address per lane.
__device__ __forceinline__ void load16_to_lds(const void *lane_address, unsigned lds_base) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" : : "v"(lane_address), "s"(lds_base) : "memory", "m0");
}
// From a wavefront-uniform 64-bit base in scalar registers + an unsigned 32-bit byte offset per lane: the offsets can be loop constants
// while the base advances with scalar arithmetic, so that a load costs no vector ALU instruction.
__device__ __forceinline__ void load16_to_lds_at(const void *base, unsigned lane_offset, unsigned lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" : : "v"(lane_offset), "s"(base), "s"(lds_base) : "memory", "m0");
}
// The same for 4 bytes per lane.
__device__ __forceinline__ void load4_to_lds_at(const void *base, unsigned lane_offset, unsigned lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1" : : "v"(lane_offset), "s"(base), "s"(lds_base) : "memory", "m0");
}
#pragma clang diagnostic pop

}  // namespace som
