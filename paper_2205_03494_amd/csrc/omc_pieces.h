// Loads straight into LDS by count, and the order of tiles, of the kernels whose workgroups take one tile after the other.
#pragma once
#include "omc_mma.h"

namespace omc {

// Direct loads into LDS (see load_to_lds): lane l's 16 bytes to `to` + TO + 16 l, in the lanes that `lanes` has; all lanes are on before and after.
template <uint32_t TO>
__device__ __forceinline__ void load_pieces(const uint8_t *base, uint32_t off, uint32_t to, uint64_t lanes) {
    asm volatile("s_add_u32 m0, %0, %3\n\ts_mov_b64 exec, %4\n\tglobal_load_lds_dwordx4 %1, %2\n\ts_mov_b64 exec, -1" ::"s"(to), "v"(off), "s"(base), "n"(TO), "s"(lanes)
                 : "memory", "m0", "scc");
}
template <uint32_t TO>
__device__ __forceinline__ void load_pieces(const uint8_t *lanes_own, uint32_t to, uint64_t lanes) {
    asm volatile("s_add_u32 m0, %0, %2\n\ts_mov_b64 exec, %3\n\tglobal_load_lds_dwordx4 %1, off\n\ts_mov_b64 exec, -1" ::"s"(to), "v"(lanes_own), "n"(TO), "s"(lanes)
                 : "memory", "m0", "scc");
}

// The same with 4 bytes of a lane, to `to` + 4 l.
__device__ __forceinline__ void load_dwords(const float *lanes_own, uint32_t to, uint64_t lanes) {
    asm volatile("s_mov_b32 m0, %0\n\ts_mov_b64 exec, %2\n\tglobal_load_lds_dword %1, off\n\ts_mov_b64 exec, -1" ::"s"(to), "v"(lanes_own), "s"(lanes) : "memory", "m0");
}

// Between a wave's writes to LDS and reads by its other lanes, and back.  The hardware takes a wave's LDS accesses in order; the compiler must not carry a value over.
__device__ __forceinline__ void lanes_exchange() { asm volatile("" ::: "memory"); }

// The same address in all lanes, in scalar registers whatever the compiler thinks of its origin.
__device__ __forceinline__ const uint8_t *in_scalars(const uint8_t *p) {
    const uint64_t v = reinterpret_cast<uintptr_t>(p);
    const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v)), hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32));
    return reinterpret_cast<const uint8_t *>(static_cast<uint64_t>(hi) << 32 | lo);
}

// Tile x of a grid of tiles: as tile_of_block deals them to the workgroups, x for the workgroup's number.
__device__ __forceinline__ void tile_of(uint32_t x, uint32_t group_rows, uint32_t tiles_m, uint32_t tiles_n, uint32_t &tm, uint32_t &tn) {
    const uint32_t total = tiles_m * tiles_n, q = total / 8, r = total % 8, die = x % 8, id = die * q + min(die, r) + x / 8;
    const uint32_t rows = min(tiles_m, group_rows), group = id / (rows * tiles_n), first = group * rows, height = min(tiles_m - first, rows), in = id - group * rows * tiles_n;
    tm = first + in % height;
    tn = in / height;
}

}  // namespace omc
