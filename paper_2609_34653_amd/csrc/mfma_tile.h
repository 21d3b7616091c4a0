// Building blocks of the attention kernels: MFMA operand types, the swizzles of K and V tiles in LDS,
// direct global -> LDS loads, transposing LDS reads and the exchange between a wave's halves.
#pragma once

#include "common.h"

namespace omnitide {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float floatx16 __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float floatx4 __attribute__((ext_vector_type(4)));

// Tiles of 64 keys for the 32x32 products, row-major [64][D]:
//   K  16-byte chunks XOR-swizzled by kswz(key), so the 8 (and 16) lanes one LDS cycle serves
//      read distinct bank groups when they fetch rows perm_key(0..31) of the S^T tile.
//   V  32-byte units XOR-swizzled by vswz(key); the V^T operand of O^T = V^T P^T is gathered
//      with the transposing 64-bit LDS read (ds_read_b64_tr_b16): within a 16-lane group, lane i
//      receives element i%4 of the 8-byte rows read by lanes i/4, 4+i/4, 8+i/4, 12+i/4, i.e.
//      one dimension of four consecutive keys.  Each group reads four rows x 32 bytes; the
//      swizzle puts them (and the neighbouring group's) in distinct banks.
// A direct load's LDS destination is lane-contiguous, so the swizzles are realised by choosing
// which global chunk each lane fetches.
__device__ inline int kswz(int key) {
  return (key & 3) | ((key >> 2) & 4) | ((key << 1) & 8);
}
template <int D>
__device__ inline int vswz(int key) {
  return D == 128 ? ((key & 3) ^ ((key & 1) << 2)) : (key & 3);
}

__device__ inline floatx16 mfma(bf16x8 a, bf16x8 b, floatx16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// S^T row r of a 32x32 MFMA tile holds key perm_key(r): lane half h, accumulator i <-> key 16h+i.
__device__ inline int perm_key(int r) { return 16 * ((r & 7) >> 2) + 4 * (r >> 3) + (r & 3); }

__device__ inline u32x4 ld16(const uint16_t* p) { return *reinterpret_cast<const u32x4*>(p); }

typedef short shortx4 __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) void lds_void;

__device__ inline shortx4 ld_tr(const uint16_t* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) shortx4*)(p));
}

__device__ inline uint32_t lds_addr(const void* p) {
  return static_cast<uint32_t>(reinterpret_cast<size_t>((const lds_void*)p));
}

// 16-byte direct global -> LDS load: lane i reads base + voff_i and writes 16 bytes at LDS byte
// address lds_base + 16 i.  Written as inline assembly (uniform base in SGPRs, per-lane 32-bit
// offset) so that issuing it costs no vector instructions and so that the compiler's wait
// insertion does not treat it as a pending LDS write (it would otherwise make later LDS reads of
// other buffers wait for it).  Callers wait for it explicitly (s_waitcnt vmcnt(0) + barrier)
// before any lane reads the buffer it fills.  One wait state is required between the M0 write
// and the load.  M0 is not listed as clobbered (the compiler reserves it and ignores such
// clobbers): the kernels that include this have no other M0 user, so no compiler value lives in M0.
__device__ inline void dma16(const void* base, uint32_t voff, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1"
               :
               : "v"(voff), "s"(base), "s"(lds_base)
               : "memory");
}
// The same for data that is read once: it is not kept in the caches at the cost of other lines.
__device__ inline void dma16_once(const void* base, uint32_t voff, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1 nt"
               :
               : "v"(voff), "s"(base), "s"(lds_base)
               : "memory");
}
// The same for 4 bytes per lane (lane i writes LDS byte address lds_base + 4 i).
__device__ inline void dma4(const void* base, uint32_t voff, uint32_t lds_base) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dword %0, %1"
               :
               : "v"(voff), "s"(base), "s"(lds_base)
               : "memory");
}

// This lane's index in its wave, recomputed (two instructions) at the point of use.  The span
// paths index by lane only now and then; a fresh value there spares the register allocator a
// long-lived copy, which it would otherwise spill and reload behind the tile prefetches.
__device__ inline int lane_now() {
  int r;   // volatile: not hoisted out of the loop (where it would be spilled again)
  asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(r));
  return r;
}

// max and sum over both 32-lane halves: v_permlane32_swap exchanges them without LDS.
__device__ inline float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ inline float sum_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false,
                                                  false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// Stores four consecutive output values as float32, or rounded to bf16 (nearest even).
__device__ inline void store_row4(void* out, size_t idx, bool out_bf16, floatx4 v) {
  if (out_bf16) {
    typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
    *reinterpret_cast<bf16x4*>(static_cast<__bf16*>(out) + idx) =
        bf16x4{static_cast<__bf16>(v[0]), static_cast<__bf16>(v[1]), static_cast<__bf16>(v[2]),
               static_cast<__bf16>(v[3])};
  } else {
    *reinterpret_cast<floatx4*>(static_cast<float*>(out) + idx) = v;
  }
}

template <int B, class T>
__device__ inline T& pick(T& a, T& b) {
  if constexpr (B == 0) return a; else return b;
}

}  // namespace
}  // namespace omnitide
