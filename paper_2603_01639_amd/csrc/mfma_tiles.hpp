// What the matrix-core attention kernels share: vector types, the row order that
// leaves a query row's scores in one lane, lane exchanges, transposed LDS reads
// and direct global->LDS loads (gfx950).
#pragma once

#include <type_traits>
#include <utility>

#include "ltd_device.hpp"

namespace ltd {
namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef int i32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
typedef __attribute__((address_space(3))) void lds_void;
typedef const __attribute__((address_space(1))) void global_cvoid;

constexpr float kLog2e = 1.4426950408889634f;

// A-row i of a 32-key block reads key sigma(i); accumulator register r of lane
// half h then holds key 16*h + r.
__device__ __forceinline__ int sigma(int i) {
  return 16 * ((i >> 2) & 1) + 4 * (i >> 3) + (i & 3);
}

__device__ __forceinline__ uint32_t pack_bf16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2){lo, hi}, bf16x2));
}
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// x of lane (l xor 32), with v_permlane32_swap (a VALU op; __shfl_xor goes
// through the LDS crossbar, where it queues behind the tile's fragment reads).
// The swap of x with itself leaves the upper half's values in the lower half
// of the second result and the lower half's in the upper half of the first.
__device__ __forceinline__ float xor32(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __builtin_bit_cast(float, (__lane_id() & 32) ? r[0] : r[1]);
}

__device__ __forceinline__ uint32_t pack_f16x2(float lo, float hi) {
  return __builtin_bit_cast(uint32_t, (f16x2){static_cast<_Float16>(lo), static_cast<_Float16>(hi)});
}
// The larger of x in lanes l and l ^ 32, in every lane: the swap of x with
// itself leaves the lower half's values in both halves of the first result and
// the upper half's in both halves of the second.
__device__ __forceinline__ float max_xor32(float x) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  // (the halves are copied out first: hipcc folds a bit-cast of element 1 of
  // the result to element 0)
  const uint32_t lo = r[0], hi = r[1];
  return __builtin_elementwise_maximum(__builtin_bit_cast(float, lo), __builtin_bit_cast(float, hi));
}

__device__ __forceinline__ lds_void* as_lds(const void* p) { return (lds_void*)(p); }
__device__ __forceinline__ global_cvoid* as_global(const void* p) { return (global_cvoid*)(p); }

// Transposed 4-key x 16-dim read of a 16-lane group (ds_read_b64_tr_b16):
// supplier lane s of the group addresses key k0 + s/4, dims d0 + 4*(s%4)..+3;
// lane p then receives keys k0..k0+3 of dim d0 + p.
__device__ __forceinline__ s16x4 lds_read_tr(const unsigned char* p) {
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)as_lds(p));
}

template <int N>
__device__ __forceinline__ void wait_vmcnt() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Direct global->LDS loads of 16 bytes per lane (global_load_lds_dwordx4;
// lane i's bytes land at M0 + 16*i).  They are issued as inline assembly on
// purpose: the compiler does not track them, so it does not put a full
// vector-memory wait in front of every later LDS read (which would drain the
// prefetch ring every tile).  The kernel waits for them itself (wait_vmcnt)
// and orders them across waves with bare barriers.  Nothing else in these
// kernels uses M0.  A load that takes its place in LDS from M0 comes one wait state
// after the write (s_nop 0), which nobody else sees to inside the assembly: without it
// the load may take the last place.
__device__ __forceinline__ uint32_t lds_addr(const void* p) {
  return __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(reinterpret_cast<uintptr_t>(as_lds(p))));
}
// Base pointer that the compiler must keep in scalar registers (the SADDR
// form of the load takes a 64-bit SGPR pair).
__device__ __forceinline__ const void* scalar_ptr(const void* p) {
  const uint64_t v = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v));
  const uint32_t hi = __builtin_amdgcn_readfirstlane(static_cast<uint32_t>(v >> 32));
  return reinterpret_cast<const void*>((static_cast<uint64_t>(hi) << 32) | lo);
}
__device__ __forceinline__ void dma16(uint32_t lds, const void* uniform_base, uint32_t lane_off) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2"
               ::"s"(lds), "v"(lane_off), "s"(scalar_ptr(uniform_base))
               : "memory");
}
__device__ __forceinline__ void dma16(uint32_t lds, const void* lane_ptr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, off" ::"s"(lds), "v"(lane_ptr)
               : "memory");
}
// Direct global->LDS load of a byte per lane (lane i's byte lands as a word at M0 + 4*i).
__device__ __forceinline__ void dma1(uint32_t lds, const void* lane_ptr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_ubyte %1, off" ::"s"(lds), "v"(lane_ptr)
               : "memory");
}
// Direct global->LDS load of 4 bytes per lane (lane i's word lands at M0 + 4*i).
__device__ __forceinline__ void dma4(uint32_t lds, const void* lane_ptr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, off" ::"s"(lds), "v"(lane_ptr)
               : "memory");
}
// Workgroup barrier without the memory fence __syncthreads() adds (that fence
// would also wait for every outstanding direct load).
__device__ __forceinline__ void barrier_only() { asm volatile("s_barrier" ::: "memory"); }

// f(0), ..., f(N - 1) with the indices as compile-time constants: arrays indexed
// by them stay in registers of their own (a loop that hipcc unrolls late leaves
// them one wide vector, copied whole at every branch).
template <int... I, class F>
__device__ __forceinline__ void for_each_of(std::integer_sequence<int, I...>, F f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void for_each_index(F f) {
  for_each_of(std::make_integer_sequence<int, N>{}, f);
}

}  // namespace
}  // namespace ltd
