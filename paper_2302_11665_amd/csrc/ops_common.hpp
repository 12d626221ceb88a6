// Shared by the operators of a served model's step (alpaserve_ops.h): operand
// types of the matrix instructions, 16-bit conversions, cross-lane steps.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <atomic>

#include "alpaserve_ops.h"
#include "sim_internal.hpp"

namespace as_ops {

typedef int v4i __attribute__((ext_vector_type(4)));
typedef float v4f __attribute__((ext_vector_type(4)));
typedef uint32_t v2u __attribute__((ext_vector_type(2)));
typedef uint32_t v4u __attribute__((ext_vector_type(4)));
typedef __bf16 v8bf __attribute__((ext_vector_type(8)));
typedef _Float16 v8h __attribute__((ext_vector_type(8)));
typedef _Float16 v2h __attribute__((ext_vector_type(2)));

constexpr float kInf = __builtin_huge_valf();

// A 16-bit value as fp32.
template <int TYPE>
__device__ __forceinline__ float to_f32(uint32_t bits16) {
  if (TYPE == AS_BF16) return __uint_as_float(bits16 << 16);
  return (float)__builtin_bit_cast(_Float16, (uint16_t)bits16);
}

// fp32 rounded to a 16-bit type (to nearest even, NaN stays NaN).
template <int TYPE>
__device__ __forceinline__ uint16_t from_f32(float x) {
  if (TYPE == AS_BF16) return __builtin_bit_cast(uint16_t, (__bf16)x);
  return __builtin_bit_cast(uint16_t, (_Float16)x);
}

// Two fp32 numbers rounded to bf16, the first in the low half.
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  typedef __bf16 v2bf __attribute__((ext_vector_type(2)));
  v2bf p = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, p);
}

// Maximum and sum over the four rows of 16 lanes of a wavefront: every lane
// gets the result of the lanes that agree with it modulo 16.  The swap of a
// register with itself pairs each row with another in one instruction.
__device__ __forceinline__ float max_over_rows(float x) {
  v2u p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
}
__device__ __forceinline__ float sum_over_rows(float x) {
  v2u p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(p[0]) + __uint_as_float(p[1]);
  p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(p[0]) + __uint_as_float(p[1]);
}

// Sum over the lanes up to and with this one: four steps within rows of 16
// lanes, then the rows' last lanes to the rows after them.
__device__ __forceinline__ uint32_t scan_lanes(uint32_t x) {
#define AS_ADD_DPP(ctrl, rows) x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, ctrl, rows, 0xf, false)
  AS_ADD_DPP(0x111, 0xf);  // row_shr:1
  AS_ADD_DPP(0x112, 0xf);
  AS_ADD_DPP(0x114, 0xf);
  AS_ADD_DPP(0x118, 0xf);
  AS_ADD_DPP(0x142, 0xa);  // row_bcast:15
  AS_ADD_DPP(0x143, 0xc);  // row_bcast:31
#undef AS_ADD_DPP
  return x;
}

// Barrier of a workgroup that orders its LDS accesses alone: loads from memory
// stay in flight across it.
__device__ __forceinline__ void lds_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// Wait until at most N of the wavefront's loads are on their way; what is read
// from LDS afterwards is read afterwards.
template <int N>
__device__ __forceinline__ void wait_loads() {
  static_assert(N < 64, "six bits");
  __builtin_amdgcn_s_waitcnt((N & 15) | (N >> 4) << 14 | 0x0f70);
  asm volatile("" ::: "memory");
}
// Wait for the wavefront's LDS reads: their place may be written again.
__device__ __forceinline__ void wait_reads() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0), nothing else
  asm volatile("" ::: "memory");
}

__host__ __device__ __forceinline__ int64_t round_up(int64_t x, int64_t to) { return (x + to - 1) / to * to; }

inline bool aligned(const void* p, size_t to) { return ((uintptr_t)p & (to - 1)) == 0; }

// Result of a launch as a status code.
inline int launched(const char* what) {
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return as_host::fail(AS_E_HIP, "%s: kernel launch failed: %s", what, hipGetErrorString(e));
  return as_host::ok();
}

// Lets a kernel have more than 64 KiB of LDS; once on each device (F is one
// kernel's type and address, so the flags are its own).
template <auto F>
int allow_lds(size_t bytes, const char* what) {
  static std::atomic<uint64_t> done{0};
  if (bytes <= 64 * 1024) return AS_OK;
  int dev = 0;
  if (hipGetDevice(&dev) != hipSuccess || dev < 0 || dev > 63) dev = 63;
  if (done.load(std::memory_order_relaxed) >> dev & 1) return AS_OK;
  const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void*>(F), hipFuncAttributeMaxDynamicSharedMemorySize,
                                           156 * 1024);  // of 160: 4 KiB for static arrays
  if (e != hipSuccess) return as_host::fail(AS_E_HIP, "%s: %s", what, hipGetErrorString(e));
  if (dev < 63) done.fetch_or((uint64_t)1 << dev, std::memory_order_relaxed);
  return AS_OK;
}

// Checks of a cache's sizes and pointers; AS_OK or the error recorded.
int check_cache(const as_cache_t* c, const char* name, bool need_pos, bool need_acc);

// A cache as kernels take it, with the strides of one page and head.
struct CacheArgs {
  uint32_t *k, *v;
  uint32_t *k_par, *v_par;  // a (scale, minimum) pair is one word
  int32_t* pos;
  float* acc;
  const int32_t* page_table;
  int32_t n_pages, n_heads, dim, group, page, n_seqs, max_pages;
};
CacheArgs cache_args(const as_cache_t* c);

// Division of a block of 32 slots' number (below 2^25) by a page's blocks (at
// most 128): the high half of a product with ceil(2^32 / blocks), which is off
// by less than blocks, so that the error stays below 2^32.
__host__ __forceinline__ uint32_t page_magic(int page) {
  const uint32_t blocks = (uint32_t)page / 32;
  return blocks > 1 ? (uint32_t)((((uint64_t)1 << 32) + blocks - 1) / blocks) : 0;
}
__device__ __forceinline__ int page_index(int block, uint32_t magic) {
  return magic ? (int)__umulhi((uint32_t)block, magic) : block;
}

// Index of the (page, head) row of a page of a sequence, or -1 where the table
// has no such page; word offsets follow by multiplication with the row's length.
__device__ __forceinline__ int64_t cache_row(const CacheArgs& c, int b, int h, int index) {
  if ((unsigned)index >= (unsigned)c.max_pages) return -1;
  const int p = c.page_table[(int64_t)b * c.max_pages + index];
  if ((unsigned)p >= (unsigned)c.n_pages) return -1;
  return (int64_t)p * c.n_heads + h;
}

}  // namespace as_ops
