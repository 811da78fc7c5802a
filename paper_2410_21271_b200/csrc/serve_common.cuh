// Helpers of the serving operators (eora_serve.h): 16-bit types, asynchronous copies and matrix fragments, argument checks.
#pragma once
#include <math.h>
#include "decode_common.cuh"
#include "../../include/eora_serve.h"

namespace eora {
namespace serve {

using dec::smem_u32;

// ---------------------------------------------------------------------------------------------- 16-bit types
struct F16 {
  using T = __half;
  static __device__ __forceinline__ float2 unpack(uint32_t v) { return __half22float2(*reinterpret_cast<__half2*>(&v)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {          // a in the low half; one rounding each
    __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
  }
};
struct BF16 {
  using T = __nv_bfloat16;
  static __device__ __forceinline__ float2 unpack(uint32_t v) { return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u)); }
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<uint32_t*>(&h);
  }
};

// ---------------------------------------------------------------------------------------------- copies and fragments
// 16 bytes to shared memory; with !there, zeros (src is then not read).
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, bool there) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t a) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(a) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
  uint32_t r;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
template <class E> __device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1);
template <> __device__ __forceinline__ void mma<F16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <> __device__ __forceinline__ void mma<BF16>(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// ---------------------------------------------------------------------------------------------- host side
inline bool aligned(const void* p, unsigned n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool x_type(int t) { return t == EORA_X_F16 || t == EORA_X_BF16; }
// A cache as eora_serve.h has it: EORA_OK, or what is wrong with it.
inline int check_cache(const eora_kv_cache& c) {
  if (!c.k || !c.v) return EORA_ERR_NULL_ARG;
  if (c.n_pages < 1 || c.page_size < 1 || (c.page_size & (c.page_size - 1)) || c.n_kv_heads < 1 || c.head_dim < 1) return EORA_ERR_BAD_SHAPE;
  if ((int64_t)c.n_pages * c.page_size > 0x7fffffff) return EORA_ERR_BAD_SHAPE;
  if (c.page_stride < 0 || c.head_stride < 0 || c.token_stride < c.head_dim) return EORA_ERR_BAD_SHAPE;
  if ((c.n_kv_heads > 1 && c.head_stride < c.head_dim) || (c.n_pages > 1 && c.page_stride < c.head_dim)) return EORA_ERR_BAD_SHAPE;
  if (!x_type(c.dtype)) return EORA_ERR_UNSUPPORTED;
  if (!aligned(c.k, 16) || !aligned(c.v, 16) || c.page_stride % 8 || c.head_stride % 8 || c.token_stride % 8) return EORA_ERR_MISALIGNED;
  return EORA_OK;
}
inline int log2i(int v) {
  int s = 0;
  while ((1 << s) < v) ++s;
  return s;
}

}  // namespace serve
}  // namespace eora
