// Low-rank adapters of many requests beside a shared projection (eora_serve.h):
//   y[i] = base[i] + s_j (x[i] . A_j) . B_j,  j = ids[i].
// Simple form: a thread block per token.
#include "serve_common.cuh"

namespace eora {
namespace serve {
namespace {

constexpr int kMaxRank = 256, kMaxAdapters = 4096, kMaxTokens = 1 << 20;

struct AdapterArgs {
  const void *x, *a, *b, *base;
  void* y;
  const int32_t *ids, *ranks;
  const float* scales;
  int64_t x_stride, base_stride, y_stride;
  int m, d_in, d_out, max_rank, n_adapters, y_dtype;
};

template <class E> __device__ __forceinline__ float elem(const void* p, int64_t i);
template <> __device__ __forceinline__ float elem<F16>(const void* p, int64_t i) { return __half2float(reinterpret_cast<const __half*>(p)[i]); }
template <> __device__ __forceinline__ float elem<BF16>(const void* p, int64_t i) { return __bfloat162float(reinterpret_cast<const __nv_bfloat16*>(p)[i]); }

template <class E>
__global__ void k_adapters_simple(const AdapterArgs p) {
  __shared__ float t[kMaxRank];
  const int i = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5, nw = blockDim.x >> 5;
  const int j = p.ids[i];
  const bool has = j >= 0 && j < p.n_adapters;
  if (!has && p.base == p.y) return;
  const int r = has ? min(max(p.ranks ? p.ranks[j] : p.max_rank, 0), p.max_rank) : 0;
  const float s = has && p.scales ? p.scales[j] : 1.f;
  for (int c = warp; c < r; c += nw) {
    float acc = 0.f;
    for (int k = lane; k < p.d_in; k += 32)
      acc = fmaf(elem<E>(p.x, i * p.x_stride + k), elem<E>(p.a, ((int64_t)j * p.d_in + k) * p.max_rank + c), acc);
    for (int o = 16; o > 0; o >>= 1) acc += __shfl_xor_sync(0xffffffffu, acc, o);
    if (lane == 0) t[c] = acc * s;
  }
  __syncthreads();
  for (int n = threadIdx.x; n < p.d_out; n += blockDim.x) {
    float acc = 0.f;
    for (int c = 0; c < r; ++c) acc = fmaf(t[c], elem<E>(p.b, ((int64_t)j * p.max_rank + c) * p.d_out + n), acc);
    if (p.base) {
      const int64_t at = i * p.base_stride + n;
      acc += p.y_dtype == EORA_Y_F32 ? reinterpret_cast<const float*>(p.base)[at] : p.y_dtype == EORA_Y_F16 ? elem<F16>(p.base, at) : elem<BF16>(p.base, at);
    }
    dec::store_y(p.y, p.y_dtype, i * p.y_stride + n, acc);
  }
}

}  // namespace
}  // namespace serve
}  // namespace eora

using namespace eora::serve;

extern "C" int eora_adapters_forward(const eora_adapters_config* cfg, const eora_adapters_weights* w, const void* x, int64_t x_stride, int32_t m,
                                     const int32_t* ids, const void* base, int64_t base_stride, void* y, int64_t y_stride, void* stream) {
  if (!cfg || !w) return EORA_ERR_NULL_ARG;
  const eora_adapters_config& c = *cfg;
  if (c.d_in <= 0 || c.d_in % 128 || c.d_out <= 0 || c.d_out % 32 || c.max_rank < 8 || c.max_rank > kMaxRank || c.max_rank % 8) return EORA_ERR_BAD_SHAPE;
  if (c.n_adapters < 1 || c.n_adapters > kMaxAdapters || m < 0 || m > kMaxTokens) return EORA_ERR_BAD_SHAPE;
  if (!x_type(c.x_dtype) || (c.y_dtype != EORA_Y_F16 && c.y_dtype != EORA_Y_BF16 && c.y_dtype != EORA_Y_F32)) return EORA_ERR_UNSUPPORTED;
  if (m == 0) return EORA_OK;
  if (!w->a || !w->b || !x || !ids || !y) return EORA_ERR_NULL_ARG;
  if (x_stride < c.d_in || y_stride < c.d_out || (base && base_stride < c.d_out)) return EORA_ERR_BAD_SHAPE;
  if (base == y && base_stride != y_stride) return EORA_ERR_BAD_SHAPE;
  if (!aligned(w->a, 16) || !aligned(w->b, 16) || !aligned(x, 16) || !aligned(y, 16) || !aligned(base, 16) || !aligned(ids, 4) || !aligned(w->ranks, 4) ||
      !aligned(w->scales, 4) || x_stride % 8 || y_stride % 8 || (base && base_stride % 8))
    return EORA_ERR_MISALIGNED;
  AdapterArgs a = {};
  a.x = x; a.a = w->a; a.b = w->b; a.base = base; a.y = y; a.ids = ids; a.ranks = w->ranks; a.scales = w->scales;
  a.x_stride = x_stride; a.base_stride = base_stride; a.y_stride = y_stride;
  a.m = m; a.d_in = c.d_in; a.d_out = c.d_out; a.max_rank = c.max_rank; a.n_adapters = c.n_adapters; a.y_dtype = c.y_dtype;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (c.x_dtype == EORA_X_F16) k_adapters_simple<F16><<<m, 256, 0, st>>>(a);
  else k_adapters_simple<BF16><<<m, 256, 0, st>>>(a);
  return cudaGetLastError() == cudaSuccess ? EORA_OK : EORA_ERR_CUDA;
}
