// Norms of queries and keys for each head, rotation by position, and the new keys and values into the paged cache
// (eora_serve.h), in one pass over q, k and v.
//
//   u = x * rsqrt(mean(x^2) + eps) * w;   (u_a, u_b) -> (u_a c - u_b s, u_b c + u_a s)
//
// What bounds it: bytes (every input read once, every output written once), and for a few tokens the latency of one chain
// token -> row -> store.  A row (one head of one token) belongs to a group of 8, 16 or 32 lanes, 16 bytes each, so that a
// load or store is one instruction per row, the norm a shuffle reduction, and a pair's other half (rot_dim/2 channels
// away, a whole number of 16-byte chunks) one shuffle.  A warp has kRows rows of one token for each of its lane groups, so that the
// token's cosines and sines (fp32, four times a row's bytes) are read once for all of them; nothing loops: what hides the
// latency of its two dependent loads (position, then the table's row) is the number of warps.
#include "serve_common.cuh"

namespace eora {
namespace serve {
namespace {

struct RotateArgs {
  const void *q, *k, *v;
  void *q_out, *k_out, *kc, *vc;
  int64_t q_stride, k_stride, v_stride, q_out_stride, k_out_stride;
  int64_t page_stride, head_stride, token_stride;
  const int32_t *positions, *slots;
  const void *q_weight, *k_weight;
  const float* cos_sin;
  int m, heads, kv_heads, head_dim, rot_dim, adjacent, n_positions;
  int n_slots, page_shift;      // n_slots = 0: no cache
  int rows;                     // of a token: heads + kv_heads + (kv_heads with a cache)
  int parts;                    // warps of a token
  float eps;
};

template <class E>
__device__ __forceinline__ void unpack8(float (&f)[8], const uint4& v) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = E::unpack(w[i]);
    f[2 * i] = p.x; f[2 * i + 1] = p.y;
  }
}

constexpr int kRows = 4;      // rows of a lane group, all loads in flight together

// LPR: lanes of a row, a power of two >= head_dim / 8.
template <class E, int LPR>
__global__ void __launch_bounds__(256, 4) k_qk_norm_rope(const RotateArgs p) {
  constexpr int GROUPS = 32 / LPR;
  using T = typename E::T;
  const int lane = threadIdx.x & 31, sub = lane / LPR, c = lane % LPR;
  const unsigned warp = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int token = (int)(warp / p.parts), row0 = (int)(warp - token * p.parts) * (GROUPS * kRows) + sub;
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (token >= p.m) return;
  const bool in_row = c * 8 < p.head_dim;

  // the rows do not wait for the token's position, whose row of the table does
  const int pos = p.positions[token];
  const int slot = p.n_slots ? p.slots[token] : -1;
  uint4 raw[kRows];
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    const int row = row0 + j * GROUPS;
    raw[j] = make_uint4(0, 0, 0, 0);
    if (row >= p.rows || !in_row) continue;
    const T* src;
    if (row < p.heads) src = reinterpret_cast<const T*>(p.q) + token * p.q_stride + row * p.head_dim;
    else if (row < p.heads + p.kv_heads) src = reinterpret_cast<const T*>(p.k) + token * p.k_stride + (row - p.heads) * p.head_dim;
    else src = reinterpret_cast<const T*>(p.v) + token * p.v_stride + (row - p.heads - p.kv_heads) * p.head_dim;
    raw[j] = *reinterpret_cast<const uint4*>(src + 8 * c);
  }
  if (pos < 0 || pos >= p.n_positions) return;
  const bool kept = slot >= 0 && slot < p.n_slots;

  // this lane's cosines and sines: half pairs: those of its 8 channels; adjacent pairs: those of its 4 pairs, twice each
  float cs[8], sn[8];
  const int half = p.rot_dim / 2;
  const bool turned = c * 8 < p.rot_dim, first = c * 8 < half;
#pragma unroll
  for (int i = 0; i < 8; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
  if (turned) {
    const float* tab = p.cos_sin + (int64_t)pos * p.rot_dim;
    if (p.adjacent) {
      const float4 a = *reinterpret_cast<const float4*>(tab + 4 * c), b = *reinterpret_cast<const float4*>(tab + half + 4 * c);
      cs[0] = cs[1] = a.x; cs[2] = cs[3] = a.y; cs[4] = cs[5] = a.z; cs[6] = cs[7] = a.w;
      sn[0] = -b.x; sn[1] = b.x; sn[2] = -b.y; sn[3] = b.y; sn[4] = -b.z; sn[5] = b.z; sn[6] = -b.w; sn[7] = b.w;
    } else {
      const int at = 8 * c - (first ? 0 : half);
      const float sign = first ? -1.f : 1.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float4 a = *reinterpret_cast<const float4*>(tab + at + 4 * i), b = *reinterpret_cast<const float4*>(tab + half + at + 4 * i);
        cs[4 * i] = a.x; cs[4 * i + 1] = a.y; cs[4 * i + 2] = a.z; cs[4 * i + 3] = a.w;
        sn[4 * i] = sign * b.x; sn[4 * i + 1] = sign * b.y; sn[4 * i + 2] = sign * b.z; sn[4 * i + 3] = sign * b.w;
      }
    }
  }
  const int partner = (lane & ~(LPR - 1)) | ((first ? c + half / 8 : c - half / 8) & (LPR - 1));
  const int64_t page_at = kept ? (int64_t)(slot >> p.page_shift) * p.page_stride + (int64_t)(slot & ((1 << p.page_shift) - 1)) * p.token_stride : 0;
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    const int row = row0 + j * GROUPS;
    if (row - sub >= p.rows) break;                       // (the same for the whole warp: the shuffles below need all of it)
    const bool is_q = row < p.heads, is_v = row >= p.heads + p.kv_heads;
    float f[8];
    unpack8<E>(f, raw[j]);
    const uint4* weight = reinterpret_cast<const uint4*>(is_q ? p.q_weight : p.k_weight);
    if (p.q_weight || p.k_weight) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(f[i], f[i], ss);
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      if (weight && in_row) {
        const float inv = rsqrtf(ss / (float)p.head_dim + p.eps);
        float w[8];
        unpack8<E>(w, __ldg(weight + c));
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] *= inv * w[i];
      }
    }
    float g[8];
    if (p.adjacent) {
#pragma unroll
      for (int i = 0; i < 8; ++i) g[i] = turned ? fmaf(f[i ^ 1], sn[i], f[i] * cs[i]) : f[i];
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float other = __shfl_sync(0xffffffffu, f[i], partner);
        g[i] = turned ? fmaf(other, sn[i], f[i] * cs[i]) : f[i];
      }
    }
    if (row >= p.rows || !in_row) continue;
    const uint4 o = make_uint4(E::pack(g[0], g[1]), E::pack(g[2], g[3]), E::pack(g[4], g[5]), E::pack(g[6], g[7]));
    if (is_q) {
      *reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.q_out) + token * p.q_out_stride + row * p.head_dim + 8 * c) = o;
    } else if (!is_v) {
      const int h = row - p.heads;
      if (p.k_out) *reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.k_out) + token * p.k_out_stride + h * p.head_dim + 8 * c) = o;
      if (kept) *reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.kc) + page_at + h * p.head_stride + 8 * c) = o;
    } else if (kept) {
      *reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.vc) + page_at + (row - p.heads - p.kv_heads) * p.head_stride + 8 * c) = raw[j];
    }
  }
}

template <class E>
cudaError_t launch(const RotateArgs& a, int lpr, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(((int64_t)a.m * a.parts + 7) / 8));
  cfg.blockDim = dim3(256);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  switch (lpr) {
    case 2: return cudaLaunchKernelEx(&cfg, k_qk_norm_rope<E, 2>, a);
    case 4: return cudaLaunchKernelEx(&cfg, k_qk_norm_rope<E, 4>, a);
    case 8: return cudaLaunchKernelEx(&cfg, k_qk_norm_rope<E, 8>, a);
    case 16: return cudaLaunchKernelEx(&cfg, k_qk_norm_rope<E, 16>, a);
    default: return cudaLaunchKernelEx(&cfg, k_qk_norm_rope<E, 32>, a);
  }
}

}  // namespace
}  // namespace serve
}  // namespace eora

using namespace eora::serve;

extern "C" int eora_qk_norm_rope(const eora_qk_config* cfg, const void* q, int64_t q_stride, const void* k, int64_t k_stride, const void* v,
                                 int64_t v_stride, const int32_t* positions, int32_t m, void* q_out, int64_t q_out_stride, void* k_out,
                                 int64_t k_out_stride, const int32_t* slots, const eora_kv_cache* cache, void* stream) {
  if (!cfg) return EORA_ERR_NULL_ARG;
  const eora_qk_config& c = *cfg;
  if (c.n_heads < 1 || c.n_kv_heads < 1 || c.n_heads > 1024 || c.n_heads % c.n_kv_heads || c.head_dim < 16 || c.head_dim > 256 || c.head_dim % 16) return EORA_ERR_BAD_SHAPE;
  if (c.rot_dim < 0 || c.rot_dim > c.head_dim || c.rot_dim % 16 || c.n_positions < 1 || m < 0 || m > (1 << 20)) return EORA_ERR_BAD_SHAPE;
  if (!(c.eps >= 0.f) || !isfinite(c.eps)) return EORA_ERR_BAD_SHAPE;
  if (!x_type(c.dtype) || (c.pairs != EORA_ROPE_HALF && c.pairs != EORA_ROPE_ADJACENT)) return EORA_ERR_UNSUPPORTED;
  if (m == 0) return EORA_OK;
  if (!q || !k || !q_out || !positions || (c.rot_dim && !c.cos_sin)) return EORA_ERR_NULL_ARG;
  if ((cache != nullptr) != (slots != nullptr) || (cache != nullptr) != (v != nullptr)) return EORA_ERR_NULL_ARG;
  const int64_t qd = (int64_t)c.n_heads * c.head_dim, kd = (int64_t)c.n_kv_heads * c.head_dim;
  if (q_stride < qd || k_stride < kd || (v && v_stride < kd) || q_out_stride < qd || (k_out && k_out_stride < kd)) return EORA_ERR_BAD_SHAPE;
  if (cache) {
    const int st = check_cache(*cache);
    if (st != EORA_OK) return st;
    if (cache->n_kv_heads != c.n_kv_heads || cache->head_dim != c.head_dim) return EORA_ERR_BAD_SHAPE;
    if (cache->dtype != c.dtype) return EORA_ERR_UNSUPPORTED;
  }
  if (!aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(q_out, 16) || !aligned(k_out, 16) || !aligned(c.q_weight, 16) ||
      !aligned(c.k_weight, 16) || !aligned(c.cos_sin, 16) || !aligned(positions, 4) || !aligned(slots, 4))
    return EORA_ERR_MISALIGNED;
  if (q_stride % 8 || k_stride % 8 || (v && v_stride % 8) || q_out_stride % 8 || (k_out && k_out_stride % 8)) return EORA_ERR_MISALIGNED;

  RotateArgs a = {};
  a.q = q; a.k = k; a.v = v; a.q_out = q_out; a.k_out = k_out;
  a.q_stride = q_stride; a.k_stride = k_stride; a.v_stride = v_stride; a.q_out_stride = q_out_stride; a.k_out_stride = k_out_stride;
  if (cache) {
    a.kc = cache->k; a.vc = cache->v;
    a.page_stride = cache->page_stride; a.head_stride = cache->head_stride; a.token_stride = cache->token_stride;
    a.n_slots = cache->n_pages * cache->page_size; a.page_shift = log2i(cache->page_size);
  }
  a.positions = positions; a.slots = slots;
  a.q_weight = c.q_weight; a.k_weight = c.k_weight; a.cos_sin = c.cos_sin;
  a.m = m; a.heads = c.n_heads; a.kv_heads = c.n_kv_heads; a.head_dim = c.head_dim; a.rot_dim = c.rot_dim;
  a.adjacent = c.pairs == EORA_ROPE_ADJACENT; a.n_positions = c.n_positions; a.eps = c.eps;
  a.rows = c.n_heads + (cache ? 2 : 1) * c.n_kv_heads;
  int lpr = 2;
  while (lpr * 8 < c.head_dim) lpr *= 2;
  a.parts = (a.rows + (32 / lpr) * kRows - 1) / ((32 / lpr) * kRows);
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = c.dtype == EORA_X_F16 ? launch<F16>(a, lpr, st) : launch<BF16>(a, lpr, st);
  return e == cudaSuccess ? EORA_OK : EORA_ERR_CUDA;
}
