// Norms of queries and keys for each head, rotation by position, and the new keys and values into the paged cache
// (eora_serve.h), in one pass over q, k and v.
//
//   u = x * rsqrt(mean(x^2) + eps) * w;   (u_a, u_b) -> (u_a c - u_b s, u_b c + u_a s)
//
// What bounds it: bytes (every input read once, every output written once), for a few tokens the latency of one chain
// position -> row of the table -> store, and in between the instructions: a lane's 16 bytes are eight values.  A row (one head of one
// token) belongs to a group of 2 to 32 lanes, 16 bytes each, so that a load or store is one instruction per row, the norm a
// shuffle reduction, and a pair's other half (rot_dim/2 channels away, a whole number of 16-byte chunks) one shuffle of 16-bit pairs.
// A warp has kRows rows of one token, all of q, all of k or all of v, for each of its lane groups: the token's cosines and sines
// (fp32, four times a row's bytes) are read once for all of them and multiplied by the weights once, values of v are only
// copied, and nothing loops: what hides the latency is the number of warps.
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
  int q_parts, kv_parts, parts; // warps of a token: for its heads of q, of k (and as many of v); all
  float eps, inv_dim;
};

template <class E>
__device__ __forceinline__ void unpack8(float (&f)[8], const uint32_t (&w)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = E::unpack(w[i]);
    f[2 * i] = p.x; f[2 * i + 1] = p.y;
  }
}
__device__ __forceinline__ void load16(uint32_t (&w)[4], const void* p) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
}

constexpr int kRows = 4;      // rows of a lane group, all loads in flight together

// LPR: lanes of a row, a power of two >= head_dim / 8.
template <class E, int LPR>
__global__ void __launch_bounds__(256, 4) k_qk_norm_rope(const RotateArgs p) {
  constexpr int GROUPS = 32 / LPR;
  using T = typename E::T;
  const int lane = threadIdx.x & 31, sub = lane / LPR, c = lane % LPR;
  const unsigned warp = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int token = (int)(warp / p.parts), part = (int)(warp - token * p.parts);
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (token >= p.m) return;
  const bool in_row = c * 8 < p.head_dim, is_q = part < p.q_parts, is_v = part >= p.q_parts + p.kv_parts;
  const int heads = is_q ? p.heads : p.kv_heads;
  const int head0 = (is_q ? part : part - p.q_parts - (is_v ? p.kv_parts : 0)) * (GROUPS * kRows) + sub;      // this lane's rows: head0 + GROUPS j

  // the rows do not wait for the token's position, whose row of the table does
  const int pos = p.positions[token];
  const int slot = p.n_slots ? p.slots[token] : -1;
  uint32_t raw[kRows][4] = {};
  {
    const T* src = reinterpret_cast<const T*>(is_q ? p.q : is_v ? p.v : p.k) + token * (is_q ? p.q_stride : is_v ? p.v_stride : p.k_stride) + head0 * p.head_dim + 8 * c;
#pragma unroll
    for (int j = 0; j < kRows; ++j)
      if (head0 + GROUPS * j < heads && in_row) load16(raw[j], src + GROUPS * j * p.head_dim);
  }
  if (pos < 0 || pos >= p.n_positions) return;
  const bool kept = slot >= 0 && slot < p.n_slots;
  const int64_t page_at = kept ? (int64_t)(slot >> p.page_shift) * p.page_stride + (int64_t)(slot & ((1 << p.page_shift) - 1)) * p.token_stride + 8 * c : 0;
  if (is_v) {
    if (!kept || !in_row) return;
#pragma unroll
    for (int j = 0; j < kRows; ++j)
      if (head0 + GROUPS * j < heads)
        *reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.vc) + page_at + (head0 + GROUPS * j) * p.head_stride) = make_uint4(raw[j][0], raw[j][1], raw[j][2], raw[j][3]);
    return;
  }

  // A lane's channels x and their partners' y become  inv (x a + y b),  a = weight cos, b = -+ partner's weight sin
  const int half = p.rot_dim / 2;
  const bool turned = c * 8 < p.rot_dim, first = c * 8 < half;
  const int partner = !turned ? lane : (lane & ~(LPR - 1)) | ((first ? c + half / 8 : c - half / 8) & (LPR - 1));
  const void* weight = is_q ? p.q_weight : p.k_weight;
  float a[8], b[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) { a[i] = 1.f; b[i] = 0.f; }
  if (turned) {
    const float* tab = p.cos_sin + (int64_t)pos * p.rot_dim;
    if (p.adjacent) {                                     // those of its 4 pairs, twice each
      const float4 u = *reinterpret_cast<const float4*>(tab + 4 * c), w = *reinterpret_cast<const float4*>(tab + half + 4 * c);
      a[0] = a[1] = u.x; a[2] = a[3] = u.y; a[4] = a[5] = u.z; a[6] = a[7] = u.w;
      b[0] = -w.x; b[1] = w.x; b[2] = -w.y; b[3] = w.y; b[4] = -w.z; b[5] = w.z; b[6] = -w.w; b[7] = w.w;
    } else {                                              // those of its 8 channels
      const int at = 8 * c - (first ? 0 : half);
      const float sign = first ? -1.f : 1.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const float4 u = *reinterpret_cast<const float4*>(tab + at + 4 * i), w = *reinterpret_cast<const float4*>(tab + half + at + 4 * i);
        a[4 * i] = u.x; a[4 * i + 1] = u.y; a[4 * i + 2] = u.z; a[4 * i + 3] = u.w;
        b[4 * i] = sign * w.x; b[4 * i + 1] = sign * w.y; b[4 * i + 2] = sign * w.z; b[4 * i + 3] = sign * w.w;
      }
    }
  }
  if (weight) {
    uint32_t w[4] = {}, wp[4];
    if (in_row) load16(w, reinterpret_cast<const T*>(weight) + 8 * c);
#pragma unroll
    for (int i = 0; i < 4; ++i) wp[i] = p.adjacent ? __funnelshift_l(w[i], w[i], 16) : __shfl_sync(0xffffffffu, w[i], partner);
    float f[8], fp[8];
    unpack8<E>(f, w);
    unpack8<E>(fp, wp);
#pragma unroll
    for (int i = 0; i < 8; ++i) { a[i] *= f[i]; b[i] *= fp[i]; }
  }
#pragma unroll
  for (int j = 0; j < kRows; ++j) {
    const int head = head0 + GROUPS * j;
    if (head - sub >= heads) break;                       // (the same for the whole warp: the shuffles below need all of it)
    float x[8], y[8];
    unpack8<E>(x, raw[j]);
    float inv = 1.f;
    if (weight) {
      float ss = 0.f;
#pragma unroll
      for (int i = 0; i < 8; ++i) ss = fmaf(x[i], x[i], ss);
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      inv = rsqrtf(fmaf(ss, p.inv_dim, p.eps));
    }
    uint32_t other[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      other[i] = p.adjacent ? __funnelshift_l(raw[j][i], raw[j][i], 16) : __shfl_sync(0xffffffffu, raw[j][i], partner);
      if (!turned) other[i] = 0;                          // (an infinity times a sine of zero would be NaN)
    }
    unpack8<E>(y, other);
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
      o[i] = E::pack(inv * fmaf(y[2 * i], b[2 * i], x[2 * i] * a[2 * i]), inv * fmaf(y[2 * i + 1], b[2 * i + 1], x[2 * i + 1] * a[2 * i + 1]));
    if (head >= heads || !in_row) continue;
    const uint4 out = make_uint4(o[0], o[1], o[2], o[3]);
    if (is_q) {
      *reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.q_out) + token * p.q_out_stride + head * p.head_dim + 8 * c) = out;
    } else {
      if (p.k_out) *reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.k_out) + token * p.k_out_stride + head * p.head_dim + 8 * c) = out;
      if (kept) *reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.kc) + page_at + head * p.head_stride) = out;
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
  a.inv_dim = 1.f / (float)c.head_dim;
  int lpr = 2;
  while (lpr * 8 < c.head_dim) lpr *= 2;
  const int rows = (32 / lpr) * kRows;                     // of a warp
  a.q_parts = (c.n_heads + rows - 1) / rows;
  a.kv_parts = (c.n_kv_heads + rows - 1) / rows;
  a.parts = a.q_parts + (cache ? 2 : 1) * a.kv_parts;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = c.dtype == EORA_X_F16 ? launch<F16>(a, lpr, st) : launch<BF16>(a, lpr, st);
  return e == cudaSuccess ? EORA_OK : EORA_ERR_CUDA;
}
