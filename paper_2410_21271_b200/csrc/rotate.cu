// Norms of queries and keys for each head, rotation by position, and the new keys and values into the paged cache
// (eora_serve.h), in one pass over q, k and v.
//
//   u = x * rsqrt(mean(x^2) + eps) * w;   (u_a, u_b) -> (u_a c - u_b s, u_b c + u_a s)
//
// What bounds it: bytes (every input read once, every output written once), for a few tokens the latency of one chain
// position -> row of the table -> store, and in between the instructions: at 16 bytes a lane and step, the first form took 1300 of
// them for 2 KB and 8192 tokens of 32 + 2 x 8 heads of 128 56 us at two thirds of the issue rate.  So
//  - a lane has two 16-byte chunks of a row (one head of one token): the two halves of its pairs (or neighbours), so that nothing
//    is exchanged or unpacked twice; the norm is a shuffle reduction over the row's 1 to 16 lanes;
//  - a warp has rows of one token, all of q, all of k or all of v: the token's cosines and sines (fp32, four times a row's bytes) are
//    read once and multiplied by the weights once for all of them; values of v are only copied;
//  - products are packed, two fp32 to an instruction.
// Nothing loops: what hides the latency is the number of warps.
// Measured (B200): 8192 tokens of 32 + 2 x 8 heads of 128 42.4 to 43.1 us (4.8 TB/s, 73 % of a copy's rate), neighbouring pairs 47.1; 333 tokens of 8 + 2
// heads of 256 2.8, one token 1.6 (1.9 with norms).
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

constexpr int kThreads = 128;
// Rows of a lane group: one where that gives fewer than so many warps (48 heads of 128 with norms, one token 1.9 us, two rows 2.1; 333 tokens 3.6 and
// 3.8), beyond, two (512 tokens 4.6 us, one row 5.7; 8192 tokens 43, one row 50, four 52).  Neighbouring pairs: one token 1.9 and 2.2, 333 tokens 4.8 and
// 4.3, 512 tokens 5.1 with two and 6.0 with one, 8192 tokens 47 and 62 (that form with two rows spills 32 to 40 bytes a thread).
constexpr int64_t kFewWarps = 4096;

__device__ __forceinline__ void load16(uint32_t (&w)[4], const void* p) {
  const uint4 v = *reinterpret_cast<const uint4*>(p);
  w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
}
// Two fp32 at a time.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
  float2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(reinterpret_cast<unsigned long long&>(d))
      : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)), "l"(reinterpret_cast<unsigned long long&>(c)));
  return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
  float2 d;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<unsigned long long&>(d)) : "l"(reinterpret_cast<unsigned long long&>(a)), "l"(reinterpret_cast<unsigned long long&>(b)));
  return d;
}
__device__ __forceinline__ float2 swapped(float2 a) { return make_float2(a.y, a.x); }

// LPR: lanes of a row, a power of two >= head_dim / 16.  ADJ: pairs of neighbours.  ROWS: rows of a lane group, all loads in flight together.
template <class E, int LPR, bool ADJ, int ROWS>
__global__ void __launch_bounds__(kThreads, 6) k_qk_norm_rope(const RotateArgs p) {
  constexpr int GROUPS = 32 / LPR;
  using T = typename E::T;
  const int lane = threadIdx.x & 31, sub = lane / LPR, l = lane % LPR;
  const unsigned warp = blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int token = (int)(warp / p.parts), part = (int)(warp - token * p.parts);
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (token >= p.m) return;
  const bool in_row = l * 16 < p.head_dim, is_q = part < p.q_parts, is_v = part >= p.q_parts + p.kv_parts;
  const int heads = is_q ? p.heads : p.kv_heads;
  const int head0 = (is_q ? part : part - p.q_parts - (is_v ? p.kv_parts : 0)) * (GROUPS * ROWS) + sub;       // this lane's rows: head0 + GROUPS j
  // this lane's channels: ch0 .. + 7 and ch1 .. + 7
  const int half = p.rot_dim / 2;
  const bool turned = l * 16 < p.rot_dim;
  const int ch0 = ADJ || !turned ? 16 * l : 8 * l, ch1 = ADJ || !turned ? 16 * l + 8 : 8 * l + half;

  // the rows do not wait for the token's position, whose row of the table does
  const int pos = p.positions[token];
  const int slot = p.n_slots ? p.slots[token] : -1;
  uint32_t raw[ROWS][2][4] = {};
  {
    const T* src = reinterpret_cast<const T*>(is_q ? p.q : is_v ? p.v : p.k) + token * (is_q ? p.q_stride : is_v ? p.v_stride : p.k_stride) + head0 * p.head_dim;
#pragma unroll
    for (int j = 0; j < ROWS; ++j)
      if (head0 + GROUPS * j < heads && in_row) {
        load16(raw[j][0], src + GROUPS * j * p.head_dim + ch0);
        load16(raw[j][1], src + GROUPS * j * p.head_dim + ch1);
      }
  }
  if (pos < 0 || pos >= p.n_positions) return;
  const bool kept = slot >= 0 && slot < p.n_slots;
  const int64_t page_at = kept ? (int64_t)(slot >> p.page_shift) * p.page_stride + (int64_t)(slot & ((1 << p.page_shift) - 1)) * p.token_stride + head0 * p.head_stride : 0;
  auto store = [&](T* to, const uint32_t (&w)[2][4]) {
    *reinterpret_cast<uint4*>(to + ch0) = make_uint4(w[0][0], w[0][1], w[0][2], w[0][3]);
    *reinterpret_cast<uint4*>(to + ch1) = make_uint4(w[1][0], w[1][1], w[1][2], w[1][3]);
  };
  if (is_v) {
    if (!kept || !in_row) return;
    T* to = reinterpret_cast<T*>(p.vc) + page_at;
#pragma unroll
    for (int j = 0; j < ROWS; ++j)
      if (head0 + GROUPS * j < heads) store(to + GROUPS * j * p.head_stride, raw[j]);
    return;
  }

  // Channels x with partners y become  inv (x a + y b),  a = weight cos, b = -+ partner's weight sin; channels that are not rotated: a = weight, b = 0
  float2 a[2][4], b[2][4];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) { a[h][i] = make_float2(1.f, 1.f); b[h][i] = make_float2(0.f, 0.f); }
  if (turned) {
    const float* tab = p.cos_sin + (int64_t)pos * p.rot_dim + 8 * l;
    float4 cs[2], sn[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) { cs[i] = *reinterpret_cast<const float4*>(tab + 4 * i); sn[i] = *reinterpret_cast<const float4*>(tab + half + 4 * i); }
    if (ADJ) {                                            // pairs 8 l .. + 7: four to a chunk
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        a[h][0] = make_float2(cs[h].x, cs[h].x); a[h][1] = make_float2(cs[h].y, cs[h].y); a[h][2] = make_float2(cs[h].z, cs[h].z); a[h][3] = make_float2(cs[h].w, cs[h].w);
        b[h][0] = make_float2(-sn[h].x, sn[h].x); b[h][1] = make_float2(-sn[h].y, sn[h].y); b[h][2] = make_float2(-sn[h].z, sn[h].z); b[h][3] = make_float2(-sn[h].w, sn[h].w);
      }
    } else {                                              // pairs 8 l .. + 7: one channel of each in either chunk
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        a[0][2 * i] = a[1][2 * i] = make_float2(cs[i].x, cs[i].y); a[0][2 * i + 1] = a[1][2 * i + 1] = make_float2(cs[i].z, cs[i].w);
        b[1][2 * i] = make_float2(sn[i].x, sn[i].y); b[1][2 * i + 1] = make_float2(sn[i].z, sn[i].w);
        b[0][2 * i] = make_float2(-sn[i].x, -sn[i].y); b[0][2 * i + 1] = make_float2(-sn[i].z, -sn[i].w);
      }
    }
  }
  const T* weight = reinterpret_cast<const T*>(is_q ? p.q_weight : p.k_weight);
  if (weight && in_row) {
    uint32_t w[2][4];
    load16(w[0], weight + ch0);
    load16(w[1], weight + ch1);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 w0 = E::unpack(w[0][i]), w1 = E::unpack(w[1][i]);
      a[0][i] = mul2(a[0][i], w0); a[1][i] = mul2(a[1][i], w1);
      b[0][i] = mul2(b[0][i], ADJ ? swapped(w0) : w1); b[1][i] = mul2(b[1][i], ADJ ? swapped(w1) : w0);
    }
  }
#pragma unroll
  for (int j = 0; j < ROWS; ++j) {
    const int head = head0 + GROUPS * j;
    if (head - sub >= heads) break;                       // (the same for the whole warp: the shuffles below need all of it)
    float2 x[2][4];
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int i = 0; i < 4; ++i) x[h][i] = E::unpack(raw[j][h][i]);
    float inv = 1.f;
    if (weight) {
      float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i) s2 = fma2(x[h][i], x[h][i], s2);
      float ss = s2.x + s2.y;
#pragma unroll
      for (int o = LPR / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      inv = rsqrtf(fmaf(ss, p.inv_dim, p.eps));
    }
    const float2 inv2 = make_float2(inv, inv);
    uint32_t out[2][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 y0 = ADJ ? swapped(x[0][i]) : x[1][i], y1 = ADJ ? swapped(x[1][i]) : x[0][i];
      float2 o0 = mul2(x[0][i], a[0][i]), o1 = mul2(x[1][i], a[1][i]);
      if (turned) { o0 = fma2(y0, b[0][i], o0); o1 = fma2(y1, b[1][i], o1); }      // (an infinity in a channel or weight that is no partner, times zero, would be NaN)
      o0 = mul2(inv2, o0);
      o1 = mul2(inv2, o1);
      out[0][i] = E::pack(o0.x, o0.y);
      out[1][i] = E::pack(o1.x, o1.y);
    }
    if (head >= heads || !in_row) continue;
    if (is_q) {
      store(reinterpret_cast<T*>(p.q_out) + token * p.q_out_stride + head * p.head_dim, out);
    } else {
      if (p.k_out) store(reinterpret_cast<T*>(p.k_out) + token * p.k_out_stride + head * p.head_dim, out);
      if (kept) store(reinterpret_cast<T*>(p.kc) + page_at + GROUPS * j * p.head_stride, out);
    }
  }
}

template <class E, int LPR, int ROWS>
cudaError_t launch(RotateArgs& a, cudaStream_t st) {
  constexpr int rows = (32 / LPR) * ROWS;                  // of a warp
  a.q_parts = (a.heads + rows - 1) / rows;
  a.kv_parts = (a.kv_heads + rows - 1) / rows;
  a.parts = a.q_parts + (a.n_slots ? 2 : 1) * a.kv_parts;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(((int64_t)a.m * a.parts + kThreads / 32 - 1) / (kThreads / 32)));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return a.adjacent ? cudaLaunchKernelEx(&cfg, k_qk_norm_rope<E, LPR, true, ROWS>, a) : cudaLaunchKernelEx(&cfg, k_qk_norm_rope<E, LPR, false, ROWS>, a);
}
template <class E, int LPR>
cudaError_t launch(RotateArgs& a, cudaStream_t st) {
  return (int64_t)a.m * (a.heads + 2 * a.kv_heads) < kFewWarps * (32 / LPR) ? launch<E, LPR, 1>(a, st) : launch<E, LPR, 2>(a, st);
}
template <class E>
cudaError_t launch(RotateArgs& a, cudaStream_t st) {
  if (a.head_dim <= 16) return launch<E, 1>(a, st);
  if (a.head_dim <= 32) return launch<E, 2>(a, st);
  if (a.head_dim <= 64) return launch<E, 4>(a, st);
  if (a.head_dim <= 128) return launch<E, 8>(a, st);
  return launch<E, 16>(a, st);
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
  if ((q_out == q && q_out_stride != q_stride) || (k_out && k_out == k && k_out_stride != k_stride)) return EORA_ERR_BAD_SHAPE;

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
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = c.dtype == EORA_X_F16 ? launch<F16>(a, st) : launch<BF16>(a, st);
  return e == cudaSuccess ? EORA_OK : EORA_ERR_CUDA;
}
