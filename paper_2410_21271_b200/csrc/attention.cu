// Attention of one new token per sequence over a paged cache (eora_serve.h):
//   out = sum_t softmax_t(scale q . k_t) v_t,  lse = log sum_t exp(scale q . k_t).
//
// What bounds it: the bytes of K and V (4 head_dim bytes per token and key head, each read once; heads / key heads flops per
// byte), so everything serves a steady stream of loads from HBM.
//  - One pass: running maximum m, sum l and accumulator O in registers, O and l scaled by exp(m_old - m_new) per step.
//  - Tokens are the 16-row operand of the matrix instruction and the query heads of one key head its 8 columns: with the few
//    heads that share a key head the other way round would leave half of each instruction (and of O's registers) empty.
//    S^T = K Q^T, O^T += V^T P^T; P^T comes from S^T's registers by an 8 x 8 transposition in the warp.
//  - A warp takes 16 tokens at a time through a ring of its own in shared memory (cp.async; rows that are not seen are filled
//    with zeros, so that NaN in them meets no arithmetic); warps meet only where a sequence's key head ends.
//  - Work is cut into units of 16 tokens per warp over all (sequence, key head) pairs, in order, and every thread block takes
//    an equal share of the units whatever the lengths are (they are read from device memory). A pair cut by the border of a
//    share is joined from partial sums in scratch memory by the block that finishes last, in the order of the blocks.
// Measured (B200; a copy reaches 6.56 TB/s): 64 sequences of 512 to 8192 tokens, 32 heads on 8 of 128 (1.14 GB) 187 to 203 us by the card, 5.6 to 6.1
// TB/s; one of 131072 tokens (537 MB) 85 to 91 us, 5.9 to 6.3 TB/s; one of 1000 8.2 us, of which 2 are the launch and 6 a chain of accesses (lengths,
// pages, K and V, the join).
#include "serve_common.cuh"

namespace eora {
namespace serve {
namespace {

struct AttnArgs {
  const void *q, *k, *v;
  void* out;
  float* lse;
  const int32_t *table, *lengths;
  int64_t q_stride, out_stride, table_stride, page_stride, head_stride, token_stride;
  int batch, kv_heads, group;          // group: query heads of a key head
  int splits, per;                     // a key head's query heads are served in `splits` parts of `per` (the last may be smaller)
  int n_pages, page_shift, max_tokens, window;
  int few;                             // no more pairs than blocks
  float scale_log2;                    // scale / ln 2
  float* part;                         // [grid][2][rows][head_dim]
  float2 *part_ml, *joined_ml;         // [grid][2][rows] each
  unsigned* arrived;                   // [batch][kv_heads * splits], zero between calls
  unsigned* arrived_group;             // [grid][2], zero between calls
};

constexpr int kTile = 16;              // tokens of a warp's step
constexpr int kOneRound = 24;          // parts that one block joins by itself, times the columns of a thread
// Probabilities enter the second product as 2^kLift exp(s - m): fp16 keeps eleven bits down to 2^-14 and nothing below 2^-25, and a hundred
// thousand tokens of 2^-26 each are not nothing.  With the lift that border lies at 2^-40 of the largest; bf16 has fp32's range.
template <class E> constexpr float kLift = 0.f;
template <> constexpr float kLift<F16> = 15.f;
// Two probabilities as 16-bit numbers in two parts each, so that the second product sums what l does: with one part the output was off by half a
// step of the type twice over (131072 tokens in bf16 1.79e-3 instead of 1.66e-3, which is the output's own rounding).  It costs little where bytes bound
// the call: 64 sequences 185.6 -> 187.4 us, 131072 tokens 84.6 -> 84.8, 13 sequences of groups of seven with a window 12.8 -> 13.2.  The high part is cut
// below p by construction: both parts are positive, and an infinity among the values meets no zero and no other sign.  What is left of p is
// 2^-15 (bf16: a low part of at most 2^-7, rounded) or 2^-20 (fp16: 2^-9, rounded; the high part is cut 2^-10 lower, for the low part to stay above fp16's 2^-24).
template <class E> __device__ __forceinline__ void two_weights(float a, float b, uint32_t& hi, uint32_t& lo);
template <> __device__ __forceinline__ void two_weights<BF16>(float a, float b, uint32_t& hi, uint32_t& lo) {
  const uint32_t ua = max(__float_as_uint(a), 1u) - 1, ub = max(__float_as_uint(b), 1u) - 1;
  hi = __byte_perm(ua, ub, 0x7632);
  lo = BF16::pack(a - __uint_as_float(ua & 0xffff0000u), b - __uint_as_float(ub & 0xffff0000u));
}
template <> __device__ __forceinline__ void two_weights<F16>(float a, float b, uint32_t& hi, uint32_t& lo) {
  constexpr uint32_t kLower = 1u << 13;
  const float fa = __uint_as_float(max(__float_as_uint(a), kLower) - kLower), fb = __uint_as_float(max(__float_as_uint(b), kLower) - kLower);
  asm("cvt.rz.f16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(fb), "f"(fa));
  const float2 h = F16::unpack(hi);
  lo = F16::pack(a - h.x, b - h.y);
}

template <int D, int NT> struct Shape {
  static constexpr int kWarps = D > 128 ? 4 : 8;
  static constexpr int kStages = D > 64 ? 2 : 4;
  static constexpr int kThreads = 32 * kWarps;
  static constexpr int kRows = 8 * NT;
  static constexpr int kUnit = kTile * kWarps;
  static constexpr int kChunks = D / 8;                       // 16-byte chunks of a row
  static constexpr int kTileBytes = kTile * D * 2;            // of K or of V
  static constexpr int kQPitch = D * 2 + 16;
  static constexpr int kOPitch = D + 4;                       // floats
  static constexpr int kRingBytes = kWarps * kStages * 2 * kTileBytes;
  static constexpr int kJoinBytes = kWarps * 8 * kOPitch * 4;
  static constexpr int kQBytes = kRows * kQPitch;
  static constexpr int kSmem = kRingBytes + kJoinBytes + kQBytes + kWarps * 8 * 8 + kWarps * kStages * 4 + 16 + kWarps * kStages * kTile * 4;
};

// chunk c of row r stands at chunk swizzled<D>(r, c) of the row: eight rows' same chunk lie in eight bank groups
template <int D> __device__ __forceinline__ int swizzled(int r, int c) {
  constexpr int NC = D / 8;
  return NC % 8 == 0 ? (c ^ (r & 7)) : (c ^ ((r >> 1) & 3));      // (12 chunks: rows two apart differ by 24 chunks, so two rows by parity)
}

// Infinities and NaN in what a sequence sees go as in the formula.  The running maximum is NaN where a score is (max_nan), and a score of -inf is held as
// the lowest number, kLowest, so that tokens that are seen and count nothing differ from tokens that are not: where they are all, the formula has 0 / 0.
constexpr float kLowest = -3.402823466e+38f;
__device__ __forceinline__ float max_nan(float a, float b) {
  float m;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(m) : "f"(a), "f"(b));
  return m;
}

struct Seq { int n, first, lo, units; };
template <int U> __device__ __forceinline__ Seq sequence(const AttnArgs& p, int b) {
  Seq s;
  s.n = min(max(p.lengths[b], 0), p.max_tokens);
  s.first = p.window && s.n > p.window ? s.n - p.window : 0;
  s.lo = s.first & ~(kTile - 1);
  s.units = (s.n - s.lo + U - 1) / U;
  return s;
}

// Where a share stands: unit u of part vh of sequence b.
struct Place {
  int b, vh, u;
  Seq s;
};
template <int U> __device__ __forceinline__ void next(const AttnArgs& p, Place& a) {
  if (++a.u < a.s.units) return;
  a.u = 0;
  if (++a.vh < p.kv_heads * p.splits) return;
  a.vh = 0;
  while (++a.b < p.batch) {
    a.s = sequence<U>(p, a.b);
    if (a.s.units) return;
  }
}

__device__ __forceinline__ float2 ld_cg2(const float2* p) {
  float2 v;
  asm volatile("ld.global.cg.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "l"(p) : "memory");
  return v;
}

// TWICE: the heads of a part, four at most, stand twice in the eight columns of the instruction, at c and 4 + c: the scores are the same, one of the two
// takes the high parts of the weights and the other the low ones, and the sums of both columns, added where the warps' sums are, are those of one
// (instead of a product for either part: 64 sequences 190.4 -> 187.4 us, one of 1000 tokens 8.30 -> 8.24, 131072 tokens 84.8 as before).
template <class E, int D, int NT, bool TWICE>
__global__ void __launch_bounds__(Shape<D, NT>::kThreads, 1) k_attention(const AttnArgs p) {
  using S = Shape<D, NT>;
  constexpr int U = S::kUnit, NC = S::kChunks;
  using T = typename E::T;
  extern __shared__ __align__(128) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
  uint8_t* join_mem = smem + S::kRingBytes;
  float* obuf = reinterpret_cast<float*>(join_mem);                                     // [warp][8][kOPitch]
  uint8_t* qmem = join_mem + S::kJoinBytes;                                             // [kRows][kQPitch]
  float2* ml = reinterpret_cast<float2*>(qmem + S::kQBytes);                            // [warp][8]
  uint32_t* seen_mem = reinterpret_cast<uint32_t*>(ml + S::kWarps * 8) + warp * S::kStages;   // bit r: row r of the stage's tile counts
  int* flag = reinterpret_cast<int*>(reinterpret_cast<uint32_t*>(ml + S::kWarps * 8) + S::kWarps * S::kStages);
  int* pages = flag + 4;                                                                // [warp][stage][16]
  const uint32_t ring = smem_u32(smem) + warp * S::kStages * 2 * S::kTileBytes, q_addr = smem_u32(qmem);
  const int HV = p.kv_heads * p.splits, heads = p.kv_heads * p.group;

  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  auto empty_ones = [&]() {                  // sequences without a token
    for (int b = blockIdx.x; b < p.batch; b += gridDim.x) {
      if (p.lengths[b] > 0) continue;
      for (int i = tid; i < heads * D / 8; i += S::kThreads)
        reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.out) + b * p.out_stride)[i] = make_uint4(0, 0, 0, 0);
      if (p.lse)
        for (int i = tid; i < heads; i += S::kThreads) p.lse[(int64_t)b * heads + i] = -INFINITY;
    }
  };

  // ---- this block's share of the units (every warp works it out for itself)
  int64_t total = 0;
  for (int b = lane; b < p.batch; b += 32) total += sequence<U>(p, b).units;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  total *= HV;
  const int grid = total < (int64_t)gridDim.x ? (int)total : (int)gridDim.x;
  if (grid == 0) return empty_ones();
  // (in 32 bits where they do: a 64-bit division is a hundred instructions)
  const bool small = total < (1 << 24);
  auto share = [&](int i) { return small ? (int64_t)((uint32_t)total * (uint32_t)i / (uint32_t)grid) : total * i / grid; };       // first unit of block i
  auto owner = [&](int64_t unit) {           // the block that has it
    return small ? (int)((((uint32_t)unit + 1) * (uint32_t)grid - 1) / (uint32_t)total) : (int)(((unit + 1) * grid - 1) / total);
  };
  // Where the pairs are few, each may have blocks of its own instead (one, and more in proportion to its units), so that no block has two pairs to
  // finish and to join: if that makes the longest share little longer (13 sequences of 33 units for 2 key heads: 7 units instead of 6,
  // 0.9 us less; one of 131072 tokens for 8: 88.3 -> 84.6).  Where there are no more units than blocks, none has two pairs anyway.
  const int spare = (int)gridDim.x - p.batch * HV;               // blocks beyond one for each pair
  auto blocks_of = [&](int u) { return min(u, 1 + (small ? (int)((uint32_t)u * (uint32_t)spare / (uint32_t)total) : (int)((int64_t)u * spare / total))); };
  bool own_blocks = false;
  if (total > (int64_t)gridDim.x && p.few) {
    int worst = 0;
    for (int b = lane; b < p.batch; b += 32) {
      const int u = sequence<U>(p, b).units;
      if (u) { const int c = blocks_of(u); worst = max(worst, (u + c - 1) / c); }
    }
    worst = __reduce_max_sync(0xffffffffu, worst);
    const int even = (int)((total + grid - 1) / grid);
    own_blocks = worst <= even + max(2, even / 16);
  }
  if (!own_blocks && (int)blockIdx.x >= grid) return empty_ones();
  // this block's first unit in the order of the units, or its place in the order of the pairs' blocks
  const int64_t lo = own_blocks ? (int64_t)blockIdx.x : share(blockIdx.x);
  Place at = {};
  int64_t before = 0;                        // units, or blocks, in front of sequence at.b
  for (int b0 = 0;; b0 += 32) {
    if (b0 >= p.batch) return empty_ones();  // (a block behind the last pair's)
    const int b = b0 + lane;
    int64_t mine = b < p.batch ? sequence<U>(p, b).units : 0;
    if (own_blocks && mine) mine = blocks_of((int)mine);
    mine *= HV;
    int64_t sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, sum, o);
      if (lane >= o) sum += v;
    }
    const unsigned behind = __ballot_sync(0xffffffffu, before + sum > lo);
    if (behind) {
      const int l = __ffs(behind) - 1;
      at.b = b0 + l;
      before += __shfl_sync(0xffffffffu, sum - mine, l);
      break;
    }
    before += __shfl_sync(0xffffffffu, sum, 31);
  }
  at.s = sequence<U>(p, at.b);
  int count, own_first = 0, own_parts = 0;   // units of this block; the pair's blocks, where it has its own
  if (own_blocks) {
    own_parts = blocks_of(at.s.units);
    const int rest = (int)(lo - before), part = rest % own_parts;
    at.vh = rest / own_parts;
    at.u = (int)((uint32_t)at.s.units * (uint32_t)part / (uint32_t)own_parts);
    count = (int)((uint32_t)at.s.units * (uint32_t)(part + 1) / (uint32_t)own_parts) - at.u;
    own_first = (int)blockIdx.x - part;
  } else {
    count = (int)(share(blockIdx.x + 1) - lo);
    if (small) {
      at.vh = (int)((uint32_t)(lo - before) / (uint32_t)at.s.units);
      at.u = (int)(lo - before) - at.vh * at.s.units;
    } else {
      at.vh = (int)((lo - before) / at.s.units);
      at.u = (int)((lo - before) % at.s.units);
    }
  }
  int64_t item_start = before + (int64_t)at.vh * at.s.units;     // first unit of the pair that is being computed (equal shares)
  int begun = at.u;                                              // the unit of it at which this block began

  // ---- loads: the producer's place `in` runs kStages units ahead, and the page numbers' place `ahead` as many more: a tile's page numbers are
  // copied together with the tile kStages before it, so that no load waits for another (each lane has the page of row lane % 16)
  Place in = at, ahead = at;
  const int row_of = warp * kTile + (lane & (kTile - 1));
  auto entry = [&](const Place& a) {         // of the page table; nullptr: this row is not seen
    const int pos = a.s.lo + a.u * U + row_of;
    return pos >= a.s.first && pos < a.s.n ? p.table + a.b * p.table_stride + (pos >> p.page_shift) : nullptr;
  };
  const uint32_t pages_at = smem_u32(pages) + (warp * S::kStages * kTile + (lane & (kTile - 1))) * 4;
  auto issue = [&](int i, int page) {        // page: this lane's, as the table has it
    if (i < count) {
      const int stage = i % S::kStages;
      const uint32_t dst = ring + stage * 2 * S::kTileBytes;
      const int pos0 = in.s.lo + in.u * U + warp * kTile, pos = in.s.lo + in.u * U + row_of;
      if (!(pos >= in.s.first && pos < in.s.n) || page >= p.n_pages) page = -1;
      const unsigned seen = __ballot_sync(0xffffffffu, page >= 0) & 0xffffu;
      if (lane == 0) seen_mem[stage] = seen;
      if (seen) {
        const int mask = (1 << p.page_shift) - 1;
        const int64_t head_at = (int64_t)(in.vh / p.splits) * p.head_stride;
#pragma unroll
        for (int j = 0; j < NC / 2; ++j) {
          const int idx = j * 32 + lane, r = idx / NC, c = idx % NC;
          const int pg = __shfl_sync(0xffffffffu, page, r);
          const int64_t off = pg >= 0 ? pg * p.page_stride + head_at + (int64_t)((pos0 + r) & mask) * p.token_stride + c * 8 : 0;
          const uint32_t d = dst + (r * NC + swizzled<D>(r, c)) * 16;
          cp16(d, reinterpret_cast<const T*>(p.k) + off, pg >= 0);
          cp16(d + S::kTileBytes, reinterpret_cast<const T*>(p.v) + off, pg >= 0);
        }
      }
      next<U>(p, in);
      if (i + S::kStages < count) {
        const int32_t* e = entry(ahead);
        if (e && lane < kTile) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(pages_at + stage * kTile * 4), "l"(e) : "memory");
        next<U>(p, ahead);
      }
    }
    cp_commit();
  };
  auto finish = [&](T* to, float* to_lse, float top, float sum, const float4& acc) {
    const float inv = top == -INFINITY ? 0.f : top == kLowest ? NAN : 1.f / sum;      // no token counted: zeros
    *reinterpret_cast<uint2*>(to) = make_uint2(E::pack(acc.x * inv, acc.y * inv), E::pack(acc.z * inv, acc.w * inv));
    if (to_lse) *to_lse = top == INFINITY ? top : top == kLowest ? -INFINITY : (top + (log2f(sum) - kLift<E>)) * 0.693147180559945309f;
  };
  auto load_q = [&](const Place& a) {        // the query heads of a place; rows behind them are zeros
    const int kvh = a.vh / p.splits, sub = a.vh % p.splits, n = min(p.per, p.group - sub * p.per);
    const T* src = reinterpret_cast<const T*>(p.q) + a.b * p.q_stride + (int64_t)(kvh * p.group + sub * p.per) * D;
    for (int i = tid; i < S::kRows * NC; i += S::kThreads) {
      const int row = i / NC, c = i % NC, r = TWICE ? row & 3 : row;
      const uint4 v = r < n ? reinterpret_cast<const uint4*>(src + (int64_t)r * D)[c] : make_uint4(0, 0, 0, 0);
      *reinterpret_cast<uint4*>(qmem + row * S::kQPitch + c * 16) = v;
    }
  };

#pragma unroll 1
  for (int i = 0; i < S::kStages && i < count; ++i) {        // the first tiles' page numbers: nothing to hide them behind
    const int32_t* e = entry(ahead);
    if (e && lane < kTile) asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(pages_at + i * kTile * 4), "l"(e) : "memory");
    next<U>(p, ahead);
  }
  cp_commit();
  load_q(at);
  empty_ones();
  cp_wait<0>();
  __syncthreads();

  float o[D / 16][NT][4];
  float m[NT][2], l[NT][2];
  auto reset = [&]() {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m[n][0] = m[n][1] = -INFINITY;
      l[n][0] = l[n][1] = 0.f;
#pragma unroll
      for (int j = 0; j < D / 16; ++j) o[j][n][0] = o[j][n][1] = o[j][n][2] = o[j][n][3] = 0.f;
    }
  };
  reset();

  // (the first kStages trips only issue copies: one place in the code for them, as little to fetch as there is)
#pragma unroll 1
  for (int i = -S::kStages; i < count; ++i) {
    const int stage = (i + S::kStages) % S::kStages;
    const uint32_t kt = ring + stage * 2 * S::kTileBytes, vt = kt + S::kTileBytes;
    unsigned seen = 0;
    if (i >= 0) {
      cp_wait<S::kStages - 1>();
      __syncwarp();
      seen = seen_mem[stage];
    }
    if (seen) {
      // ---- S^T = K Q^T
      float s[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) s[n][0] = s[n][1] = s[n][2] = s[n][3] = 0.f;
      const int kr = lane & 15, kc = lane >> 4;                   // ldmatrix: rows 0-7, 8-15 of chunk 2j, then of chunk 2j + 1
      const int qr = lane & 7, qc = lane >> 3;                    // eight heads, chunks 4j .. 4j + 3
#pragma unroll
      for (int j = 0; j < D / 32; ++j) {
        uint32_t a0[4], a1[4];
        ldsm4(a0, kt + (kr * NC + swizzled<D>(kr, 4 * j + kc)) * 16);
        ldsm4(a1, kt + (kr * NC + swizzled<D>(kr, 4 * j + 2 + kc)) * 16);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          uint32_t b[4];
          ldsm4(b, q_addr + (8 * n + qr) * S::kQPitch + (4 * j + qc) * 16);
          mma<E>(s[n], a0, b[0], b[1]);
          mma<E>(s[n], a1, b[2], b[3]);
        }
      }
      // ---- running maximum, probabilities
      const bool s0 = (seen >> g) & 1, s1 = (seen >> (g + 8)) & 1;
      uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float alpha[2], base[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          s[n][c] = s0 ? max_nan(s[n][c] * p.scale_log2, kLowest) : -INFINITY;
          s[n][2 + c] = s1 ? max_nan(s[n][2 + c] * p.scale_log2, kLowest) : -INFINITY;
          float top = max_nan(s[n][c], s[n][2 + c]);
          top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 4));
          top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 8));
          top = max_nan(top, __shfl_xor_sync(0xffffffffu, top, 16));
          const float now = max_nan(m[n][c], top);
          base[c] = now == -INFINITY ? 0.f : now;                 // nothing seen so far: every exponent is -inf - 0
          alpha[c] = exp2f(m[n][c] - base[c]);
          base[c] -= kLift<E>;
          m[n][c] = now;
          s[n][c] = exp2f(s[n][c] - base[c]);
          s[n][2 + c] = exp2f(s[n][2 + c] - base[c]);
          l[n][c] = l[n][c] * alpha[c] + s[n][c] + s[n][2 + c];
        }
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          two_weights<E>(s[n][2 * c], s[n][2 * c + 1], hi[n][c], lo[n][c]);
          if (TWICE && t4 >= 2) hi[n][c] = lo[n][c];
          hi[n][c] = transpose8x8(hi[n][c]);
          if (!TWICE) lo[n][c] = transpose8x8(lo[n][c]);
        }
#pragma unroll
        for (int j = 0; j < D / 16; ++j) {
          o[j][n][0] *= alpha[0]; o[j][n][1] *= alpha[1]; o[j][n][2] *= alpha[0]; o[j][n][3] *= alpha[1];
        }
      }
      // ---- O^T += V^T P^T
      const int vr = (lane & 7) + ((lane >> 4) << 3), vc = (lane >> 3) & 1;   // transposed: tokens 0-7 of chunks 2j, 2j + 1, then tokens 8-15
#pragma unroll
      for (int j = 0; j < D / 16; j += 2) {
        uint32_t a0[4], a1[4];
        ldsm4_t(a0, vt + (vr * NC + swizzled<D>(vr, 2 * j + vc)) * 16);
        ldsm4_t(a1, vt + (vr * NC + swizzled<D>(vr, 2 * j + 2 + vc)) * 16);
#pragma unroll
        for (int n = 0; n < NT; ++n) { mma<E>(o[j][n], a0, hi[n][0], hi[n][1]); mma<E>(o[j + 1][n], a1, hi[n][0], hi[n][1]); }
        if (TWICE) continue;
#pragma unroll
        for (int n = 0; n < NT; ++n) { mma<E>(o[j][n], a0, lo[n][0], lo[n][1]); mma<E>(o[j + 1][n], a1, lo[n][0], lo[n][1]); }
      }
    }
    __syncwarp();
    int page;
    asm volatile("ld.shared.s32 %0, [%1];" : "=r"(page) : "r"(pages_at + stage * kTile * 4) : "memory");
    issue(i + S::kStages, page);
    if (i < 0) continue;

    const bool ends = at.u + 1 == at.s.units;
    if (!ends && i + 1 < count) { ++at.u; continue; }

    // ---- the pair, or this block's share of it, is through: the warps' sums become one
    const bool whole = ends && begun == 0;
    const int slot = blockIdx.x * 2 + (begun ? 0 : 1);
    const int kvh = at.vh / p.splits, sub = at.vh % p.splits, n_heads = min(p.per, p.group - sub * p.per);
    const int head0 = kvh * p.group + sub * p.per;
    T* out = reinterpret_cast<T*>(p.out) + at.b * p.out_stride + (int64_t)head0 * D;
    float* lse = p.lse ? p.lse + (int64_t)at.b * heads + head0 : nullptr;
    Place to = at;
    next<U>(p, to);
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int here = min(8, n_heads - 8 * n);
      if (here <= 0) break;
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        float sum = l[n][c];
        sum += __shfl_xor_sync(0xffffffffu, sum, 4);
        sum += __shfl_xor_sync(0xffffffffu, sum, 8);
        sum += __shfl_xor_sync(0xffffffffu, sum, 16);
        const int h = 2 * t4 + c;
        if (TWICE || h < here) {
          if (g == 0) ml[warp * 8 + h] = make_float2(m[n][c], sum);
          float* dst = obuf + (warp * 8 + h) * S::kOPitch + g;
#pragma unroll
          for (int j = 0; j < D / 16; ++j) { dst[16 * j] = o[j][n][c]; dst[16 * j + 8] = o[j][n][2 + c]; }
        }
      }
      __syncthreads();
      for (int idx = tid; idx < here * (D / 4); idx += S::kThreads) {
        const int h = idx / (D / 4), d = idx % (D / 4);
        float top = -INFINITY;
#pragma unroll
        for (int w = 0; w < S::kWarps; ++w) top = max_nan(top, ml[w * 8 + h].x);
        const float base = top == -INFINITY ? 0.f : top;
        float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
        float sum = 0.f;
#pragma unroll
        for (int w = 0; w < S::kWarps; ++w) {
          const float2 v = ml[w * 8 + h];
          const float k = exp2f(v.x - base);
          float4 x = *reinterpret_cast<const float4*>(obuf + (w * 8 + h) * S::kOPitch + 4 * d);
          if (TWICE) {
            const float4 low = *reinterpret_cast<const float4*>(obuf + (w * 8 + 4 + h) * S::kOPitch + 4 * d);
            x.x += low.x; x.y += low.y; x.z += low.z; x.w += low.w;
          }
          sum = fmaf(k, v.y, sum);
          acc.x = fmaf(k, x.x, acc.x); acc.y = fmaf(k, x.y, acc.y); acc.z = fmaf(k, x.z, acc.z); acc.w = fmaf(k, x.w, acc.w);
        }
        if (whole) {
          finish(out + (int64_t)(8 * n + h) * D + 4 * d, lse && d == 0 ? lse + 8 * n + h : nullptr, top, sum, acc);
        } else {
          __stcg(reinterpret_cast<float4*>(p.part + ((int64_t)slot * S::kRows + 8 * n + h) * D) + d, acc);
          if (d == 0) __stcg(p.part_ml + (int64_t)slot * S::kRows + 8 * n + h, make_float2(top, sum));
        }
      }
      if (n == (n_heads - 1) / 8 && i + 1 < count) load_q(to);
      __syncthreads();
    }
    if (!whole) {
      // the blocks that share this pair: those that own its first and its last unit, and all between
      const int c0 = own_parts ? own_first : owner(item_start), n_parts = own_parts ? own_parts : owner(item_start + at.s.units - 1) - c0 + 1;
      const int columns = n_heads * (D / 4);
      // Parts start, start + step, ... of the pair, n of them, become one: the result, or (in the first one's place) a part for the next round.
      auto join = [&](int start, int step, int n, const float2* from_ml, bool final) {
        for (int idx = tid; idx < columns; idx += S::kThreads) {
          const int h = idx / (D / 4), d = idx % (D / 4);
          // eight parts' values in flight together, their maximum, then what they add
          float top = -INFINITY, sum = 0.f;
          float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 1
          for (int c = 0; c < n; c += 8) {
            float2 v[8];
            float4 x[8];
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const int part = start + (c + q) * step;
              const int64_t row = (int64_t)(2 * part + (part == c0)) * S::kRows + h;
              v[q] = make_float2(-INFINITY, 0.f);
              x[q] = make_float4(0.f, 0.f, 0.f, 0.f);
              if (c + q < n) {
                v[q] = ld_cg2(from_ml + row);
                x[q] = __ldcg(reinterpret_cast<const float4*>(p.part + row * D) + d);
              }
            }
            float now = top;
#pragma unroll
            for (int q = 0; q < 8; ++q) now = max_nan(now, v[q].x);
            const float base = now == -INFINITY ? 0.f : now, k0 = exp2f(top - base);
            sum *= k0; acc.x *= k0; acc.y *= k0; acc.z *= k0; acc.w *= k0;
#pragma unroll
            for (int q = 0; q < 8; ++q) {
              const float k = exp2f(v[q].x - base);
              sum = fmaf(k, v[q].y, sum);
              acc.x = fmaf(k, x[q].x, acc.x); acc.y = fmaf(k, x[q].y, acc.y); acc.z = fmaf(k, x[q].z, acc.z); acc.w = fmaf(k, x[q].w, acc.w);
            }
            top = now;
          }
          if (final) {
            finish(out + (int64_t)h * D + 4 * d, lse && d == 0 ? lse + h : nullptr, top, sum, acc);
          } else {                               // (each thread overwrites what it alone has read; the statistics, which all read, go elsewhere)
            const int64_t row = (int64_t)(2 * start + (start == c0)) * S::kRows + h;
            __stcg(reinterpret_cast<float4*>(p.part + row * D) + d, acc);
            if (d == 0) __stcg(p.joined_ml + row, make_float2(top, sum));
          }
        }
      };
      // Whether this block is the last of n that count up there (which it then leaves as the next call expects it).
      auto last_of = [&](unsigned* counter, int n) {
        if (tid == 0) {
          __threadfence();
          const bool is_last = atomicAdd(counter, 1u) == (unsigned)(n - 1);
          if (is_last) *counter = 0;
          __threadfence();
          *flag = is_last;
        }
        __syncthreads();
        const bool is = *flag;
        __syncthreads();
        return is;
      };
      // Many parts are joined in two rounds, eight blocks' first: one block would read them all through one SM (74 parts of 12 heads of 128: 16 us)
      unsigned* arrived = p.arrived + (int64_t)at.b * HV + at.vh;
      if (n_parts * ((columns + S::kThreads - 1) / S::kThreads) <= kOneRound) {
        if (last_of(arrived, n_parts)) join(c0, 1, n_parts, p.part_ml, true);
      } else {
        const int mine = ((int)blockIdx.x - c0) / 8, start = c0 + 8 * mine, n = min(8, n_parts - 8 * mine);
        if (last_of(p.arrived_group + 2 * start + (start == c0), n)) {
          join(start, 1, n, p.part_ml, false);
          __syncthreads();
          const int groups = (n_parts + 7) / 8;
          if (last_of(arrived, groups)) join(c0, 8, groups, p.joined_ml, true);
        }
      }
    }
    if (i + 1 < count) {
      item_start += at.s.units;                                    // (sequences that lie between have no units)
      at = to;
      begun = 0;
      reset();
    }
  }
}

constexpr int kMaxGrid = 160;         // partial sums are kept for so many blocks (a B200 has 148 SMs)

// How the query heads of a key head are served: in `splits` parts of at most 8 nt, as even as they come.  More per part reads K and V
// less often; what an accumulator of head_dim x 8 nt leaves of the registers ends it (32 heads up to 128 channels, 16 at 256).
struct Plan {
  int nt, splits, per, unit;
  size_t counters, groups, part, stats; // bytes
  size_t bytes() const { return groups + counters + part + 2 * stats; }
};
Plan make_plan(const eora_attention_config& c) {
  Plan p;
  const int group = c.n_heads / c.n_kv_heads, most = c.head_dim <= 128 ? 32 : 16;
  p.splits = (group + most - 1) / most;
  p.per = (group + p.splits - 1) / p.splits;
  p.splits = (group + p.per - 1) / p.per;
  p.nt = p.per <= 8 ? 1 : p.per <= 16 ? 2 : 4;
  p.unit = kTile * (c.head_dim > 128 ? 4 : 8);
  const size_t rows = 2 * (size_t)kMaxGrid * 8 * p.nt;
  p.counters = ((size_t)c.max_batch * c.n_kv_heads * p.splits * 4 + 255) / 256 * 256;
  p.groups = 2 * kMaxGrid * 4;
  p.part = rows * c.head_dim * 4;
  p.stats = rows * 8;
  return p;
}

template <class E, int D, int NT, bool TWICE = false>
cudaError_t launch_one(const AttnArgs& a, int grid, int device, cudaStream_t st) {
  using S = Shape<D, NT>;
  static int set_up[16] = {};           // per device; benign if two threads do it at once
  if (device >= 16 || !set_up[device]) {
    const cudaError_t e = cudaFuncSetAttribute(k_attention<E, D, NT, TWICE>, cudaFuncAttributeMaxDynamicSharedMemorySize, S::kSmem);
    if (e != cudaSuccess) return e;
    if (device < 16) set_up[device] = 1;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(S::kThreads);
  cfg.dynamicSmemBytes = S::kSmem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, k_attention<E, D, NT, TWICE>, a);
}
template <class E, int D>
cudaError_t launch_nt(int nt, const AttnArgs& a, int grid, int device, cudaStream_t st) {
  if (nt == 1) return a.per <= 4 ? launch_one<E, D, 1, true>(a, grid, device, st) : launch_one<E, D, 1>(a, grid, device, st);
  if constexpr (D <= 128) {
    if (nt == 4) return launch_one<E, D, 4>(a, grid, device, st);
  }
  return launch_one<E, D, 2>(a, grid, device, st);
}
template <class E>
cudaError_t launch(int head_dim, int nt, const AttnArgs& a, int grid, int device, cudaStream_t st) {
  switch (head_dim) {
    case 64: return launch_nt<E, 64>(nt, a, grid, device, st);
    case 96: return launch_nt<E, 96>(nt, a, grid, device, st);
    case 128: return launch_nt<E, 128>(nt, a, grid, device, st);
    default: return launch_nt<E, 256>(nt, a, grid, device, st);
  }
}

int check(const eora_attention_config& c) {
  if (c.n_heads < 1 || c.n_heads > 1024 || c.n_kv_heads < 1 || c.n_heads % c.n_kv_heads) return EORA_ERR_BAD_SHAPE;
  if (c.head_dim != 64 && c.head_dim != 96 && c.head_dim != 128 && c.head_dim != 256) return EORA_ERR_BAD_SHAPE;
  if (c.page_size < 1 || (c.page_size & (c.page_size - 1)) || c.max_pages < 1 || (int64_t)c.max_pages * c.page_size > (1 << 30)) return EORA_ERR_BAD_SHAPE;
  if (c.max_batch < 1 || c.max_batch > 65536 || c.window < 0 || !(c.scale > 0.f) || !isfinite(c.scale)) return EORA_ERR_BAD_SHAPE;
  return x_type(c.dtype) ? EORA_OK : EORA_ERR_UNSUPPORTED;
}

}  // namespace
}  // namespace serve
}  // namespace eora

using namespace eora::serve;

extern "C" {

size_t eora_attention_workspace_bytes(const eora_attention_config* cfg) { return cfg && check(*cfg) == EORA_OK ? make_plan(*cfg).bytes() : 0; }

int eora_attention_forward(const eora_attention_config* cfg, const void* q, int64_t q_stride, const eora_kv_cache* cache, const int32_t* page_table,
                           int64_t table_stride, const int32_t* lengths, int32_t batch, void* out, int64_t out_stride, float* lse, void* workspace,
                           size_t workspace_bytes, void* stream) {
  if (!cfg || !cache) return EORA_ERR_NULL_ARG;
  const eora_attention_config& c = *cfg;
  int st = check(c);
  if (st != EORA_OK) return st;
  if (batch < 0) return EORA_ERR_BAD_SHAPE;
  if (batch > c.max_batch) return EORA_ERR_M_TOO_LARGE;
  if (batch == 0) return EORA_OK;
  if (!q || !page_table || !lengths || !out || !workspace) return EORA_ERR_NULL_ARG;
  st = check_cache(*cache);
  if (st != EORA_OK) return st;
  if (cache->n_kv_heads != c.n_kv_heads || cache->head_dim != c.head_dim || cache->page_size != c.page_size) return EORA_ERR_BAD_SHAPE;
  if (cache->dtype != c.dtype) return EORA_ERR_UNSUPPORTED;
  const int64_t row = (int64_t)c.n_heads * c.head_dim;
  const Plan plan = make_plan(c);
  if (q_stride < row || out_stride < row || table_stride < c.max_pages || workspace_bytes < plan.bytes()) return EORA_ERR_BAD_SHAPE;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(page_table, 4) || !aligned(lengths, 4) || !aligned(workspace, 16) || q_stride % 8 || out_stride % 8)
    return EORA_ERR_MISALIGNED;
  if (out == q && batch > 1 && out_stride != q_stride) return EORA_ERR_BAD_SHAPE;      // (a pair's queries are read before its result is stored, other rows' are not)
  int device = 0, sms = 0;
  if (cudaGetDevice(&device) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device) != cudaSuccess) return EORA_ERR_CUDA;

  AttnArgs a = {};
  a.q = q; a.k = cache->k; a.v = cache->v; a.out = out; a.lse = lse; a.table = page_table; a.lengths = lengths;
  a.q_stride = q_stride; a.out_stride = out_stride; a.table_stride = table_stride;
  a.page_stride = cache->page_stride; a.head_stride = cache->head_stride; a.token_stride = cache->token_stride;
  a.batch = batch; a.kv_heads = c.n_kv_heads; a.group = c.n_heads / c.n_kv_heads; a.splits = plan.splits; a.per = plan.per;
  a.n_pages = cache->n_pages; a.page_shift = log2i(c.page_size); a.max_tokens = c.max_pages * c.page_size;
  a.window = c.window;
  a.scale_log2 = c.scale * 1.44269504088896341f;
  char* ws = static_cast<char*>(workspace);
  a.arrived_group = reinterpret_cast<unsigned*>(ws);
  a.arrived = reinterpret_cast<unsigned*>(ws + plan.groups);
  ws += plan.groups + plan.counters;
  a.part = reinterpret_cast<float*>(ws);
  a.part_ml = reinterpret_cast<float2*>(ws + plan.part);
  a.joined_ml = reinterpret_cast<float2*>(ws + plan.part + plan.stats);
  // a block per SM, but no more blocks than there can be units
  const int64_t most = c.window && c.window < a.max_tokens ? (int64_t)c.window + kTile : a.max_tokens;
  const int64_t units = (most + plan.unit - 1) / plan.unit * batch * c.n_kv_heads * plan.splits;
  int grid = sms < kMaxGrid ? sms : kMaxGrid;
  if (units < grid) grid = (int)units;
  a.few = (int64_t)batch * c.n_kv_heads * plan.splits <= grid;
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const cudaError_t e = c.dtype == EORA_X_F16 ? launch<F16>(c.head_dim, plan.nt, a, grid, device, s) : launch<BF16>(c.head_dim, plan.nt, a, grid, device, s);
  return e == cudaSuccess ? EORA_OK : EORA_ERR_CUDA;
}

}  // extern "C"
