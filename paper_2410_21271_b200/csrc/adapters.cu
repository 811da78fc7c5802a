// Low-rank adapters of many requests beside a shared projection (eora_serve.h):
//   y[i] = base[i] + s_j (x[i] . A_j) . B_j,  j = ids[i].
//
// What bounds it: few tokens: the bytes of the adapters that are named (r (d_in + d_out) 16-bit values each) and the latency of
// two products of which the second needs all of the first; prompts: the bytes of x, base and y, while an adapter's A and B, read
// once per tile of tokens, come from L2.
//  - A thread block cluster per tile: an adapter and up to 16 (few tokens) or 32 (many) of its tokens.  Its blocks share d_in in the
//    first product and d_out in the second, and exchange t = x . A through distributed shared memory.  So one launch does both
//    products, t never leaves the chip, nothing is kept between calls, and the sums have a fixed order.
//  - Which tokens a cluster has, every block works out for itself from ids (counts per adapter, then the tile's tokens in order).
//  - The order in which the reduction axis is taken is free, so that neither product needs its operands rearranged: a lane takes
//    rows 8 t .. 8 t + 7 (t = lane % 4) of 32 and eight consecutive columns of each, and pairs of rows are interleaved with a byte
//    permute.  Column g of the instruction is then column 8 block_of(g) + i of the matrix, and a lane ends with runs of eight
//    consecutive result columns.  x, A, B (and base, with many tokens) come by asynchronous copies into slots of shared memory from
//    which each warp reads its own: no two warps of a block load the same byte of A or B.
// Measured (B200, of the copy rate of 6.56 TB/s): 32 requests of 30 adapters of rank 64, 32 and 16 on 4096 x 4096 10.3 us (1.9 TB/s of
// 19 MB); 61 tokens, 5 adapters of rank 128 on 4096 x 14336, fp32 out 15.8 us (2.0 TB/s); prompts of 2048 tokens, rank 64 on
// 14336 x 4096 47 us (2.3 TB/s; 95 TFLOP/s); one token, rank 16 6.0 us.  What is left is latency: ids -> adapter -> A -> exchange -> B is
// a chain of some 5 us, and 40 % of a prompt's time lies outside the two products.
#include <algorithm>
#include "serve_common.cuh"

namespace eora {
namespace serve {
namespace {

constexpr int kMaxRank = 256, kMaxAdapters = 4096, kMaxTokens = 1 << 20;
constexpr int kStaged = 7680;                   // tokens of a launch: their ids stand in shared memory (and looking through them stays short)
constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kPitch = 68;                      // floats of a row of 64 partial sums in shared memory

struct AdapterArgs {
  const void *x, *a, *b, *base;
  void* y;
  const int32_t *ids, *ranks;
  const float* scales;
  int64_t x_stride, base_stride, y_stride;
  int m, d_in, d_out, max_rank, n_adapters, y_dtype;
  int skip_none;                                // rows without an adapter are in place already
  int t_at, t_pitch;                            // t's parts in shared memory: byte offset, bytes of a row
};

__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ void st_cluster(uint32_t addr, uint2 v, uint2 w) {
  asm volatile("st.shared::cluster.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(v.x), "r"(v.y), "r"(w.x), "r"(w.y) : "memory");
}
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Weights go through the ring in pieces of four rows x 64 columns: in the copy, lane L brings columns 8 (L % 8) .. + 7 of row L / 8, so that eight
// neighbouring lanes read 128 consecutive bytes (in the consumers' order, 4 rows x 32 bytes per eight lanes, a copy took 21 cycles instead of 8);
// the consumer (g, t) of row t takes column block block_of(g).  That order of the blocks gives a lane two runs of eight result columns, 8 t and
// 32 + 8 (t ^ 1), so that four lanes store 64 consecutive bytes of a row.  A row's 128 bytes stay together in shared memory, swizzled in pairs of
// blocks; both sides are free of bank conflicts.
__device__ __forceinline__ int block_of(int g) { return (g & 1) ? 4 + ((g >> 1) ^ 1) : g >> 1; }
__device__ __forceinline__ uint32_t piece_at(int block, int t) { return (uint32_t)(8 * t + (block ^ (2 * t))) * 16; }

// Eight columns of two rows, as eight pairs (row 0, row 1).
__device__ __forceinline__ uint32_t pair_of(const uint4& r0, const uint4& r1, int i) {
  return __byte_perm(word(r0, i >> 1), word(r1, i >> 1), (i & 1) ? 0x7632 : 0x5410);
}

// Rank and scale of adapter j.  Ordinary loads: this launch may begin before the one in front has written them, and the read-only path is for what
// nobody writes from a kernel's begin on.
__device__ __forceinline__ int2 kind_of(const AdapterArgs& p, int j) {
  return make_int2(p.ranks ? p.ranks[j] : p.max_rank, __float_as_int(p.scales ? p.scales[j] : 1.f));
}

// The tile of cluster `c`: its adapter (n_adapters: none) and, in tok, its tokens in order of their place in ids.  Returns how many,
// 0 if there is no such tile.  counts: n_adapters + 1 + kStaged + a thread's each ints, aux: WARPS + 4 ints.
template <int TM, int WARPS>
__device__ __forceinline__ int find_tile(const AdapterArgs& p, int c, int& adapter, int* tok, int* counts, int* aux) {
  constexpr int kThr = 32 * WARPS;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = p.n_adapters;
  // A thread looks through `1 << shift` neighbouring ids, which come to shared memory first, all loads in flight, each thread's an odd number of words
  // from the next one's.
  int shift = 0;
  while ((kThr << shift) < p.m) ++shift;
  int* staged = counts + n + 1;
#pragma unroll 8
  for (int i = tid; i < p.m; i += kThr) {
    const int j = p.ids[i];
    staged[i + (i >> shift)] = j >= 0 && j < n ? j : n;
  }
  for (int i = tid; i <= n; i += kThr) counts[i] = 0;
  __syncthreads();
  const int lo = min(tid << shift, p.m), hi = min(lo + (1 << shift), p.m);
  const int* mine = staged + tid;               // (id i of this thread is at mine[i])
  {
    int run = 0, last = n;                      // neighbouring tokens are often of one request: one addition for a run
#pragma unroll 1
    for (int i = lo; i < hi; i += 8) {
      int key[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) key[q] = i + q < hi ? mine[i + q] : -1;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        if (key[q] < 0) break;
        if (key[q] != last && run) { atomicAdd(&counts[last], run); run = 0; }
        last = key[q];
        ++run;
      }
    }
    if (run) atomicAdd(&counts[last], run);
  }
  __syncthreads();
  if (warp == 0) {                              // which adapter owns tile c: a lane adds up a run of adapters, the warp the lanes
    const int per = (n + 32) / 32, first = lane * per, end = min(first + per, n + 1);
    auto tiles = [&](int j) { return j == n && p.skip_none ? 0 : (counts[j] + TM - 1) / TM; };
    int sum = 0;
    for (int j = first; j < end; ++j) sum += tiles(j);
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    if (lane == 31) aux[WARPS] = upto;          // all tiles
    if (c >= upto - sum && c < upto) {
      int left = c - (upto - sum), j = first;
      while (left >= tiles(j)) left -= tiles(j++);
      aux[WARPS + 1] = j;
      aux[WARPS + 2] = left;
    }
  }
  __syncthreads();
  if (c >= aux[WARPS]) return 0;
  adapter = aux[WARPS + 1];
  const int from = aux[WARPS + 2] * TM;
  // its tokens: how many each thread has, how many are in front of those, then their places
  int found = 0;
#pragma unroll 4
  for (int i = lo; i < hi; ++i) found += mine[i] == adapter;
  int upto = found;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 31) aux[warp] = upto;
  __syncthreads();
  int at = upto - found - from;
  for (int w = 0; w < warp; ++w) at += aux[w];
  if (found && at < TM && at + found > 0) {
#pragma unroll 4
    for (int i = lo; i < hi; ++i) {
      const bool is = mine[i] == adapter;
      if (is && at >= 0 && at < TM) tok[at] = i;
      at += is;
    }
  }
  const int n_tok = min(TM, counts[adapter] - from);
  __syncthreads();
  return n_tok;
}

// Eight columns (those of half k = 2 h + c of a fragment) or four of them, added to base's and stored.
template <class E>
__device__ __forceinline__ void put8(void* y, int64_t at, const float (&acc)[8][4], int k, float undo, const uint4& base) {
  uint32_t o[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const float2 v = E::unpack(word(base, q));
    o[q] = E::pack(fmaf(acc[2 * q][k], undo, v.x), fmaf(acc[2 * q + 1][k], undo, v.y));
  }
  *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(y) + at) = make_uint4(o[0], o[1], o[2], o[3]);
}
__device__ __forceinline__ void put4(void* y, int64_t at, const float (&acc)[8][4], int k, int q, float undo, const uint4& base) {
  *reinterpret_cast<float4*>(reinterpret_cast<float*>(y) + at) =
      make_float4(fmaf(acc[4 * q][k], undo, __uint_as_float(base.x)), fmaf(acc[4 * q + 1][k], undo, __uint_as_float(base.y)),
                  fmaf(acc[4 * q + 2][k], undo, __uint_as_float(base.z)), fmaf(acc[4 * q + 3][k], undo, __uint_as_float(base.w)));
}

// y's and base's columns of a lane: eight from at_c[c] on, of its tile's rows g and 8 + g; all loads before the first store (y may be base).
__device__ __forceinline__ void add_store(const AdapterArgs& p, const int64_t (&token)[2], const int (&at_c)[2], const bool (&there)[4], const float (&acc)[8][4], const float (&undo)[2]) {
  uint4 b[8] = {};
  if (p.y_dtype == EORA_Y_F32) {
    if (p.base) {
#pragma unroll
      for (int k = 0; k < 8; ++k)
        if (there[k >> 1]) b[k] = *reinterpret_cast<const uint4*>(reinterpret_cast<const float*>(p.base) + token[k >> 2] * p.base_stride + at_c[(k >> 1) & 1] + 4 * (k & 1));
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (there[k >> 1]) put4(p.y, token[k >> 2] * p.y_stride + at_c[(k >> 1) & 1] + 4 * (k & 1), acc, k >> 1, k & 1, undo[k >> 2], b[k]);
    return;
  }
  if (p.base) {
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (there[k]) b[k] = *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(p.base) + token[k >> 1] * p.base_stride + at_c[k & 1]);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (!there[k]) continue;
    const int64_t at = token[k >> 1] * p.y_stride + at_c[k & 1];
    if (p.y_dtype == EORA_Y_F16) put8<F16>(p.y, at, acc, k, undo[k >> 1], b[k]);
    else put8<BF16>(p.y, at, acc, k, undo[k >> 1], b[k]);
  }
}

// The second product's ring: for each 64 columns of a warp, B's pieces (32 ranks a stage), then base's (eight pieces a stage: a lane's own eight
// columns of 16 bits, or four of 32, per piece, in its own slot).  Base is on its way while B is multiplied; y may be base, each byte of which is
// read by the lane that writes it, before that.
template <class T, int STAGES>
struct Columns {
  const AdapterArgs& p;
  const T* b;                          // of the adapter, at this lane's columns
  const int* tok;
  int n_tok, r, n1, step, chunks, bases;
  uint32_t ring, to;
  int lane, g, ct, at0, at1;           // a lane's two runs of eight columns in the 64
  int c0, ch, stage;                   // what is copied next
  __device__ __forceinline__ void issue() {
    const uint32_t d = ring + stage * 8 * 512;
    stage = stage + 1 == STAGES ? 0 : stage + 1;
    if (c0 < n1) {
      if (ch < chunks) {
        const bool in_n = c0 + 8 * (lane & 7) < n1;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int c = 32 * ch + 16 * (q >> 2) + 4 * ct + (q & 3);
          const bool there = in_n && c < r;
          cp16(d + q * 512 + to, there ? b + (int64_t)c * p.d_out + c0 : reinterpret_cast<const T*>(p.b), there);
        }
      } else if (p.y_dtype == EORA_Y_F32) {
        const int i = ch - chunks;
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int row = 16 * i + 8 * (q >> 2) + g, at = c0 + ((q & 2) ? at1 : at0);
          const bool there = row < n_tok && at < n1;
          cp16(d + q * 512 + lane * 16, reinterpret_cast<const float*>(p.base) + (there ? tok[row] * p.base_stride + at + 4 * (q & 1) : 0), there);
        }
      } else {
        const int i = 2 * (ch - chunks);
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          const int row = 16 * (i + (q >> 2)) + 8 * ((q >> 1) & 1) + g, at = c0 + ((q & 1) ? at1 : at0);
          const bool there = row < n_tok && at < n1;
          cp16(d + q * 512 + lane * 16, reinterpret_cast<const uint16_t*>(p.base) + (there ? tok[row] * p.base_stride + at : 0), there);
        }
      }
      if (++ch >= chunks + bases) { ch = 0; c0 += step; }
    }
    cp_commit();
  }
};
// How many stages base takes for 64 columns of 32 tokens.
__device__ __forceinline__ int base_stages(const AdapterArgs& p) { return p.base ? (p.y_dtype == EORA_Y_F32 ? 2 : 1) : 0; }

// The power of two that brings `top`, which is finite, to [2^9, 2^10) (1 for zero), and its inverse.
__device__ __forceinline__ void powers(float top, float& up, float& down) {
  const int e = (int)(__float_as_uint(top) >> 23);                  // biased exponent
  const int lift = top == 0.f ? 0 : min(9 + 127 - e, 126);
  up = __uint_as_float((uint32_t)(127 + lift) << 23);
  down = __uint_as_float((uint32_t)(127 - lift) << 23);
}
template <class E> __device__ __forceinline__ void two_parts(const float (&v)[4], float up, uint2& hi, uint2& lo) {
  float f[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = v[i] * up;
  hi = make_uint2(E::pack(f[0], f[1]), E::pack(f[2], f[3]));
  const float2 h0 = E::unpack(hi.x), h1 = E::unpack(hi.y);
  const float rest[4] = {f[0] - h0.x, f[1] - h0.y, f[2] - h1.x, f[3] - h1.y};
#pragma unroll
  for (int i = 0; i < 4; ++i) f[i] = isinf(f[i]) ? 0.f : rest[i];        // (nothing is left of an infinity; inf - inf would make it NaN)
  lo = make_uint2(E::pack(f[0], f[1]), E::pack(f[2], f[3]));
}

// t of the tile from the blocks' sums (at `part` in each block's shared memory; S: distance of two column blocks there), a row per 16 lanes (32 where
// the rank is above 64), four columns per lane.  A token's values share a power of two that brings the largest to [2^9, 2^10): fp16 has room on
// both sides there.  High part and low part each rounded to nearest: 2^-22 (fp16), 2^-16 (bf16) of a value is left.
// Four values' high parts and their low parts stand side by side.  With `spread`, a row is added up by one block only, which sends the parts to all:
// every block pulling all rows is one exchange less, but 16 blocks that pull 12 rows of 128 from each other took 4 us, the two exchanges take 1.5.
template <class E, int WARPS, int TM>
__device__ __forceinline__ void gather_t(const AdapterArgs& p, uint32_t part, int S, int r, int n_tok, float scale, uint32_t size, uint32_t rank_in, bool spread,
                                         uint32_t parts, float* undo) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int r16 = (r + 15) & ~15, lanes = r <= 64 ? 16 : 32, sub = lane & (lanes - 1), rows = 32 / lanes;
  const int stride = spread ? (int)size : 1, first = spread ? (int)rank_in : 0;
  for (int i0 = warp * rows; first + i0 * stride < n_tok; i0 += WARPS * rows) {
    const int row = first + (i0 + (lanes == 16 ? lane >> 4 : 0)) * stride;
    float v[2][4];
    float top = 0.f;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int c = 4 * sub + 128 * q;
      v[q][0] = v[q][1] = v[q][2] = v[q][3] = 0.f;
      if (c < r && row < n_tok) {
        const uint32_t at = part + ((c / 64 * S * TM + row) * kPitch + c % 64) * 4;
        for (uint32_t s0 = 0; s0 < size; s0 += 8) {
          float4 o[8];
#pragma unroll
          for (uint32_t s = 0; s < 8; ++s) o[s] = s0 + s < size ? ld_cluster4(dec::mapa(at, s0 + s)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
          for (uint32_t s = 0; s < 8; ++s) { v[q][0] += o[s].x; v[q][1] += o[s].y; v[q][2] += o[s].z; v[q][3] += o[s].w; }
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          v[q][e] = c + e < r ? v[q][e] * scale : 0.f;              // (columns behind the rank hold anything)
          top = fmaxf(top, isfinite(v[q][e]) ? fabsf(v[q][e]) : 0.f);
        }
      }
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      if (o < lanes) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    float up, down;
    powers(top, up, down);
    if (row >= n_tok) continue;
#pragma unroll
    for (int q = 0; q < 2; ++q) {
      const int c = 4 * sub + 128 * q;
      if (c >= r16) continue;
      uint2 hi, lo;
      two_parts<E>(v[q], up, hi, lo);
      const uint32_t at = parts + row * p.t_pitch + 4 * c;
      for (uint32_t s = 0; s < (spread ? size : 1); ++s) st_cluster(dec::mapa(at, spread ? s : rank_in), hi, lo);
    }
    if (sub != 0) continue;
    if (!spread) undo[row] = down;
    else
      for (uint32_t s = 0; s < size; ++s) asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(dec::mapa(smem_u32(undo + row), s)), "f"(down) : "memory");
  }
}

// ---- few tokens: a cluster per (adapter, up to sixteen of its tokens)
// Two blocks of eight warps per SM (a warp alone, or two on a quarter of an SM, leave gaps between its loads, its matrix instructions and its
// epilogue: 61 tokens, rank 128, 24 us with one block of three stages).
constexpr int kSpread = 8192;                  // floats that every block would pull
constexpr int kFewWarps = 8, kFewThreads = 256, kFewStages = 2, kFewPieces = 10;
constexpr int kFewRing = kFewWarps * kFewStages * kFewPieces * 512, kFewSums = kFewWarps / 2 * 16 * kPitch * 4;

// The tile of cluster c among at most 64 tokens: every warp has all ids in its lanes and works it out for itself.  Tiles are numbered by the
// place of their first token.  Returns the number of tokens (0: no such tile), their places in tok (written by every warp alike, into rows of its own).
__device__ __forceinline__ int find_tile_few(const AdapterArgs& p, int c, int& adapter, int* tok) {
  const int lane = threadIdx.x & 31, n = p.n_adapters;
  const unsigned below = (1u << lane) - 1;
  int key[2], rank[2];
  unsigned same[2] = {0, 0}, lead[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int i = lane + 32 * h;
    key[h] = -1 - i;                                              // (no token: like no other)
    if (i < p.m) {
      const int j = p.ids[i];
      key[h] = j >= 0 && j < n ? j : n;
    }
  }
  same[0] = __match_any_sync(0xffffffffu, key[0]);
  rank[0] = __popc(same[0] & below);
  rank[1] = 0;
  if (p.m > 32) {
    same[1] = __match_any_sync(0xffffffffu, key[1]);
    rank[1] = __popc(same[1] & below);
#pragma unroll
    for (int s = 0; s < 32; ++s) rank[1] += __shfl_sync(0xffffffffu, key[0], s) == key[1];
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) lead[h] = __ballot_sync(0xffffffffu, key[h] >= 0 && rank[h] % 16 == 0 && !(key[h] == n && p.skip_none));
  const int in0 = __popc(lead[0]);
  if (c >= in0 + __popc(lead[1])) return 0;
  const int h = c >= in0, nth = c - (h ? in0 : 0);
  const unsigned leads = h ? lead[1] : lead[0];
  const int who = __ffs(__ballot_sync(0xffffffffu, ((leads >> lane) & 1) && __popc(leads & below) == nth)) - 1;
  adapter = __shfl_sync(0xffffffffu, h ? key[1] : key[0], who);
  const int first = __shfl_sync(0xffffffffu, h ? rank[1] : rank[0], who);
  int count = 0;
#pragma unroll
  for (int q = 0; q < 2; ++q) {
    const bool mine = key[q] == adapter;
    if (mine && rank[q] >= first && rank[q] < first + 16) tok[rank[q] - first] = lane + 32 * q;
    count += __popc(__ballot_sync(0xffffffffu, mine));
  }
  __syncwarp();
  return min(16, count - first);
}

// One stream of copies through each warp's ring: its runs of A (with x) first, then its columns of B, whose first stages are on their way
// while the blocks exchange t.
// LANES: m <= 64, ids in the lanes of every warp (a kernel of its own: with the general search in it as well, one token took 0.7 us more).
template <class E, bool LANES>
__global__ void __launch_bounds__(kFewThreads, 2) k_adapters_few(const AdapterArgs p) {
  using T = typename E::T;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int tok_of[kFewWarps][16], aux[kFewWarps + 4];
  __shared__ float undo[16];
  __shared__ int2 kinds[kFewThreads];                               // rank and scale of the first adapters
  float* part = reinterpret_cast<float*>(smem + kFewRing);
  const uint32_t parts = smem_u32(smem) + kFewRing + kFewSums;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
  uint32_t rank_in, size;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank_in));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
  const uint32_t nb = (uint32_t)p.d_out / 32, kb = (uint32_t)p.d_in / 32;
  const int n0 = (int)(nb * rank_in / size) * 32, n1 = (int)(nb * (rank_in + 1) / size) * 32;
  const int k0 = (int)(kb * rank_in / size), k1 = (int)(kb * (rank_in + 1) / size);
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  auto kind = [&](int j) { return kind_of(p, j); };
  if (tid < p.n_adapters) kinds[tid] = kind(tid);                   // (in flight together with ids)
  int j = 0;
  int* tok = tok_of[LANES ? warp : 0];
  int n_tok;
  if constexpr (LANES) n_tok = find_tile_few(p, blockIdx.x / size, j, tok);
  else n_tok = find_tile<16, kFewWarps>(p, blockIdx.x / size, j, tok, reinterpret_cast<int*>(smem), aux);
  if (n_tok == 0) return;                                           // (the whole cluster)
  __syncthreads();
  const int2 mine = j >= p.n_adapters ? make_int2(0, 0) : j < kFewThreads ? kinds[j] : kind(j);
  const int r = min(max(mine.x, 0), p.max_rank);
  const float scale = __int_as_float(mine.y);
  const bool spread = n_tok * r * (int)size > kSpread;

  // this warp's part: 64 columns of A over every S-th run of 32 of this block's share of d_in; every eighth 64 columns of its share of d_out
  const int ncb = (r + 63) / 64, S = kFewWarps / (ncb <= 1 ? 1 : ncb == 2 ? 2 : 4), cb = warp / S, ks = warp % S;
  const int trips = r > 0 && cb < ncb && k0 + ks < k1 ? (k1 - k0 - ks + S - 1) / S : 0;
  const int chunks = (r + 31) / 32;                                 // of 32 ranks, for each of its column blocks of B
  const int cl = 8 * (lane & 7), ct = lane >> 3;                    // what this lane copies: columns, row of a piece
  const bool col = cb * 64 + cl < r;
  const T* a_next = reinterpret_cast<const T*>(p.a) + ((int64_t)j * p.d_in + (k0 + ks) * 32 + 8 * ct) * p.max_rank + (col ? cb * 64 + cl : 0);
  const T* x_next[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) x_next[i] = reinterpret_cast<const T*>(p.x) + tok[8 * i + g < n_tok ? 8 * i + g : 0] * p.x_stride + 8 * t4 + (k0 + ks) * 32;
  const T* bj = reinterpret_cast<const T*>(p.b) + (int64_t)j * p.max_rank * p.d_out + cl;
  const uint32_t ring = smem_u32(smem) + warp * kFewStages * kFewPieces * 512, to = piece_at(lane & 7, lane >> 3), from = piece_at(block_of(g), t4);
  int in = 0, in_c0 = n0 + 64 * warp, in_ch = 0, in_stage = 0;
  auto issue = [&]() {
    const uint32_t d = ring + in_stage * kFewPieces * 512;
    in_stage = in_stage + 1 == kFewStages ? 0 : in_stage + 1;
    if (in < trips) {
      ++in;
#pragma unroll
      for (int q = 0; q < 8; ++q) cp16(d + q * 512 + to, a_next + (int64_t)q * p.max_rank, col);
#pragma unroll
      for (int i = 0; i < 2; ++i) { cp16(d + (8 + i) * 512 + lane * 16, x_next[i], 8 * i + g < n_tok); x_next[i] += 32 * S; }
      a_next += (int64_t)32 * S * p.max_rank;
    } else if (in_c0 < n1 && chunks) {
      const bool in_n = in_c0 + cl < n1;
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const int c = 32 * in_ch + 16 * (q >> 2) + 4 * ct + (q & 3);
        const bool there = in_n && c < r;
        cp16(d + q * 512 + to, there ? bj + (int64_t)c * p.d_out + in_c0 : reinterpret_cast<const T*>(p.b), there);
      }
      if (++in_ch == chunks) { in_ch = 0; in_c0 += 64 * kFewWarps; }
    }
    cp_commit();
  };
#pragma unroll 1
  for (int i = 0; i < kFewStages; ++i) issue();
  int stage = 0;
  auto slot = [&]() { return ring + stage * kFewPieces * 512; };
  auto done = [&]() { __syncwarp(); issue(); stage = stage + 1 == kFewStages ? 0 : stage + 1; };

  float acc[8][4];
  auto clear = [&]() {
#pragma unroll
    for (int n = 0; n < 8; ++n) acc[n][0] = acc[n][1] = acc[n][2] = acc[n][3] = 0.f;
  };
  if (r > 0) {
    clear();
#pragma unroll 1
    for (int it = 0; it < trips; ++it) {
      cp_wait<kFewStages - 1>();
      __syncwarp();
      uint4 w[8], xv[2];
#pragma unroll
      for (int q = 0; q < 8; ++q) w[q] = dec::lds_u4(slot() + q * 512 + from);
#pragma unroll
      for (int i = 0; i < 2; ++i) xv[i] = dec::lds_u4(slot() + (8 + i) * 512 + lane * 16);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        const uint32_t a[4] = {word(xv[0], 2 * s), word(xv[1], 2 * s), word(xv[0], 2 * s + 1), word(xv[1], 2 * s + 1)};
#pragma unroll
        for (int n = 0; n < 8; ++n) mma<E>(acc[n], a, pair_of(w[4 * s], w[4 * s + 1], n), pair_of(w[4 * s + 2], w[4 * s + 3], n));
      }
      done();
    }
    // The sums of the S warps that share a column block, in S / 2 places: one half of them writes, the other adds.  A lane's columns of row
    // 8 h + g: 8 t4 .. + 7 (from the even half of a fragment) and 32 + 8 (t4 ^ 1) .. + 7 (from the odd).
    const int half = S / 2;
    float* dst = part + (cb * half + ks % half) * 16 * kPitch;
    auto place = [&](bool add) {
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            float4* at = reinterpret_cast<float4*>(dst + (8 * h + g) * kPitch + (c ? 32 + 8 * (t4 ^ 1) : 8 * t4) + 4 * q);
            float4 v = make_float4(acc[4 * q][2 * h + c], acc[4 * q + 1][2 * h + c], acc[4 * q + 2][2 * h + c], acc[4 * q + 3][2 * h + c]);
            if (add) { const float4 o = *at; v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w; }
            *at = v;
          }
    };
    if (cb < ncb && ks >= half) place(false);
    __syncthreads();
    if (cb < ncb && ks < half) place(true);
    __syncthreads();
    // the block's sum stands in the first of a column block's places
    for (int idx = tid; idx < ncb * n_tok * 16 && half > 1; idx += kFewThreads) {
      const int q = idx & 15, at_row = idx >> 4, c = at_row / n_tok, row = at_row - c * n_tok;
      float4* at = reinterpret_cast<float4*>(part + (c * half * 16 + row) * kPitch) + q;
      float4 v = *at;
#pragma unroll
      for (int s = 1; s < kFewWarps / 2; ++s) {
        if (s >= half) break;
        const float4 o = at[s * 16 * kPitch / 4];
        v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
      }
      *at = v;
    }
    dec::cluster_arrive();
    dec::cluster_wait();
    gather_t<E, kFewWarps, 16>(p, smem_u32(part), half, r, n_tok, scale, size, rank_in, spread, parts, undo);
    dec::cluster_arrive();                                          // (the others have read this block's sums when the wait at the end is over)
    if (spread) dec::cluster_wait();                                // (all of t is there)
  }
  __syncthreads();

  // ---- y = base + t . B.  Rows of t behind the tile's tokens hold anything; what they give is not stored.
  const int64_t token[2] = {g < n_tok ? tok[g] : 0, 8 + g < n_tok ? tok[8 + g] : 0};
  const float un[2] = {g < n_tok && r > 0 ? undo[g] : 0.f, 8 + g < n_tok && r > 0 ? undo[8 + g] : 0.f};
  for (int c0 = n0 + 64 * warp; c0 < n1; c0 += 64 * kFewWarps) {
    clear();
    for (int ch = 0; ch < chunks; ++ch) {
      cp_wait<kFewStages - 1>();
      __syncwarp();
      uint4 w[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) w[q] = dec::lds_u4(slot() + q * 512 + from);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (32 * ch + 16 * s >= r) break;
        const uint32_t at = parts + g * p.t_pitch + 4 * (32 * ch + 16 * s + 4 * t4);
        const uint4 t0 = dec::lds_u4(at), t1 = dec::lds_u4(at + 8 * p.t_pitch);
        const uint32_t hi[4] = {t0.x, t1.x, t0.y, t1.y}, lo[4] = {t0.z, t1.z, t0.w, t1.w};
        uint32_t b[8][2];
#pragma unroll
        for (int n = 0; n < 8; ++n) {
          b[n][0] = pair_of(w[4 * s], w[4 * s + 1], n); b[n][1] = pair_of(w[4 * s + 2], w[4 * s + 3], n);
          mma<E>(acc[n], hi, b[n][0], b[n][1]);
        }
#pragma unroll
        for (int n = 0; n < 8; ++n) mma<E>(acc[n], lo, b[n][0], b[n][1]);
      }
      done();
    }
    const int at_c[2] = {c0 + 8 * t4, c0 + 32 + 8 * (t4 ^ 1)};
    const bool there[4] = {g < n_tok && at_c[0] < n1, g < n_tok && at_c[1] < n1, 8 + g < n_tok && at_c[0] < n1, 8 + g < n_tok && at_c[1] < n1};
    add_store(p, token, at_c, there, acc, un);
  }
  if (r > 0 && !spread) dec::cluster_wait();
}

// ---- many tokens: a cluster per (adapter, up to 32 of its tokens), four blocks of four warps an SM.  (Tiles of 64 with two blocks an SM read A
// and B half as often, but 418 tokens of rank 128 took 41 us instead of 23, prompts of 2048 67 instead of 40.)
// Dynamic shared memory: the counts; then the warps' rings; then in their place the partial sums [kWarps][TM][kPitch] fp32 (the block's sums take the
// place of the first) and t's parts [TM][t_pitch]; then B's rings in the place of the sums.
constexpr int MT = 2, TM = 16 * MT;
struct Ring {
  static constexpr int kPieces = 8 + 2 * MT;                   // 16 bytes per lane each: eight rows of A, 2 MT rows of x
  static constexpr int kStages = 2;
  static constexpr int kBytes = kWarps * kStages * kPieces * 512;
  static constexpr int kSums = kWarps * TM * kPitch * 4;
  static constexpr int kBStages = 2;                           // of B's ring, eight pieces each
  static_assert(kWarps * kBStages * 8 * 512 <= kSums, "t stands behind them");
};

template <class E>
__global__ void __launch_bounds__(kThreads, 4) k_adapters_many(const AdapterArgs p) {
  using T = typename E::T;
  using R = Ring;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int tok[TM], aux[kWarps + 4];
  __shared__ float undo[TM];
  __shared__ int2 kinds[kThreads];                             // rank and scale of the first adapters
  float* part = reinterpret_cast<float*>(smem);
  const uint32_t parts = smem_u32(smem) + p.t_at;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
  uint32_t rank_in, size;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank_in));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  auto kind = [&](int j) { return kind_of(p, j); };
  if (tid < p.n_adapters) kinds[tid] = kind(tid);              // (in flight together with ids)
  int j = 0;
  const int n_tok = find_tile<TM, kWarps>(p, blockIdx.x / size, j, tok, reinterpret_cast<int*>(smem), aux);
  if (n_tok == 0) return;                                           // (the whole cluster)
  const int2 mine = j >= p.n_adapters ? make_int2(0, 0) : j < kThreads ? kinds[j] : kind(j);
  const int r = min(max(mine.x, 0), p.max_rank);
  const float scale = __int_as_float(mine.y);
  const int n0 = (int)((uint32_t)(p.d_out / 32) * rank_in / size) * 32, n1 = (int)((uint32_t)(p.d_out / 32) * (rank_in + 1) / size) * 32;

  if (r > 0) {
    // ---- t = x . A over this block's share of d_in: a warp takes 64 columns of A and every S-th run of 32 of the reduction axis.  What a lane
    // needs goes through slots of its own in shared memory (the ring is a register file with copies in flight: no lane reads another's).
    const int ncb = (r + 63) / 64, S = kWarps / (ncb <= 1 ? 1 : ncb == 2 ? 2 : 4), cb = warp / S, ks = warp % S;
    const int k0 = (int)((uint32_t)(p.d_in / 32) * rank_in / size), k1 = (int)((uint32_t)(p.d_in / 32) * (rank_in + 1) / size);
    const int trips = cb < ncb && k0 + ks < k1 ? (k1 - k0 - ks + S - 1) / S : 0;
    const int cl = 8 * (lane & 7), ct = lane >> 3;                  // what this lane copies: columns, row of a piece
    const bool col = cb * 64 + cl < r;
    const T* a_next = reinterpret_cast<const T*>(p.a) + ((int64_t)j * p.d_in + (int64_t)(k0 + ks) * 32 + 8 * ct) * p.max_rank + (col ? cb * 64 + cl : 0);
    const T* xr[2 * MT];
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) xr[i] = reinterpret_cast<const T*>(p.x) + tok[8 * i + g < n_tok ? 8 * i + g : 0] * p.x_stride + 8 * t4 + (k0 + ks) * 32;
    const uint32_t ring = smem_u32(smem) + warp * R::kStages * R::kPieces * 512, to = piece_at(lane & 7, lane >> 3), from = piece_at(block_of(g), t4);
    int in = 0;
    auto issue = [&](int stage) {
      if (in < trips) {
        const uint32_t d = ring + stage * R::kPieces * 512;
#pragma unroll
        for (int q = 0; q < 8; ++q) cp16(d + q * 512 + to, a_next + (int64_t)q * p.max_rank, col);
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) cp16(d + (8 + i) * 512 + lane * 16, xr[i] + (int64_t)in * 32 * S, 8 * i + g < n_tok);
        a_next += (int64_t)32 * S * p.max_rank;
        ++in;
      }
      cp_commit();
    };
#pragma unroll
    for (int i = 0; i < R::kStages; ++i) issue(i);
    float acc[MT][8][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int n = 0; n < 8; ++n) acc[i][n][0] = acc[i][n][1] = acc[i][n][2] = acc[i][n][3] = 0.f;
    int stage = 0;
#pragma unroll 1
    for (int it = 0; it < trips; ++it) {
      cp_wait<R::kStages - 1>();
      __syncwarp();
      const uint32_t at = ring + stage * R::kPieces * 512;
      uint4 w[8], xv[2 * MT];
#pragma unroll
      for (int q = 0; q < 8; ++q) w[q] = dec::lds_u4(at + q * 512 + from);
#pragma unroll
      for (int i = 0; i < 2 * MT; ++i) xv[i] = dec::lds_u4(at + (8 + i) * 512 + lane * 16);
#pragma unroll
      for (int s = 0; s < 2; ++s)
#pragma unroll
        for (int n = 0; n < 8; ++n) {
          const uint32_t b0 = pair_of(w[4 * s], w[4 * s + 1], n), b1 = pair_of(w[4 * s + 2], w[4 * s + 3], n);
#pragma unroll
          for (int i = 0; i < MT; ++i) {
            const uint32_t a[4] = {word(xv[2 * i], 2 * s), word(xv[2 * i + 1], 2 * s), word(xv[2 * i], 2 * s + 1), word(xv[2 * i + 1], 2 * s + 1)};
            mma<E>(acc[i][n], a, b0, b1);
          }
        }
      __syncwarp();
      issue(stage);
      stage = stage + 1 == R::kStages ? 0 : stage + 1;
    }
    __syncthreads();                                                // (the sums take the rings' place; trips over, no copy is in flight)
    // The sums of the S warps that share a column block (S / 2 places: one half of them writes, the other adds; alone, it writes).  A lane's
    // columns of row 8 i + g: 8 t4 .. + 7 (from the even half of a fragment) and 32 + 8 (t4 ^ 1) .. + 7 (from the odd).
    const int half = S > 1 ? S / 2 : 1;
    float* dst = part + (cb * half + ks % half) * TM * kPitch;
    auto place = [&](bool add) {
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
              float4* at = reinterpret_cast<float4*>(dst + (16 * i + 8 * h + g) * kPitch + (c ? 32 + 8 * (t4 ^ 1) : 8 * t4) + 4 * q);
              float4 v = make_float4(acc[i][4 * q][2 * h + c], acc[i][4 * q + 1][2 * h + c], acc[i][4 * q + 2][2 * h + c], acc[i][4 * q + 3][2 * h + c]);
              if (add) { const float4 o = *at; v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w; }
              *at = v;
            }
    };
    if (cb < ncb && ks < half) place(false);
    __syncthreads();
    if (cb < ncb && ks >= half) place(true);
    __syncthreads();
    if (half > 1)                                                   // (four warps: two places)
      for (int idx = tid; idx < n_tok * 16; idx += kThreads) {
        float4* at = reinterpret_cast<float4*>(part + (idx >> 4) * kPitch) + (idx & 15);
        float4 v = *at;
        const float4 o = at[TM * kPitch / 4];
        v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
        *at = v;
      }
    dec::cluster_arrive();
    dec::cluster_wait();
    gather_t<E, kWarps, TM>(p, smem_u32(part), half, r, n_tok, scale, size, rank_in, true, parts, undo);
    dec::cluster_arrive();
    dec::cluster_wait();                                            // (all of t is there, and nobody reads this block's sums any more)
  }
  __syncthreads();

  // ---- y = base + t . B over this block's share of d_out: a warp takes 64 columns and all of the rank.  Rows of t behind the tile's tokens hold
  // anything; what they give is not stored.
  const uint32_t ring = smem_u32(smem) + warp * R::kBStages * 8 * 512, to = piece_at(lane & 7, lane >> 3), from = piece_at(block_of(g), t4);
  Columns<T, R::kBStages> cols = {p, reinterpret_cast<const T*>(p.b) + (int64_t)j * p.max_rank * p.d_out + 8 * (lane & 7), tok, n_tok, r, n1, 64 * kWarps, (r + 31) / 32,
                                         base_stages(p), ring, to, lane, g, lane >> 3, 8 * t4, 32 + 8 * (t4 ^ 1), n0 + 64 * warp, 0, 0};
  const int chunks = cols.chunks;
  if (chunks + cols.bases == 0) cols.c0 = n1;
  int stage = 0;
  auto slot = [&]() { return ring + stage * 8 * 512; };
  auto done = [&]() { __syncwarp(); cols.issue(); stage = stage + 1 == R::kBStages ? 0 : stage + 1; };
#pragma unroll 1
  for (int i = 0; i < R::kBStages; ++i) cols.issue();
  for (int c0 = n0 + 64 * warp; c0 < n1; c0 += 64 * kWarps) {
    float acc[MT][8][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int n = 0; n < 8; ++n) acc[i][n][0] = acc[i][n][1] = acc[i][n][2] = acc[i][n][3] = 0.f;
#pragma unroll 1
    for (int ch = 0; ch < chunks; ++ch) {
      cp_wait<R::kBStages - 1>();
      __syncwarp();
      uint4 w[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) w[q] = dec::lds_u4(slot() + q * 512 + from);
#pragma unroll
      for (int s = 0; s < 2; ++s) {
        if (32 * ch + 16 * s >= r) break;
        uint32_t b[8][2];
#pragma unroll
        for (int n = 0; n < 8; ++n) { b[n][0] = pair_of(w[4 * s], w[4 * s + 1], n); b[n][1] = pair_of(w[4 * s + 2], w[4 * s + 3], n); }
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const uint32_t at = parts + (16 * i + g) * p.t_pitch + 4 * (32 * ch + 16 * s + 4 * t4);
          const uint4 t0 = dec::lds_u4(at), t1 = dec::lds_u4(at + 8 * p.t_pitch);
          const uint32_t hi[4] = {t0.x, t1.x, t0.y, t1.y}, lo[4] = {t0.z, t1.z, t0.w, t1.w};
#pragma unroll
          for (int n = 0; n < 8; ++n) mma<E>(acc[i][n], hi, b[n][0], b[n][1]);
#pragma unroll
          for (int n = 0; n < 8; ++n) mma<E>(acc[i][n], lo, b[n][0], b[n][1]);
        }
      }
      done();
    }
    const bool f32 = p.y_dtype == EORA_Y_F32;
#pragma unroll
    for (int i = 0; i < MT; ++i) {
      uint4 base[8] = {};                                           // 16-bit: the first four
      if (cols.bases) {
        if (f32 || i % 2 == 0) cp_wait<R::kBStages - 1>();
#pragma unroll
        for (int q = 0; q < 8; ++q) base[q] = dec::lds_u4(slot() + (f32 ? q : 4 * (i % 2) + (q & 3)) * 512 + lane * 16);
        if (f32 || i % 2 == 1) done();
      }
#pragma unroll
      for (int k = 0; k < 4; ++k) {                                 // half k = 2 h + c of the fragments
        const int row = 16 * i + 8 * (k >> 1) + g, at_c = c0 + ((k & 1) ? cols.at1 : cols.at0);
        if (row >= n_tok || at_c >= n1) continue;
        const float un = r > 0 ? undo[row] : 0.f;
        const int64_t at = tok[row] * p.y_stride + at_c;
        if (f32) {
          put4(p.y, at, acc[i], k, 0, un, base[2 * k]);
          put4(p.y, at + 4, acc[i], k, 1, un, base[2 * k + 1]);
        } else if (p.y_dtype == EORA_Y_F16) {
          put8<F16>(p.y, at, acc[i], k, un, base[k]);
        } else {
          put8<BF16>(p.y, at, acc[i], k, un, base[k]);
        }
      }
    }
  }
}

// Clusters of 1 .. 16 blocks that a B200 holds at once, with one block on an SM and with two (cudaOccupancyMaxActiveClusters: a cluster stays
// within a group of 16 to 20 SMs).  Above rank 192 few tokens have one block on an SM, above rank 128 many have three instead of four (t's parts take
// the shared memory), which the rule below does not count with: clusters then run in two waves where it expects one.
constexpr int kFit1[17] = {0, 148, 74, 45, 33, 26, 22, 15, 15, 15, 11, 7, 7, 7, 7, 7, 7};
constexpr int kFit2[17] = {0, 296, 148, 93, 71, 56, 45, 37, 33, 30, 26, 21, 21, 17, 14, 14, 14};

template <class K>
cudaError_t launch(K kernel, int* set_up, AdapterArgs& a, int tiles, int cluster, int threads, size_t smem, cudaStream_t st) {
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  if (device >= 16 || !set_up[device]) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 * 1024);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    if (device < 16) set_up[device] = 1;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * cluster));
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, a);
}

template <class E>
cudaError_t launch(AdapterArgs& a, cudaStream_t st) {
  // as many tiles as there can be: one that is not full for each adapter that can occur, and full ones
  const bool few = a.m <= 256;
  const int tm = few ? 16 : TM, kinds = a.m < a.n_adapters + 1 ? a.m : a.n_adapters + 1, tiles = kinds + (a.m - kinds) / tm;
  // The cluster as large as lets all tiles run at once.  How many there will be is not known here: few tokens: as with as many tokens of each
  // adapter; many: half way from that to the most (a guess that only speed goes by).
  const int even = kinds * ((a.m + tm * kinds - 1) / (tm * kinds)), likely = few ? even : (even + tiles) / 2;
  const bool alone = few && likely <= 7;     // (every block an SM to itself, where the largest clusters still fit: 64 tokens of two adapters 8.5 -> 7.8 us)
  int cluster = 16;
  while (cluster > 1 && (alone ? kFit1 : kFit2)[cluster] * (few ? 1 : 2) < likely) --cluster;
  a.t_pitch = 4 * ((a.max_rank + 15) & ~15) + 64;         // (rows an odd number of four 16-byte units apart: no bank conflicts)
  if (a.t_pitch % 128 == 0) a.t_pitch += 64;
  const size_t t_bytes = (size_t)tm * a.t_pitch;
  static int set_up[3][16] = {};                 // per device; benign if two threads do it at once
  if (few) {
    const size_t smem = std::max<size_t>(kFewRing + kFewSums + t_bytes, alone ? 120 * 1024 : 0);
    return a.m <= 64 ? launch(k_adapters_few<E, true>, set_up[0], a, tiles, cluster, kFewThreads, smem, st)
                     : launch(k_adapters_few<E, false>, set_up[2], a, tiles, cluster, kFewThreads, smem, st);
  }
  a.t_at = Ring::kSums;
  const size_t after = (size_t)a.t_at + t_bytes;
  return launch(k_adapters_many<E>, set_up[1], a, tiles, cluster, kThreads, after > (size_t)Ring::kBytes ? after : (size_t)Ring::kBytes, st);
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
  a.skip_none = base == y;
  const cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  // more tokens than a launch takes: equal parts, one after the other
  const int parts = (m + kStaged - 1) / kStaged, step = (m + parts - 1) / parts;
  const int yb = c.y_dtype == EORA_Y_F32 ? 4 : 2;
  for (int i = 0; i < m; i += step) {
    AdapterArgs part = a;
    part.m = m - i < step ? m - i : step;
    part.x = static_cast<const char*>(x) + i * x_stride * 2;
    part.y = static_cast<char*>(y) + i * y_stride * yb;
    if (base) part.base = static_cast<const char*>(base) + i * base_stride * yb;
    part.ids = ids + i;
    const cudaError_t e = c.x_dtype == EORA_X_F16 ? launch<F16>(part, st) : launch<BF16>(part, st);
    if (e != cudaSuccess) return EORA_ERR_CUDA;
  }
  return EORA_OK;
}
