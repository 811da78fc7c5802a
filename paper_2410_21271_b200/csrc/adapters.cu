// Low-rank adapters of many requests beside a shared projection (eora_serve.h):
//   y[i] = base[i] + s_j (x[i] . A_j) . B_j,  j = ids[i].
//
// What bounds it: few tokens: the bytes of the adapters that are named (r (d_in + d_out) 16-bit values each) and the latency of
// two products of which the second needs all of the first; prompts: the bytes of x, base and y, while an adapter's A and B, read
// once per tile of tokens, come from L2.
//  - A thread block cluster per (adapter, up to 16 MT of its tokens): its blocks share d_in in the first product and d_out in the
//    second, and exchange t = x . A (16 MT x r) through distributed shared memory.  So one launch does both products, t never
//    leaves the chip, nothing is kept between calls, and the sums have a fixed order.
//  - Which tokens a cluster has, every block works out for itself from ids (counts per adapter, then the tile's tokens in order).
//  - Weights go from global memory to the matrix instruction's registers without shared memory in between: the order in which the
//    reduction axis is taken is free, so a lane takes rows 8t .. 8t + 7 (t = lane % 4) of 32 and of each 8 consecutive columns
//    (16 bytes; 8 lanes read 128 consecutive bytes of a row), and pairs of rows are interleaved with a byte permute.  Column n of
//    the instruction is then column 8n + i of the matrix, and a lane ends with 16 consecutive columns of its rows.  Every byte of
//    A, B, x, base and y is loaded by one warp of one block only.
#include "serve_common.cuh"

namespace eora {
namespace serve {
namespace {

constexpr int kMaxRank = 256, kMaxAdapters = 4096, kMaxTokens = 1 << 20;
constexpr int kWarps = 4, kThreads = 32 * kWarps;
constexpr int kAhead = 1024;                    // 128-byte lines of B and of base that a block has brought to L2 ahead of their use
constexpr int kPitch = 68;                      // floats of a row of 64 partial sums in shared memory

struct AdapterArgs {
  const void *x, *a, *b, *base;
  void* y;
  const int32_t *ids, *ranks;
  const float* scales;
  int64_t x_stride, base_stride, y_stride;
  int m, d_in, d_out, max_rank, n_adapters, y_dtype;
  int skip_none;                                // rows without an adapter are in place already
  int t_at, t_pitch;                            // t's parts in shared memory: byte offset, 16-bit elements of a row
};

__device__ __forceinline__ float4 ld_cluster4(uint32_t addr) {
  float4 v;
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(addr) : "memory");
  return v;
}
__device__ __forceinline__ uint4 ld_u4(const void* p) { return __ldg(reinterpret_cast<const uint4*>(p)); }
__device__ __forceinline__ uint32_t word(const uint4& v, int i) { return i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w; }

// Eight columns of two rows, as eight pairs (row 0, row 1).
__device__ __forceinline__ uint32_t pair_of(const uint4& r0, const uint4& r1, int i) {
  return __byte_perm(word(r0, i >> 1), word(r1, i >> 1), (i & 1) ? 0x7632 : 0x5410);
}

// The tile of cluster `c`: its adapter (n_adapters: none) and, in tok, its tokens in order of their place in ids.  Returns how many,
// 0 if there is no such tile.  counts: n_adapters + 1 ints, aux: kWarps + 4 ints.
template <int TM>
__device__ __forceinline__ int find_tile(const AdapterArgs& p, int c, int& adapter, int* tok, int* counts, int* aux) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, n = p.n_adapters;
  auto key_of = [&](int i) {
    const int j = p.ids[i];
    return j >= 0 && j < n ? j : n;
  };
  if (p.m <= 32) {                              // one warp's lanes hold all ids: no counting (every warp for itself, writing the same)
    const int key = lane < p.m ? key_of(lane) : n + 1 + lane;
    const unsigned same = __match_any_sync(0xffffffffu, key);
    const int rank = __popc(same & ((1u << lane) - 1));
    const bool leads = lane < p.m && rank % TM == 0 && !(key == n && p.skip_none);
    const unsigned leaders = __ballot_sync(0xffffffffu, leads);
    if (c >= __popc(leaders)) return 0;
    const int leader = __fns(leaders, 0, c + 1);
    adapter = __shfl_sync(0xffffffffu, key, leader);
    const int first = __shfl_sync(0xffffffffu, rank, leader);
    const unsigned mine = __shfl_sync(0xffffffffu, same, leader);
    if (((mine >> lane) & 1) && rank >= first && rank < first + TM && warp == 0) tok[rank - first] = lane;
    __syncthreads();
    return min(TM, __popc(mine) - first);
  }
  for (int i = tid; i <= n; i += kThreads) counts[i] = 0;
  __syncthreads();
  for (int i = tid; i < p.m; i += kThreads) atomicAdd(&counts[key_of(i)], 1);
  __syncthreads();
  if (warp == 0) {                              // which adapter owns tile c: a lane adds up a run of adapters, the warp the lanes
    const int per = (n + 32) / 32, lo = lane * per, hi = min(lo + per, n + 1);
    auto tiles = [&](int j) { return j == n && p.skip_none ? 0 : (counts[j] + TM - 1) / TM; };
    int sum = 0;
    for (int j = lo; j < hi; ++j) sum += tiles(j);
    int upto = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int v = __shfl_up_sync(0xffffffffu, upto, o);
      if (lane >= o) upto += v;
    }
    if (lane == 31) aux[kWarps] = upto;         // all tiles
    if (c >= upto - sum && c < upto) {
      int left = c - (upto - sum), j = lo;
      while (left >= tiles(j)) left -= tiles(j++);
      aux[kWarps + 1] = j;
      aux[kWarps + 2] = left;
    }
  }
  __syncthreads();
  if (c >= aux[kWarps]) return 0;
  adapter = aux[kWarps + 1];
  const int first = aux[kWarps + 2] * TM;
  // the tokens: a warp looks through its eighth of ids, first counting, then placing
  const int lo = (int)((int64_t)p.m * warp / kWarps), hi = (int)((int64_t)p.m * (warp + 1) / kWarps);
  int found = 0;
  for (int i = lo; i < hi; i += 32) found += __popc(__ballot_sync(0xffffffffu, i + lane < hi && key_of(i + lane) == adapter));
  if (lane == 0) aux[warp] = found;
  __syncthreads();
  int rank = 0;
  for (int w = 0; w < warp; ++w) rank += aux[w];
  if (rank < first + TM && rank + found > first) {
    for (int i = lo; i < hi && rank < first + TM; i += 32) {
      const bool is = i + lane < hi && key_of(i + lane) == adapter;
      const unsigned b = __ballot_sync(0xffffffffu, is);
      const int at = rank + __popc(b & ((1u << lane) - 1)) - first;
      if (is && at >= 0 && at < TM) tok[at] = i + lane;
      rank += __popc(b);
    }
  }
  const int n_tok = min(TM, counts[adapter] - first);
  __syncthreads();
  return n_tok;
}

// y's and base's rows of a lane: 16 t4 + 8 c .. + 7 of row 8 h + g of MB row groups of 16, all loads before the first store (y may be base).
template <class E, int MB>
__device__ __forceinline__ void add_store(const AdapterArgs& p, const int64_t (&base_at)[MB][2], const int64_t (&y_at)[MB][2], const bool (&row)[MB][2], const bool (&col)[2],
                                          const float (&acc)[MB][8][4], const float (&undo)[MB][2]) {
  if (p.y_dtype == EORA_Y_F32) {
    float4 b[MB][2][2][2];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int q = 0; q < 2; ++q)
            b[i][h][c][q] = p.base && row[i][h] && col[c] ? *reinterpret_cast<const float4*>(reinterpret_cast<const float*>(p.base) + base_at[i][h] + 8 * c + 4 * q)
                                                          : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h)
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
          for (int q = 0; q < 2; ++q) {
            const float4 v = b[i][h][c][q];
            const int k = 2 * h + c;
            if (row[i][h] && col[c])
              *reinterpret_cast<float4*>(reinterpret_cast<float*>(p.y) + y_at[i][h] + 8 * c + 4 * q) =
                  make_float4(fmaf(acc[i][4 * q][k], undo[i][h], v.x), fmaf(acc[i][4 * q + 1][k], undo[i][h], v.y), fmaf(acc[i][4 * q + 2][k], undo[i][h], v.z),
                              fmaf(acc[i][4 * q + 3][k], undo[i][h], v.w));
          }
    return;
  }
  uint4 b[MB][2][2];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < 2; ++c)
        b[i][h][c] = p.base && row[i][h] && col[c] ? *reinterpret_cast<const uint4*>(reinterpret_cast<const uint16_t*>(p.base) + base_at[i][h] + 8 * c) : make_uint4(0, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int c = 0; c < 2; ++c) {
        const int k = 2 * h + c;
        uint32_t o[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float2 v = E::unpack(word(b[i][h][c], q));
          o[q] = E::pack(fmaf(acc[i][2 * q][k], undo[i][h], v.x), fmaf(acc[i][2 * q + 1][k], undo[i][h], v.y));
        }
        if (row[i][h] && col[c]) *reinterpret_cast<uint4*>(reinterpret_cast<uint16_t*>(p.y) + y_at[i][h] + 8 * c) = make_uint4(o[0], o[1], o[2], o[3]);
      }
}

// MT: tokens of a tile / 16.  Dynamic shared memory: the counts; then the warps' rings; then in their place the partial sums
// [kWarps][16 MT][kPitch] fp32 (the block's sums take the place of the first) and t's high and low parts [2][16 MT][t_pitch].
template <int MT> struct Ring {
  static constexpr int kPieces = 8 + 2 * MT;                   // 16 bytes per lane each: eight rows of A, 2 MT rows of x
  static constexpr int kStages = 3;
  static constexpr int kBytes = kWarps * kStages * kPieces * 512;
  static constexpr int kSums = kWarps * 16 * MT * kPitch * 4;
};

template <class E, int MT>
__global__ void __launch_bounds__(kThreads, MT == 1 ? 3 : 2) k_adapters(const AdapterArgs p) {
  constexpr int TM = 16 * MT;
  using T = typename E::T;
  using R = Ring<MT>;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int tok[TM], aux[kWarps + 4];
  __shared__ float undo[TM];
  __shared__ int2 kinds[kThreads];                             // rank and scale of the first adapters
  float* part = reinterpret_cast<float*>(smem);
  T* t_hi = reinterpret_cast<T*>(smem + p.t_at);
  T* t_lo = t_hi + TM * p.t_pitch;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
  uint32_t rank_in, size;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(rank_in));
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(size));
  asm volatile("griddepcontrol.launch_dependents;");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  auto kind = [&](int j) { return make_int2(p.ranks ? __ldg(p.ranks + j) : p.max_rank, __float_as_int(p.scales ? __ldg(p.scales + j) : 1.f)); };
  if (tid < p.n_adapters) kinds[tid] = kind(tid);              // (in flight together with ids)
  int j = 0;
  const int n_tok = find_tile<TM>(p, blockIdx.x / size, j, tok, reinterpret_cast<int*>(smem), aux);
  if (n_tok == 0) return;                                           // (the whole cluster)
  const int2 mine = j >= p.n_adapters ? make_int2(0, 0) : j < kThreads ? kinds[j] : kind(j);
  const int r = min(max(mine.x, 0), p.max_rank);
  const float scale = __int_as_float(mine.y);
  const int n0 = (int)((int64_t)(p.d_out / 32) * rank_in / size) * 32, n1 = (int)((int64_t)(p.d_out / 32) * (rank_in + 1) / size) * 32;
  const T* bj = reinterpret_cast<const T*>(p.b) + (int64_t)j * p.max_rank * p.d_out;

  // B's and base's share on their way into L2 while t is computed (128 bytes each; as much as L2 holds for all blocks)
  auto ahead = [&]() {
    const int lines = ((n1 - n0) * 2 + 127) / 128;
    for (int i = tid; i < min(r * lines, kAhead); i += kThreads) {
      const int row = i / lines, l = i - row * lines;
      asm volatile("prefetch.global.L2 [%0];" ::"l"(bj + (int64_t)row * p.d_out + min(n0 + 64 * l, n1 - 1)));
    }
    if (!p.base) return;
    const int yb = p.y_dtype == EORA_Y_F32 ? 4 : 2, bl = ((n1 - n0) * yb + 127) / 128;
    for (int i = tid; i < min(n_tok * bl, kAhead); i += kThreads) {
      const int row = i / bl, l = i - row * bl;
      asm volatile("prefetch.global.L2 [%0];" ::"l"(reinterpret_cast<const char*>(p.base) + (tok[row] * p.base_stride + min(n0 + 128 / yb * l, n1 - 1)) * yb));
    }
  };

  if (r > 0) {
    // ---- t = x . A over this block's share of d_in: a warp takes 64 columns of A and every S-th run of 32 of the reduction axis.  What a lane
    // needs goes through slots of its own in shared memory (the ring is a register file with copies in flight: no lane reads another's).
    const int ncb = (r + 63) / 64, S = kWarps / (ncb <= 1 ? 1 : ncb == 2 ? 2 : 4), cb = warp / S, ks = warp % S;
    const int k0 = (int)((int64_t)(p.d_in / 32) * rank_in / size), k1 = (int)((int64_t)(p.d_in / 32) * (rank_in + 1) / size);
    const int trips = cb < ncb && k0 + ks < k1 ? (k1 - k0 - ks + S - 1) / S : 0;
    const bool col = cb * 64 + 8 * g < r;
    const T* a_next = reinterpret_cast<const T*>(p.a) + ((int64_t)j * p.d_in + (int64_t)(k0 + ks) * 32 + 8 * t4) * p.max_rank + (col ? cb * 64 + 8 * g : 0);
    const T* xr[2 * MT];
#pragma unroll
    for (int i = 0; i < 2 * MT; ++i) xr[i] = reinterpret_cast<const T*>(p.x) + tok[8 * i + g < n_tok ? 8 * i + g : 0] * p.x_stride + 8 * t4 + (k0 + ks) * 32;
    const uint32_t ring = smem_u32(smem) + warp * R::kStages * R::kPieces * 512 + lane * 16;
    int in = 0;
    auto issue = [&](int stage) {
      if (in < trips) {
        const uint32_t d = ring + stage * R::kPieces * 512;
#pragma unroll
        for (int q = 0; q < 8; ++q) cp16(d + q * 512, a_next + (int64_t)q * p.max_rank, col);
#pragma unroll
        for (int i = 0; i < 2 * MT; ++i) cp16(d + (8 + i) * 512, xr[i] + (int64_t)in * 32 * S, 8 * i + g < n_tok);
        a_next += (int64_t)32 * S * p.max_rank;
        ++in;
      }
      cp_commit();
    };
#pragma unroll
    for (int i = 0; i < R::kStages; ++i) issue(i);
    ahead();
    float acc[MT][8][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int n = 0; n < 8; ++n) acc[i][n][0] = acc[i][n][1] = acc[i][n][2] = acc[i][n][3] = 0.f;
    int stage = 0;
#pragma unroll 1
    for (int it = 0; it < trips; ++it) {
      cp_wait<R::kStages - 1>();
      const uint32_t at = ring + stage * R::kPieces * 512;
      uint4 w[8], xv[2 * MT];
#pragma unroll
      for (int q = 0; q < 8; ++q) w[q] = dec::lds_u4(at + q * 512);
#pragma unroll
      for (int i = 0; i < 2 * MT; ++i) xv[i] = dec::lds_u4(at + (8 + i) * 512);
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
      issue(stage);
      stage = stage + 1 == R::kStages ? 0 : stage + 1;
    }
    __syncthreads();                                                // (the sums take the rings' place; trips over, no copy is in flight)
    // a lane's columns of row 8 i + g: 16 t4 .. 16 t4 + 15 (n of the even half of a fragment, then of the odd)
    if (cb < ncb) {
      float* mine = part + warp * TM * kPitch;
#pragma unroll
      for (int i = 0; i < MT; ++i)
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int q = 0; q < 2; ++q)
              *reinterpret_cast<float4*>(mine + (16 * i + 8 * h + g) * kPitch + 16 * t4 + 8 * c + 4 * q) =
                  make_float4(acc[i][4 * q][2 * h + c], acc[i][4 * q + 1][2 * h + c], acc[i][4 * q + 2][2 * h + c], acc[i][4 * q + 3][2 * h + c]);
    }
    __syncthreads();
    // the block's sum stands where the first of the warps that share a column block has its own
    for (int idx = tid; idx < ncb * n_tok * 16 && S > 1; idx += kThreads) {
      const int q = idx % 16, row = idx / 16 % n_tok, c = idx / 16 / n_tok;
      float4* at = reinterpret_cast<float4*>(part + (c * S * TM + row) * kPitch) + q;
      float4 v = *at;
#pragma unroll
      for (int s = 1; s < kWarps; ++s) {
        if (s >= S) break;
        const float4 o = at[s * TM * kPitch / 4];
        v.x += o.x; v.y += o.y; v.z += o.z; v.w += o.w;
      }
      *at = v;
    }
    dec::cluster_arrive();
    dec::cluster_wait();
    // ---- every block adds up the blocks' sums, a row per 16 lanes (32 where the rank is above 64), four columns per lane.  A token's values
    // share a power of two that brings the largest to [2^9, 2^10): fp16 has room on both sides there.  High part and low part each rounded to
    // nearest: 2^-22 (fp16), 2^-16 (bf16) of a value is left.
    const uint32_t part_at = smem_u32(part);
    const int r16 = (r + 15) & ~15, lanes = r <= 64 ? 16 : 32, sub = lane & (lanes - 1), rows = 32 / lanes;
    for (int row0 = warp * rows; row0 < n_tok; row0 += kWarps * rows) {
      const int row = row0 + (lanes == 16 ? lane >> 4 : 0);
      float v[2][4];
      float top = 0.f;
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int c = 4 * sub + 128 * q;
        v[q][0] = v[q][1] = v[q][2] = v[q][3] = 0.f;
        if (c < r && row < n_tok) {
          const uint32_t at = part_at + ((c / 64 * S * TM + row) * kPitch + c % 64) * 4;
          for (uint32_t s0 = 0; s0 < size; s0 += 8) {
            float4 o[8];
#pragma unroll
            for (uint32_t s = 0; s < 8; ++s) o[s] = s0 + s < size ? ld_cluster4(dec::mapa(at, s0 + s)) : make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
            for (uint32_t s = 0; s < 8; ++s) { v[q][0] += o[s].x; v[q][1] += o[s].y; v[q][2] += o[s].z; v[q][3] += o[s].w; }
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            v[q][e] = c + e < r ? v[q][e] * scale : 0.f;            // (columns behind the rank hold anything)
            top = fmaxf(top, fabsf(v[q][e]));
          }
        }
      }
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        if (o < lanes) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
      const int e = (int)(__float_as_uint(top) >> 23);              // biased exponent
      const int lift = top == 0.f || e == 255 ? 0 : min(9 + 127 - e, 126);
      const float up = __uint_as_float((uint32_t)(127 + lift) << 23);
      if (sub == 0 && row < n_tok) undo[row] = __uint_as_float((uint32_t)(127 - lift) << 23);
#pragma unroll
      for (int q = 0; q < 2; ++q) {
        const int c = 4 * sub + 128 * q;
        if (c < r16 && row < n_tok) {
          float f[4], rest[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) f[i] = v[q][i] * up;
          const uint2 hi = make_uint2(E::pack(f[0], f[1]), E::pack(f[2], f[3]));
          const float2 h0 = E::unpack(hi.x), h1 = E::unpack(hi.y);
          rest[0] = f[0] - h0.x; rest[1] = f[1] - h0.y; rest[2] = f[2] - h1.x; rest[3] = f[3] - h1.y;
          *reinterpret_cast<uint2*>(t_hi + row * p.t_pitch + c) = hi;
          *reinterpret_cast<uint2*>(t_lo + row * p.t_pitch + c) = make_uint2(E::pack(rest[0], rest[1]), E::pack(rest[2], rest[3]));
        }
      }
    }
    dec::cluster_arrive();                                          // (the others have read this block's sums when the wait at the end is over)
  }
  __syncthreads();

  // ---- y = base + t . B over this block's share of d_out: a warp takes 64 columns and all of the rank.  Rows of t behind the tile's tokens hold
  // anything; what they give is not stored.
  const int steps = (r + 15) / 16;
  for (int c0 = n0 + 64 * warp; c0 < n1; c0 += 64 * kWarps) {
    float acc[MT][8][4];
#pragma unroll
    for (int i = 0; i < MT; ++i)
#pragma unroll
      for (int n = 0; n < 8; ++n) acc[i][n][0] = acc[i][n][1] = acc[i][n][2] = acc[i][n][3] = 0.f;
    const bool in_n = c0 + 8 * g < n1;
    constexpr int CH = MT == 1 ? 4 : 2;                             // steps whose loads are in flight together
    for (int s0 = 0; s0 < steps; s0 += CH) {
      uint4 w[CH][4];
#pragma unroll
      for (int s = 0; s < CH; ++s)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int c = 16 * (s0 + s) + 4 * t4 + q;
          w[s][q] = in_n && c < r ? ld_u4(bj + (int64_t)c * p.d_out + c0 + 8 * g) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
      for (int s = 0; s < CH; ++s) {
        if (s0 + s >= steps) break;
#pragma unroll
        for (int i = 0; i < MT; ++i) {
          const int at = (16 * i + g) * p.t_pitch + 16 * (s0 + s) + 4 * t4;
          const uint2 h0 = *reinterpret_cast<const uint2*>(t_hi + at), h1 = *reinterpret_cast<const uint2*>(t_hi + at + 8 * p.t_pitch);
          const uint2 l0 = *reinterpret_cast<const uint2*>(t_lo + at), l1 = *reinterpret_cast<const uint2*>(t_lo + at + 8 * p.t_pitch);
          const uint32_t hi[4] = {h0.x, h1.x, h0.y, h1.y}, lo[4] = {l0.x, l1.x, l0.y, l1.y};
#pragma unroll
          for (int n = 0; n < 8; ++n) {
            const uint32_t b0 = pair_of(w[s][0], w[s][1], n), b1 = pair_of(w[s][2], w[s][3], n);
            mma<E>(acc[i][n], hi, b0, b1);
            mma<E>(acc[i][n], lo, b0, b1);
          }
        }
      }
    }
    const bool col[2] = {c0 + 16 * t4 < n1, c0 + 16 * t4 + 8 < n1};
    constexpr int MB = MT == 1 ? 1 : 2;
#pragma unroll
    for (int i0 = 0; i0 < MT; i0 += MB) {
      int64_t base_at[MB][2], y_at[MB][2];
      bool row[MB][2];
      float un[MB][2], part_acc[MB][8][4];
#pragma unroll
      for (int i = 0; i < MB; ++i) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int at = 16 * (i0 + i) + 8 * h + g;
          row[i][h] = at < n_tok;
          const int64_t token = row[i][h] ? tok[at] : 0;
          un[i][h] = row[i][h] && r > 0 ? undo[at] : 0.f;
          base_at[i][h] = token * p.base_stride + c0 + 16 * t4;
          y_at[i][h] = token * p.y_stride + c0 + 16 * t4;
        }
#pragma unroll
        for (int n = 0; n < 8; ++n)
#pragma unroll
          for (int k = 0; k < 4; ++k) part_acc[i][n][k] = acc[i0 + i][n][k];
      }
      if (p.y_dtype == EORA_Y_BF16) add_store<BF16, MB>(p, base_at, y_at, row, col, part_acc, un);
      else add_store<F16, MB>(p, base_at, y_at, row, col, part_acc, un);
    }
  }
  if (r > 0) dec::cluster_wait();
}

template <class E, int MT>
cudaError_t launch(AdapterArgs& a, cudaStream_t st) {
  constexpr int TM = 16 * MT;
  // as many tiles as there can be: one that is not full for each adapter that can occur, and full ones
  const int kinds = a.m < a.n_adapters + 1 ? a.m : a.n_adapters + 1;
  const int tiles = kinds + (a.m - kinds) / TM;
  const int want = (MT == 1 ? 3 : 2) * 148 / tiles;
  const int cluster = want >= 16 ? 16 : want >= 8 ? 8 : want >= 1 ? want : 1;
  a.t_pitch = ((a.max_rank + 15) & ~15) + 8;
  static_assert(Ring<MT>::kSums >= (kMaxAdapters + 1) * 4 || Ring<MT>::kBytes >= (kMaxAdapters + 1) * 4, "room for the counts");
  a.t_at = Ring<MT>::kSums;
  const size_t after = (size_t)a.t_at + (size_t)2 * TM * a.t_pitch * 2;
  const size_t smem = after > (size_t)Ring<MT>::kBytes ? after : (size_t)Ring<MT>::kBytes;
  static int set_up[16] = {};                    // per device; benign if two threads do it at once
  int device = 0;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  if (device >= 16 || !set_up[device]) {
    e = cudaFuncSetAttribute(k_adapters<E, MT>, cudaFuncAttributeMaxDynamicSharedMemorySize, 224 * 1024);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_adapters<E, MT>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    if (device < 16) set_up[device] = 1;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * cluster));
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cluster; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, k_adapters<E, MT>, a);
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
  const bool f16 = c.x_dtype == EORA_X_F16;
  const cudaError_t e = m <= 64 ? (f16 ? launch<F16, 1>(a, st) : launch<BF16, 1>(a, st)) : (f16 ? launch<F16, 4>(a, st) : launch<BF16, 4>(a, st));
  return e == cudaSuccess ? EORA_OK : EORA_ERR_CUDA;
}
