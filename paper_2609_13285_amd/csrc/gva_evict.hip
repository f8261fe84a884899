// libgva.so -- the attention weight that cached rows have drawn, and eviction
// of rows by it.
//
// A row's weight is the sum, over the queries that saw it and over the heads,
// of its softmax weight exp(x - lse), x the scaled score that the attention
// calls use.  The streams of a sequence share one positional key per row and one
// length, so rows are kept or evicted for all of its heads together.

#include "gva_common.h"
#include "gva_q4.h"

namespace {

// ========================================================= accumulate
struct WeightParams {
  const void* v;
  const uint8_t* scales;
  const void* kr;
  const float* q_abs;     // [B][N][H][d_v], fp32
  const float* q_rot;
  const float* lse;       // [B][N][H]
  const int32_t* lens;
  const float* weights;   // may be NULL with decay 0
  float* new_weights;
  float* part;            // [G][B][T]: row sums of a group, before they are joined
  int32_t B, H, G, N, d_v, d_r, t_max, chunk;
  float scale_log2, decay;
};

constexpr int kWeightWaves = 8;
constexpr int kWeightChunk = 512;              // most rows of a workgroup

// The cached rows as matrix-core operands: 32 rows, K-chunk c of the products.
template <int DV, int NRC, bool Q4>
struct WeightRows {
  u32x4 v[Q4 ? DV / 64 : DV / 16];             // [half][chunk], or codes
  unsigned s;
  bf16x8 k[2][NRC > 0 ? NRC : 1];
};

template <int DV, int NRC, bool Q4>
struct WeightStream {
  static constexpr int NC = DV / 32, NS = DV / kScaleCols;
  __amdgpu_buffer_rsrc_t vres, sres, kres;
  int k_lane[NRC > 0 ? NRC : 1];
  int lane, n, qd, d_r;

  // rows [0, r1) of stream (b, g); loads past their last tile read zeros
  __device__ __forceinline__ WeightStream(const WeightParams& p, int b, int g, int r1, int lane_)
      : lane(lane_), n(lane_ & 15), qd(lane_ >> 4), d_r(p.d_r) {
    const int64_t stream = (int64_t)b * p.G + g;
    const int r1k = (r1 + 15) / 16 * 16, r1c = (r1 + 31) / 32 * 32;
    const uint8_t* v = static_cast<const uint8_t*>(p.v) + stream * p.t_max * (Q4 ? DV / 2 : DV * 2);
    const uint8_t* sc = Q4 ? p.scales + stream * p.t_max * NS : v;
    const uint16_t* k = static_cast<const uint16_t*>(p.kr) + (int64_t)b * p.t_max * p.d_r;
    vres = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(v), (short)0, Q4 ? r1c * (DV / 2) : r1k * DV * 2, kBufferWord3);
    sres = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(sc), (short)0, Q4 ? r1c * NS : 0, kBufferWord3);
    kres = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint16_t*>(k), (short)0, r1k * p.d_r * 2, kBufferWord3);
#pragma unroll
    for (int rc = 0; rc < NRC; ++rc) k_lane[rc] = min(4 * rc + qd, p.d_r / 8 - 1) * 256 + n * 16;
  }
  template <int AUX>
  __device__ __forceinline__ void load(WeightRows<DV, NRC, Q4>& t, int row0) const {
    if constexpr (Q4) {
#pragma unroll
      for (int u = 0; u < DV / 64; ++u)
        t.v[u] = __builtin_amdgcn_raw_buffer_load_b128(vres, lane * 16 + u * kBlockBytes, row0 * (DV / 2), AUX);
      t.s = __builtin_amdgcn_raw_buffer_load_b16(sres, (qd * NS / 4 * 16 + n) * 2, row0 * NS, AUX);
    } else {
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int c = 0; c < NC; ++c)
          t.v[hf * NC + c] = __builtin_amdgcn_raw_buffer_load_b128(vres, qd * 256 + n * 16 + 1024 * c, (row0 + 16 * hf) * DV * 2, AUX);
    }
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int rc = 0; rc < NRC; ++rc)
        t.k[hf][rc] = as_bf16x8(__builtin_amdgcn_raw_buffer_load_b128(kres, k_lane[rc], (row0 + 16 * hf) * d_r * 2, 0));
  }
  __device__ __forceinline__ static bf16x8 chunk(const WeightRows<DV, NRC, Q4>& t, int hf, int c) {
    if constexpr (Q4)
      return dequant8(t.v[DV == 128 ? hf : 0][DV == 128 ? c : 2 * hf + c], hf ? t.s >> 8 : t.s & 255u);
    else
      return as_bf16x8(t.v[hf * NC + c]);
  }
  // The absorbed query at qa and the rotated one at qr in the columns of the
  // lane: requested (request), then scaled and split as chunk c (NC on: the
  // positional ones).
  struct Query {
    f32x4 x[NC + NRC][2];
  };
  __device__ __forceinline__ void request(Query& q, const float* qa, const float* qr) const {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const f32x4* src = reinterpret_cast<const f32x4*>(qa + (Q4 ? qd * (DV / 4) + 8 * c : 32 * c + 8 * qd));
      q.x[c][0] = src[0];
      q.x[c][1] = src[1];
    }
#pragma unroll
    for (int rc = 0; rc < NRC; ++rc) {
      const f32x4* src = reinterpret_cast<const f32x4*>(qr + min(32 * rc + 8 * qd, d_r - 8));
      q.x[NC + rc][0] = src[0];
      q.x[NC + rc][1] = src[1];
    }
  }
  __device__ __forceinline__ bf16x8 part(const Query& q, int c, float scale, bool lo) const {
    const bool in = c < NC || 32 * (c - NC) + 8 * qd < d_r;
    float x[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = in ? q.x[c][j >> 2][j & 3] * scale : 0.f;
    return split_hi_lo(x, lo);
  }
};

// What the score products start from, -log2(e) lse.  -inf, whose weights are 0, for a
// query with nothing to see: lse is -inf, or so low that rows hidden by a large finite
// value are all there is.  Scores are as large then, and x - lse would be their
// rounding (past 2^20 over 2^-4, at a type's lowest value anything: weights of 1e27
// and infinity, which no later one outweighs).  A NaN stays.
constexpr float kNothingSeen = -1048576.f;
__device__ __forceinline__ float weight_start(float lse) { return lse < kNothingSeen ? -INFINITY : -lse * (float)kLog2e; }

// One query per sequence (a decode step).  The workgroup takes `chunk` rows of
// one sequence; wave w scores group w % GP of a round of GP = min(G, 8) groups (a
// power of two), every (8 / GP)-th tile of the chunk.  A head has two columns of
// the products, its query's bf16 high and low parts; the high column's lanes add
// the pair for the tile's first 16 rows and the low column's for the others, so
// that every exponential is taken once.  A wave's sums over the heads go to its
// group's array of row sums, which are added in order at the end: the result
// does not depend on timing.  The log-sum-exp is the products' initial value.  With
// the query in two parts a sum over 32 heads is off by 3e-8 of its size (an
// evaluation in fp32: 4e-8), over two by up to 2.2e-6; three parts cost 3%.
// Bound by HBM: B32 T8K H32 G8 d 128/16 in 4 bits (154 MB) 28.2 us, 5.5 TB/s, and
// 4.6 before it for the absorbed queries.
template <int HPG, int DV, int NRC, bool Q4>
__global__ void __launch_bounds__(64 * kWeightWaves, Q4 || DV == 64 ? 4 : 2) weights_step_kernel(WeightParams p) {
  using Stream = WeightStream<DV, NRC, Q4>;
  constexpr int NC = Stream::NC, DEPTH = NRC == 2 ? 2 : 3;
  __shared__ __attribute__((aligned(16))) float sums[kWeightWaves][kWeightChunk];
  const int nchunks = (p.t_max + p.chunk - 1) / p.chunk;
  const int item = xcd_remap(blockIdx.x, p.B * nchunks);
  const int b = item / nchunks, r0 = item % nchunks * p.chunk;
  const int L = clamp_len(p.lens, b, p.t_max);
  if (r0 >= L) return;
  const int r1 = min(r0 + p.chunk, L);
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, qd = lane >> 4;
  const bool active = n < 2 * HPG, is_lo = n >= HPG;
  const int head = !active ? 0 : (is_lo ? 2 * HPG - 1 - n : n);
  int GP = 1;
  while (2 * GP <= min(p.G, kWeightWaves)) GP *= 2;
  const int TS = kWeightWaves / GP;            // waves that share a group's tiles
  const int ntiles = (r1 - r0 + kTileRows - 1) / kTileRows;
  const int my_tiles = ntiles > w / GP ? (ntiles - w / GP + TS - 1) / TS : 0;
  // The waves of the launch keep step with each other, and streams lie whole powers
  // of two apart: from the first tile on, all of them would ask the same memory
  // channels at once.  So each starts at a tile of its own and goes round (B32 T8K
  // H32 G8 d 128/16 in 4 bits 39.1 -> 32.5 us).
  int turn = 0;
  auto tile_row = [&](int j) {
    if (j >= my_tiles) return r0 + p.chunk;    // past the end: zeros, no traffic
    const int t = j + turn >= my_tiles ? j + turn - my_tiles : j + turn;
    return r0 + (w / GP + TS * t) * kTileRows;
  };
  const bf16x8 zero8 = as_bf16x8(u32x4{0u, 0u, 0u, 0u});
  // the lane that holds a row's sum, and the place of its four rows
  const bool puts = n == 0 || n == HPG;
  float* const put = &sums[w % GP][(n == HPG ? 16 : 0) + 4 * qd];
  for (int g = w % GP; g < p.G; g += GP) {
    const Stream in(p, b, g, r1, lane);
    turn = my_tiles > 0 ? (item + 2 * g) % my_tiles : 0;
    // the query before the tiles: loads are waited for in the order of their issue
    const int64_t qrow = (int64_t)b * p.H + g * HPG + head;
    typename Stream::Query q;
    in.request(q, p.q_abs + qrow * DV, p.q_rot + qrow * p.d_r);
    const float ls = p.lse[qrow];
    __builtin_amdgcn_sched_barrier(0);
    WeightRows<DV, NRC, Q4> buf[DEPTH];
#pragma unroll
    for (int d = 0; d < DEPTH - 1; ++d) {
      in.template load<kAuxNT>(buf[d], tile_row(d));
      __builtin_amdgcn_sched_barrier(0);
    }
    const float init = is_lo ? 0.f : weight_start(ls);
    bf16x8 bq[NC], bk[NRC > 0 ? NRC : 1];
#pragma unroll
    for (int c = 0; c < NC; ++c) bq[c] = active ? in.part(q, c, p.scale_log2, is_lo) : zero8;
#pragma unroll
    for (int rc = 0; rc < NRC; ++rc) bk[rc] = active ? in.part(q, NC + rc, p.scale_log2, is_lo) : zero8;
    const bool first = g < GP;
    for (int jt = 0; jt < my_tiles; jt += DEPTH) {
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        const int j = jt + d;
        if (j >= my_tiles) break;
        in.template load<kAuxNT>(buf[(d + DEPTH - 1) % DEPTH], tile_row(j + DEPTH - 1));
        __builtin_amdgcn_sched_barrier(0);
        f32x4 sc[2] = {f32x4{init, init, init, init}, f32x4{init, init, init, init}};
#pragma unroll
        for (int rc = 0; rc < NRC; ++rc)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) sc[hf] = mfma16(buf[d].k[hf][rc], bk[rc], sc[hf]);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf) sc[hf] = mfma16(Stream::chunk(buf[d], hf, c), bq[c], sc[hf]);
        f32x4 e;
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          const float mine = is_lo ? sc[1][jj] : sc[0][jj], other = is_lo ? sc[0][jj] : sc[1][jj];
          e[jj] = __builtin_amdgcn_exp2f(mine + mirror<HPG>(other));
          if constexpr (HPG >= 2) e[jj] = dpp_add<0xB1>(e[jj]);     // over the heads' lanes
          if constexpr (HPG >= 4) e[jj] = dpp_add<0x1B>(e[jj]);
          if constexpr (HPG >= 8) e[jj] = dpp_add<0x141>(e[jj]);
        }
        if (puts) {
          f32x4* at = reinterpret_cast<f32x4*>(put + (tile_row(j) - r0));
          *at = first ? e : *at + e;
        }
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < r1 - r0; i += 64 * kWeightWaves) {
    float s = 0.f;
    for (int g = 0; g < GP; ++g) s += sums[g][i];
    const int64_t at = (int64_t)b * p.t_max + r0 + i;
    p.new_weights[at] = p.decay != 0.f ? fmaf(p.decay, p.weights[at], s) : s;
  }
}

// Many queries, or any number of heads per group.  The workgroup takes one group
// and `chunk` rows of one sequence; a column of the products is one (query,
// head) pair, its query once as bf16 high parts and once as low parts into the
// same sums, 32 columns a wave.  The waves are dealt first over the columns and
// then over the tiles.  Sums over the columns go through LDS in a fixed order to
// the group's row sums in the workspace, which weights_join_kernel adds up.  Bound
// by the matrix products (twice the algorithm's, for the low parts) where there
// are many rows, 32 queries on B8 T16K H32 G8 d 128/16 bf16 in 100 us, 0.77
// PFLOP/s of them, and by latency where there are few: B2 of 4K to 8K rows 18.7 us,
// and 5 and 4 for the absorption before and the join behind it (sums over 1024
// queries and heads off by 3.2e-8, as in fp32; 4-bit rows 24.4 us in all).
constexpr int kWindowRows = 512, kWindowCols = 32;   // most rows of a workgroup; columns of a wave

template <int DV, int NRC, bool Q4>
__global__ void __launch_bounds__(kThreads, 2) weights_window_kernel(WeightParams p) {
  using Stream = WeightStream<DV, NRC, Q4>;
  constexpr int NC = Stream::NC, NK = NC + NRC;
  __shared__ __attribute__((aligned(16))) float sums[kWaves][kWindowRows];
  const int nchunks = (p.t_max + p.chunk - 1) / p.chunk;
  const int item = xcd_remap(blockIdx.x, p.B * nchunks * p.G);
  const int g = item % p.G, b = item / p.G / nchunks, r0 = item / p.G % nchunks * p.chunk;
  const int L = clamp_len(p.lens, b, p.t_max);
  if (r0 >= L) return;
  const int r1 = min(r0 + p.chunk, L);
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, qd = lane >> 4;
  const int hpg = p.H / p.G, cols = p.N * hpg;
  const int nsets = (cols + kWindowCols - 1) / kWindowCols;
  const int WC = nsets >= 4 ? 4 : (nsets >= 2 ? 2 : 1), WT = kWaves / WC;   // waves over columns, over tiles
  const int ntiles = (r1 - r0 + kTileRows - 1) / kTileRows;
  const Stream in(p, b, g, r1, lane);
  float* const mine = sums[w % WC];
  for (int set = w % WC; set < nsets; set += WC) {
    typename Stream::Query q[2];
    float ls[2];
    int last[2];                               // the last row that the column's query sees
#pragma unroll
    for (int cb = 0; cb < 2; ++cb) {
      const int col = set * kWindowCols + 16 * cb + n;
      const bool active = col < cols;
      const int qi = active ? col / hpg : 0;
      const int64_t qrow = ((int64_t)b * p.N + qi) * p.H + g * hpg + (active ? col % hpg : 0);
      in.request(q[cb], p.q_abs + qrow * DV, p.q_rot + qrow * p.d_r);
      ls[cb] = active ? p.lse[qrow] : -INFINITY;
      last[cb] = active ? L - p.N + qi : -1;
    }
    __builtin_amdgcn_sched_barrier(0);
    WeightRows<DV, NRC, Q4> buf[2];
    in.template load<0>(buf[0], r0 + w / WC * kTileRows);
    __builtin_amdgcn_sched_barrier(0);
    bf16x8 hi[2][NK], lo[2][NK];
    float init[2];
#pragma unroll
    for (int cb = 0; cb < 2; ++cb) {
      init[cb] = weight_start(ls[cb]);
#pragma unroll
      for (int c = 0; c < NK; ++c) {
        hi[cb][c] = in.part(q[cb], c, p.scale_log2, false);
        lo[cb][c] = in.part(q[cb], c, p.scale_log2, true);
      }
    }
    for (int j0 = w / WC; j0 < ntiles; j0 += 2 * WT)
#pragma unroll
    for (int d = 0; d < 2; ++d) {
      const int j = j0 + d * WT;
      if (j >= ntiles) break;
      const int row0 = r0 + j * kTileRows;
      const WeightRows<DV, NRC, Q4>& t = buf[d];
      in.template load<0>(buf[1 - d], row0 + WT * kTileRows);   // (past the last tile: zeros, no traffic)
      __builtin_amdgcn_sched_barrier(0);
      f32x4 sc[2][2];
#pragma unroll
      for (int cb = 0; cb < 2; ++cb)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) sc[cb][hf] = f32x4{init[cb], init[cb], init[cb], init[cb]};
#pragma unroll
      for (int c = 0; c < NK; ++c)
#pragma unroll
        for (int hf = 0; hf < 2; ++hf) {
          const bf16x8 a = c < NC ? Stream::chunk(t, hf, c) : t.k[hf][c < NC ? 0 : c - NC];
#pragma unroll
          for (int cb = 0; cb < 2; ++cb) sc[cb][hf] = mfma16(a, lo[cb][c], sc[cb][hf]);
#pragma unroll
          for (int cb = 0; cb < 2; ++cb) sc[cb][hf] = mfma16(a, hi[cb][c], sc[cb][hf]);
        }
      // a tile that some query sees only in part, or that holds rows past the end
      // (where anything may stand): those rows count as not seen
      const bool edge = row0 + kTileRows > L - p.N + 1 || cols < (set + 1) * kWindowCols;
      f32x4 e[2];
#pragma unroll
      for (int hf = 0; hf < 2; ++hf)
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          float v[2];
#pragma unroll
          for (int cb = 0; cb < 2; ++cb) {
            v[cb] = __builtin_amdgcn_exp2f(sc[cb][hf][jj]);
            if (edge) v[cb] = row0 + 16 * hf + 4 * qd + jj <= last[cb] ? v[cb] : 0.f;
          }
          e[hf][jj] = sum16(v[0] + v[1]);
        }
      if (n < 2) {                             // lane 0: the first 16 rows' sums, lane 1 the others'
        f32x4* at = reinterpret_cast<f32x4*>(mine + j * kTileRows + 16 * n + 4 * qd);
        const f32x4 mine4 = n ? e[1] : e[0];
        *at = set < WC ? mine4 : *at + mine4;
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < r1 - r0; i += kThreads) {
    float s = 0.f;
    for (int c = 0; c < WC; ++c) s += sums[c][i];
    p.part[((int64_t)g * p.B + b) * p.t_max + r0 + i] = s;
  }
}

__global__ void __launch_bounds__(kThreads) weights_join_kernel(WeightParams p) {
  const int b = blockIdx.y, t = blockIdx.x * kThreads + threadIdx.x;
  if (t >= clamp_len(p.lens, b, p.t_max)) return;
  const int64_t at = (int64_t)b * p.t_max + t;
  float s = 0.f;
#pragma unroll 8
  for (int g = 0; g < p.G; ++g) s += p.part[(int64_t)g * p.B * p.t_max + at];
  p.new_weights[at] = p.decay != 0.f ? fmaf(p.decay, p.weights[at], s) : s;
}

// fp32 storage: the same on the fp32 products, 16-row tiles, any d_v and d_r
// that the tiled layout takes.  Bound by the products and their loads' latency, the
// rows read again for every 16 columns: a checking path, not a serving one (H32 G8 d
// 128/16: a token of B8 T8K, 275 MB, 87 us, 32 queries on B2 of 4K to 8K rows 117).
__global__ void __launch_bounds__(64 * kWeightWaves) weights_f32_kernel(WeightParams p) {
  __shared__ float sums[kWeightWaves][kWeightChunk];
  const int nchunks = (p.t_max + p.chunk - 1) / p.chunk;
  const int item = xcd_remap(blockIdx.x, p.B * nchunks);
  const int b = item / nchunks, r0 = item % nchunks * p.chunk;
  const int L = clamp_len(p.lens, b, p.t_max);
  if (r0 >= L) return;
  const int r1 = min(r0 + p.chunk, L);
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, qd = lane >> 4;
  const int hpg = p.H / p.G, cols = p.N * hpg;
  int GP = 1;
  while (2 * GP <= min(p.G, kWeightWaves)) GP *= 2;
  const int TS = kWeightWaves / GP;
  float* const mine = sums[w];
  for (int i = lane; i < p.chunk; i += 64) mine[i] = 0.f;
  const int ntiles = (r1 - r0 + 15) / 16;
  const f32x4 zero4 = {0.f, 0.f, 0.f, 0.f};
  const float* kr = static_cast<const float*>(p.kr) + (int64_t)b * p.t_max * p.d_r;
  for (int g = w % GP; g < p.G; g += GP) {
    const float* v = static_cast<const float*>(p.v) + ((int64_t)b * p.G + g) * p.t_max * p.d_v;
    for (int c0 = 0; c0 < cols; c0 += 16) {
      const int col = c0 + n;
      const bool active = col < cols;
      const int qi = active ? col / hpg : 0;
      const int64_t qrow = ((int64_t)b * p.N + qi) * p.H + g * hpg + (active ? col % hpg : 0);
      const float ls = active ? p.lse[qrow] : -INFINITY;
      const float start = weight_start(ls);
      const bool live = start != -INFINITY;
      const int last = L - p.N + qi;
      const float init = live ? start : 0.f;
      for (int j = w / GP; j < ntiles; j += TS) {
        const int64_t row0 = r0 + j * 16;
        f32x4 sc = {init, init, init, init};
        auto add = [&](const float* stream, const float* query, int D) {
          for (int c = 0; c < D; c += 16) {
            const bool in = c + 4 * qd < D;
            const f32x4 x = in ? *reinterpret_cast<const f32x4*>(stream + row0 * D + ((c / 4 + qd) * 16 + n) * 4) : zero4;
            const f32x4 y = in && active ? *reinterpret_cast<const f32x4*>(query + c + 4 * qd) * p.scale_log2 : zero4;
#pragma unroll
            for (int e = 0; e < 4; ++e) sc = __builtin_amdgcn_mfma_f32_16x16x4f32(x[e], y[e], sc, 0, 0, 0);
          }
        };
        add(v, p.q_abs + qrow * p.d_v, p.d_v);
        add(kr, p.q_rot + qrow * p.d_r, p.d_r);
        float sum[4];
#pragma unroll
        for (int jj = 0; jj < 4; ++jj) {
          const int row = (int)row0 + 4 * qd + jj;
          sum[jj] = sum16(live && row <= last && row < r1 ? __builtin_amdgcn_exp2f(sc[jj]) : 0.f);
        }
        if (n == 0) {
#pragma unroll
          for (int jj = 0; jj < 4; ++jj) mine[j * 16 + 4 * qd + jj] += sum[jj];
        }
      }
    }
  }
  __syncthreads();
  for (int i = tid; i < r1 - r0; i += 64 * kWeightWaves) {
    float s = 0.f;
#pragma unroll
    for (int ww = 0; ww < kWeightWaves; ++ww) s += sums[ww][i];
    const int64_t at = (int64_t)b * p.t_max + r0 + i;
    p.new_weights[at] = p.decay != 0.f ? fmaf(p.decay, p.weights[at], s) : s;
  }
}

using WeightFn = void (*)(WeightParams);

template <int DV, int NRC, bool Q4>
WeightFn pick_weights_hpg(int hpg) {           // 0: the window kernel
  switch (hpg) {
    case 1: return weights_step_kernel<1, DV, NRC, Q4>;
    case 2: return weights_step_kernel<2, DV, NRC, Q4>;
    case 4: return weights_step_kernel<4, DV, NRC, Q4>;
    case 8: return weights_step_kernel<8, DV, NRC, Q4>;
  }
  return weights_window_kernel<DV, NRC, Q4>;
}

template <bool Q4>
WeightFn pick_weights(int hpg, int dv, int nrc) {
  const bool wide = dv == 128;
  switch (nrc) {
    case 0: return wide ? pick_weights_hpg<128, 0, Q4>(hpg) : pick_weights_hpg<64, 0, Q4>(hpg);
    case 1: return wide ? pick_weights_hpg<128, 1, Q4>(hpg) : pick_weights_hpg<64, 1, Q4>(hpg);
    case 2: return wide ? pick_weights_hpg<128, 2, Q4>(hpg) : pick_weights_hpg<64, 2, Q4>(hpg);
  }
  return nullptr;
}

// A decode step's query with a supported number of heads per group goes to the
// step kernel (0 otherwise); fp32 has one kernel.
int step_heads(const gva_dims* d, int n_new) {
  const int hpg = d->n_heads / d->n_groups;
  return n_new == 1 && (hpg == 1 || hpg == 2 || hpg == 4 || hpg == 8) ? hpg : 0;
}
bool weights_joined(const gva_dims* d, int n_new) { return d->dtype == GVA_DTYPE_BF16 && step_heads(d, n_new) == 0; }

// =============================================================== evict
constexpr int kEvictThreads = 1024, kEvictWaves = kEvictThreads / 64;
constexpr int kEvictRows = 4;                  // rows of a thread
constexpr int kEvictBlock = kEvictThreads * kEvictRows;
constexpr int kDigit0 = 12, kDigit12 = 10;     // bits of the key's digits, from the top

struct EvictParams {
  const int32_t* lens;
  const int32_t* seen;
  const float* weights;
  const int32_t* row_pos;
  int32_t* new_lens;
  float* new_weights;
  int32_t* new_row_pos;
  int32_t* count;         // [B]: rows that move
  int32_t* hole;          // [B][room]: the rows they go to, ascending
  int32_t* move;          // [B][room]: and come from, ascending
  int32_t* state;         // [B][4]: the border's first digit and the rank left in it; the second and its
  int32_t* above;         // [2][B][blocks]: keys above the border's first digit; above its second in the first
  uint16_t* hist0;        // [B][blocks][2^12]: keys by first digit
  uint16_t* hist1;        // [B][blocks][2^10]: by second digit, of those with the border's first
  uint16_t* hist2;        // [B][blocks][2^10]: by third digit, of those with the border's first two
  int32_t B, t_max, keep, first, recent, room, blocks, low;   // low: blocks of the rows below the budget
};

// The order of rows: larger keys stay.  Protected rows before all, NaN
// after all, -0 like +0.
__device__ __forceinline__ unsigned evict_key(const EvictParams& p, int pos, float weight, int seen) {
  const float x = weight + 0.f;
  const unsigned u = __float_as_uint(x);
  const unsigned order = x != x ? 0u : (u >> 31 ? ~u : u | 0x80000000u);
  return pos < p.first || (int64_t)pos >= (int64_t)seen - p.recent ? 0xFFFFFFFFu : order;
}

// The selection runs in four launches over blocks of 4096 rows, one workgroup
// each; the rows below the budget and those from it on have blocks of their own,
// so that places to fill and rows to move are numbered per block.  Three launches
// find the border, the keep-th largest key, digit by digit (12, 10 and 10 bits:
// the first takes in the exponent and three bits more, so that keys of like weight
// spread over many counters): every block counts its own keys, and the next launch
// adds up the blocks' counters, each workgroup for itself.  The fourth numbers the
// rows.  No counter is shared, so nothing has to be cleared.  Bound by latency: four
// sequences of 32K rows 4.7, 4.7, 4.7 and 6.6 us.
template <int N>
struct EvictRows {
  int t[N];
  bool in[N];             // a cached row of the block
  float weight[N];
  int pos[N];
  unsigned key[N];
};

// Rows t0 .. t1 - 1, N a thread; a wave's are contiguous.
template <int N>
__device__ __forceinline__ void evict_rows(const EvictParams& p, int b, int t0, int t1, int L, EvictRows<N>& r) {
  const int seen = p.seen != nullptr ? p.seen[b] : L;
  const int64_t base = (int64_t)b * p.t_max;
  const int first = t0 + (int)(threadIdx.x >> 6) * 64 * N + (int)(threadIdx.x & 63);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    r.t[i] = first + 64 * i;
    r.in[i] = r.t[i] < t1;
    const int t = r.in[i] ? r.t[i] : 0;
    r.weight[i] = p.weights[base + t];
    r.pos[i] = p.row_pos != nullptr ? p.row_pos[base + t] : t;
  }
#pragma unroll
  for (int i = 0; i < N; ++i) r.key[i] = evict_key(p, r.pos[i], r.weight[i], seen);
}

__device__ __forceinline__ void evict_block_rows(const EvictParams& p, int b, int blk, int L, EvictRows<kEvictRows>& r) {
  const int t0 = blk < p.low ? blk * kEvictBlock : p.keep + (blk - p.low) * kEvictBlock;
  evict_rows(p, b, t0, min(blk < p.low ? min(t0 + kEvictBlock, p.keep) : t0 + kEvictBlock, L), L, r);
}

// The sum over the lanes up to this one, by shifts within 16 lanes and then the
// row's and the half's last lane broadcast to those behind (wave_incl_scan goes
// through LDS six times).
__device__ __forceinline__ int lane_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xF, 0xF, true);    // row_shr 1, 2, 4, 8
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xF, 0xF, true);
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xA, 0xF, false);   // row_bcast 15 to rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xC, 0xF, false);   // row_bcast 31 to rows 2 and 3
  return v;
}

// Sums over the workgroup: of the threads before this one, and of all.  Every
// call has a row of counters of its own, so that one barrier is enough, and reads
// them at once (a loop up to the own wave waits for each).
struct WaveCounts {
  int n[kEvictWaves];
};
__device__ __forceinline__ int block_before(int v, WaveCounts& c) {
  const int incl = lane_scan(v), w = (int)(threadIdx.x >> 6);
  if ((threadIdx.x & 63) == 63) c.n[w] = incl;
  __syncthreads();
  const WaveCounts all = c;
  int before = incl - v;
#pragma unroll
  for (int i = 0; i < kEvictWaves; ++i) before += i < w ? all.n[i] : 0;
  return before;
}
__device__ __forceinline__ int block_sum(int v, WaveCounts& c) {
  const int s = lane_scan(v);
  if ((threadIdx.x & 63) == 63) c.n[threadIdx.x >> 6] = s;
  __syncthreads();
  const WaveCounts all = c;
  int sum = 0;
#pragma unroll
  for (int i = 0; i < kEvictWaves; ++i) sum += all.n[i];
  return sum;
}

// The counter that holds the rest-th key from the top, and the rank left in it:
// thread t holds the t-th N counters from there (its first one `top`).
template <int N>
__device__ __forceinline__ void pick_digit(const int (&c)[N], int top, int& rest, int& bin, WaveCounts& counts, int* picked) {
  int sum = 0;
#pragma unroll
  for (int k = 0; k < N; ++k) sum += c[k];
  int above = block_before(sum, counts);
#pragma unroll
  for (int k = 0; k < N; ++k) {
    if (above < rest && rest <= above + c[k]) {
      picked[0] = top - k;
      picked[1] = rest - above;
    }
    above += c[k];
  }
  __syncthreads();
  bin = picked[0];
  rest = picked[1];
}

// Digit STAGE of the keys that match the border's digits before it.
template <int STAGE>
__global__ void __launch_bounds__(kEvictThreads) evict_count_kernel(EvictParams p) {
  constexpr int BITS = STAGE == 0 ? kDigit0 : kDigit12, SHIFT = STAGE == 0 ? 20 : (STAGE == 1 ? 10 : 0);
  constexpr int PER = (1 << BITS) / kEvictThreads;
  __shared__ __attribute__((aligned(16))) int hist[1 << BITS];
  __shared__ __attribute__((aligned(16))) WaveCounts counts[2];
  __shared__ int picked[2];
  const int b = blockIdx.y, blk = blockIdx.x, tid = threadIdx.x;
  const int L = clamp_len(p.lens, b, p.t_max);
  if (L <= p.keep) return;
  const int64_t at = (int64_t)b * p.blocks + blk;
  EvictRows<kEvictRows> r;
  evict_block_rows(p, b, blk, L, r);
#pragma unroll
  for (int k = 0; k < PER; ++k) hist[tid + k * kEvictThreads] = 0;
  unsigned prefix = 0u;
  if constexpr (STAGE == 1) {
    const int top = (1 << kDigit0) - 1 - 4 * tid;
    int c[4] = {0, 0, 0, 0}, rest = p.keep, bin;
    const uint16_t* h = p.hist0 + ((int64_t)b * p.blocks << kDigit0) + top - 3;
#pragma unroll 8
    for (int i = 0; i < p.blocks; ++i) {
      const uint64_t x = *reinterpret_cast<const uint64_t*>(h + ((int64_t)i << kDigit0));
#pragma unroll
      for (int k = 0; k < 4; ++k) c[k] += (int)(x >> (16 * (3 - k)) & 0xFFFFu);
    }
    pick_digit(c, top, rest, bin, counts[0], picked);
    if (blk == 0 && tid == 0) {
      p.state[4 * b] = bin;
      p.state[4 * b + 1] = rest;
    }
    prefix = (unsigned)bin;
  }
  if constexpr (STAGE == 2) {
    int rest = p.state[4 * b + 1], bin, c[1] = {0};
    const int top = kEvictThreads - 1 - tid;
    const uint16_t* h = p.hist1 + ((int64_t)b * p.blocks << kDigit12) + top;
#pragma unroll 8
    for (int i = 0; i < p.blocks; ++i) c[0] += h[(int64_t)i << kDigit12];
    pick_digit(c, top, rest, bin, counts[0], picked);
    if (blk == 0 && tid == 0) {
      p.state[4 * b + 2] = bin;
      p.state[4 * b + 3] = rest;
    }
    prefix = (unsigned)p.state[4 * b] << kDigit12 | (unsigned)bin;
  }
  __syncthreads();                             // the counters are clear
  int above = 0;
#pragma unroll
  for (int i = 0; i < kEvictRows; ++i) {
    if (!r.in[i]) continue;
    const unsigned x = r.key[i] >> SHIFT;
    if (STAGE == 0 || x >> BITS == prefix) atomicAdd(&hist[x & ((1u << BITS) - 1u)], 1);
    // above the border's last digit known so far, alike in those before it
    if (STAGE == 1) above += x >> BITS > prefix ? 1 : 0;
    if (STAGE == 2) above += x >> BITS > prefix && x >> (BITS + kDigit12) == prefix >> kDigit12 ? 1 : 0;
  }
  if constexpr (STAGE > 0) {
    above = block_sum(above, counts[1]);
    if (tid == 0) p.above[(int64_t)(STAGE - 1) * p.B * p.blocks + at] = above;
  }
  __syncthreads();
  if constexpr (STAGE == 0) {
    uint64_t x = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) x |= (uint64_t)hist[4 * tid + k] << (16 * k);
    *reinterpret_cast<uint64_t*>(p.hist0 + (at << kDigit0) + 4 * tid) = x;
  } else {
    (STAGE == 1 ? p.hist1 : p.hist2)[(at << kDigit12) + tid] = (uint16_t)hist[tid];
  }
}

__global__ void __launch_bounds__(kEvictThreads) evict_number_kernel(EvictParams p) {
  __shared__ __attribute__((aligned(16))) WaveCounts counts[5];
  __shared__ int picked[2], eq_n[2];
  const int b = blockIdx.y, blk = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int L = clamp_len(p.lens, b, p.t_max), K = p.keep;
  const int64_t base = (int64_t)b * p.t_max;
  EvictRows<kEvictRows> r;
  evict_block_rows(p, b, blk, L, r);
  if (blk == 0 && tid == 0) p.new_lens[b] = min(L, K);
  auto store = [&](int i, float weight, int pos) {
    if (r.t[i] >= (blk < p.low ? min(K, p.t_max) : p.t_max)) return;
    p.new_weights[base + r.t[i]] = weight;
    if (p.new_row_pos != nullptr) p.new_row_pos[base + r.t[i]] = pos;
  };
  if (L <= K) {                                // every row stays
    if (blk == 0 && tid == 0) p.count[b] = 0;
#pragma unroll
    for (int i = 0; i < kEvictRows; ++i) store(i, r.in[i] ? r.weight[i] : 0.f, r.in[i] ? r.pos[i] : -1);
    return;
  }
  // the third digit; its counters in the blocks before this one, and in those
  // below the budget
  int rest = p.state[4 * b + 3], bin, c[1] = {0}, before = 0, low = 0;
  const int top = kEvictThreads - 1 - tid;
  const uint16_t* h = p.hist2 + ((int64_t)b * p.blocks << kDigit12) + top;
#pragma unroll 8
  for (int i = 0; i < p.blocks; ++i) {
    const int x = h[(int64_t)i << kDigit12];
    c[0] += x;
    before += i < blk ? x : 0;
    low += i < p.low ? x : 0;
  }
  pick_digit(c, top, rest, bin, counts[0], picked);
  const unsigned border = ((unsigned)p.state[4 * b] << kDigit12 | (unsigned)p.state[4 * b + 2]) << kDigit12 | (unsigned)bin;
  if (top == bin) {
    eq_n[0] = before;
    eq_n[1] = low;
  }
  int more = 0, more_low = 0;                  // keys above the border's earlier digits: a block's to a thread
  for (int i = tid; i < p.low || i < blk; i += kEvictThreads) {
    const int64_t at = (int64_t)b * p.blocks + i;
    const int x = p.above[at] + p.above[(int64_t)p.B * p.blocks + at];
    more += i < blk ? x : 0;
    more_low += i < p.low ? x : 0;
  }
  const int gt = block_sum(more + (top > bin ? before : 0), counts[1]);
  const int gt_low = block_sum(more_low + (top > bin ? low : 0), counts[2]);
  // rows above the border stay, and the first `rest` of those on it
  const int eq = eq_n[0];
  const int kept_low = gt_low + min(rest, eq_n[1]), kept = gt + min(rest, eq);
  if (blk == 0 && tid == 0) p.count[b] = K - kept_low;
  const unsigned long long below = (1ull << lane) - 1ull;
  // a wave's rows are contiguous: its numbers go on from those of the waves before
  unsigned long long on[kEvictRows], stay[kEvictRows];
  int n_on = 0;
#pragma unroll
  for (int i = 0; i < kEvictRows; ++i) {
    on[i] = __ballot(r.in[i] && r.key[i] == border);
    n_on += __popcll(on[i]);
  }
  int at_eq = eq + __builtin_amdgcn_readfirstlane(block_before(lane == 0 ? n_on : 0, counts[3]));
  int n_stay = 0, n_go = 0;
#pragma unroll
  for (int i = 0; i < kEvictRows; ++i) {
    const bool me = r.in[i] && (r.key[i] > border || (r.key[i] == border && at_eq + __popcll(on[i] & below) < rest));
    at_eq += __popcll(on[i]);
    stay[i] = __ballot(me);
    n_stay += __popcll(stay[i]);
    n_go += __popcll(__ballot(r.in[i]) & ~stay[i]);
  }
  const bool is_low = blk < p.low;
  int at = block_before(lane == 0 ? (is_low ? n_go : n_stay) : 0, counts[4]);
  at = __builtin_amdgcn_readfirstlane(at) + (is_low ? blk * kEvictBlock - kept : kept - kept_low);
  int32_t* const list = (is_low ? p.hole : p.move) + (int64_t)b * p.room;
#pragma unroll
  for (int i = 0; i < kEvictRows; ++i) {
    const unsigned long long m = is_low ? __ballot(r.in[i]) & ~stay[i] : stay[i];
    const bool listed = m >> lane & 1ull;
    if (listed) list[at + __popcll(m & below)] = r.t[i];
    at += __popcll(m);
    // a row to fill gets its weight and position with the row that moves there
    if (!is_low)
      store(i, 0.f, -1);
    else if (!listed)
      store(i, r.weight[i], r.pos[i]);
  }
}

// The whole selection of a sequence in one workgroup, N rows a thread: up to 8K
// rows it takes less than the four launches above (4K rows, B = 32: 9.6 us against
// 20; 32K rows, whose keys do not fit the registers beside the rest: 84 against 20).
template <int N>
__global__ void __launch_bounds__(kEvictThreads) evict_select_kernel(EvictParams p) {
  __shared__ __attribute__((aligned(16))) int hist[1 << kDigit0];
  __shared__ __attribute__((aligned(16))) WaveCounts counts[5];
  __shared__ int picked[2];
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int L = clamp_len(p.lens, b, p.t_max), K = p.keep;
  const int64_t base = (int64_t)b * p.t_max;
  EvictRows<N> r;
  evict_rows(p, b, 0, L, L, r);
  auto store = [&](int i, float weight, int pos) {
    if (r.t[i] >= p.t_max) return;
    p.new_weights[base + r.t[i]] = weight;
    if (p.new_row_pos != nullptr) p.new_row_pos[base + r.t[i]] = pos;
  };
  if (tid == 0) p.new_lens[b] = min(L, K);
  if (L <= K) {                                // every row stays
    if (tid == 0) p.count[b] = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) store(i, r.in[i] ? r.weight[i] : 0.f, r.in[i] ? r.pos[i] : -1);
    return;
  }
  // (the counters of a digit are cleared while the digit before is being settled:
  // three barriers a digit)
  unsigned border = 0u;
  int rest = K;
#pragma unroll
  for (int k = 0; k < 4; ++k) hist[tid + k * kEvictThreads] = 0;
  __syncthreads();
#pragma unroll
  for (int digit = 0; digit < 3; ++digit) {
    const int bits = digit == 0 ? kDigit0 : kDigit12, shift = digit == 0 ? 20 : (digit == 1 ? 10 : 0);
    constexpr int kMost = (1 << kDigit0) / kEvictThreads;
    const int per = digit == 0 ? kMost : 1;    // counters a thread holds
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const unsigned x = r.key[i] >> shift;
      if (r.in[i] && (digit == 0 || x >> bits == border)) atomicAdd(&hist[x & ((1u << bits) - 1u)], 1);
    }
    __syncthreads();
    const int top = (1 << bits) - 1 - per * tid;
    int c[kMost], sum = 0;
#pragma unroll
    for (int k = 0; k < per; ++k) {
      c[k] = hist[top - k];
      sum += c[k];
    }
    int above = block_before(sum, counts[digit]);
#pragma unroll
    for (int k = 0; k < per; ++k) {
      if (above < rest && rest <= above + c[k]) {
        picked[0] = top - k;
        picked[1] = rest - above;
      }
      above += c[k];
    }
    if (digit < 2) hist[tid] = 0;              // the next digits have 1024 counters
    __syncthreads();
    border = border << bits | (unsigned)picked[0];
    rest = picked[1];
  }
  // rows above the border stay, and the first `rest` of those on it
  const unsigned long long below = (1ull << lane) - 1ull;
  unsigned long long on[N], stay[N];
  int n_on = 0, n_hole = 0, n_move = 0;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    on[i] = __ballot(r.in[i] && r.key[i] == border);
    n_on += __popcll(on[i]);
  }
  int at_eq = __builtin_amdgcn_readfirstlane(block_before(lane == 0 ? n_on : 0, counts[3]));
#pragma unroll
  for (int i = 0; i < N; ++i) {
    stay[i] = __ballot(r.in[i] && (r.key[i] > border || (r.key[i] == border && at_eq + __popcll(on[i] & below) < rest)));
    at_eq += __popcll(on[i]);
    n_hole += __popcll(__ballot(r.in[i] && r.t[i] < K) & ~stay[i]);
    n_move += __popcll(stay[i] & __ballot(r.t[i] >= K));
  }
  // both numbers in one scan (each below 2^14)
  const int both = __builtin_amdgcn_readfirstlane(block_before(lane == 0 ? n_hole << 16 | n_move : 0, counts[4]));
  int hole = both >> 16, move = both & 0xFFFF;
  if (tid == kEvictThreads - 1) p.count[b] = move + n_move;
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const unsigned long long hm = __ballot(r.in[i] && r.t[i] < K) & ~stay[i], mm = stay[i] & __ballot(r.t[i] >= K);
    if (hm >> lane & 1ull) p.hole[(int64_t)b * p.room + hole + __popcll(hm & below)] = r.t[i];
    if (mm >> lane & 1ull) p.move[(int64_t)b * p.room + move + __popcll(mm & below)] = r.t[i];
    hole += __popcll(hm);
    move += __popcll(mm);
    // a row to fill gets its weight and position with the row that moves there
    if (r.t[i] >= K)
      store(i, 0.f, -1);
    else if (stay[i] >> lane & 1ull)
      store(i, r.weight[i], r.pos[i]);
  }
}

struct MoveParams {
  const float* weights;
  const int32_t* row_pos;
  float* new_weights;
  int32_t* new_row_pos;
  const int32_t* count;
  const int32_t* hole;
  const int32_t* move;
  uint8_t* v;
  uint8_t* scales;
  uint8_t* kr;
  int32_t B, G, t_max, d_v, room;
  int32_t v_pieces, kr_pieces;   // 16-byte pieces of a row in a tiled stream
};

// Rows move from at or past the budget to below it, so no row is both read and
// written and the moves need no order.  A wave takes 16 moves of one stream and
// 16 of its 16-byte pieces, lane (n, qd) pieces qd, qd + 4, ... of move n, all
// requested before the first is stored: moves next to each other come from, and
// go to, nearby rows of a tile, whose pieces lie side by side.  Half the rows of
// four sequences of 32K go (G8 d 128/24 bf16): 85 us for 139 MB read and written,
// but every line below the budget is rewritten in part and every line behind it
// read: with the former read too 410 MB, 78 us at a copy's pace (whole tiles read,
// filled in LDS and written took 77 us, and a map of the moves more).
template <bool Q4>
__global__ void __launch_bounds__(kThreads) evict_move_kernel(MoveParams p) {
  const int b = blockIdx.z, nseg = Q4 ? 1 : (p.v_pieces + 15) / 16;
  const int g = blockIdx.y / nseg, c0 = blockIdx.y % nseg * 16;
  const int lane = threadIdx.x & 63, n = lane & 15, qd = lane >> 4;
  const int i = ((int)blockIdx.x * kWaves + (int)(threadIdx.x >> 6)) * 16 + n;
  if (i >= p.count[b]) return;
  const int to = p.hole[(int64_t)b * p.room + i], from = p.move[(int64_t)b * p.room + i];
  auto tiled = [&](uint8_t* stream, int pieces) {
    const u32x4* src = reinterpret_cast<const u32x4*>(stream) + (int64_t)(from / 16) * 16 * pieces + from % 16;
    u32x4* dst = reinterpret_cast<u32x4*>(stream) + (int64_t)(to / 16) * 16 * pieces + to % 16;
    u32x4 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c0 + qd + 4 * k < pieces) x[k] = __builtin_nontemporal_load(src + (c0 + qd + 4 * k) * 16);
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (c0 + qd + 4 * k < pieces) __builtin_nontemporal_store(x[k], dst + (c0 + qd + 4 * k) * 16);
  };
  if (g == p.G) {                              // what the groups share (a positional key has at most 16 pieces)
    if (p.kr_pieces > 0) tiled(p.kr + (int64_t)b * p.t_max * p.kr_pieces * 16, p.kr_pieces);
    if (qd == 0) {
      const int64_t base = (int64_t)b * p.t_max;
      p.new_weights[base + to] = p.weights[base + from];
      if (p.new_row_pos != nullptr) p.new_row_pos[base + to] = p.row_pos[base + from];
    }
    return;
  }
  const int64_t stream = (int64_t)b * p.G + g;
  if constexpr (Q4) {
    uint8_t* codes = p.v + stream * p.t_max * (p.d_v / 2);
    if (p.d_v == 128)
      *reinterpret_cast<u32x4*>(codes + code_off(to, qd, 128)) = *reinterpret_cast<const u32x4*>(codes + code_off(from, qd, 128));
    else
      *reinterpret_cast<u32x2*>(codes + code_off(to, qd, 64)) = *reinterpret_cast<const u32x2*>(codes + code_off(from, qd, 64));
    uint8_t* sc = p.scales + stream * p.t_max * (p.d_v / kScaleCols);
    if (qd < p.d_v / kScaleCols) sc[scale_off(to, qd, p.d_v)] = sc[scale_off(from, qd, p.d_v)];
  } else {
    tiled(p.v + stream * p.t_max * p.v_pieces * 16, p.v_pieces);
  }
}

struct WeightLayout {
  size_t q_rot, part, bytes;
};

int weight_layout(const gva_dims* d, int32_t n_new, WeightLayout& L) {
  const int st = check_dims(d);
  if (st != GVA_OK) return st;
  if (n_new < 1 || n_new > d->t_max) return GVA_ERR_INVALID_ARG;
  const size_t rows = (size_t)d->batch * n_new * d->n_heads;
  L.q_rot = round256(rows * d->d_v * 4);
  L.part = L.q_rot + round256(rows * d->d_r * 4);
  L.bytes = L.part + (weights_joined(d, n_new) ? round256((size_t)d->n_groups * d->batch * d->t_max * 4) : 0);
  return GVA_OK;
}

struct EvictLayout {
  size_t hole, move, state, above, hist0, hist1, hist2, bytes;
  int room, blocks;
};

// The workspace for any budget: at most min(keep, t_max - keep) rows move, and
// the rows below the budget and from it on make at most one block more.
int evict_layout(const gva_dims* d, EvictLayout& L) {
  const int st = check_dims(d);
  if (st != GVA_OK) return st;
  L.room = d->t_max / 2 + 1;
  L.blocks = (d->t_max + kEvictBlock - 1) / kEvictBlock + 1;
  const size_t B = (size_t)d->batch, n = B * (size_t)L.blocks;
  size_t off = 0;
  auto take = [&](size_t bytes) {
    const size_t at = off;
    off += round256(bytes);
    return at;
  };
  take(B * 4);                                 // count, at 0
  L.hole = take(B * L.room * 4);
  L.move = take(B * L.room * 4);
  L.state = take(B * 16);
  L.above = take(2 * n * 4);
  L.hist0 = take(n << (kDigit0 + 1));
  L.hist1 = take(n << (kDigit12 + 1));
  L.hist2 = take(n << (kDigit12 + 1));
  L.bytes = off;
  return GVA_OK;
}

}  // namespace

extern "C" {

int gva_weights_workspace_size(const gva_dims* dims, int32_t n_new, size_t* bytes) {
  if (bytes == nullptr) return GVA_ERR_INVALID_ARG;
  WeightLayout L;
  const int st = weight_layout(dims, n_new, L);
  if (st != GVA_OK) return st;
  *bytes = L.bytes;
  return GVA_OK;
}

int gva_accumulate_weights(const gva_dims* dims, int32_t n_new, const void* q, const void* m, const void* v_cache,
                           const void* v4_scale, const void* kr_cache, const int32_t* lens, const int32_t* seen,
                           const float* lse, double decay, const float* weights, float* new_weights, void* workspace,
                           size_t workspace_bytes, void* stream) {
  WeightLayout L;
  int st = weight_layout(dims, n_new, L);
  if (st != GVA_OK) return st;
  if (!q || !m || !v_cache || !lens || !lse || !new_weights) return GVA_ERR_INVALID_ARG;
  if (dims->d_r > 0 && !kr_cache) return GVA_ERR_INVALID_ARG;
  if (!(decay >= 0.0) || !isfinite((float)decay) || (decay != 0.0 && !weights)) return GVA_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(m, 16) || !aligned(v_cache, 16) || !aligned(v4_scale, 16) || !aligned(lens, 4) ||
      !aligned(seen, 4) || !aligned(lse, 4) || !aligned(weights, 4) || !aligned(new_weights, 4) ||
      (dims->d_r > 0 && !aligned(kr_cache, 16)))
    return GVA_ERR_INVALID_ARG;
  if (workspace == nullptr || workspace_bytes < L.bytes || !aligned(workspace, 256)) return GVA_ERR_INVALID_ARG;
  const bool q4 = v4_scale != nullptr, f32 = dims->dtype == GVA_DTYPE_F32;
  st = q4 ? check_q4_dims(dims) : check_cache_layout(dims);
  if (st != GVA_OK) return st;
  WeightFn fn = weights_f32_kernel;
  if (!f32) {
    if ((dims->d_v != 64 && dims->d_v != 128) || dims->d_r % 8 != 0 || dims->d_r > 64) return GVA_ERR_UNSUPPORTED;
    const int nrc = (dims->d_r + 31) / 32, heads = step_heads(dims, n_new);
    fn = q4 ? pick_weights<true>(heads, dims->d_v, nrc) : pick_weights<false>(heads, dims->d_v, nrc);
  }
  const bool joined = weights_joined(dims, n_new);
  if ((long long)n_new * (dims->n_heads / dims->n_groups) > 0x7FFFFF00LL || dims->batch > 65535) return GVA_ERR_UNSUPPORTED;
  // rows per workgroup: few enough for two workgroups per CU, whole tiles
  const long long streams = (long long)dims->batch * (joined ? dims->n_groups : 1);
  int chunk = joined ? kWindowRows : kWeightChunk;
  auto count = [&]() { return streams * ((dims->t_max + chunk - 1) / chunk); };
  while (chunk > 32 && count() < 2LL * device_cu_count()) chunk /= 2;
  const long long items = count();
  if (items > 0x7FFFFFFFLL) return GVA_ERR_UNSUPPORTED;
  float* q_abs = static_cast<float*>(workspace);
  float* q_rot = dims->d_r > 0 ? reinterpret_cast<float*>(static_cast<char*>(workspace) + L.q_rot) : nullptr;
  gva_dims at = *dims;                         // the queries' positions count the tokens seen, not the rows left
  if (seen != nullptr) at.t_max = 0x7FFFFFFF;
  st = gva_prefill_absorb(&at, n_new, q, m, seen != nullptr ? seen : lens, q_abs, q_rot, stream);
  if (st != GVA_OK) return st;
  float* part = reinterpret_cast<float*>(static_cast<char*>(workspace) + L.part);
  WeightParams p{v_cache, static_cast<const uint8_t*>(v4_scale), kr_cache, q_abs, q_rot, lse, lens, weights, new_weights, part,
                 dims->batch, dims->n_heads, dims->n_groups, n_new, dims->d_v, dims->d_r, dims->t_max, chunk,
                 scale_log2(dims), (float)decay};
  hipStream_t s = static_cast<hipStream_t>(stream);
  hipLaunchKernelGGL(fn, dim3((unsigned)items), dim3(joined ? kThreads : 64 * kWeightWaves), 0, s, p);
  st = launch_status();
  if (st != GVA_OK || !joined) return st;
  hipLaunchKernelGGL(weights_join_kernel, dim3((unsigned)((dims->t_max + kThreads - 1) / kThreads), (unsigned)dims->batch),
                     dim3(kThreads), 0, s, p);
  return launch_status();
}

int gva_evict_workspace_size(const gva_dims* dims, size_t* bytes) {
  if (bytes == nullptr) return GVA_ERR_INVALID_ARG;
  EvictLayout L;
  const int st = evict_layout(dims, L);
  if (st != GVA_OK) return st;
  *bytes = L.bytes;
  return GVA_OK;
}

int gva_evict_rows(const gva_dims* dims, int32_t n_keep, int32_t n_first, int32_t n_recent, void* v_cache,
                   void* v4_scale, void* kr_cache, const int32_t* lens, const int32_t* seen, const float* weights,
                   const int32_t* row_pos, int32_t* new_lens, float* new_weights, int32_t* new_row_pos,
                   void* workspace, size_t workspace_bytes, void* stream) {
  EvictLayout L;
  int st = evict_layout(dims, L);
  if (st != GVA_OK) return st;
  if (n_keep < 1 || n_first < 0 || n_recent < 0 || (long long)n_first + n_recent > n_keep) return GVA_ERR_INVALID_ARG;
  if (!v_cache || !lens || !weights || !new_lens || !new_weights) return GVA_ERR_INVALID_ARG;
  if (dims->d_r > 0 && !kr_cache) return GVA_ERR_INVALID_ARG;
  if ((row_pos == nullptr) != (new_row_pos == nullptr)) return GVA_ERR_INVALID_ARG;
  if (!aligned(v_cache, 16) || !aligned(v4_scale, 16) || !aligned(lens, 4) || !aligned(seen, 4) || !aligned(weights, 4) ||
      !aligned(row_pos, 4) || !aligned(new_lens, 4) || !aligned(new_weights, 4) || !aligned(new_row_pos, 4) ||
      (dims->d_r > 0 && !aligned(kr_cache, 16)))
    return GVA_ERR_INVALID_ARG;
  if (new_lens == lens || new_lens == seen || new_weights == weights || (row_pos != nullptr && new_row_pos == row_pos))
    return GVA_ERR_INVALID_ARG;
  if (workspace == nullptr || workspace_bytes < L.bytes || !aligned(workspace, 256)) return GVA_ERR_INVALID_ARG;
  const bool q4 = v4_scale != nullptr;
  st = q4 ? check_q4_dims(dims) : check_cache_layout(dims);
  if (st != GVA_OK) return st;
  const long long segs = q4 ? 1 : ((long long)dims->d_v * (long long)elem_size(dims) / 16 + 15) / 16;
  if (dims->batch > 65535 || segs * dims->n_groups >= 65535) return GVA_ERR_UNSUPPORTED;
  char* ws = static_cast<char*>(workspace);
  auto ints = [&](size_t off) { return reinterpret_cast<int32_t*>(ws + off); };
  auto shorts = [&](size_t off) { return reinterpret_cast<uint16_t*>(ws + off); };
  int32_t *count = ints(0), *hole = ints(L.hole), *move = ints(L.move);
  const int low = ((n_keep < dims->t_max ? n_keep : dims->t_max) + kEvictBlock - 1) / kEvictBlock;
  const int high = n_keep < dims->t_max ? (dims->t_max - n_keep + kEvictBlock - 1) / kEvictBlock : 0;
  const EvictParams p{lens, seen, weights, row_pos, new_lens, new_weights, new_row_pos, count, hole, move,
                      ints(L.state), ints(L.above), shorts(L.hist0), shorts(L.hist1), shorts(L.hist2),
                      dims->batch, dims->t_max, n_keep, n_first, n_recent, L.room, low + high, low};
  hipStream_t s = static_cast<hipStream_t>(stream);
  const dim3 blocks((unsigned)(low + high), (unsigned)dims->batch);
  if (dims->t_max <= 2 * kEvictBlock) {
    hipLaunchKernelGGL((dims->t_max <= kEvictBlock ? evict_select_kernel<4> : evict_select_kernel<8>),
                       dim3((unsigned)dims->batch), dim3(kEvictThreads), 0, s, p);
  } else {
    hipLaunchKernelGGL(evict_count_kernel<0>, blocks, dim3(kEvictThreads), 0, s, p);
    hipLaunchKernelGGL(evict_count_kernel<1>, blocks, dim3(kEvictThreads), 0, s, p);
    hipLaunchKernelGGL(evict_count_kernel<2>, blocks, dim3(kEvictThreads), 0, s, p);
    hipLaunchKernelGGL(evict_number_kernel, blocks, dim3(kEvictThreads), 0, s, p);
  }
  st = launch_status();
  const int most = n_keep < dims->t_max - n_keep ? n_keep : dims->t_max - n_keep;   // rows of a sequence that can move
  if (st != GVA_OK || most <= 0) return st;
  const int piece = (int)(16 / elem_size(dims));
  const int nseg = q4 ? 1 : (dims->d_v / piece + 15) / 16;
  const MoveParams mp{weights, row_pos, new_weights, new_row_pos, count, hole, move,
                      static_cast<uint8_t*>(v_cache), static_cast<uint8_t*>(v4_scale), static_cast<uint8_t*>(kr_cache),
                      dims->batch, dims->n_groups, dims->t_max, dims->d_v, L.room, dims->d_v / piece, dims->d_r / piece};
  const dim3 grid((unsigned)((most + 16 * kWaves - 1) / (16 * kWaves)), (unsigned)(dims->n_groups * nseg + 1), (unsigned)dims->batch);
  hipLaunchKernelGGL((q4 ? evict_move_kernel<true> : evict_move_kernel<false>), grid, dim3(kThreads), 0, s, mp);
  return launch_status();
}

}  // extern "C"
