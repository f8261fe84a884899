// libgva.so -- a value cache held in 4 bits: append, unpack, decode.
//
// A cached value row is kept as e2m1 codes (sign and one of 0, .5, 1, 1.5, 2,
// 3, 4, 6) with one power-of-two scale byte per 32 columns, the element and
// scale types that the matrix cores' converters read:
//   value = code * 2^(byte - 127),   byte 255: NaN
// The scale is the smallest 2^e with amax <= 7 * 2^e, -119 <= e <= 125: up to
// 7 an element that saturates at 6 is off by at most 2^e, no more than one
// between 4 and 6 is, and the finer scale pays for it (rms error of N(0, 1)
// rows 0.112; 0.115 with amax <= 6 * 2^e and with floor(log2 amax) - 2).  Every
// value is exactly a bf16: codes have two significant bits, and the bounds on e
// keep 0.5 * 2^e normal and 6 * 2^e finite.
// A row takes 4.25 bits an element, 576 B at G = 8, d_v = 128, d_r = 16 against
// 2080 B in bf16 (the positional key, 1/16 of a bf16 row, stays bf16).
//
// Layout.  Codes in blocks of 1 KB, which a wave reads as 16 bytes a lane: lane
// (n, p) = (lane % 16, lane / 16) receives piece p, d_v / 4 columns, of row n
// of the block (16 rows at d_v = 128, one scale block a lane; 32 rows at d_v =
// 64, the piece of row n and then that of row n + 16).  Scale bytes in tiles of
// 32 rows, [32-column block][row % 16][row / 16 % 2]: one 2-byte load per lane
// and tile.  A matrix-core product over columns may take them in any order as
// long as both operands do, so the 32 columns of product c are the eight columns
// 8 c .. 8 c + 7 of every piece: one 32-bit word of each lane.

#include "gva_common.h"
#include "gva_q4.h"

namespace {

// ================================================================ append
struct Q4AppendParams {
  uint8_t* codes;
  uint8_t* scales;
  uint16_t* kr_cache;
  const uint16_t* v_new;
  const uint16_t* kr_new;
  const int32_t* seq;
  const int32_t* row;
  const int32_t* pos;
  int32_t* row_pos;
  int32_t B, G, t_max, d_r, n_rows;
  double inv_freq[kMaxPairs];
};

// A wave takes one group's values of the rows of one 1 KB block, a lane one
// scale block (32 columns) of a row: rows at consecutive places of a stream are
// then stored as whole blocks.  The positional pairs, an fp64 rotation each,
// have workgroups of their own.
template <int DV>
__global__ void __launch_bounds__(kThreads) q4_append_kernel(Q4AppendParams p) {
  constexpr int R = block_rows(DV), NS = DV / kScaleCols;
  const int r0 = blockIdx.x * R, tid = threadIdx.x;
  const int gblocks = (p.G + kWaves - 1) / kWaves;
  if ((int)blockIdx.y < gblocks) {
    const int g = blockIdx.y * kWaves + (tid >> 6), lane = tid & 63;
    const int c = lane / R, r = r0 + lane % R;
    if (g >= p.G || r >= p.n_rows) return;
    const u32x4* src = reinterpret_cast<const u32x4*>(p.v_new + ((int64_t)r * p.G + g) * DV + c * kScaleCols);
    u32x4 x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) x[k] = src[k];
    const int b = p.seq[r], t = p.row[r];
    if (b < 0 || b >= p.B || t < 0 || t >= p.t_max) return;
    if (p.row_pos != nullptr && g == 0 && c == 0) p.row_pos[(int64_t)b * p.t_max + t] = p.pos != nullptr ? p.pos[r] : t;
    // the magnitudes of bf16 numbers are ordered as their bits are
    unsigned amax = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const unsigned lo = x[k][j] & 0x7FFFu, hi = x[k][j] >> 16 & 0x7FFFu;
        amax = max(amax, max(lo, hi));
      }
    // amax = 1.m * 2^(E - 127): 2^(E - 129) * 7 reaches it up to m = 3/4
    int byte = (int)(amax >> 7) - ((amax & 127u) <= 96u ? 2 : 1);
    byte = min(max(byte, kScaleLow), kScaleHigh);
    const float s = scale_of((unsigned)byte);
    u32x4 code = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const bf16x8 v = as_bf16x8(x[k]);
      unsigned w = 0u;
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_shufflevector(v, v, 0, 1), s, 0);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_shufflevector(v, v, 2, 3), s, 1);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_shufflevector(v, v, 4, 5), s, 2);
      w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, __builtin_shufflevector(v, v, 6, 7), s, 3);
      code[k] = w;
    }
    if (amax >= 0x7F80u) {                     // a NaN or an infinity: the block stands for NaN
      byte = kScaleNaN;
      code = u32x4{0u, 0u, 0u, 0u};
    }
    const int64_t stream = (int64_t)b * p.G + g;
    uint8_t* cs = p.codes + stream * p.t_max * (DV / 2);
    if constexpr (DV == 128) {
      *reinterpret_cast<u32x4*>(cs + code_off(t, c, DV)) = code;
    } else {                                   // two pieces of 16 columns
      *reinterpret_cast<u32x2*>(cs + code_off(t, 2 * c, DV)) = u32x2{code[0], code[1]};
      *reinterpret_cast<u32x2*>(cs + code_off(t, 2 * c + 1, DV)) = u32x2{code[2], code[3]};
    }
    p.scales[stream * p.t_max * NS + scale_off(t, c, DV)] = (uint8_t)byte;
    return;
  }
  const int npair = p.d_r / 2;
  const int task = ((int)blockIdx.y - gblocks) * kThreads + tid;
  if (task >= R * npair) return;
  const int r = r0 + task / npair, i = task % npair;
  if (r >= p.n_rows) return;
  const uint32_t two = *reinterpret_cast<const uint32_t*>(p.kr_new + (int64_t)r * p.d_r + 2 * i);
  const int b = p.seq[r], t = p.row[r];
  const int at = p.pos != nullptr ? p.pos[r] : t;
  if (b < 0 || b >= p.B || t < 0 || t >= p.t_max) return;
  double y0, y1;
  rotate_pair(bf16_bits_to_f32(two & 0xFFFFu), bf16_bits_to_f32(two >> 16), (double)at * p.inv_freq[i], y0, y1);
  uint16_t* k = p.kr_cache + (int64_t)b * p.t_max * p.d_r + tiled_off<uint16_t>(t, 2 * i, p.d_r);
  *reinterpret_cast<uint32_t*>(k) = (uint32_t)f64_to_bf16_rne(y0) | (uint32_t)f64_to_bf16_rne(y1) << 16;
}

// ================================================================ unpack
struct Q4UnpackParams {
  const uint8_t* codes;
  const uint8_t* scales;
  const int32_t* lens;
  uint16_t* v;
  int32_t B, G, t_max;
};

// A wave per 1 KB block of codes: 4 KB of bf16 rows, in 16-byte pieces of 16
// consecutive rows.
template <int DV>
__global__ void __launch_bounds__(kThreads) q4_unpack_kernel(Q4UnpackParams p) {
  constexpr int R = block_rows(DV), NS = DV / kScaleCols, NH = R / 16, NW = 4 / NH;   // NW words per row and piece
  const int stream = blockIdx.y;
  const int b = stream / p.G;
  const int lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
  const int blk = blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int t0 = blk * R;
  const int L = clamp_len(p.lens, b, p.t_max);
  if (t0 >= L) return;
  const u32x4 w = *reinterpret_cast<const u32x4*>(p.codes + (int64_t)stream * p.t_max * (DV / 2) + (int64_t)blk * kBlockBytes + lane * 16);
  const uint8_t* sc = p.scales + (int64_t)stream * p.t_max * NS;
  uint16_t* out = p.v + (int64_t)stream * p.t_max * DV;
#pragma unroll
  for (int hf = 0; hf < NH; ++hf) {
    const int t = t0 + 16 * hf + n;
    if (t >= L) continue;
    const unsigned byte = sc[scale_off(t, q * (DV / 4) / kScaleCols, DV)];
#pragma unroll
    for (int k = 0; k < NW; ++k)
      *reinterpret_cast<bf16x8*>(out + tiled_off<uint16_t>(t, q * (DV / 4) + 8 * k, DV)) = dequant8(w[hf * NW + k], byte);
  }
}

// ================================================================ decode
struct Q4DecodeParams {
  DecodeArgs a;                                // a.v: the codes
  const uint8_t* scales;
};

template <int DV, int NRC>
struct Q4Tile {
  u32x4 w[DV / 64];                            // codes of 32 rows
  unsigned s;                                  // scale bytes of rows n (low) and n + 16
  bf16x8 k[2][NRC > 0 ? NRC : 1];
};

// One (sequence, group, split) per workgroup; its waves take interleaved tiles
// of 32 rows.  As in the bf16 kernel a head has two columns of the products, its
// absorbed query (and its softmax weights) as bf16 high and low parts.
template <int HPG, int DV, int NRC>
__global__ void __launch_bounds__(kThreads) q4_decode_kernel(Q4DecodeParams p) {
  const DecodeArgs& a = p.a;
  constexpr int NC = DV / 32, NB = DV / 16, NS = DV / kScaleCols, DEPTH = 4, NW = kWaves;
  constexpr int RS = DV + 2;
  using TileT = Q4Tile<DV, NRC>;
  __shared__ __attribute__((aligned(16))) float red[NW * HPG * RS];
  int b, s, g;
  bool empty_slot;
  if (!work_item(a, b, s, g, empty_slot)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, qd = lane >> 4;
  const int h0 = g * HPG;
  const bool active = n < 2 * HPG;
  const bool is_lo = n >= HPG;
  const int hq = h0 + (!active ? 0 : (is_lo ? 2 * HPG - 1 - n : n));
  const bf16x8 zero8 = as_bf16x8(u32x4{0u, 0u, 0u, 0u});
  const int L = clamp_len(a.lens, b, a.t_max);
  int r0, r1;
  split_rows(L, a.S, a.split_rows, s, r0, r1);
  if ((empty_slot || r0 >= r1) && s > 0) {
    if (tid < HPG) a.lse_part[((int64_t)b * a.H + h0 + tid) * a.S + s] = -INFINITY;
    return;
  }
  const int r1c = (r1 + 31) / 32 * 32;         // descriptors end with the split's last tile

  const int64_t stream = (int64_t)b * a.G + g;
  const __amdgpu_buffer_rsrc_t vres = __builtin_amdgcn_make_buffer_rsrc(
      static_cast<uint8_t*>(a.v) + stream * a.t_max * (DV / 2), (short)0, r1c * (DV / 2), kBufferWord3);
  const __amdgpu_buffer_rsrc_t sres = __builtin_amdgcn_make_buffer_rsrc(
      const_cast<uint8_t*>(p.scales) + stream * a.t_max * NS, (short)0, r1c * NS, kBufferWord3);
  const int r1k = (r1 + 15) / 16 * 16;
  const __amdgpu_buffer_rsrc_t kres = __builtin_amdgcn_make_buffer_rsrc(
      static_cast<uint16_t*>(a.kr) + (int64_t)b * a.t_max * a.d_r, (short)0, r1k * a.d_r * 2, kBufferWord3);
  int k_lane[NRC > 0 ? NRC : 1];
#pragma unroll
  for (int rc = 0; rc < NRC; ++rc) k_lane[rc] = min(4 * rc + qd, a.d_r / 8 - 1) * 256 + n * 16;
  const int s_lane = (qd * NS / 4 * 16 + n) * 2;
  const int ntiles = (r1 - r0 + kTileRows - 1) / kTileRows;
  const int my_tiles = ntiles > w ? (ntiles - w + NW - 1) / NW : 0;
  auto tile_row = [&](int j) { return r0 + (w + NW * j) * kTileRows; };
  auto load_tile = [&](TileT& t, int row0) {
#pragma unroll
    for (int u = 0; u < DV / 64; ++u)
      t.w[u] = __builtin_amdgcn_raw_buffer_load_b128(vres, lane * 16 + u * kBlockBytes, row0 * (DV / 2), kAuxNT);
    t.s = __builtin_amdgcn_raw_buffer_load_b16(sres, s_lane, row0 * NS, kAuxNT);
#pragma unroll
    for (int hf = 0; hf < 2; ++hf)
#pragma unroll
      for (int rc = 0; rc < NRC; ++rc)
        t.k[hf][rc] = as_bf16x8(__builtin_amdgcn_raw_buffer_load_b128(kres, k_lane[rc], (row0 + 16 * hf) * a.d_r * 2, 0));
  };
  TileT buf[DEPTH];
#pragma unroll
  for (int d = 0; d < DEPTH - 1; ++d) {
    load_tile(buf[d], tile_row(d));
    __builtin_amdgcn_sched_barrier(0);
  }

  // the query operands, columns in the codes' order
  bf16x8 bq[NC], bk[NRC > 0 ? NRC : 1];
  {
    const float* qa = a.q_abs + ((int64_t)b * a.H + hq) * DV + qd * (DV / 4);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = qa[8 * c + j] * a.scale_log2;
      bq[c] = active ? split_hi_lo(x, is_lo) : zero8;
    }
#pragma unroll
    for (int rc = 0; rc < NRC; ++rc) {
      const bool in_range = 32 * rc + 8 * qd < a.d_r;
      const float* qr = a.q_rot + ((int64_t)b * a.H + hq) * a.d_r + min(32 * rc + 8 * qd, a.d_r - 8);
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = qr[j] * a.scale_log2;
      bk[rc] = (active && in_range) ? split_hi_lo(x, is_lo) : zero8;
    }
  }
  // identity selectors for the V transpose
  bf16x8 esel[2];
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    u32x4 u = {0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (8 * qd + j == n + 16 * half) u[j >> 1] |= 0x3F80u << (16 * (j & 1));
    esel[half] = as_bf16x8(u);
  }

  float m_run = -__FLT_MAX__, l_run = 0.f;
  f32x4 acc[NB];
#pragma unroll
  for (int ib = 0; ib < NB; ++ib) acc[ib] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto compute_tile = [&](TileT& t, int row0) {
    bf16x8 v[2][NC];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      const unsigned byte = hf ? t.s >> 8 & 255u : t.s & 255u;
#pragma unroll
      for (int c = 0; c < NC; ++c) v[hf][c] = dequant8(t.w[DV == 128 ? hf : 0][DV == 128 ? c : 2 * hf + c], byte);
    }
    const bool tail = row0 + kTileRows > r1;
    if (tail) {                                // rows past the end may hold anything
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const bool dead = row0 + 16 * hf + n >= r1;
#pragma unroll
        for (int c = 0; c < NC; ++c) v[hf][c] = dead ? zero8 : v[hf][c];
#pragma unroll
        for (int rc = 0; rc < NRC; ++rc) t.k[hf][rc] = dead ? zero8 : t.k[hf][rc];
      }
    }
    float x[8];
#pragma unroll
    for (int hf = 0; hf < 2; ++hf) {
      f32x4 sc = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int c = 0; c < NC; ++c) sc = mfma16(v[hf][c], bq[c], sc);
#pragma unroll
      for (int rc = 0; rc < NRC; ++rc) sc = mfma16(t.k[hf][rc], bk[rc], sc);
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        x[4 * hf + jj] = sc[jj] + mirror<HPG>(sc[jj]);
        if (tail && row0 + 16 * hf + 4 * qd + jj >= r1) x[4 * hf + jj] = -INFINITY;
      }
    }
    float mt = x[0];
#pragma unroll
    for (int k = 1; k < 8; ++k) mt = fmaxf(mt, x[k]);
    mt = max_over_rows(mt);
    const float m_new = fmaxf(m_run, mt);
    if (__ballot(m_new > m_run) != 0) {
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int ib = 0; ib < NB; ++ib) acc[ib] *= alpha;
      m_run = m_new;
    }
    float pr[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      pr[k] = __builtin_amdgcn_exp2f(x[k] - m_run);
      l_run += pr[k];
    }
    const bf16x8 bp = active ? split_hi_lo(pr, is_lo) : zero8;
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        const f32x4 z = {0.f, 0.f, 0.f, 0.f};
        const f32x4 t0 = mfma16(v[0][c], esel[half], z);
        const f32x4 t1 = mfma16(v[1][c], esel[half], z);
        bf16x8 at;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          at[j] = (__bf16)t0[j];
          at[4 + j] = (__bf16)t1[j];
        }
        acc[2 * c + half] = mfma16(at, bp, acc[2 * c + half]);
      }
  };
  for (int jt = 0; jt < my_tiles; jt += DEPTH) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) {
      const int j = jt + d;
      if (j >= my_tiles) break;
      load_tile(buf[(d + DEPTH - 1) % DEPTH], tile_row(j + DEPTH - 1));
      __builtin_amdgcn_sched_barrier(0);
      compute_tile(buf[d], tile_row(j));
    }
  }

  // ---- merge the waves and write this split's partial
  l_run = sum_over_rows(l_run);
  if (l_run == 0.f) m_run = -INFINITY;         // no row counted
#pragma unroll
  for (int ib = 0; ib < NB; ++ib)
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) acc[ib][jj] += mirror<HPG>(acc[ib][jj]);
  if (n < HPG) {
    float* rec = red + (w * HPG + n) * RS;
    if (qd == 0) {
      rec[0] = m_run;
      rec[1] = l_run;
    }
    // output row k = 4 qd + jj + 16 half of product c is column 8 c + k % 8 of piece k / 8
#pragma unroll
    for (int ib = 0; ib < NB; ++ib)
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) {
        const int k = 4 * qd + jj + 16 * (ib & 1);
        rec[2 + (k >> 3) * (DV / 4) + 8 * (ib >> 1) + (k & 7)] = acc[ib][jj];
      }
  }
  __syncthreads();
  for (int idx = tid; idx < HPG * DV; idx += kThreads) {
    const int hl = idx / DV, i = idx % DV;
    float mx = -INFINITY;
#pragma unroll
    for (int ww = 0; ww < NW; ++ww) mx = fmaxf(mx, red[(ww * HPG + hl) * RS]);
    float o = 0.f, lsum = 0.f;
    if (mx != -INFINITY) {
#pragma unroll
      for (int ww = 0; ww < NW; ++ww) {
        const float* rec = red + (ww * HPG + hl) * RS;
        const float sc = rec[0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(rec[0] - mx);
        lsum += rec[1] * sc;
        o += rec[2 + i] * sc;
      }
      o /= lsum;
    }
    const int64_t row = ((int64_t)b * a.H + h0 + hl) * a.S + s;
    a.o_part[row * DV + i] = o;
    if (i == 0) a.lse_part[row] = mx == -INFINITY ? -INFINITY : (mx + log2f(lsum)) * kLn2;
  }
}

using Q4DecodeFn = void (*)(Q4DecodeParams);

template <int HPG, int DV>
Q4DecodeFn pick_q4_nrc(int nrc) {
  switch (nrc) {
    case 0: return q4_decode_kernel<HPG, DV, 0>;
    case 1: return q4_decode_kernel<HPG, DV, 1>;
    case 2: return q4_decode_kernel<HPG, DV, 2>;
  }
  return nullptr;
}

Q4DecodeFn pick_q4_decode(int hpg, int dv, int nrc) {
  const bool wide = dv == 128;
  switch (hpg) {
    case 1: return wide ? pick_q4_nrc<1, 128>(nrc) : pick_q4_nrc<1, 64>(nrc);
    case 2: return wide ? pick_q4_nrc<2, 128>(nrc) : pick_q4_nrc<2, 64>(nrc);
    case 4: return wide ? pick_q4_nrc<4, 128>(nrc) : pick_q4_nrc<4, 64>(nrc);
    case 8: return wide ? pick_q4_nrc<8, 128>(nrc) : pick_q4_nrc<8, 64>(nrc);
  }
  return nullptr;
}

struct Q4StepLayout {
  size_t q_abs, q_rot, o_part, lse_part, bytes;   // offsets into the workspace
};

int q4_step_layout(const gva_dims* d, int32_t num_splits, int32_t split_rows, Q4StepLayout& L) {
  int st = check_q4_dims(d);
  if (st != GVA_OK) return st;
  if (num_splits < 1 || num_splits > GVA_MAX_SPLITS || split_rows < 0 || split_rows % kTileRows != 0)
    return GVA_ERR_INVALID_ARG;
  const size_t rows = (size_t)d->batch * (size_t)d->n_heads;
  L = Q4StepLayout{};
  size_t off = round256(rows * (size_t)d->d_v * 4);
  L.q_rot = off;
  off += round256(rows * (size_t)d->d_r * 4);
  if (num_splits > 1) {
    L.o_part = off;
    off += round256(rows * (size_t)num_splits * (size_t)d->d_v * 4);
    L.lse_part = off;
    off += round256(rows * (size_t)num_splits * 4);
  }
  L.bytes = off;
  return GVA_OK;
}

}  // namespace

extern "C" {

int gva_q4_append_kv(const gva_dims* dims, void* v4_cache, void* v4_scale, void* kr_cache, const void* v_new,
                     const void* kr_new, const int32_t* seq, const int32_t* row, const int32_t* pos, int32_t n_rows,
                     int32_t* row_pos, void* stream) {
  int st = check_dims(dims);
  if (st != GVA_OK) return st;
  if (n_rows < 0) return GVA_ERR_INVALID_ARG;
  if (n_rows == 0) return GVA_OK;
  if (!v4_cache || !v4_scale || !v_new || !seq || !row) return GVA_ERR_INVALID_ARG;
  if (dims->d_r > 0 && (!kr_cache || !kr_new)) return GVA_ERR_INVALID_ARG;
  if (!aligned(v4_cache, 16) || !aligned(v4_scale, 16) || !aligned(v_new, 16) || !aligned(seq, 4) || !aligned(row, 4) ||
      !aligned(pos, 4) || !aligned(row_pos, 4))
    return GVA_ERR_INVALID_ARG;
  if (dims->d_r > 0 && (!aligned(kr_cache, 16) || !aligned(kr_new, 4))) return GVA_ERR_INVALID_ARG;
  st = check_q4_dims(dims);
  if (st != GVA_OK) return st;
  Q4AppendParams p{};
  p.codes = static_cast<uint8_t*>(v4_cache);
  p.scales = static_cast<uint8_t*>(v4_scale);
  p.kr_cache = static_cast<uint16_t*>(kr_cache);
  p.v_new = static_cast<const uint16_t*>(v_new);
  p.kr_new = static_cast<const uint16_t*>(kr_new);
  p.seq = seq;
  p.row = row;
  p.pos = pos;
  p.row_pos = row_pos;
  p.B = dims->batch;
  p.G = dims->n_groups;
  p.t_max = dims->t_max;
  p.d_r = dims->d_r;
  p.n_rows = n_rows;
  fill_inv_freq(dims, p.inv_freq);
  const int R = block_rows(dims->d_v);
  const long long gblocks = (dims->n_groups + kWaves - 1) / kWaves;
  const long long pairs = (R * (dims->d_r / 2) + kThreads - 1) / kThreads;
  if (gblocks + pairs > 65535) return GVA_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)((n_rows + (long long)R - 1) / R), (unsigned)(gblocks + pairs));
  hipLaunchKernelGGL((dims->d_v == 128 ? q4_append_kernel<128> : q4_append_kernel<64>), grid, dim3(kThreads), 0,
                     static_cast<hipStream_t>(stream), p);
  return launch_status();
}

int gva_q4_unpack_kv(const gva_dims* dims, const void* v4_cache, const void* v4_scale, const int32_t* lens,
                     void* v_cache, void* stream) {
  int st = check_dims(dims);
  if (st != GVA_OK) return st;
  if (!v4_cache || !v4_scale || !lens || !v_cache) return GVA_ERR_INVALID_ARG;
  if (!aligned(v4_cache, 16) || !aligned(v4_scale, 16) || !aligned(lens, 4) || !aligned(v_cache, 16))
    return GVA_ERR_INVALID_ARG;
  st = check_q4_dims(dims);
  if (st != GVA_OK) return st;
  const long long streams = (long long)dims->batch * dims->n_groups;
  if (streams > 65535) return GVA_ERR_UNSUPPORTED;
  Q4UnpackParams p{static_cast<const uint8_t*>(v4_cache), static_cast<const uint8_t*>(v4_scale), lens,
                   static_cast<uint16_t*>(v_cache), dims->batch, dims->n_groups, dims->t_max};
  const int blocks = dims->t_max / block_rows(dims->d_v);
  const dim3 grid((unsigned)((blocks + kWaves - 1) / kWaves), (unsigned)streams);
  hipLaunchKernelGGL((dims->d_v == 128 ? q4_unpack_kernel<128> : q4_unpack_kernel<64>), grid, dim3(kThreads), 0,
                     static_cast<hipStream_t>(stream), p);
  return launch_status();
}

int gva_q4_pick_splits(const gva_dims* dims, int32_t max_len, int64_t total_len, int32_t n_cu, int32_t* split_rows) {
  return gva_pick_splits(dims, max_len, total_len, n_cu, split_rows);
}

int gva_q4_decode_workspace_size(const gva_dims* dims, int32_t num_splits, int32_t split_rows, size_t* bytes) {
  if (bytes == nullptr) return GVA_ERR_INVALID_ARG;
  Q4StepLayout L;
  const int st = q4_step_layout(dims, num_splits, split_rows, L);
  if (st != GVA_OK) return st;
  *bytes = L.bytes;
  return GVA_OK;
}

int gva_q4_decode_step(const gva_dims* dims, const void* q, const void* m, const void* v4_cache, const void* v4_scale,
                       const void* kr_cache, const int32_t* lens, const int32_t* seen, int32_t num_splits,
                       int32_t split_rows, void* workspace, size_t workspace_bytes, float* o, float* lse,
                       void* stream) {
  Q4StepLayout L;
  int st = q4_step_layout(dims, num_splits, split_rows, L);
  if (st != GVA_OK) return st;
  if (!q || !m || !v4_cache || !v4_scale || !lens || !o || !lse) return GVA_ERR_INVALID_ARG;
  if (dims->d_r > 0 && !kr_cache) return GVA_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(m, 16) || !aligned(v4_cache, 16) || !aligned(v4_scale, 16) || !aligned(lens, 4) ||
      !aligned(seen, 4) || !aligned(o, 16) || !aligned(lse, 4) || (dims->d_r > 0 && !aligned(kr_cache, 16)))
    return GVA_ERR_INVALID_ARG;
  if (L.bytes > 0 && (workspace == nullptr || workspace_bytes < L.bytes || !aligned(workspace, 256)))
    return GVA_ERR_INVALID_ARG;
  if (dims->d_c % 32 != 0 || dims->d_c < 32 || dims->d_c > 512) return GVA_ERR_UNSUPPORTED;
  const int hpg = dims->n_heads / dims->n_groups;
  const Q4DecodeFn fn = pick_q4_decode(hpg, dims->d_v, (dims->d_r + 31) / 32);
  const long long n_items = decode_grid(dims, num_splits, split_rows);
  if (fn == nullptr || n_items > 0x7FFFFFFFLL) return GVA_ERR_UNSUPPORTED;
  char* ws = static_cast<char*>(workspace);
  float* q_abs = reinterpret_cast<float*>(ws + L.q_abs);
  float* q_rot = dims->d_r > 0 ? reinterpret_cast<float*>(ws + L.q_rot) : nullptr;
  const int S = num_splits;
  gva_dims at = *dims;                         // the query's position counts the tokens seen, not the rows left
  if (seen != nullptr) at.t_max = 0x7FFFFFFF;
  st = gva_absorb_query(&at, q, m, seen != nullptr ? seen : lens, q_abs, q_rot, stream);
  if (st != GVA_OK) return st;
  Q4DecodeParams p{};
  p.a.q_abs = q_abs;
  p.a.q_rot = q_rot;
  p.a.v = const_cast<void*>(v4_cache);
  p.a.kr = const_cast<void*>(kr_cache);
  p.a.lens = lens;
  p.a.o_part = S > 1 ? reinterpret_cast<float*>(ws + L.o_part) : o;
  p.a.lse_part = S > 1 ? reinterpret_cast<float*>(ws + L.lse_part) : lse;
  p.a.B = dims->batch;
  p.a.H = dims->n_heads;
  p.a.G = dims->n_groups;
  p.a.d_v = dims->d_v;
  p.a.d_c = dims->d_c;
  p.a.d_r = dims->d_r;
  p.a.t_max = dims->t_max;
  p.a.S = S;
  p.a.split_rows = split_rows;
  p.a.scale_log2 = scale_log2(dims);
  p.scales = static_cast<const uint8_t*>(v4_scale);
  hipLaunchKernelGGL(fn, dim3((unsigned)n_items), dim3(kThreads), 0, static_cast<hipStream_t>(stream), p);
  st = launch_status();
  if (st != GVA_OK || S == 1) return st;
  return gva_combine(dims, p.a.o_part, p.a.lse_part, S, o, lse, stream);
}

}  // extern "C"
