// libgva.so -- a value cache held in 4 bits: append, unpack, decode.
//
// A cached value row is kept as e2m1 codes (sign and one of 0, .5, 1, 1.5, 2,
// 3, 4, 6) with one power-of-two scale byte per 32 columns, the element and
// scale types that the matrix cores' converters read:
//   value = code * 2^(byte - 127),   byte 255: NaN
// The scale is the smallest 2^e with amax <= 7 * 2^e, -119 <= e <= 125: up to
// 7 an element that saturates at 6 is off by at most 2^e, no more than one
// between 4 and 6 is, and the finer scale pays for it (rms error of N(0, 1)
// rows 0.112; 0.115 with amax <= 6 * 2^e and with floor(log2 amax) - 2).  (Past 7 *
// 2^125 there is no larger scale, and the last bf16 numbers are off by up to twice
// that.)  Every
// value is exactly a bf16: codes have two significant bits, and the bounds on e
// keep 0.5 * 2^e normal and 6 * 2^e finite.
// A row takes 4.25 bits an element, 576 B at G = 8, d_v = 128, d_r = 16 against
// 2080 B in bf16 (the positional key, 1/65 of a bf16 row, stays bf16).
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
// have workgroups of their own.  A few rows are bound by the launch (8 rows of
// G4 d 64: 2.5 us), a prompt by that and HBM: 8192 rows of G8 d 128/16 (22 MB) in
// 6.7 us, 3.3 TB/s.
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
// consecutive rows.  Bound by HBM: 8 sequences of 4K to 8K rows, G8 d 128 (127 MB),
// 20.2 us, 6.3 TB/s, with streaming stores (25.5 without).
template <int DV>
__global__ void __launch_bounds__(kThreads) q4_unpack_kernel(Q4UnpackParams p) {
  constexpr int R = block_rows(DV), NS = DV / kScaleCols, NH = R / 16, NW = 4 / NH;   // NW words per row and piece
  const int per = (p.t_max / R + kWaves - 1) / kWaves;   // workgroups of a stream
  const int stream = blockIdx.x / per;
  const int b = stream / p.G;
  const int lane = threadIdx.x & 63, n = lane & 15, q = lane >> 4;
  const int blk = blockIdx.x % per * kWaves + (threadIdx.x >> 6);
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
      __builtin_nontemporal_store(__builtin_bit_cast(u32x4, dequant8(w[hf * NW + k], byte)),
                                  reinterpret_cast<u32x4*>(out + tiled_off<uint16_t>(t, q * (DV / 4) + 8 * k, DV)));
  }
}

// ================================================================ decode
struct Q4DecodeParams {
  DecodeArgs a;                                // a.v: the codes
  const uint8_t* scales;
  double inv_freq[kMaxPairs];
};

// The leading scalar arguments, in registers before a wave starts (see
// GVA_DECODE_HEAD_ARGS): what the first memory requests need.  head_q, head_m:
// the raw query and the maps, or the absorbed and the rotated query.  head_seen:
// NULL, or the tokens that each sequence has had.
#define GVA_Q4_HEAD_ARGS                                                                                       \
  const int32_t *head_lens, const int32_t *head_seen, const void *head_q, const void *head_m, void *head_codes, \
      int32_t head_dims, int32_t head_B, int32_t head_G, int32_t head_split_rows

template <int HPG, int DV, int NRC, int NW>
struct Q4Cfg {
  // tiles in registers (two leave room for a third workgroup of four waves on a CU
  // at d_v = 128: B64 to 8K rows H32 G8, chunks of 2560, 35.5 -> 29.6 us); waves
  // per SIMD at least
  static constexpr int DEPTH = NW > kWaves || DV == 128 ? 2 : 3, OCC = 2;
  // absorption: loads of four map rows (of 128 columns) per round, so that the
  // heads' maps are one round over the waves where registers allow it
  static constexpr int AR0 = DV * HPG / (4 * NW);
  static constexpr int AR = AR0 < 4 ? 4 : (AR0 > 16 ? 16 : AR0);
  static constexpr int QS = DV + 4, QR = 32 * NRC + 4;   // padded rows of the query in LDS (floats)
  static constexpr int PITCH = DV * 2 + 16;    // bytes of a row of the wave's tile in LDS
};

template <int DV, int NRC>
struct Q4Tile {
  u32x4 w[DV / 64];                            // codes of 32 rows
  unsigned s;                                  // scale bytes of rows n (low) and n + 16
  bf16x8 k[2][NRC > 0 ? NRC : 1];
};

// Eight bf16 of column n of an LDS tile: four rows at p and four at p + step.
// Within 16 lanes ds_read_b64_tr_b16 takes four values from each lane's address,
// lanes 4 r .. 4 r + 3 a row of 16, and hands lane n column n of the four rows.
__device__ __forceinline__ bf16x8 read_transposed(const uint8_t* p, int step) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4* Lds;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + step));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

// Part k of eight floats as a sum of three bf16, each rounded to nearest.
__device__ __forceinline__ bf16x8 split_part(const float* x, int k) {
  bf16x8 out;
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    f32x2 v = {x[j], x[j + 1]};
    bf16x2 h = __builtin_convertvector(v, bf16x2);
#pragma unroll
    for (int i = 1; i < 3; ++i)
      if (k >= i) {
        v = v - __builtin_convertvector(h, f32x2);
        h = __builtin_convertvector(v, bf16x2);
      }
    out[j] = h[0];
    out[j + 1] = h[1];
  }
  return out;
}

// The largest of three (a NaN among them is passed over); fmaxf chains quiet every
// operand with an instruction of its own first.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(d) : "v"(a), "v"(b), "v"(c));
  return d;
}

// One (sequence, group, split) per workgroup; its waves take interleaved tiles
// of 32 rows.  As in the bf16 kernel a head has two columns of the products, its
// absorbed query (and its softmax weights) as bf16 high and low parts, and with
// FUSED the workgroup absorbs its heads' queries itself while its first tiles
// are on their way.  Up to four heads a group leave columns 8 .. 15 free: column
// 15 - n takes the query's third part for high column n, one more addition a
// score (o is off by 5e-7 of its norm at B32 T8K H32 G8 d 128/16, by 2.5e-6 without;
// 36.1 against 34.9 us).  Eight heads would need products of their own for it, and
// the registers of a third workgroup (6 to 9% of the time): they have two parts.
// The weights have a third part in the same columns where a wave has at most four
// tiles: the roundings of few rows show most (256 rows of H8 G2 d 64: 1.2e-6 with
// two parts, 1.3e-7 with three; 5.7 and 5.9 us), and in every tile of a long split
// it costs 2 to 5% for an error that is below 1e-6 already.
//
// A tile is converted once, in the score products' operand order, and goes
// through the wave's LDS for the transposed operand of P.V, a tile later.  At d_v
// = 128 a tile takes the loop about 235 cycles of a CU, which nothing fills alone: HBM's
// share is 177, LDS 176 (8 KB written, 8 KB read), vector work 134, matrix products
// 77.  What is lost is overlap, with one workgroup of eight waves on a CU (V^T by
// products with an identity, which need no LDS, was slower: 16 more of them a tile).
// B32 T8K H32 G8 d 128/16 (153 MB): 36.4 to 38.9 us on different GPUs, 3.9 to 4.2 TB/s,
// of which about 7.5 are the start, the absorption and the end, which nothing hides;
// B4 of 64K to 128K rows (240 MB) 51 to 52 and 5 for the combine.
template <int HPG, int DV, int NRC, int NW, bool FUSED>
__global__ void __launch_bounds__(64 * NW, (Q4Cfg<HPG, DV, NRC, NW>::OCC)) q4_decode_kernel(GVA_Q4_HEAD_ARGS,
                                                                                            Q4DecodeParams p) {
  using Cfg = Q4Cfg<HPG, DV, NRC, NW>;
  using TileT = Q4Tile<DV, NRC>;
  constexpr int NC = DV / 32, NB = DV / 16, NS = DV / kScaleCols, DEPTH = Cfg::DEPTH, NT = 64 * NW;
  constexpr int RS = DV + 2, PITCH = Cfg::PITCH, AR = Cfg::AR, QS = Cfg::QS, QR = Cfg::QR;
  constexpr int LDS_TR = NW * 32 * PITCH, LDS_RED = NW * HPG * RS * 4;
  __shared__ __attribute__((aligned(16))) uint8_t lds[LDS_TR > LDS_RED ? LDS_TR : LDS_RED];
  __shared__ __attribute__((aligned(16))) float qlds[FUSED ? HPG * (QS + QR) : 1];
  DecodeArgs a = p.a;
  a.lens = head_lens;
  a.v = head_codes;
  a.d_c = head_dims & 1023;
  a.d_r = head_dims >> 10 & 127;
  a.S = head_dims >> 17 & 511;
  a.B = head_B;
  a.G = head_G;
  a.H = head_G * HPG;
  a.split_rows = head_split_rows;

  int b, s, g;
  bool empty_slot;
  if (!work_item(a, b, s, g, empty_slot)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, qd = lane >> 4;
  const int h0 = g * HPG;
  const bool third = HPG <= 4 && n >= 8;       // the mirror column's third part
  const int col = third ? 15 - n : n;
  const bool active = col < 2 * HPG;
  const bool is_lo = col >= HPG;
  const int col_head = !active ? 0 : (is_lo ? 2 * HPG - 1 - col : col);
  auto query_part = [&](const float* x) {
    return !active || (third && is_lo) ? as_bf16x8(u32x4{0u, 0u, 0u, 0u}) : split_part(x, third ? 2 : (is_lo ? 1 : 0));
  };
  const bf16x8 zero8 = as_bf16x8(u32x4{0u, 0u, 0u, 0u});
  const int len_b = *(const __attribute__((address_space(4))) int32_t*)(head_lens + b);
  const int32_t* const seen_at = head_seen != nullptr ? head_seen : head_lens;
  const int seen_b = *(const __attribute__((address_space(4))) int32_t*)(seen_at + b);
  if (empty_slot && s > 0) {                   // bounded chunks: a split with no rows
    if (tid < HPG) a.lse_part[((int64_t)b * a.H + h0 + tid) * a.S + s] = -INFINITY;
    return;
  }

  // ---- the query's loads, which need no length.  Absorption, q~[i] = sum_k
  // q[k] M_h[i][k]: a job is 4 AR rows of a head's map, wave w taking jobs w, w +
  // NW, ...; a load covers four whole rows of 128 columns (16 lanes of 16 bytes).
  constexpr int ARB = DV / 4 / AR, NJOB = HPG * ARB;
  const int W = a.d_c + a.d_r;
  const int a_row = lane >> 4, a_col = 8 * (lane & 15);
  u32x4 am[FUSED ? AR : 1], xq = {0u, 0u, 0u, 0u};
  f32x4 xa[FUSED ? 1 : NC][2], xr[NRC > 0 ? NRC : 1][2];
  const int npair = a.d_r / 2, ptid = NT - 1 - tid;
  const bool has_pair = FUSED && ptid < HPG * npair;
  const int pair_h = npair > 0 ? ptid / npair : 0, pair_i = npair > 0 ? ptid % npair : 0;
  uint32_t rq_bits = 0u;
  double qfreq = 0.0;
  auto load_round = [&](int job, int seg) {    // columns past d_c: a valid piece, against zeros of the query
    const int h = h0 + job / ARB, i0 = (job % ARB) * 4 * AR + a_row, col = min(128 * seg + a_col, a.d_c - 8);
    const uint16_t* mh = static_cast<const uint16_t*>(head_m) + ((int64_t)h * DV + i0) * a.d_c + col;
    xq = *reinterpret_cast<const u32x4*>(static_cast<const uint16_t*>(head_q) + ((int64_t)b * a.H + h) * W + col);
#pragma unroll
    for (int r = 0; r < AR; ++r) am[r] = *reinterpret_cast<const u32x4*>(mh + (int64_t)(4 * r) * a.d_c);
  };
  if constexpr (FUSED) {
    if (has_pair) {
      rq_bits = *reinterpret_cast<const uint32_t*>(static_cast<const uint16_t*>(head_q) +
                                                   ((int64_t)b * a.H + h0 + pair_h) * W + a.d_c + 2 * pair_i);
      qfreq = p.inv_freq[pair_i];
    }
    if (w < NJOB) load_round(w, 0);
  } else {
    const int hq = h0 + col_head;
    const float* qa = static_cast<const float*>(head_q) + ((int64_t)b * a.H + hq) * DV + qd * (DV / 4);
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      xa[c][0] = *reinterpret_cast<const f32x4*>(qa + 8 * c);
      xa[c][1] = *reinterpret_cast<const f32x4*>(qa + 8 * c + 4);
    }
#pragma unroll
    for (int rc = 0; rc < NRC; ++rc) {
      const float* qr = static_cast<const float*>(head_m) + ((int64_t)b * a.H + hq) * a.d_r + min(32 * rc + 8 * qd, a.d_r - 8);
      xr[rc][0] = *reinterpret_cast<const f32x4*>(qr);
      xr[rc][1] = *reinterpret_cast<const f32x4*>(qr + 4);
    }
  }
  __builtin_amdgcn_sched_barrier(0);
  request_args(a);
  asm volatile("" ::"s"(p.scales) : "memory");

  const int L = len_b < 0 ? 0 : (len_b > a.t_max ? a.t_max : len_b);
  int r0, r1;
  split_rows(L, a.S, a.split_rows, s, r0, r1);
  if (r0 >= r1 && s > 0) {                     // an empty split past the first: lse only
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
  const bool fine = ntiles <= 4 * NW;          // the weights in three parts
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

  // ---- the query operands, scaled, columns in the codes' order
  bf16x8 bq[NC], bk[NRC > 0 ? NRC : 1];
  if constexpr (FUSED) {
    float* const qs = qlds;                    // [HPG][QS]
    float* const qrs = qlds + HPG * QS;        // [HPG][QR]
    const int nseg = (a.d_c + 127) / 128;
    auto absorb_job = [&](int job, bool loaded) {
      float v[AR];
#pragma unroll
      for (int r = 0; r < AR; ++r) v[r] = 0.f;
      for (int seg = 0; seg < nseg; ++seg) {
        if (!(loaded && seg == 0)) load_round(job, seg);
        const u32x4 qv = 128 * seg + a_col < a.d_c ? xq : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int r = 0; r < AR; ++r) v[r] += dot8_bf16(am[r], qv);
      }
      float* dst = qs + job / ARB * QS + (job % ARB) * 4 * AR + a_row;
#pragma unroll
      for (int r = 0; r < AR; ++r) dst[4 * r] = sum16(v[r]) * a.scale_log2;   // every lane of a row the same value
    };
    if (w < NJOB) absorb_job(w, true);
    for (int job = w + NW; job < NJOB; job += NW) absorb_job(job, false);
    if (has_pair) {                            // the positional slice at the token's position
      const int at = head_seen != nullptr ? seen_b : L;
      float y0, y1;
      rotate_query_pair(bf16_bits_to_f32(rq_bits & 0xFFFFu), bf16_bits_to_f32(rq_bits >> 16),
                        (double)(at > 0 ? at - 1 : 0) * qfreq, a.scale_log2, y0, y1);
      qrs[pair_h * QR + 2 * pair_i] = y0;
      qrs[pair_h * QR + 2 * pair_i + 1] = y1;
    }
    if constexpr (NRC > 0) {
      for (int i = tid; i < HPG * 32 * NRC; i += NT)
        if (i % (32 * NRC) >= a.d_r) qrs[i / (32 * NRC) * QR + i % (32 * NRC)] = 0.f;
    }
    __syncthreads();
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const float* src = qs + col_head * QS + qd * (DV / 4) + 8 * c;
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = src[j];
      bq[c] = query_part(x);
    }
#pragma unroll
    for (int rc = 0; rc < NRC; ++rc) {
      const float* src = qrs + col_head * QR + 32 * rc + 8 * qd;
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = src[j];
      bk[rc] = query_part(x);
    }
  } else {
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = xa[c][j >> 2][j & 3] * a.scale_log2;
      bq[c] = query_part(x);
    }
#pragma unroll
    for (int rc = 0; rc < NRC; ++rc) {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = xr[rc][j >> 2][j & 3] * a.scale_log2;
      bk[rc] = 32 * rc + 8 * qd < a.d_r ? query_part(x) : zero8;
    }
  }
  // the wave's tile: where the lane writes its pieces, and where it reads V^T
  uint8_t* const tr = lds + w * 32 * PITCH;
  uint8_t* const tr_put = tr + n * PITCH + qd * (DV / 2);
  // The transposing LDS read hands lane (n, qd) column n of rows 4 qd .. 4 qd +
  // 3 (and 16 more), the order in which the score product returns the weights.
  const uint8_t* const tr_get = tr + (4 * qd + (n >> 2)) * PITCH + 8 * (n & 3);

  // no tile before the first: rows and weights of 0
  for (int i = lane * 16; i < 32 * PITCH; i += 64 * 16) *reinterpret_cast<u32x4*>(tr + i) = u32x4{0u, 0u, 0u, 0u};
  bf16x8 bp = zero8;
  float m_run = 0.f, m_limit = -INFINITY;      // no maximum yet: any score sets it
  f32x4 start = {0.f, 0.f, 0.f, 0.f};          // of the score products: -m_run in the high columns
  f32x4 l_run = {0.f, 0.f, 0.f, 0.f};          // the sum of a column's weights, four times
  // x - y, exact where y is x rounded: a dot product with (-1, 0) and (0, -1) each,
  // one instruction where a conversion and a subtraction are two (36.4 against 36.7
  // us at B32 T8K on one GPU).  The pairs are held in registers: as constants they came out as
  // the bits of an fp32 -1, the wrong half of a pair for one of them.
  uint32_t minus_first = 0x0000BF80u, minus_second = 0xBF800000u;
  asm volatile("" : "+s"(minus_first), "+s"(minus_second));
  auto less = [&](f32x2 x, bf16x2 y) {
    return f32x2{__builtin_amdgcn_fdot2_f32_bf16(y, __builtin_bit_cast(bf16x2, minus_first), x[0], false),
                 __builtin_amdgcn_fdot2_f32_bf16(y, __builtin_bit_cast(bf16x2, minus_second), x[1], false)};
  };
  const bf16x8 ones = as_bf16x8(u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
  f32x4 acc[NB];
#pragma unroll
  for (int ib = 0; ib < NB; ++ib) acc[ib] = f32x4{0.f, 0.f, 0.f, 0.f};

  auto compute_tile = [&](TileT& t, int row0) {
    const bool tail = row0 + kTileRows > r1;
    unsigned scales = t.s;
    if (tail) {
      // Rows past the end may hold anything.  Codes are finite under a finite
      // scale, and those rows' weights are 0, so only the scales are replaced
      // (the key's NaN would reach only the row's own scores).
      __builtin_amdgcn_sched_barrier(0);
      if (row0 + n >= r1) scales = scales & ~255u | 127u;
      if (row0 + 16 + n >= r1) scales = scales & 255u | 127u << 8;
      __builtin_amdgcn_sched_barrier(0);
    }
    // V^T of the tile before; its P.V products go between this tile's
    // conversions and score products
    bf16x8 vt[NB];
#pragma unroll
    for (int ib = 0; ib < NB; ++ib) vt[ib] = read_transposed(tr_get + 32 * ib, 16 * PITCH);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();           // this tile is written after those reads
    f32x4 sc[2] = {start, start};
#pragma unroll
    for (int rc = 0; rc < NRC; ++rc)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) sc[hf] = mfma16(t.k[hf][rc], bk[rc], sc[hf]);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int hf = 0; hf < 2; ++hf) {
        const bf16x8 v = dequant8(t.w[DV == 128 ? hf : 0][DV == 128 ? c : 2 * hf + c], hf ? scales >> 8 : scales & 255u);
        *reinterpret_cast<bf16x8*>(tr_put + 16 * hf * PITCH + 16 * c) = v;
        sc[hf] = mfma16(v, bq[c], sc[hf]);
        acc[2 * c + hf] = mfma16(vt[2 * c + hf], bp, acc[2 * c + hf]);
      }
    l_run = mfma16(ones, bp, l_run);
    // Each of a head's two lanes takes the sum of the parts, and the exponential,
    // for one half of the rows: the high column's lane the first 16.
    float x[4];
    auto take_scores = [&]() {                   // and the largest of the lane's
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        x[j] = (is_lo ? sc[1][j] : sc[0][j]) + mirror<HPG>(is_lo ? sc[0][j] : sc[1][j]);
        if constexpr (HPG <= 4) x[j] = dpp_add<0x140>(x[j]);     // and the third part's, or to it
      }
      if (tail) {
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (row0 + (is_lo ? 16 : 0) + 4 * qd + j >= r1) x[j] = -INFINITY;
        __builtin_amdgcn_sched_barrier(0);
      }
      return max3(max3(x[0], x[1], x[2]), x[3], x[3]);
    };
    // The scores come less the running maximum (the products start from it), which
    // moves only when a column's score passes it by 8 (log2), or its first one
    // comes: until then weights stay below 2^8, and most tiles need neither the
    // maximum over the lanes nor the rescaling.
    const float mt = take_scores();
    if (__ballot(mt > m_limit) != 0) {
      const float top = max_over_rows(fmaxf(mt, mirror<HPG>(mt)));
      const bool moves = top > m_limit, some = m_limit != -INFINITY;
      float by = moves ? top : 0.f, next = m_run + by;
      if (__ballot(moves && some && top > 64.f) == 0) {
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] -= by;
      } else {
        // Started from a maximum far below them, scores have lost what tells them
        // apart (all of it, where the rows before were hidden by the lowest value
        // of a type): they are taken again, from 0.
        sc[0] = sc[1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int rc = 0; rc < NRC; ++rc)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
            sc[hf] = mfma16(as_bf16x8(__builtin_amdgcn_raw_buffer_load_b128(kres, k_lane[rc], (row0 + 16 * hf) * a.d_r * 2, 0)), bk[rc], sc[hf]);
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int hf = 0; hf < 2; ++hf)
            sc[hf] = mfma16(*reinterpret_cast<const bf16x8*>(tr_put + 16 * hf * PITCH + 16 * c), bq[c], sc[hf]);
        const float most = take_scores();
        const float again = max_over_rows(fmaxf(most, mirror<HPG>(most)));
        next = moves ? again : m_run;
        by = next - m_run;
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] -= next;
      }
      const float alpha = moves && some ? __builtin_amdgcn_exp2f(-by) : 1.f;
      l_run *= alpha;
#pragma unroll
      for (int ib = 0; ib < NB; ++ib) acc[ib] *= alpha;
      m_run = next;
      m_limit = moves ? 8.f : m_limit;
      const float s0 = is_lo || third ? 0.f : -m_run;
      start = f32x4{s0, s0, s0, s0};
    }
    // Weights as bf16 parts, each rounded to nearest: the high columns' own, in the
    // low columns that of what the high part leaves, and in the mirror columns, where
    // a split is short, that of the rest (two parts are together off by at most
    // 2^-17, three hold an fp32 number; a single one, 2^-8, would show in o at 1e-3).
    // The two lanes of a pair exchange what the other needs.  The sum of the weights
    // is a product with ones.
    u32x4 parts;
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const f32x2 e = {__builtin_amdgcn_exp2f(x[2 * j]), __builtin_amdgcn_exp2f(x[2 * j + 1])};
      const bf16x2 h = __builtin_convertvector(e, bf16x2);
      const f32x2 r = less(e, h);
      const bf16x2 l = __builtin_convertvector(r, bf16x2);
      uint32_t hb = __builtin_bit_cast(uint32_t, h), lb = __builtin_bit_cast(uint32_t, l);
      if constexpr (HPG <= 4) {
        if (fine) {
          const bf16x2 rest = __builtin_convertvector(less(r, l), bf16x2);
          hb = third ? __builtin_bit_cast(uint32_t, rest) : hb;
          lb = third ? __builtin_bit_cast(uint32_t, rest) : lb;
        }
      }
      if constexpr (HPG >= 4) {
        // high and low columns are whole banks of four lanes: each takes the other's
        // part where it is the one that lacks it
        constexpr int LO = HPG == 4 ? 6 : 12;
        parts[j] = (uint32_t)__builtin_amdgcn_update_dpp((int)hb, (int)lb, Mirror<HPG>::ctrl, 0xF, LO, false);
        parts[2 + j] = (uint32_t)__builtin_amdgcn_update_dpp((int)lb, (int)hb, Mirror<HPG>::ctrl, 0xF, 15 - LO, false);
      } else {
        const uint32_t keep = is_lo ? lb : hb, got = __float_as_uint(mirror<HPG>(__uint_as_float(is_lo ? hb : lb)));
        parts[j] = is_lo ? got : keep;
        parts[2 + j] = is_lo ? keep : got;
      }
    }
    bp = as_bf16x8(parts);
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();           // the tile's rows, written by the other lanes
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
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
#pragma unroll
  for (int ib = 0; ib < NB; ++ib) acc[ib] = mfma16(read_transposed(tr_get + 32 * ib, 16 * PITCH), bp, acc[ib]);
  l_run = mfma16(ones, bp, l_run);

  // ---- merge the waves and write this split's partial
  auto all_parts = [&](float y) {              // of a high column
    const float two = y + mirror<HPG>(y);
    return HPG <= 4 && fine ? two + mirror<8>(y) : two;
  };
  const float l_sum = all_parts(l_run[0]);
  if (l_sum == 0.f) m_run = -INFINITY;         // no row counted
#pragma unroll
  for (int ib = 0; ib < NB; ++ib)
#pragma unroll
    for (int jj = 0; jj < 4; ++jj) acc[ib][jj] = all_parts(acc[ib][jj]);
  __syncthreads();                             // the tiles' LDS holds the records from here on
  float* const red = reinterpret_cast<float*>(lds);
  if (n < HPG) {
    float* rec = red + (w * HPG + n) * RS;
    if (qd == 0) {
      rec[0] = m_run;
      rec[1] = l_sum;
    }
#pragma unroll
    for (int ib = 0; ib < NB; ++ib)
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) rec[2 + 16 * ib + 4 * qd + jj] = acc[ib][jj];
  }
  __syncthreads();
  for (int idx = tid; idx < HPG * DV; idx += 64 * NW) {
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

using Q4DecodeFn = void (*)(GVA_Q4_HEAD_ARGS, Q4DecodeParams);

template <int HPG, int DV, int NW, bool FUSED>
Q4DecodeFn pick_q4_nrc(int nrc) {
  switch (nrc) {
    case 0: return q4_decode_kernel<HPG, DV, 0, NW, FUSED>;
    case 1: return q4_decode_kernel<HPG, DV, 1, NW, FUSED>;
    case 2: return q4_decode_kernel<HPG, DV, 2, NW, FUSED>;
  }
  return nullptr;
}

// Eight waves absorb inside but for chunks of 4096 <= split_rows < 4 (H/G) d_c (see
// q4_waves, q4_fused), which takes four heads a group at least (d_c <= 512).
template <int HPG, int DV>
Q4DecodeFn pick_q4_waves(int nrc, int nw, bool fused) {
  if (nw == 8 && fused) return pick_q4_nrc<HPG, DV, 8, true>(nrc);
  if (nw == 8) {
    if constexpr (HPG >= 4) return pick_q4_nrc<HPG, DV, 8, false>(nrc);
    return nullptr;
  }
  return fused ? pick_q4_nrc<HPG, DV, 4, true>(nrc) : pick_q4_nrc<HPG, DV, 4, false>(nrc);
}

Q4DecodeFn pick_q4_decode(int hpg, int dv, int nrc, int nw, bool fused) {
  const bool wide = dv == 128;
  switch (hpg) {
    case 1: return wide ? pick_q4_waves<1, 128>(nrc, nw, fused) : pick_q4_waves<1, 64>(nrc, nw, fused);
    case 2: return wide ? pick_q4_waves<2, 128>(nrc, nw, fused) : pick_q4_waves<2, 64>(nrc, nw, fused);
    case 4: return wide ? pick_q4_waves<4, 128>(nrc, nw, fused) : pick_q4_waves<4, 64>(nrc, nw, fused);
    case 8: return wide ? pick_q4_waves<8, 128>(nrc, nw, fused) : pick_q4_waves<8, 64>(nrc, nw, fused);
  }
  return nullptr;
}

// The shapes that the step takes: a 4-bit cache's, the absorption's widths, and
// the heads per group that the kernel has columns for.
int check_q4_step_dims(const gva_dims* d) {
  const int st = check_q4_dims(d);
  if (st != GVA_OK) return st;
  const int hpg = d->n_heads / d->n_groups;
  if (hpg != 1 && hpg != 2 && hpg != 4 && hpg != 8) return GVA_ERR_UNSUPPORTED;
  return d->d_c % 32 != 0 || d->d_c < 32 || d->d_c > 512 ? GVA_ERR_UNSUPPORTED : GVA_OK;
}

// Workgroups that a CU holds at once, at least, by the registers of a lane: at d_v
// = 128 up to 164, 191 with a second chunk of the positional key (d_r > 32); at d_v
// = 64 up to 120 with eight waves and 144 with four, 143 and 170 with that chunk (168,
// which a third workgroup of four waves would fit, with the absorption outside or one
// head a group).
inline int q4_resident(const gva_dims* d, int nw) {
  const bool two_chunks = d->d_r > 32;
  if (nw == 8) return d->d_v == 128 || two_chunks ? 1 : 2;
  return two_chunks ? 2 : 3;
}

// Waves per workgroup: eight while the workgroups are resident at once; with
// bounded chunks (whose empty splits count among them) while a chunk is long and
// the streams are no more than the CUs.  us per step, eight and four waves: B32
// T8K H32 G8 d 128, 256 workgroups, 35.4 and 43.1; B64 T2K, 512, 28.0 and 23.5; B4
// of 64K to 128K rows, chunks of 13024, 54.8 and 67.4; B64 to 32K rows, H16 G2,
// chunks of 4096 30.0 and 33.0, of 2048 39.2 and 30.5; B64 to 8K rows, G8, chunks
// of 4096 41.4 and 30.8.  Even splits at d_v = 64, H32 G8: d_r = 16, 320 workgroups
// of T4K 21.3 and 23.7, 512 of T2K 16.1 and 16.0; d_r = 64, 320 of T4K 30.7 and 27.8,
// 512 of T2K 22.3 and 18.7, of T256 11.5 and 8.5.
int q4_waves(const gva_dims* d, int num_splits, int split_rows, int n_cu) {
  if (split_rows > 0) return split_rows >= 4096 && (long long)d->batch * d->n_groups <= n_cu ? 8 : kWaves;
  return decode_grid(d, num_splits, 0) <= (long long)n_cu * q4_resident(d, 8) ? 8 : kWaves;
}

// Whether the workgroups absorb their queries themselves: while they are resident
// at once, or a chunk's rows outweigh the (H/G) d_c map rows that its workgroup
// reads for it (us, inside and apart: B64 to 32K rows, H16 G2 d 128, chunks of
// 2048 rows against 1024 map rows, 30.6 and 29.7; B16 to 32K rows, H16 G4 d 64,
// 2048 against 256, 15.5 and 18.5; B128 T1K H32 G8 d 128, even, 29.1 and 27.9).
bool q4_fused(const gva_dims* d, int num_splits, int split_rows, int n_cu) {
  if (decode_grid(d, num_splits, split_rows) <= 2LL * n_cu) return true;
  return split_rows > 0 && split_rows >= 4LL * (d->n_heads / d->n_groups) * d->d_c;
}

// What a plan costs in microseconds, from the times above: a workgroup's start and
// end, its rows at the pace of its CU (which the workgroups there share), the
// absorption where it is a launch before, and the combine.  Only the order of two
// plans matters.  (With the absorption, and the workgroups that fit at d_r > 32,
// against without: B53 of 1K to 2K rows, H4 G1 d 128/16, 4 splits with it inside
// 12.0 us, 10 with it before 18.1; B17 to 10K rows, H32 G8 d 64/16, 14.2 and 17.2;
// B40 of 2K to 4K rows, H32 G8 d 128/40, chunks of 2912 30.8, of 1632 39.0.)
struct Q4Cost {
  int n_cu, groups, d_v;
  double us(const gva_dims* d, const int32_t* lens, int S, int c) const {
    const int nw = q4_waves(d, S, c, n_cu), most = q4_resident(d, nw);
    long long items = 0, rows = 0, longest = 0;
    for (int b = 0; b < d->batch; ++b) {
      const long long L = lens != nullptr ? (lens[b] < 0 ? 0 : (lens[b] > d->t_max ? d->t_max : lens[b])) : d->t_max;
      if (L == 0) continue;
      const long long n = c <= 0 ? S : ((L + c - 1) / c > S ? S : (L + c - 1) / c);
      const long long per = ((L + n - 1) / n + kTileRows - 1) / kTileRows * kTileRows;
      items += (L + per - 1) / per * groups;
      rows += L * groups;
      if (per > longest) longest = per;
    }
    const long long here = (items + n_cu - 1) / n_cu;
    const long long resident = here < 1 ? 1 : (here > most ? most : here);
    const double pace = d_v == 128 ? 290.0 : 500.0;      // rows per us of a CU with eight waves or more, 0.68 with four
    const double mean = (double)rows / n_cu / (pace * (resident * nw >= 8 ? 1.0 : 0.68));
    // the longest chunk, whose neighbours on the CU end before it
    const double last = (double)longest / (pace * (nw == 8 ? 1.0 : 0.68)) * (1.0 + 0.35 * (double)(resident - 1));
    const double rounds = (double)items / ((double)n_cu * most);
    double t = rounds <= 1.0 ? 7.0 + (last > mean ? last : mean) : 7.0 + 4.0 * (rounds - 1.0) + mean + last / 2;
    const double idle = (double)(decode_grid(d, S, c) - items) / ((double)n_cu * most);      // empty splits
    if (!q4_fused(d, S, c, n_cu)) t += 4.0;
    return t + (idle > 0 ? idle * 1.2 : 0.0) + (S > 1 ? 4.5 + 0.05 * S + (S > 16 ? 3.0 : 0.0) : 0.0);
  }
};

struct Q4StepLayout {
  bool fused;
  size_t q_abs, q_rot, o_part, lse_part, bytes;   // offsets into the workspace
};

int q4_step_layout(const gva_dims* d, int32_t num_splits, int32_t split_rows, Q4StepLayout& L) {
  const int st = check_q4_step_dims(d);
  if (st != GVA_OK) return st;
  if (num_splits < 1 || num_splits > GVA_MAX_SPLITS || split_rows < 0 || split_rows % kTileRows != 0)
    return GVA_ERR_INVALID_ARG;
  const size_t rows = (size_t)d->batch * (size_t)d->n_heads;
  L = Q4StepLayout{};
  L.fused = q4_fused(d, num_splits, split_rows, device_cu_count());
  size_t off = 0;
  if (!L.fused) {
    L.q_rot = off = round256(rows * (size_t)d->d_v * 4);
    off += round256(rows * (size_t)d->d_r * 4);
  }
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
  const int R = block_rows(dims->d_v);
  const long long grid = (long long)dims->batch * dims->n_groups * ((dims->t_max / R + kWaves - 1) / kWaves);
  if (grid > 0x7FFFFFFFLL) return GVA_ERR_UNSUPPORTED;
  Q4UnpackParams p{static_cast<const uint8_t*>(v4_cache), static_cast<const uint8_t*>(v4_scale), lens,
                   static_cast<uint16_t*>(v_cache), dims->batch, dims->n_groups, dims->t_max};
  hipLaunchKernelGGL((dims->d_v == 128 ? q4_unpack_kernel<128> : q4_unpack_kernel<64>), dim3((unsigned)grid), dim3(kThreads), 0,
                     static_cast<hipStream_t>(stream), p);
  return launch_status();
}

int gva_q4_pick_splits(const gva_dims* dims, const int32_t* lens, int32_t n_cu, int32_t* split_rows) {
  if (split_rows != nullptr) *split_rows = 0;
  if (check_q4_step_dims(dims) != GVA_OK) return 1;
  if (n_cu <= 0) n_cu = device_cu_count();
  const Q4Cost cost{n_cu, dims->n_groups, dims->d_v};
  int longest = 0;
  for (int b = 0; b < dims->batch; ++b) {
    const int L = lens != nullptr ? lens[b] : dims->t_max;
    if (L > longest) longest = L;
  }
  if (longest > dims->t_max) longest = dims->t_max;
  int best_s = 1, best_c = 0;
  double best = cost.us(dims, lens, 1, 0);
  auto look = [&](int S, int c) {
    const double t = cost.us(dims, lens, S, c);
    if (t < best) {
      best = t;
      best_s = S;
      best_c = c;
    }
  };
  for (int S = 2; S <= 32; ++S) look(S, 0);
  // bounded chunks, a 24th shorter each time
  if (split_rows != nullptr)
    for (int c = longest; c >= 256; c -= c / 24) {
      const int rows = (c + kTileRows - 1) / kTileRows * kTileRows, S = (longest + rows - 1) / rows;
      if (S > GVA_MAX_SPLITS) break;
      if (S > 1) look(S, rows);
    }
  if (split_rows != nullptr) *split_rows = best_c;
  return best_s;
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
  const int hpg = dims->n_heads / dims->n_groups;
  const int nw = q4_waves(dims, num_splits, split_rows, device_cu_count());
  const Q4DecodeFn fn = pick_q4_decode(hpg, dims->d_v, (dims->d_r + 31) / 32, nw, L.fused);
  const long long n_items = decode_grid(dims, num_splits, split_rows);
  if (fn == nullptr || n_items > 0x7FFFFFFFLL) return GVA_ERR_UNSUPPORTED;
  char* ws = static_cast<char*>(workspace);
  const int S = num_splits;
  float *q_abs = nullptr, *q_rot = nullptr;
  if (!L.fused) {
    q_abs = reinterpret_cast<float*>(ws + L.q_abs);
    q_rot = dims->d_r > 0 ? reinterpret_cast<float*>(ws + L.q_rot) : nullptr;
    gva_dims at = *dims;                       // the query's position counts the tokens seen, not the rows left
    if (seen != nullptr) at.t_max = 0x7FFFFFFF;
    st = gva_absorb_query(&at, q, m, seen != nullptr ? seen : lens, q_abs, q_rot, stream);
    if (st != GVA_OK) return st;
  }
  Q4DecodeParams p{};
  p.a.kr = const_cast<void*>(kr_cache);
  p.a.o_part = S > 1 ? reinterpret_cast<float*>(ws + L.o_part) : o;
  p.a.lse_part = S > 1 ? reinterpret_cast<float*>(ws + L.lse_part) : lse;
  p.a.t_max = dims->t_max;
  p.a.scale_log2 = scale_log2(dims);
  p.scales = static_cast<const uint8_t*>(v4_scale);
  fill_inv_freq(dims, p.inv_freq);
  const int packed = dims->d_c | dims->d_r << 10 | S << 17;
  hipLaunchKernelGGL(fn, dim3((unsigned)n_items), dim3(64 * nw), 0, static_cast<hipStream_t>(stream), lens, seen,
                     L.fused ? q : static_cast<const void*>(q_abs), L.fused ? m : static_cast<const void*>(q_rot),
                     const_cast<void*>(v4_cache), packed, dims->batch, dims->n_groups, split_rows, p);
  st = launch_status();
  if (st != GVA_OK || S == 1) return st;
  return gva_combine(dims, p.a.o_part, p.a.lse_part, S, o, lse, stream);
}

}  // extern "C"
