// libgva.so -- attention of packed windows of queries, the last rows of each
// sequence: prompts of different lengths (gva_packed_prefill) and trees of
// drafted tokens (gva_tree_attention), on contiguous or paged caches.

#include <cfloat>
#include <map>
#include <new>
#include <type_traits>

#include "gva_window.h"

namespace {

// ============================================================== the kernel
// Sequence b has n_b query rows, packed at cu[b] .. cu[b+1] - 1, which are its
// last n_b cached rows; P = L_b - n_b rows are before them.  A workgroup takes
// 32 CW (row, head) columns of one group, 32 CW / hpg consecutive rows times
// the H/G heads that share the group's value rows, and one split of the keys.
// Its waves are KW sets of CW (one or two of four, three or four of one or two):
// a set walks every KW-th tile of 32 keys, a wave of it scores its own 32 columns;
// the sets are merged at the end.
//
// Per tile, on 32x32x16 products (lane = column, registers = rows):
//  - the tile's value and positional-key rows go straight to LDS, copied by the
//    set's waves, NBUF - 2 tiles ahead.  A lane may fetch any 16 bytes but puts
//    them in lane order, so the rows of piece k are fetched in the order
//    row ^ 4 (k mod 4): both readers below are then free of bank conflicts;
//  - scores S^T = [V | kr] q^T from rows read as they lie; the query's bf16
//    high and low parts are B operands in registers (x = hi + lo to 2^-17).  The
//    first tile takes a third part (to 2^-24), whose registers the accumulators
//    have afterwards: the log-sum-exp of a few rows is off by their scores'
//    roundings, that of many by the roundings' weighted mean, which is far less;
//  - the online softmax; scores come back with rows 8 (r/4) + 4 h + r % 4 in
//    register r, the order in which the transposing LDS read hands out V^T, so
//    the weights, rounded to bf16, are the B operand of P.V as they are.  A
//    weight is then off by at most 2^-8 of itself, what the output's own
//    rounding to bf16 may add again; the sum of the weights, which lse needs, is
//    of the unrounded ones in fp32.
//  - the exponentials and P.V run one tile behind the scores, between this
//    tile's products.
// Tiles with rows that some column does not see (the last rows of a block of a
// prompt, a tree's own rows) are masked, and, because 0 x NaN is NaN, their
// infinities and NaN are set to 0 in LDS after the scores have been taken:
// a column that sees such a row has the NaN (or infinite) score, one that does
// not is none the wiser.  Rows past the last key are set to 0 whole.
//
// Bound by the matrix cores: the parts of the queries make it 26 products for every
// 17 of the formulas (d 128/16; 28 for 18 at 128/32).  They run at 1.02 PFLOP/s in
// 15 K packed prompt rows (484 us, 323 GFLOP of the formulas) and at 1.20 in 860 rows
// behind up to 32 K (375 us of the kernel), where a library product of 8192 cubed has
// 1.18: the pipes are busy in 50 and 63% of the cycles, at 1.76 GHz.  Small calls are a chain of latencies: the
// item, copies, queries, tiles and end of 8 drafts behind 400 rows take 2, 2, 3, 4
// and 2 us.  A wave has 32 columns and a SIMD two waves, so that one's
// exponentials run beside the other's products: 64 columns a wave, which halves the
// LDS reads, leave registers for one wave and took 625 us and more.  Several sets
// where a sequence has few columns: 16 drafts behind 8 K rows (32 sequences, 549
// MB) 131 us against 156 with one (131 to 136 on different GPUs); of it the loop
// without its copies takes 80, the copies into LDS add 24, HBM 9.
struct WindowParams {
  const int32_t* cu;            // [B + 1] packed offsets
  const int32_t* lens;          // [B]
  const int32_t* parent;        // trees: [n_rows]; NULL: causal
  const int32_t* block_table;   // paged: [B][max_pages]; NULL: contiguous (page b, of t_max rows)
  const void* q;                // [n_rows][H][d_c + d_r]
  const void* m;                // [H][d_v][d_c]
  const float* q_abs;           // [n_rows][H][d_v], or NULL: absorbed here
  const void* v;
  const void* kr;
  void* o;                      // [n_rows][H][d_v] in the storage type (one split)
  float* lse;                   // [n_rows][H], may be NULL
  float* o_part;                // [n_rows][H][S][d_v] (more splits)
  float* lse_part;              // [n_rows][H][S]
  int32_t B, H, G, d_c, d_r, t_max, n_rows, S, split_rows;
  int32_t rows_log2;            // query rows of a workgroup
  int32_t page_rows, max_pages, n_pages;
  float scale_log2;
  double quarters[kMaxPairs];   // a pair's frequency, in quarter turns a position
};

// What a workgroup's first instructions need comes ahead of the block as scalar
// arguments, which are in registers before a wave starts (see decode_args).
#define WINDOW_HEAD_ARGS                                                                                         \
  const int32_t *head_cu, const int32_t *head_lens, int32_t head_B, int32_t head_G, int32_t head_rows_log2,       \
      int32_t head_S, int32_t head_n_rows, int32_t head_t_max, int32_t head_split_rows
#define WINDOW_HEAD_NAMES \
  head_cu, head_lens, head_B, head_G, head_rows_log2, head_S, head_n_rows, head_t_max, head_split_rows
struct WindowHead {
  const int32_t* cu;
  const int32_t* lens;
  int32_t B, G, rows_log2, S, n_rows, t_max, split_rows;
};

// A sequence's window: its first packed row, rows and cached rows.
struct Window {
  int first, n, L;
};
__device__ __forceinline__ Window window_of(const WindowHead& p, int b) {
  const int a = min(max(p.cu[b], 0), p.n_rows), e = min(max(p.cu[b + 1], 0), p.n_rows);
  return Window{a, max(e - a, 0), clamp_len(p.lens, b, p.t_max)};
}

// blocks of query rows
__device__ __forceinline__ int window_blocks_of(const WindowHead& p, int n) {
  return (int)(((unsigned)n + (1u << p.rows_log2) - 1) >> p.rows_log2);
}

__device__ __forceinline__ int window_splits(const WindowHead& p, int L) {
  return p.S == 1 ? 1 : max(1, min(p.S, split_count(L, p.S, p.split_rows)));
}

__device__ __forceinline__ int wave_sum_dpp(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x1B, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x140, 0xF, 0xF, false);
  const auto a = __builtin_amdgcn_permlane32_swap((unsigned)v, (unsigned)v, false, false);
  v = (int)(a[0] + a[1]);
  const auto c = __builtin_amdgcn_permlane16_swap((unsigned)v, (unsigned)v, false, false);
  return __builtin_amdgcn_readfirstlane((int)(c[0] + c[1]));
}

__device__ __forceinline__ int wave_max_dpp(int v) {
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x1B, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x141, 0xF, 0xF, false));
  v = max(v, __builtin_amdgcn_update_dpp(0, v, 0x140, 0xF, 0xF, false));
  const auto a = __builtin_amdgcn_permlane32_swap((unsigned)v, (unsigned)v, false, false);
  v = max((int)a[0], (int)a[1]);
  const auto c = __builtin_amdgcn_permlane16_swap((unsigned)v, (unsigned)v, false, false);
  return __builtin_amdgcn_readfirstlane(max((int)c[0], (int)c[1]));
}

// Item i of the (sequence, block of query rows, split) triples that exist.
//  - One split, up to 256 sequences: the blocks with most key tiles first.  The
//    number of blocks with at least t tiles is a sum over the sequences, four
//    of them a lane; the i-th block's t is found by bisection, then the
//    sequence among those that have a block of exactly t tiles.
//  - Otherwise sequence by sequence, splits in order, a split's blocks (which
//    read the same keys) next to each other.
__device__ __forceinline__ bool window_item(const WindowHead& p, int i, int& b, int& blk, int& s, Window& win) {
  const int lane = threadIdx.x & 63;
  if (p.S == 1 && p.B <= 256) {
    int P[4], n[4], first[4];
    int hi = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int bb = lane + 64 * k;
      const Window w = bb < p.B ? window_of(p, bb) : Window{0, 0, 0};
      n[k] = w.n;
      P[k] = w.L - w.n;
      first[k] = w.first;
      hi = max(hi, w.n > 0 ? w.L : 0);
    }
    // blocks of a sequence below the first with at least t tiles (all, if none)
    auto below = [&](int k, int t) {
      const int key = kTileRows * (t - 1) + 1;            // keys that make t tiles
      if (t <= 0) return 0;
      if (key > P[k] + n[k]) return window_blocks_of(p, n[k]);
      const int need = key - P[k];                        // rows of the window up to the last
      return need <= 0 ? 0 : (need - 1) >> p.rows_log2;
    };
    auto at_least = [&](int t) {
      int c = 0;
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (64 * k < p.B) c += window_blocks_of(p, n[k]) - below(k, t);
      return wave_sum_dpp(c);
    };
    if (i >= at_least(0)) return false;
    int lo = 0;                                // at_least(lo) > i >= at_least(hi)
    hi = (wave_max_dpp(hi) + kTileRows - 1) / kTileRows + 1;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (at_least(mid) > i) lo = mid;
      else hi = mid;
    }
    int rest = i - at_least(lo + 1);
    b = blk = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int base = below(k, lo), cnt = below(k, lo + 1) - base;
      const int incl = wave_incl_scan(cnt);
      const unsigned long long hit = __ballot(cnt > 0 && incl > rest && incl - cnt <= rest);
      if (hit != 0ull) {
        const int l = __builtin_ctzll(hit);
        b = 64 * k + l;
        blk = __builtin_amdgcn_readlane(base, l) + rest - __builtin_amdgcn_readlane(incl - cnt, l);
        win.first = __builtin_amdgcn_readlane(first[k], l);
        win.n = __builtin_amdgcn_readlane(n[k], l);
        win.L = __builtin_amdgcn_readlane(P[k], l) + win.n;
        break;
      }
      rest -= __builtin_amdgcn_readlane(incl, 63);
    }
    s = 0;
    return true;
  }
  const int k = (p.B + 63) >> 6;
  auto items = [&](int bb) {
    if (bb >= p.B) return 0;
    const Window w = window_of(p, bb);
    return window_blocks_of(p, w.n) * window_splits(p, w.L);
  };
  int sum = 0;
  for (int j = 0; j < k; ++j) sum += items(lane * k + j);
  const int incl = wave_incl_scan(sum);
  if (i >= __builtin_amdgcn_readlane(incl, 63)) return false;
  const int j1 = min(__popcll(__ballot(incl <= i)), 63);
  int local = i - __builtin_amdgcn_readlane(incl - sum, j1);
  b = __builtin_amdgcn_readfirstlane(j1 * k);
  for (int c = 0; c < k; c += 64) {            // the sequence among the lane's
    const int cnt = c + lane < k ? items(j1 * k + c + lane) : 0;
    const int in2 = wave_incl_scan(cnt);
    const int j2 = __popcll(__ballot(in2 <= local));
    if (j2 < 64) {
      b = __builtin_amdgcn_readfirstlane(j1 * k + c + j2);
      local -= __builtin_amdgcn_readlane(in2 - cnt, j2);
      break;
    }
    local -= __builtin_amdgcn_readlane(in2, 63);
  }
  win = window_of(p, b);
  const int nb = window_blocks_of(p, win.n);
  s = __builtin_amdgcn_readfirstlane(local / nb);
  blk = __builtin_amdgcn_readfirstlane(local % nb);
  return true;
}

// Workgroup -> item and group.  One split: groups fastest, so that with G a
// multiple of 8 an XCD keeps to its groups' streams, which the blocks of a
// sequence share.  More splits: the groups of an item on one XCD (see
// work_item), as they share the positional keys.
__device__ __forceinline__ bool window_work(const WindowHead& p, int& b, int& blk, int& s, int& g, Window& win) {
  const int x = blockIdx.x;
  if (p.S == 1) {
    g = x % p.G;
    return window_item(p, x / p.G, b, blk, s, win);
  }
  const int slot = x >> 3;
  g = slot % p.G;
  return window_item(p, 8 * (slot / p.G) + (x & 7), b, blk, s, win);
}

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0);
}

// One wave copies 1 KB into LDS, 16 bytes a lane in lane order, from byte soff +
// OFF behind the descriptor to m0 + OFF (zeros past the descriptor's end).  In asm so
// that the compiler does not drain the copies in flight before each LDS read (see the
// prompt kernel); it writes no register but m0, and the copies of a tile that lie
// one behind the other share one setting of it.  NT: rows that are read once, kept
// out of the caches' normal replacement.
__device__ __forceinline__ void copy_to(uint32_t dst) { asm volatile("s_mov_b32 m0, %0\n\ts_nop 0" ::"s"(dst) : "memory", "m0"); }
template <int OFF, bool NT>
__device__ __forceinline__ void copy_kb(i32x4 desc, int voff, int soff) {
  if constexpr (NT)
    asm volatile("buffer_load_dwordx4 %0, %1, %2 offen offset:%3 nt lds" ::"v"(voff), "s"(desc), "s"(soff), "n"(OFF) : "memory");
  else
    asm volatile("buffer_load_dwordx4 %0, %1, %2 offen offset:%3 lds" ::"v"(voff), "s"(desc), "s"(soff), "n"(OFF) : "memory");
}
// N KB in a row.
template <int N, bool NT>
__device__ __forceinline__ void copy_run(i32x4 desc, uint32_t dst, int voff, int soff) {
  copy_to(dst);
  copy_kb<0, NT>(desc, voff, soff);
  if constexpr (N > 1) copy_kb<1024, NT>(desc, voff, soff);
  if constexpr (N > 2) copy_kb<2048, NT>(desc, voff, soff);
  if constexpr (N > 3) copy_kb<3 * 1024, NT>(desc, voff, soff);
  if constexpr (N > 4) copy_run<N - 4, NT>(desc, dst + 4096, voff, soff + 4096);
}
template <int N>
__device__ __forceinline__ void wait_copies() {   // until at most N of this wave's copies are in flight
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
__device__ __forceinline__ void tile_barrier() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void wave_fence() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

// Eight bf16 of one column, rows 4 h .. + 3 and 8 more: within 16 lanes the
// transposing read takes four values from each lane's address, lanes 4 r .. 4 r
// + 3 a row of 16, and hands lane n column n of the four rows.
__device__ __forceinline__ bf16x8 read_transposed(const char* p0, const char* p1) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) s16x4* Lds;
  const s16x4 a = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p0));
  const s16x4 b = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p1));
  return __builtin_bit_cast(bf16x8, __builtin_shufflevector(a, b, 0, 1, 2, 3, 4, 5, 6, 7));
}

__device__ __forceinline__ bf16x8 to_bf16x8(const float* x) {
  bf16x8 out;
#pragma unroll
  for (int j = 0; j < 8; j += 2) {
    const bf16x2 h = __builtin_convertvector((f32x2{x[j], x[j + 1]}), bf16x2);
    out[j] = h[0];
    out[j + 1] = h[1];
  }
  return out;
}

// The bf16 nearest to each of eight floats, which keep what is left.
__device__ __forceinline__ bf16x8 take_part(float* x) {
  const bf16x8 part = to_bf16x8(x);
#pragma unroll
  for (int j = 0; j < 8; ++j) x[j] -= (float)part[j];
  return part;
}

// row of a 32-row tile in score register r of a lane in half h
__device__ __forceinline__ constexpr int score_row(int r, int h) { return 8 * (r >> 2) + 4 * h + (r & 3); }

// A pair rotated by an angle in quarter turns.  The whole quarters come off in 64
// bits, exactly; sine and cosine of the rest, at most pi/4, are their power series up
// to x^9 and x^10 (what follows is below 2e-9 of either), in fp32 as the scores are.
__device__ __forceinline__ void rotate_quarters(float x0, float x1, double quarters, float& y0, float& y1) {
  const double whole = rint(quarters);
  const float x = (float)(quarters - whole) * 1.57079632679489661923f, z = x * x;
  const float si = x + x * z * fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f);
  const float co = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const int k = (int)(whole - 4.0 * floor(0.25 * whole));     // of any size: a base below 1 turns fast
  float s = (k & 1) ? co : si, c = (k & 1) ? si : co;
  if (k & 2) s = -s;
  if ((k + 1) & 2) c = -c;
  y0 = x0 * c - x1 * s;
  y1 = x0 * s + x1 * c;
}

// -inf for the scores whose row has no bit in `sees`, the tile's rows from the
// lane's first on.
__device__ __forceinline__ void hide(f32x16& sn, uint32_t sees) {
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)sees, score_row(r, 0), 1);      // all ones or none
    sn[r] = __uint_as_float((__float_as_uint(sn[r]) & keep) | (0xFF800000u & ~keep));
  }
}

// A running maximum moves when a column's tile maximum exceeds it by more
// than this (log2 units): weights stay below 2^8, which costs a sum in fp32 and
// a weight in bf16 nothing, and the accumulators are rescaled on few tiles.
constexpr float kWindowLazyMax = 8.f;

// A tree's masks: bit j of word w + 1 of node i: node 32 w + j is i or an
// ancestor of i.  A word of ones is ahead of them (the prefix), one of zeros behind.
constexpr int kTreeWords = kMaxTree / 32 + 2;

// Masks and depths of the rows i0 .. of a block (ppb at most), by all threads of
// the workgroup: a thread per row walks up to the root.
__device__ __forceinline__ void tree_masks(const WindowParams& p, const Window& win, int i0, int ppb, int cols, int threads,
                                           uint32_t* masks, int16_t* up, int16_t* depths) {
  const int tid = threadIdx.x;
  for (int i = tid; i < win.n; i += threads) {
    const int a = p.parent[win.first + i];
    up[i] = (int16_t)(a >= 0 && a < i ? a : -1);
  }
  for (int i = tid; i < cols * kTreeWords; i += threads) masks[i] = i % kTreeWords == 0 ? ~0u : 0u;
  __syncthreads();
  if (tid < ppb && i0 + tid < win.n) {
    uint32_t* const mine = masks + tid * kTreeWords + 1;
    int depth = -1;
    for (int i = i0 + tid; i >= 0; i = up[i]) {
      mine[i >> 5] |= 1u << (i & 31);
      ++depth;
    }
    depths[tid] = (int16_t)depth;
  }
  __syncthreads();
}

// The 32 bits of a row's masks from row `at` of the window on (negative: the prefix).
__device__ __forceinline__ uint32_t tree_sees(const uint32_t* mine, int at) {
  const int bit = min(max(at + 32, 0), 32 * (kTreeWords - 2) + 31);
  const uint32_t* const w = mine + (bit >> 5);
  return (uint32_t)((((uint64_t)w[1] << 32) | w[0]) >> (bit & 31));
}

template <int DV, int NRC, int CW, int KW>
struct WindowCfg {
  static constexpr int COLS = 32 * CW;
  static constexpr int NCH = DV / 16;                      // 16-wide K-chunks of a value row
  static constexpr int NIB = DV / 32;                      // 32-wide output blocks
  static constexpr int V_BYTES = kTileRows * DV * 2;
  static constexpr int KB = V_BYTES / 1024;                // KB per value tile
  static constexpr int TILE_BYTES = V_BYTES + NRC * 1024;
  static constexpr int NBUF = 4;                           // tiles: weighted, scored, scored next, in flight
  static constexpr int KCOPIES = (NRC + CW - 1) / CW;      // of the positional tile, per wave
  static constexpr int SET_BYTES = NBUF * TILE_BYTES;
  static constexpr int MERGE_BYTES = (KW - 1) * CW * 64 * (NIB * 16 + 2) * 4;
  static constexpr int OUT_PITCH = DV * 2 + 16;            // bytes of a column's outputs in LDS
  static constexpr int OUT_BYTES = CW * 32 * OUT_PITCH;
  static constexpr int PART_PITCH = 36;                    // floats of a column's 32-wide block of partials
  static constexpr int PART_BYTES = CW * 32 * PART_PITCH * 4;
  static constexpr int MAX1 = KW * SET_BYTES > MERGE_BYTES ? KW * SET_BYTES : MERGE_BYTES;
  static constexpr int MAX2 = OUT_BYTES > PART_BYTES ? OUT_BYTES : PART_BYTES;
  static constexpr int LDS = MAX1 > MAX2 ? MAX1 : MAX2;
  static constexpr int READ_AHEAD = DV >= 128 && NRC > 1 ? 3 : 4;
};

template <int DV, int NRC, int CW, int KW>
__global__ void __launch_bounds__(64 * CW * KW, CW == 1 ? 1 : 2) window_kernel(WINDOW_HEAD_ARGS, WindowParams p) {
  const WindowHead hd{WINDOW_HEAD_NAMES};
  using Cfg = WindowCfg<DV, NRC, CW, KW>;
  constexpr int NCH = Cfg::NCH, NIB = Cfg::NIB, RA = Cfg::READ_AHEAD, NBUF = Cfg::NBUF;
  __shared__ __attribute__((aligned(1024))) char lds[Cfg::LDS];
  __shared__ uint32_t masks[Cfg::COLS * kTreeWords];
  __shared__ int16_t tree_parent[kMaxTree];
  __shared__ int16_t tree_depth[Cfg::COLS];

  const int hpg = p.H / p.G;
  int b, blk, split, g;
  Window win;
  if (!window_work(hd, b, blk, split, g, win)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int grp = wave / CW, w = wave % CW;
  const int n = lane & 31, h = lane >> 5;      // column, and half of the rows / K-chunk
  const bf16x8 zero8 = as_bf16x8(u32x4{0u, 0u, 0u, 0u});

  const int P = win.L - win.n;                 // rows before the window (negative: some of it has no row)
  const int lg = p.rows_log2, ppb = 1 << lg;   // query rows of the block
  const int i0 = blk << lg, i1 = min(win.n, i0 + ppb);
  const bool tree = p.parent != nullptr;
  const bool too_large = tree && win.n > kMaxTree;

  // ---- this wave's columns: row i of the window, head.  Head by head, the
  // block's rows of each.
  const int col = 32 * w + n;
  const int i_col = i0 + (col & (ppb - 1));
  const int head = g * hpg + (col >> lg);
  const bool live_col = i_col < win.n;
  const bool live = i0 + ((32 * w) & (ppb - 1)) < win.n;   // some column of the wave is
  const int own_row = P + i_col;
  const bool has_row = live_col && own_row >= 0 && !too_large;
  const int packed = win.first + min(i_col, win.n - 1);
  const int64_t qrow = (int64_t)packed * p.H + head;

  // ---- keys of this split, and from which row on some column may not see
  int kbeg = 0, kend = P + i1;                 // rows that the block's last one sees
  if (p.S > 1) {
    int r0, r1;
    split_rows(win.L, p.S, p.split_rows, split, r0, r1);
    kbeg = r0;
    kend = min(kend, r1);
  }
  if (too_large) kend = kbeg;
  const int masked_from = tree ? P : P + i0 + 1;
  const int wave_masked_from = tree ? P : P + i0 + ((32 * w) & (ppb - 1)) + 1;
  const int ntiles = kend > kbeg ? (kend - kbeg + kTileRows - 1) / kTileRows : 0;
  const int nit = (ntiles + KW - 1) / KW;      // the same for all sets (they share the barriers)
  auto tile_row = [&](int j) { return kbeg + (KW * j + grp) * kTileRows; };

  // ---- tile copies, through the block table.  Lane l of `ids` holds the id of
  // the set's page id_base + l.
  const bool paged = p.block_table != nullptr;
  const int page_rows = paged ? p.page_rows : p.t_max;
  const int tiles_per_page = (page_rows + kTileRows - 1) / kTileRows;
  const int32_t* const table = p.block_table + (paged ? (int64_t)b * p.max_pages : 0);
  int page = (kbeg / kTileRows + grp) / tiles_per_page;    // of the next tile to copy
  int in_page = (kbeg / kTileRows + grp) % tiles_per_page;
  const int page_step = KW / tiles_per_page, tile_step = KW % tiles_per_page;
  int next_copy = 0, id_base = page, ids = b;
  auto load_ids = [&]() {
    id_base = page;
    const int id = table[min(id_base + lane, p.max_pages - 1)];
    ids = min(max(id, 0), p.n_pages - 1);
  };
  if (paged) load_ids();
  char* const set_lds = lds + grp * Cfg::SET_BYTES;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)set_lds;
  const int v_voff = (lane >> 4) * 256 + (((lane & 15) ^ (4 * (lane >> 4))) << 4);
  // Where the next tile is: the page's descriptors, which past the last tile
  // are empty, and the tile's place behind them.  (A stream is below 2 GiB, a page
  // of G streams may be of any size.)
  const uint32_t v_page = (uint32_t)page_rows * (DV / 8), k_page = (uint32_t)page_rows * (uint32_t)p.d_r / 8;   // 16-byte pieces
  i32x4 vdesc, kdesc;
  int v_soff, k_soff;
  auto aim = [&]() __attribute__((always_inline)) {
    if (paged && page - id_base >= 64) load_ids();
    const bool in = KW * next_copy + grp < ntiles;
    const uint32_t id = paged ? (uint32_t)__builtin_amdgcn_readlane(ids, min(max(page - id_base, 0), 63)) : (uint32_t)b;
    const uint64_t va = (uint64_t)(uintptr_t)p.v + ((((uint64_t)id * (uint32_t)p.G + (uint32_t)g) * v_page) << 4);
    const uint64_t ka = (uint64_t)(uintptr_t)p.kr + (((uint64_t)id * k_page) << 4);
    vdesc = i32x4{(int)(uint32_t)va, (int)(uint32_t)(va >> 32) & 0xFFFF, in ? (int)(v_page * 16) : 0, kBufferWord3};
    kdesc = i32x4{(int)(uint32_t)ka, (int)(uint32_t)(ka >> 32) & 0xFFFF, in ? (int)(k_page * 16) : 0, kBufferWord3};
    v_soff = in_page * (kTileRows * DV * 2);
    k_soff = in_page * (kTileRows * 2) * p.d_r;
  };
  aim();
  auto copy_next = [&](int buf) __attribute__((always_inline)) {
    const uint32_t dst = lds0 + buf * Cfg::TILE_BYTES;
    constexpr int KBW = Cfg::KB / CW;
    copy_run<KBW, (KW > 2)>(vdesc, dst + w * (KBW * 1024), v_voff, v_soff + w * (KBW * 1024));
    // the positional tile is 32 d_r 2 bytes <= NRC KB: whole KBs (what follows
    // it lands in padding); waves past NRC repeat one, so that all copy alike
    const int kb = w * Cfg::KCOPIES % NRC;
    copy_run<Cfg::KCOPIES, false>(kdesc, dst + Cfg::V_BYTES + kb * 1024, lane * 16, k_soff + kb * 1024);
    ++next_copy;
    page += page_step;
    in_page += tile_step;
    bool moved = page_step > 0 || KW * next_copy + grp >= ntiles;
    if (in_page >= tiles_per_page) {
      in_page -= tiles_per_page;
      ++page;
      moved = true;
    }
    if (moved) {
      aim();
    } else {
      v_soff += KW * kTileRows * DV * 2;
      k_soff += KW * kTileRows * 2 * p.d_r;
    }
  };
  copy_next(0);
  copy_next(1);

  // ---- a tree's masks and depths
  if (tree && !too_large) tree_masks(p, win, i0, ppb, Cfg::COLS, 64 * CW * KW, masks, tree_parent, tree_depth);
  const int pos = has_row ? max(0, tree ? P + tree_depth[i_col - i0] : own_row) : 0;

  // ---- the queries as bf16 high and low B operands: lane (n, h) holds
  // entries 16 c + 8 h .. + 7 of its column's query
  bf16x8 qh[NCH], ql[NCH], q3[NCH], rh[NRC], rl[NRC], r3[NRC];
  auto put_query = [&](bf16x8& hi, bf16x8& lo, bf16x8& third, float* xv) {
#pragma unroll
    for (int j = 0; j < 8; ++j) xv[j] *= p.scale_log2;
    hi = take_part(xv);
    lo = take_part(xv);
    third = take_part(xv);
  };
  const int W = p.d_c + p.d_r;
  const uint16_t* const qraw = static_cast<const uint16_t*>(p.q) + qrow * W;
  if (p.q_abs == nullptr) {
    // The absorption on the same products: q~^T[i][col] = sum_k M_h[i][k]
    // q[col][k].  Row m of an A operand is row i(m) of M_h, bits 2 and 3 of m
    // swapped, so that a lane's 16 results of a block are two B operands of the
    // score product as they lie.  One pass per head of the wave's columns, each
    // with the loads of CS chunks of 16 columns ahead of the products.
    const int mrow = (n & 19) | ((n & 4) << 1) | ((n & 8) >> 1);
    auto absorb = [&](auto cs_tag, int hm, int ib0, auto& e) __attribute__((always_inline)) {
      constexpr int CS = decltype(cs_tag)::value, NB = sizeof(e) / sizeof(f32x16);
      const uint16_t* const mh = static_cast<const uint16_t*>(p.m) + ((int64_t)hm * DV + 32 * ib0 + mrow) * p.d_c;
      const int nround = (p.d_c + 16 * CS - 1) / (16 * CS);
      u32x4 xq[2][CS], xm[2][CS][NB];
      auto load = [&](int ro, int at) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < CS; ++c) {         // columns past d_c: any valid ones against zeros
          const int kc = min(16 * (CS * ro + c) + 8 * h, p.d_c - 8);
          xq[at][c] = *reinterpret_cast<const u32x4*>(qraw + kc);
#pragma unroll
          for (int ib = 0; ib < NB; ++ib)
            xm[at][c][ib] = *reinterpret_cast<const u32x4*>(mh + (int64_t)(32 * ib) * p.d_c + kc);
        }
        __builtin_amdgcn_sched_barrier(0);
      };
      auto multiply = [&](int ro, int at) __attribute__((always_inline)) {
#pragma unroll
        for (int c = 0; c < CS; ++c) {
          const bf16x8 bq = 16 * (CS * ro + c) < p.d_c ? as_bf16x8(xq[at][c]) : zero8;
#pragma unroll
          for (int ib = 0; ib < NB; ++ib) e[ib] = mfma32(as_bf16x8(xm[at][c][ib]), bq, e[ib]);
        }
        __builtin_amdgcn_sched_barrier(0);
      };
#pragma unroll
      for (int ib = 0; ib < NB; ++ib)
#pragma unroll
        for (int r = 0; r < 16; ++r) e[ib][r] = 0.f;
      load(0, 0);
#pragma unroll 1
      for (int ro = 0; ro < nround; ro += 2) {
        if (ro + 1 < nround) load(ro + 1, 1);
        multiply(ro, 0);
        if (ro + 1 < nround) {
          if (ro + 2 < nround) load(ro + 2, 0);
          multiply(ro + 1, 1);
        }
      }
    };
    const int h_first = g * hpg + (32 * w >> lg), npass = ppb >= 32 ? 1 : 32 >> lg;
    if constexpr (KW < 3) {                    // each set for itself: two of four waves have no room to share
      f32x16 d[NIB];
      if (npass == 1) {
        absorb(std::integral_constant<int, 4>{}, h_first, 0, d);
      } else {
#pragma unroll 1
        for (int ps = 0; ps < npass; ++ps) {
          f32x16 e[NIB];
          absorb(std::integral_constant<int, 2>{}, h_first + ps, 0, e);
          const bool mine = (n >> lg) == ps;
#pragma unroll
          for (int ib = 0; ib < NIB; ++ib)
#pragma unroll
            for (int r = 0; r < 16; ++r) d[ib][r] = ps == 0 || mine ? e[ib][r] : d[ib][r];
        }
      }
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        float xv[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) xv[j] = d[c >> 1][8 * (c & 1) + j];
        put_query(qh[c], ql[c], q3[c], xv);
      }
    } else {
      // The sets share the work, blocks of 32 rows of a head's map in turn, and
      // pass the parts on through LDS that no tile has reached yet: part k of chunk
      // c of column wave w at share(k, c), a lane's 16 bytes in place.
      static_assert(2 * Cfg::TILE_BYTES * KW >= 3 * CW * NCH * 1024, "the queries pass through buffers not yet in use");
      constexpr int ROOM = 2 * Cfg::TILE_BYTES / 1024;       // KB of a set's free buffers
      auto share = [&](int part, int c) {
        const int kb = (part * CW + w) * NCH + c;
        return reinterpret_cast<bf16x8*>(lds + kb / ROOM * Cfg::SET_BYTES + 2 * Cfg::TILE_BYTES + kb % ROOM * 1024 + lane * 16);
      };
      constexpr int NU = 2;                    // blocks of a turn
#pragma unroll 1
      for (int u = grp; u < npass * (NIB / NU); u += KW) {
        const int ps = u / (NIB / NU), ib0 = u % (NIB / NU) * NU;
        f32x16 e[NU];
        absorb(std::integral_constant<int, 4>{}, h_first + ps, ib0, e);
        if (npass == 1 || (n >> lg) == ps) {
#pragma unroll
          for (int c = 0; c < 2 * NU; ++c) {
            float xv[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) xv[j] = e[c >> 1][8 * (c & 1) + j];
            bf16x8 hi, lo, third;
            put_query(hi, lo, third, xv);
            *share(0, 2 * ib0 + c) = hi;
            *share(1, 2 * ib0 + c) = lo;
            *share(2, 2 * ib0 + c) = third;
          }
        }
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      tile_barrier();
#pragma unroll
      for (int c = 0; c < NCH; ++c) {
        qh[c] = *share(0, c);
        ql[c] = *share(1, c);
        q3[c] = *share(2, c);
      }
      // Sets of one wave meet no other set before a set's third tile is copied over the
      // parts in its buffers: all of them have been read by then.  (Larger sets meet at
      // their barriers, which are the workgroup's.)
      if constexpr (CW == 1) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        tile_barrier();
      }
    }
  } else {
    const float* qa = p.q_abs + qrow * DV + 8 * h;
#pragma unroll
    for (int c = 0; c < NCH; ++c) {
      const f32x4 u0 = *reinterpret_cast<const f32x4*>(qa + 16 * c);
      const f32x4 u1 = *reinterpret_cast<const f32x4*>(qa + 16 * c + 4);
      float xv[8] = {u0[0], u0[1], u0[2], u0[3], u1[0], u1[1], u1[2], u1[3]};
      put_query(qh[c], ql[c], q3[c], xv);
    }
  }
#pragma unroll
  for (int rc = 0; rc < NRC; ++rc) {
    const int piece = 2 * rc + h;
    float xv[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
    if (8 * piece < p.d_r) {
      const u32x4 raw = *reinterpret_cast<const u32x4*>(qraw + p.d_c + 8 * piece);
#pragma unroll
      for (int k = 0; k < 4; ++k)
        rotate_quarters(bf16_bits_to_f32(raw[k] & 0xFFFFu), __uint_as_float(raw[k] & 0xFFFF0000u),
                        (double)pos * p.quarters[4 * piece + k], xv[2 * k], xv[2 * k + 1]);
    }
    put_query(rh[rc], rl[rc], r3[rc], xv);
  }

  // ---- LDS offsets of this lane's operands in a tile
  int v_off[2];                                // piece 2 c + h of row n, c even and odd
#pragma unroll
  for (int c = 0; c < 2; ++c) v_off[c] = (n >> 4) * (DV * 32) + h * 256 + (((n & 15) ^ (4 * (2 * c + h))) << 4);
  int k_off[NRC];
#pragma unroll
  for (int rc = 0; rc < NRC; ++rc) {           // pieces past d_r: any valid one against a zero query
    const int piece = 8 * (2 * rc + h) < p.d_r ? 2 * rc + h : 0;
    k_off[rc] = Cfg::V_BYTES + (n >> 4) * 32 * p.d_r + piece * 256 + (n & 15) * 16;
  }
  const int tl = lane & 15, tk = 2 * ((lane >> 4) & 1) + ((tl & 3) >> 1);
  const int tr_off = tk * 256 + (((4 * h + (tl >> 2)) ^ (4 * tk)) << 4) + (tl & 1) * 8;

  f32x16 acc[NIB];
  // the running maximum starts below every score but -inf: an exponential
  // against it is 0, and the first score that counts replaces it
  float m_run = -FLT_MAX, l_run = 0.f, tile_sum = 0.f;
#pragma unroll
  for (int ib = 0; ib < NIB; ++ib)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[ib][r] = 0.f;

  auto vt_piece = [&](int buf, int k) {        // A operand k = 2 ib + c of a tile's V^T
    const char* t = set_lds + buf * Cfg::TILE_BYTES + (k & 1) * (DV * 32) + (k >> 1) * 1024;
    return read_transposed(t + tr_off, t + (tr_off ^ 128));
  };
  auto exps = [&](const f32x16& sc, float (&pr)[16], int r) {
    pr[r] = __builtin_amdgcn_exp2f(sc[r] - m_run);
    tile_sum = r == 0 ? pr[r] : tile_sum + pr[r];
    if (r == 15) l_run += tile_sum;
  };
  // Between the waves of a set, which meet once a tile.  A set of one needs no
  // barrier: its copies, reads and writes of its own tiles are in order.
  auto set_barrier = [&]() __attribute__((always_inline)) {
    if constexpr (CW > 1) tile_barrier();
    else asm volatile("" ::: "memory");
  };
  // (the same answer for all sets, which share the barriers)
  auto is_masked = [&](int j) { return kbeg + (KW * j + KW) * kTileRows > masked_from; };
  // Set to 0 in a masked tile: rows past the keys, infinities and NaN.
  auto clean = [&](int j, int buf) {
    const int row0 = tile_row(j);
    char* const t = set_lds + buf * Cfg::TILE_BYTES + lane * 16;
#pragma unroll
    for (int k = 0; k < Cfg::KB / CW; ++k) {
      const int kb = w * (Cfg::KB / CW) + k;
      u32x4* const at = reinterpret_cast<u32x4*>(t + kb * 1024);
      u32x4 u = *at;
      const bool past = row0 + 16 * (kb / (DV / 32)) + ((lane & 15) ^ (4 * (lane >> 4))) >= kend;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        uint32_t x = u[e];
        x = (x & 0x7F800000u) == 0x7F800000u ? x & 0xFFFFu : x;
        x = (x & 0x7F80u) == 0x7F80u ? x & 0xFFFF0000u : x;
        u[e] = past ? 0u : x;
      }
      *at = u;
    }
  };
  // scores of rows that the column does not see, and of those past the keys
  auto mask = [&](f32x16& sn, int row0) __attribute__((always_inline)) {
    if (row0 + kTileRows <= wave_masked_from && row0 + kTileRows <= kend) return;
    const int last = (tree ? kend : min(own_row + 1, kend)) - row0;       // rows of the tile up to it
    uint32_t sees = last >= 32 ? ~0u : last <= 0 ? 0u : (1u << last) - 1u;
    if (tree) sees &= tree_sees(masks + (col & (ppb - 1)) * kTreeWords, row0 - P);
    hide(sn, sees >> (4 * h));
  };
  constexpr int NA = NCH + NRC;
  bf16x8 a[NA];                                // a tile's score operands; the first RA are read ahead of its step
  auto operand = [&](int buf, int k) __attribute__((always_inline)) {
    const char* const tile = set_lds + buf * Cfg::TILE_BYTES;
    if (k < NCH) return *reinterpret_cast<const bf16x8*>(tile + v_off[k & 1] + k * 512);
    return *reinterpret_cast<const bf16x8*>(tile + k_off[k >= NCH ? k - NCH : 0]);
  };
  float mt = -INFINITY;                        // the maximum of a lane's scores of the tile before
  auto move_max = [&](bool first) __attribute__((always_inline)) {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mt), __float_as_uint(mt), false, false);
    mt = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
    if (first || __ballot(mt > m_run + kWindowLazyMax) != 0) {
      const float m_new = fmaxf(mt, m_run);
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int ib = 0; ib < NIB; ++ib) acc[ib] *= alpha;
      m_run = m_new;
    }
  };
  // One tile j: its scores sn, beside them the softmax weights of the tile
  // before (scores sp); then the waves meet; then that tile's P.V, beside it tile
  // j's maxima and the reads of tile j + 1.  What the meeting stands for: tile j + 1
  // has landed (every wave has waited for its own copies), tile j - 1 is clean, and
  // the P.V of tile j - 2 is over, so that tile j + 2 may be copied over it.  The
  // orders are pinned (scheduling barriers): on these matrix cores a few vector
  // instructions between two products are nearly free, a run of them is not.
  // FIRST: the workgroup's first tile, with none before it.
  auto step = [&](auto first_tag, int j, int buf, const f32x16& sp, f32x16& sn) __attribute__((always_inline)) {
    constexpr bool FIRST = decltype(first_tag)::value;
    const int row0 = tile_row(j);
    const int pbuf = (buf + NBUF - 1) % NBUF;
    const bool cleaned = !FIRST && is_masked(j - 1);
    if (cleaned) clean(j - 1, pbuf);
    bf16x8 av[2 * NIB];
    float pr[16];
    bf16x8 bn[2];
    if (live) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sn[r] = 0.f;
      constexpr int NM = 2 * NA;               // products of this phase
      __builtin_amdgcn_s_setprio(1);           // ahead of another wave's P.V, which has less to interleave
#pragma unroll
      for (int i = 0; i < NM; ++i) {
        const int k = i / 2;
        if (k < NCH) sn = mfma32(a[k], (i & 1) ? ql[k < NCH ? k : 0] : qh[k < NCH ? k : 0], sn);
        else sn = mfma32(a[k], (i & 1) ? rl[k >= NCH ? k - NCH : 0] : rh[k >= NCH ? k - NCH : 0], sn);
        if constexpr (FIRST) {
          if ((i & 1) == 1) sn = mfma32(a[k], k < NCH ? q3[k < NCH ? k : 0] : r3[k >= NCH ? k - NCH : 0], sn);
        }
        if ((i & 1) == 1) {
          if (k + RA < NA) a[k + RA] = operand(buf, k + RA);
          else if (!FIRST) av[k + RA - NA] = vt_piece(pbuf, k + RA - NA);
        }
        if constexpr (!FIRST) {
          if (i == 0) {
            __builtin_amdgcn_sched_barrier(0);
            move_max(false);                   // of the tile before, beside the first products
          }
          // sixteen exponentials over the products from the second on
#pragma unroll
          for (int r = i == 0 ? 16 : (i - 1) * 16 / (NM - 1); r < i * 16 / (NM - 1); ++r) {
            exps(sp, pr, r);
            if (r == 7) bn[0] = to_bf16x8(pr);
            if (r == 15) bn[1] = to_bf16x8(pr + 8);
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (!FIRST) asm volatile("" ::"v"(bn[0]), "v"(bn[1]), "v"(l_run));   // formed here, beside the products
      __builtin_amdgcn_sched_barrier(0);
      mask(sn, row0);
      __builtin_amdgcn_s_setprio(0);
    }
    if (cleaned) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    wait_copies<0>();
    set_barrier();
    copy_next((buf + 2) % NBUF);
    if (live) {
      if (cleaned) {                           // what was read ahead was not clean yet
#pragma unroll
        for (int k = 0; k < RA; ++k) av[k] = vt_piece(pbuf, k);
      }
      const int nbuf = (buf + 1) % NBUF;
      mt = -INFINITY;
#pragma unroll
      for (int k = 0; k < 2 * NIB; ++k) {
        if constexpr (!FIRST) {
          acc[k >> 1] = mfma32(av[k], bn[k & 1], acc[k >> 1]);
          if (k + RA < 2 * NIB) av[k + RA] = vt_piece(pbuf, k + RA);
        }
        if (k >= 2 * NIB - RA) a[k - (2 * NIB - RA)] = operand(nbuf, k - (2 * NIB - RA));
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int r = k * (8 / NIB); r < (k + 1) * (8 / NIB); ++r) mt = fmaxf(mt, sn[r]);
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (FIRST) move_max(true);
    }
  };
  auto last = [&](int j, int buf, const f32x16& sp) {   // the last tile's weights and P.V
    if (is_masked(j)) {
      clean(j, buf);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      set_barrier();
    }
    if (!live) return;
    if (j > 0) move_max(false);
    float pr[16];
    bf16x8 bn[2];
#pragma unroll
    for (int r = 0; r < 16; ++r) exps(sp, pr, r);
    bn[0] = to_bf16x8(pr);
    bn[1] = to_bf16x8(pr + 8);
#pragma unroll
    for (int k = 0; k < 2 * NIB; ++k) acc[k >> 1] = mfma32(vt_piece(buf, k), bn[k & 1], acc[k >> 1]);
  };

  wait_copies<0>();
  set_barrier();
  if (nit > 0) {
    f32x16 s0, s1;                             // the scores of even and odd tiles
    if (live) {
#pragma unroll
      for (int k = 0; k < RA; ++k) a[k] = operand(0, k);
    }
    step(std::true_type{}, 0, 0, s0, s0);
    int j = 1;
    for (; j + 1 < nit; j += 2) {
      step(std::false_type{}, j, j % NBUF, s0, s1);
      step(std::false_type{}, j + 1, (j + 1) % NBUF, s1, s0);
    }
    if (j < nit) {
      step(std::false_type{}, j, j % NBUF, s0, s1);
      s0 = s1;
      ++j;
    }
    last(j - 1, (j - 1) % NBUF, s0);
  }

  // ---- merge the sets, normalise, write
  {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
    l_run = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  }
  wait_copies<0>();                            // copies past the end still write LDS
  __syncthreads();                             // every wave is done with the tiles
  if constexpr (KW > 1) {
    constexpr int REC = 64 * (NIB * 16 + 2);   // floats of a wave
    float* const recs = reinterpret_cast<float*>(lds) + lane;
    if (grp > 0) {
      float* const rec = recs + ((grp - 1) * CW + w) * REC;
      rec[0] = m_run;
      rec[64] = l_run;
#pragma unroll
      for (int ib = 0; ib < NIB; ++ib)
#pragma unroll
        for (int r = 0; r < 16; ++r) rec[64 * (2 + 16 * ib + r)] = acc[ib][r];
    }
    __syncthreads();
    if (grp == 0) {
#pragma unroll 1
      for (int k = 1; k < KW; ++k) {
        const float* const rec = recs + ((k - 1) * CW + w) * REC;
        const float m1 = rec[0], l1 = rec[64];
        const bool has0 = !(l_run == 0.f), has1 = !(l1 == 0.f);
        const float mx = has0 && has1 ? fmaxf(m_run, m1) : (has0 ? m_run : m1);
        const float a0 = has0 ? __builtin_amdgcn_exp2f(m_run - mx) : 0.f;
        const float a1 = has1 ? __builtin_amdgcn_exp2f(m1 - mx) : 0.f;
        l_run = l_run * a0 + l1 * a1;
        m_run = mx;
#pragma unroll
        for (int ib = 0; ib < NIB; ++ib)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[ib][r] = acc[ib][r] * a0 + rec[64 * (2 + 16 * ib + r)] * a1;
      }
    }
    __syncthreads();                           // the records have been read
    if (grp > 0) return;
  }
  // The outputs pass through the wave's LDS and leave as whole lines.
  const bool seen = has_row && !(l_run == 0.f);
  const float inv = seen ? 1.f / l_run : 0.f;
  const float lse = seen ? (m_run + log2f(l_run)) * kLn2 : -INFINITY;
  if (p.S == 1) {
    char* const ob = lds + w * 32 * Cfg::OUT_PITCH;
#pragma unroll
    for (int ib = 0; ib < NIB; ++ib)
#pragma unroll
      for (int r4 = 0; r4 < 4; ++r4) {
        uint32_t two[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          f32x2 x = {acc[ib][4 * r4 + 2 * e] * inv, acc[ib][4 * r4 + 2 * e + 1] * inv};
          if (!seen) x = f32x2{0.f, 0.f};
          two[e] = __builtin_bit_cast(uint32_t, __builtin_convertvector(x, bf16x2));
        }
        *reinterpret_cast<uint64_t*>(ob + n * Cfg::OUT_PITCH + (32 * ib + 8 * r4 + 4 * h) * 2) =
            (uint64_t)two[1] << 32 | two[0];
      }
    wave_fence();
    constexpr int LPR = DV / 8;                // lanes a row of outputs
#pragma unroll
    for (int it = 0; it < 32 * LPR / 64; ++it) {
      const int c = it * (64 / LPR) + lane / LPR, e = lane % LPR;
      const u32x4 u = *reinterpret_cast<const u32x4*>(ob + c * Cfg::OUT_PITCH + e * 16);
      const int cc = 32 * w + c, i = i0 + (cc & (ppb - 1));
      if (i < win.n)
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.o) +
                                  ((int64_t)(win.first + i) * p.H + g * hpg + (cc >> lg)) * DV + 8 * e) = u;
    }
    if (p.lse != nullptr && h == 0 && live_col) p.lse[qrow] = lse;
    return;
  }
  float* const ob = reinterpret_cast<float*>(lds) + w * 32 * Cfg::PART_PITCH;
#pragma unroll
  for (int ib = 0; ib < NIB; ++ib) {
    wave_fence();                              // the block before has been read
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      f32x4 o;
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) o[jj] = seen ? acc[ib][4 * r4 + jj] * inv : 0.f;
      *reinterpret_cast<f32x4*>(ob + n * Cfg::PART_PITCH + 8 * r4 + 4 * h) = o;
    }
    wave_fence();
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int c = 8 * it + (lane >> 3);
      const f32x4 o = *reinterpret_cast<const f32x4*>(ob + c * Cfg::PART_PITCH + 4 * (lane & 7));
      const int cc = 32 * w + c, i = i0 + (cc & (ppb - 1));
      if (i < win.n)
        *reinterpret_cast<f32x4*>(
            p.o_part + (((int64_t)(win.first + i) * p.H + g * hpg + (cc >> lg)) * p.S + split) * DV + 32 * ib + 4 * (lane & 7)) = o;
    }
  }
  if (h == 0 && live_col) {
    float* const lp = p.lse_part + qrow * p.S;
    lp[split] = lse;
    if (split == 0)                            // splits that no workgroup takes
      for (int k = window_splits(hd, win.L); k < p.S; ++k) lp[k] = -INFINITY;
  }
}

// ------------------------------------------------------------- fp32 storage
// The same walk on fp32 products (32x32x2; 157 TFLOP/s are what bounds it), four
// waves of 32 columns over every tile.  The k-order of a product is free as long as
// both operands have it: a lane takes entries 8 c + 4 h .. + 3 of a row with one
// 16-byte read for four products, the order in which the absorption's product
// leaves q~.  The weights in register r are rows score_row(r, h), and P.V reads
// those rows' entries from LDS, single ones of 32 columns: the rows of piece k are
// stored in the order row ^ (k mod 8), so that eight pieces of a row lie in
// different banks.  Two prompts of 300 to 1000 rows, H32 G8 d 128/16: 143 us.
template <int DV, int NRC>
__global__ void __launch_bounds__(kThreads, 2) window_f32_kernel(WINDOW_HEAD_ARGS, WindowParams p) {
  const WindowHead hd{WINDOW_HEAD_NAMES};
  constexpr int NC = DV / 8, NR = 2 * NRC, NIB = DV / 32;  // 8-wide chunks, 32-wide output blocks
  constexpr int V_BYTES = kTileRows * DV * 4, TILE_BYTES = V_BYTES + NR * 1024;
  constexpr int PITCH = 36;                    // floats of a column's 32-wide block of outputs
  constexpr int OUT_BYTES = kWaves * 32 * PITCH * 4;
  __shared__ __attribute__((aligned(1024))) char lds[2 * TILE_BYTES > OUT_BYTES ? 2 * TILE_BYTES : OUT_BYTES];
  __shared__ uint32_t masks[128 * kTreeWords];
  __shared__ int16_t tree_parent[kMaxTree];
  __shared__ int16_t tree_depth[128];

  const int hpg = p.H / p.G;
  int b, blk, split, g;
  Window win;
  if (!window_work(hd, b, blk, split, g, win)) return;
  const int tid = threadIdx.x, lane = tid & 63;
  const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 31, h = lane >> 5;

  const int P = win.L - win.n;
  const int lg = p.rows_log2, ppb = 1 << lg;   // query rows of the block
  const int i0 = blk << lg, i1 = min(win.n, i0 + ppb);
  const bool tree = p.parent != nullptr;
  const bool too_large = tree && win.n > kMaxTree;
  const int col = 32 * w + n;
  const int i_col = i0 + (col & (ppb - 1));
  const int head = g * hpg + (col >> lg);
  const bool live_col = i_col < win.n;
  const bool live = i0 + ((32 * w) & (ppb - 1)) < win.n;
  const int own_row = P + i_col;
  const bool has_row = live_col && own_row >= 0 && !too_large;
  const int64_t qrow = (int64_t)(win.first + min(i_col, win.n - 1)) * p.H + head;
  int kbeg = 0, kend = P + i1;
  if (p.S > 1) {
    int r0, r1;
    split_rows(win.L, p.S, p.split_rows, split, r0, r1);
    kbeg = r0;
    kend = min(kend, r1);
  }
  if (too_large) kend = kbeg;
  const int masked_from = tree ? P : P + i0 + 1;
  const int ntiles = kend > kbeg ? (kend - kbeg + kTileRows - 1) / kTileRows : 0;

  const bool paged = p.block_table != nullptr;
  const int page_rows = paged ? p.page_rows : p.t_max;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) char*)lds;
  auto copy_tile = [&](int j) {
    const bool in = j < ntiles;
    const int row = in ? kbeg + j * kTileRows : 0;
    int64_t id = b;
    if (paged) id = min(max(p.block_table[(int64_t)b * p.max_pages + row / page_rows], 0), p.n_pages - 1);
    const int at = row % page_rows;
    const uint64_t va = (uint64_t)(uintptr_t)p.v + (uint64_t)((id * p.G + g) * page_rows) * (DV * 4);
    const uint64_t ka = (uint64_t)(uintptr_t)p.kr + (uint64_t)(id * page_rows) * (uint64_t)(p.d_r * 4);
    const i32x4 vdesc = {__builtin_amdgcn_readfirstlane((int)(uint32_t)va),
                         __builtin_amdgcn_readfirstlane((int)(uint32_t)(va >> 32) & 0xFFFF), in ? page_rows * DV * 4 : 0,
                         kBufferWord3};
    const i32x4 kdesc = {__builtin_amdgcn_readfirstlane((int)(uint32_t)ka),
                         __builtin_amdgcn_readfirstlane((int)(uint32_t)(ka >> 32) & 0xFFFF), in ? page_rows * p.d_r * 4 : 0,
                         kBufferWord3};
    const uint32_t dst = lds0 + (j & 1) * TILE_BYTES;
#pragma unroll
    for (int k = 0; k < V_BYTES / 4096; ++k) {
      const int kb = w * (V_BYTES / 4096) + k;             // pieces 4 kb .. 4 kb + 3 of a layout tile
      const int f = 4 * (kb & 1) + (lane >> 4);
      copy_run<1, false>(vdesc, dst + kb * 1024, (lane >> 4) * 256 + (((lane & 15) ^ f) << 4), at * DV * 4 + kb * 1024);
    }
    for (int kb = w; kb < NR * 2; kb += kWaves)            // 32 d_r 4 bytes, in whole KBs
      if (kb < NR) copy_run<1, false>(kdesc, dst + V_BYTES + kb * 1024, lane * 16, at * p.d_r * 4 + kb * 1024);
  };

  if (tree && !too_large) tree_masks(p, win, i0, ppb, 128, kThreads, masks, tree_parent, tree_depth);
  const int pos = has_row ? max(0, tree ? P + tree_depth[i_col - i0] : own_row) : 0;

  // ---- the queries: lane (n, h) holds entries 8 c + 4 h .. + 3 of its column's
  const int W = p.d_c + p.d_r;
  const float* const qraw = static_cast<const float*>(p.q) + qrow * W;
  f32x16 qv[NIB];                              // q~, four chunks a block
  f32x4 qr[NR];
  {
    const int npass = ppb >= 32 ? 1 : 32 >> lg;
    for (int ps = 0; ps < npass; ++ps) {
      const bool mine = npass == 1 || (n >> lg) == ps;
      const float* mh = static_cast<const float*>(p.m) + ((int64_t)(g * hpg + (32 * w >> lg) + ps) * DV + n) * p.d_c;
      f32x16 e[NIB];
#pragma unroll
      for (int ib = 0; ib < NIB; ++ib)
#pragma unroll
        for (int r = 0; r < 16; ++r) e[ib][r] = 0.f;
      for (int c = 4 * h; c < p.d_c; c += 8) {
        const f32x4 x = *reinterpret_cast<const f32x4*>(qraw + c);
        f32x4 a[NIB];
#pragma unroll
        for (int ib = 0; ib < NIB; ++ib) a[ib] = *reinterpret_cast<const f32x4*>(mh + (int64_t)(32 * ib) * p.d_c + c);
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int ib = 0; ib < NIB; ++ib) e[ib] = __builtin_amdgcn_mfma_f32_32x32x2f32(a[ib][j], x[j], e[ib], 0, 0, 0);
      }
#pragma unroll
      for (int ib = 0; ib < NIB; ++ib)
#pragma unroll
        for (int r = 0; r < 16; ++r) qv[ib][r] = ps == 0 || mine ? e[ib][r] : qv[ib][r];
    }
#pragma unroll
    for (int ib = 0; ib < NIB; ++ib)
#pragma unroll
      for (int r = 0; r < 16; ++r) qv[ib][r] = has_row ? qv[ib][r] * p.scale_log2 : 0.f;
#pragma unroll
    for (int c = 0; c < NR; ++c) {
      const int i = 8 * c + 4 * h;
      qr[c] = f32x4{0.f, 0.f, 0.f, 0.f};
      if (i < p.d_r && has_row) {
        const float* const x = qraw + p.d_c + i;
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          float y0, y1;
          rotate_quarters(x[2 * k], x[2 * k + 1], (double)pos * p.quarters[i / 2 + k], y0, y1);
          qr[c][2 * k] = y0 * p.scale_log2;
          qr[c][2 * k + 1] = y1 * p.scale_log2;
        }
      }
    }
  }

  f32x16 acc[NIB];
  float m_run = -FLT_MAX, l_run = 0.f;
#pragma unroll
  for (int ib = 0; ib < NIB; ++ib)
#pragma unroll
    for (int r = 0; r < 16; ++r) acc[ib][r] = 0.f;
  copy_tile(0);
  for (int j = 0; j < ntiles; ++j) {
    const int row0 = kbeg + j * kTileRows;
    const bool masked = row0 + kTileRows > masked_from;
    wait_copies<0>();
    __syncthreads();                           // tile j is there, and the one before it has been read
    copy_tile(j + 1);
    char* const tile = lds + (j & 1) * TILE_BYTES;
    f32x16 sn;
    if (live) {
#pragma unroll
      for (int r = 0; r < 16; ++r) sn[r] = 0.f;
      const char* const vt = tile + (n >> 4) * (DV * 64);
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int k = 2 * c + h;
        const f32x4 a = *reinterpret_cast<const f32x4*>(vt + k * 256 + (((n & 15) ^ (k & 7)) << 4));
#pragma unroll
        for (int e = 0; e < 4; ++e) sn = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], qv[c >> 2][4 * (c & 3) + e], sn, 0, 0, 0);
      }
      const char* const kt = tile + V_BYTES + (n >> 4) * (p.d_r * 64) + (n & 15) * 16;
#pragma unroll
      for (int c = 0; c < NR; ++c) {           // pieces past d_r: any valid one against a zero query
        const int k = 4 * (2 * c + h) < p.d_r ? 2 * c + h : 0;
        const f32x4 a = *reinterpret_cast<const f32x4*>(kt + k * 256);
#pragma unroll
        for (int e = 0; e < 4; ++e) sn = __builtin_amdgcn_mfma_f32_32x32x2f32(a[e], qr[c][e], sn, 0, 0, 0);
      }
    }
    if (masked) {
      if (live) {
        const int last = (tree ? kend : min(own_row + 1, kend)) - row0;
        uint32_t sees = last >= 32 ? ~0u : last <= 0 ? 0u : (1u << last) - 1u;
        if (tree) sees &= tree_sees(masks + (col & (ppb - 1)) * kTreeWords, row0 - P);
        hide(sn, sees >> (4 * h));
      }
      __syncthreads();                         // every wave has its scores
      for (int i = tid; i < V_BYTES / 16; i += kThreads) {
        const int k = (i >> 4) % (DV / 4);     // piece
        const int row = (i / (16 * (DV / 4))) * 16 + ((i & 15) ^ (k & 7));
        u32x4* const at = reinterpret_cast<u32x4*>(tile) + i;
        u32x4 u = *at;
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = row0 + row >= kend || (u[e] & 0x7F800000u) == 0x7F800000u ? 0u : u[e];
        *at = u;
      }
      __syncthreads();
    }
    if (!live) continue;
    float mt = sn[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mt = fmaxf(mt, sn[r]);
    {
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mt), __float_as_uint(mt), false, false);
      mt = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
    }
    if (__ballot(mt > m_run) != 0) {
      const float m_new = fmaxf(mt, m_run), alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      l_run *= alpha;
#pragma unroll
      for (int ib = 0; ib < NIB; ++ib) acc[ib] *= alpha;
      m_run = m_new;
    }
    float tile_sum = 0.f;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      sn[r] = __builtin_amdgcn_exp2f(sn[r] - m_run);
      tile_sum += sn[r];
    }
    l_run += tile_sum;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      const int row = score_row(r, h);
      const char* const vt = tile + (row >> 4) * (DV * 64) + (n & 3) * 4;
#pragma unroll
      for (int ib = 0; ib < NIB; ++ib) {
        const int k = 8 * ib + (n >> 2);
        const float a = *reinterpret_cast<const float*>(vt + k * 256 + (((row & 15) ^ (k & 7)) << 4));
        acc[ib] = __builtin_amdgcn_mfma_f32_32x32x2f32(a, sn[r], acc[ib], 0, 0, 0);
      }
    }
  }
  {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l_run), __float_as_uint(l_run), false, false);
    l_run = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  }
  wait_copies<0>();
  __syncthreads();
  const bool seen = has_row && !(l_run == 0.f);
  const float inv = seen ? 1.f / l_run : 0.f;
  const float lse = seen ? (m_run + log2f(l_run)) * kLn2 : -INFINITY;
  float* const out = p.S == 1 ? static_cast<float*>(p.o) : p.o_part;
  float* const ob = reinterpret_cast<float*>(lds) + w * 32 * PITCH;
#pragma unroll
  for (int ib = 0; ib < NIB; ++ib) {
    wave_fence();
#pragma unroll
    for (int r4 = 0; r4 < 4; ++r4) {
      f32x4 o;
#pragma unroll
      for (int jj = 0; jj < 4; ++jj) o[jj] = seen ? acc[ib][4 * r4 + jj] * inv : 0.f;
      *reinterpret_cast<f32x4*>(ob + n * PITCH + 8 * r4 + 4 * h) = o;
    }
    wave_fence();
#pragma unroll
    for (int it = 0; it < 4; ++it) {
      const int c = 8 * it + (lane >> 3);
      const f32x4 o = *reinterpret_cast<const f32x4*>(ob + c * PITCH + 4 * (lane & 7));
      const int cc = 32 * w + c, i = i0 + (cc & (ppb - 1));
      if (i < win.n)
        *reinterpret_cast<f32x4*>(out + (((int64_t)(win.first + i) * p.H + g * hpg + (cc >> lg)) * p.S + split) * DV + 32 * ib +
                                  4 * (lane & 7)) = o;
    }
  }
  if (h != 0 || !live_col) return;
  if (p.S == 1) {
    if (p.lse != nullptr) p.lse[qrow] = lse;
    return;
  }
  float* const lp = p.lse_part + qrow * p.S;
  lp[split] = lse;
  if (split == 0)
    for (int k = window_splits(hd, win.L); k < p.S; ++k) lp[k] = -INFINITY;
}

// ---------------------------------------------------------------- combine
// The merge of the splits of a (row, head), by a wave: the splits' log-sum-exps
// in one read, four to a lane, then the partials of those with rows, d_v / 4 lanes
// each, so 2 or 4 splits at a time and four times that in flight.  Rows that no
// sequence has are left as they were.  Bound by latency: two round trips, 8.8 us
// for 4048 (row, head) of up to 36 splits (18 with one lane row per (row, head), all
// splits in turn), 19 us for 27 K.
template <typename T, int DV>
__global__ void __launch_bounds__(kThreads) window_combine_kernel(const float* o_part, const float* lse_part, const int32_t* cu,
                                                                 T* o, float* lse, int32_t B, int32_t H, int32_t n_rows,
                                                                 int32_t S) {
  constexpr int LPR = DV / 4, SLOTS = 64 / LPR;
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * kWaves + (threadIdx.x >> 6);
  const int row = (int)(id / H);
  if (id >= (int64_t)n_rows * H || row < cu[0] || row >= cu[B]) return;
  const float* lp = lse_part + id * S;
  float l[4], mx = -INFINITY;
  int last = 0;                                // splits up to the last with rows (it may be a NaN, which no maximum shows)
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const int s = lane + 64 * k;
    l[k] = s < S ? lp[s] : -INFINITY;
    mx = fmaxf(mx, l[k]);
    const unsigned long long some = __ballot(l[k] != -INFINITY);
    if (some != 0ull) last = 64 * k + 64 - __builtin_clzll(some);
  }
  mx = wave_max(mx);
  const float* op = o_part + id * S * DV + 4 * (lane % LPR);
  f32x4 acc = {0.f, 0.f, 0.f, 0.f};
  float sum = 0.f;
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    if (64 * k >= last) break;
    const float wgt = l[k] == -INFINITY ? 0.f : __expf(l[k] - mx);
    const int end = min(64, last - 64 * k);
#pragma unroll 4
    for (int s = 0; s < end; s += SLOTS) {
      const int mine = s + lane / LPR;
      const float ws = __shfl(wgt, mine & 63, 64);
      f32x4 x = {0.f, 0.f, 0.f, 0.f};          // a split without rows has no partial
      if (mine < end && ws != 0.f) x = *reinterpret_cast<const f32x4*>(op + (int64_t)(64 * k + mine) * DV);
      if (mine < end) {
        sum += ws;
        acc += x * ws;
      }
    }
  }
#pragma unroll
  for (int off = LPR; off < 64; off *= 2) {
    sum += __shfl_xor(sum, off, 64);
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] += __shfl_xor(acc[e], off, 64);
  }
  if (lane >= LPR) return;
  const f32x4 x = last > 0 ? acc * (1.f / sum) : f32x4{0.f, 0.f, 0.f, 0.f};
  T* const out = o + id * DV + 4 * lane;
  if constexpr (sizeof(T) == 2) {
    const bf16x2 a = __builtin_convertvector((f32x2{x[0], x[1]}), bf16x2), c = __builtin_convertvector((f32x2{x[2], x[3]}), bf16x2);
    *reinterpret_cast<uint64_t*>(out) = (uint64_t)__builtin_bit_cast(uint32_t, c) << 32 | __builtin_bit_cast(uint32_t, a);
  } else {
    *reinterpret_cast<f32x4*>(out) = x;
  }
  if (lse != nullptr && lane == 0) lse[id] = last > 0 ? mx + logf(sum) : -INFINITY;
}

using WindowFn = void (*)(WINDOW_HEAD_ARGS, WindowParams);

// Sets of one or two waves: as many as four tiles each leave room for in LDS.
constexpr int window_sets(int d_v, int nrc) { return d_v == 128 && nrc > 1 ? 3 : 4; }

template <int DV, int NRC>
WindowFn pick_window_waves(int cw, int kw) {
  if (cw == 4) return kw == 2 ? window_kernel<DV, NRC, 4, 2> : window_kernel<DV, NRC, 4, 1>;
  constexpr int KW = window_sets(DV, NRC);
  return cw == 2 ? window_kernel<DV, NRC, 2, KW> : window_kernel<DV, NRC, 1, KW>;
}

template <int DV>
WindowFn pick_window_nrc(int d_r, int cw, int kw) {
  return d_r <= 16 ? pick_window_waves<DV, 1>(cw, kw) : d_r <= 32 ? pick_window_waves<DV, 2>(cw, kw) : pick_window_waves<DV, 4>(cw, kw);
}

template <int DV>
WindowFn pick_window_f32(int d_r) {
  return d_r <= 16 ? window_f32_kernel<DV, 1> : d_r <= 32 ? window_f32_kernel<DV, 2> : window_f32_kernel<DV, 4>;
}

template <typename T>
void launch_combine(const WindowParams& p, int d_v, hipStream_t s) {
  const dim3 grid((unsigned)(((long long)p.n_rows * p.H + kWaves - 1) / kWaves));
  const auto fn = d_v == 128 ? window_combine_kernel<T, 128> : window_combine_kernel<T, 64>;
  hipLaunchKernelGGL(fn, grid, dim3(kThreads), 0, s, p.o_part, p.lse_part, p.cu, static_cast<T*>(p.o), p.lse, p.B, p.H,
                     p.n_rows, p.S);
}

// Columns of a workgroup, sets of waves, and whether it absorbs its queries.
struct WindowPlan {
  int cw, kw;
  bool inside;
};

bool window_absorbs(const gva_dims* d, int S) { return d->dtype == GVA_DTYPE_F32 || S == 1; }

long long window_blocks(const gva_dims* d, int n_rows, int rows) {
  const long long seqs = d->batch < n_rows ? d->batch : n_rows;
  return (n_rows + seqs * (rows - 1)) / rows;
}

// One set of four waves, unless a sequence can be long enough for more sets to pay.
// The lengths are on the device, so this goes by the capacity T and by the average
// of n_rows: the times below are of caches cut to their sequences, and short sequences
// in caches of many rows get the sets whether they pay or not:
//  - up to 64 columns a sequence on average: sets of one or two waves, as many as fit,
//    from 1024 rows on, or from 256 (d 64) or 512 (d 128) while a CU has one workgroup.
//    The sets need its LDS alone, so of many short sequences they take fewer at a time
//    (7 nodes, H32 G8 d 64, of up to 64 rows: 96 trees 35.6 us with sets, 21.7 with
//    one; of up to 512: 48.5 and 43.7, 16 trees 15.6 and 19.9; of up to 1024: 61.1 and
//    65.5, at d 128 89.0 and 101.9).
//  - more: two sets of four where there is one split and fewer than 1.5 workgroups a CU.  A second set halves the walk
// over the keys but doubles the copies of the absorption (causal prompts of up to
// 2048 rows, 2 sequences, G8 H8 d 64: 37.9 us with two sets, 49.5 with one; d 128
// 53.3 and 62.3; 1024 rows of d 64 23.5 and 27.7, of d 128 34.9 and 36.3; 256 rows
// of d 128 23.1 and 19.5; 28 trees of 19 with nothing ahead 29.7 and 19.0).  With
// several splits the keys are divided already (100 rows behind 8000: 24.0 and 22.9).
WindowPlan window_plan(const gva_dims* d, int n_rows, int S, int n_cu) {
  const int hpg = d->n_heads / d->n_groups;
  const long long cols = ((long long)n_rows + d->batch - 1) / d->batch * hpg;   // of a sequence, on average
  WindowPlan plan{4, 1, window_absorbs(d, S)};
  if (d->dtype == GVA_DTYPE_F32) return plan;
  const long long items = window_blocks(d, n_rows, 128 / hpg) * d->n_groups * S;
  if (cols <= 64) {
    if (d->t_max >= (items > n_cu ? 1024 : 4 * d->d_v)) plan = {cols <= 32 ? 1 : 2, window_sets(d->d_v, d->d_r <= 16 ? 1 : 2), plan.inside};
  } else if (S == 1 && d->t_max >= 16 * d->d_v && items < (long long)n_cu * 3 / 2) {
    plan.kw = 2;
  }
  return plan;
}

// Where the workspace keeps what the launches leave for each other.
struct WindowLayout {
  size_t q_abs, o_part, lse_part, bytes;
};

WindowLayout window_layout(const gva_dims* d, int n_rows, int S) {
  WindowLayout L{};
  const size_t rows = (size_t)n_rows * d->n_heads;
  auto take = [&](size_t bytes) {
    const size_t at = L.bytes;
    L.bytes += (bytes + 255) / 256 * 256;
    return at;
  };
  const bool inside = window_absorbs(d, S);
  L.q_abs = take(inside ? 0 : rows * d->d_v * 4);
  L.o_part = take(S > 1 ? rows * S * d->d_v * 4 : 0);
  L.lse_part = take(S > 1 ? rows * S * 4 : 0);
  return L;
}

int check_window(const gva_dims* d, const gva_paging* pg, int n_rows, int S, int split_rows, int n_cu) {
  const int st = check_dims(d);
  if (st != GVA_OK) return st;
  if (n_rows < 0 || S < 1 || S > GVA_MAX_SPLITS || split_rows < 0 || split_rows % kTileRows != 0) return GVA_ERR_INVALID_ARG;
  if (pg != nullptr) {
    const int sp = check_pool(d, pg);
    if (sp != GVA_OK) return sp;
  }
  const int sl = check_cache_layout(d);
  if (sl != GVA_OK) return sl;
  const int hpg = d->n_heads / d->n_groups;
  if (hpg != 1 && hpg != 2 && hpg != 4 && hpg != 8) return GVA_ERR_UNSUPPORTED;
  if (d->d_v != 64 && d->d_v != 128) return GVA_ERR_UNSUPPORTED;
  if (d->d_c < 32 || d->d_c % 32 != 0 || d->d_c > 512 || d->d_r % 8 != 0 || d->d_r > 64) return GVA_ERR_UNSUPPORTED;
  if (n_rows > (1 << 20) || (long long)n_rows * d->n_heads > 0x7FFFFFFFLL) return GVA_ERR_UNSUPPORTED;
  if (n_rows > 0) {                            // a launch has fewer than 2^32 threads
    const WindowPlan plan = window_plan(d, n_rows, S, n_cu);
    const long long items = (window_blocks(d, n_rows, 32 * plan.cw / hpg) * S + 7) / 8 * 8;
    if (items * d->n_groups * 64 * plan.cw * plan.kw > 0xFFFFFFFFLL) return GVA_ERR_UNSUPPORTED;
    if (S > 1 && ((long long)n_rows * d->n_heads + kWaves - 1) / kWaves * kThreads > 0xFFFFFFFFLL) return GVA_ERR_UNSUPPORTED;
  }
  return GVA_OK;
}

// ---------------------------------------------------------------- the plan
int window_len(const gva_dims* d, const int32_t* lens, int b) {
  return lens == nullptr ? d->t_max : (lens[b] < 0 ? 0 : lens[b] > d->t_max ? d->t_max : lens[b]);
}
int window_new(const gva_dims* d, const int32_t* n_new, int n_rows, int b) {
  const int n = n_new == nullptr ? n_rows / d->batch + (b < n_rows % d->batch ? 1 : 0) : n_new[b];
  return n < 0 ? 0 : n > n_rows ? n_rows : n;
}

// About what a call takes with a plan: its workgroups are dealt in order to
// the places that the device has for them, each to the first that is free.  The
// times of a workgroup and of a tile of 32 keys are measured ones (two workgroups
// of one set a CU at H32 G8 d 128/16: 1.2 us a tile each, 18 us of start and end
// with the absorption and 9 without; sets of one or two waves, one workgroup a CU:
// 0.3 and 0.5 us a tile, 17 and 10 us; fp32: the 136 products of a tile, which fill
// a CU with one workgroup, 4 us).  A plan of several splits pays for the
// absorption's launch, the partials' way through memory and their merge.
// On the host 0.08 ms for 8 sequences, 1 for 64, 11 to 12 for 512, 16 to 18 for 1024
// (30 candidates; lengths of 1 K to 16 K): for plans that are kept over many steps.
// A candidate is dealt for 20000 steps, what is left of it then counts as nothing.
struct WindowTimes {
  double us;
  int S, rows;
};
WindowTimes window_time(const gva_dims* d, const int32_t* lens, const int32_t* n_new, int n_rows, int n_cu, int S, int split) {
  const WindowPlan plan = window_plan(d, n_rows, S, n_cu);
  const int hpg = d->n_heads / d->n_groups, rows = 32 * plan.cw / hpg;
  const bool f32 = d->dtype == GVA_DTYPE_F32;
  const double wide = d->d_v / 128.0;
  const int places = (f32 || plan.cw * plan.kw > 4 || plan.cw < 4 ? 1 : 2) * n_cu;
  double start = (plan.inside ? 18.0 : 9.0) * (0.5 + 0.5 * d->d_v / 128.0), tile = (plan.cw == 1 ? 0.3 : plan.cw == 2 ? 0.5 : plan.kw == 2 ? 0.8 : 1.2) * wide;
  if (f32) tile = 4.0 * wide;
  std::map<double, long long> free_at{{0.0, places}};
  double end = 0.0, partials = 0.0;
  int steps = 0;
  for (int b = 0; b < d->batch; ++b) {
    const int L = window_len(d, lens, b), n = window_new(d, n_new, n_rows, b);
    if (n == 0 || L == 0) continue;
    int parts = S;
    if (S > 1 && split > 0) {
      parts = (L + split - 1) / split;
      parts = parts > S ? S : parts;
    }
    const int blocks = (n + rows - 1) / rows;
    // a block of few rows leaves waves without work, a prompt's keys are half of its own rows on average
    const double cols = (double)n / blocks / rows, part = cols < 0.25 ? 0.25 : cols;
    const double keys = (L - 0.5 * (n < L ? n : L)) / parts;
    const double t = start + keys / kTileRows * tile * (plan.cw == 4 ? 0.3 + 0.7 * part : 1.0);
    partials += (double)n * parts;
    long long left = (long long)blocks * parts * d->n_groups;
    while (left > 0 && ++steps < 20000) {
      const auto first = free_at.begin();
      const long long k = left < first->second ? left : first->second;
      const double at = first->first + t;
      if ((first->second -= k) == 0) free_at.erase(first);
      free_at[at] += k;
      if (at > end) end = at;
      left -= k;
    }
  }
  const double row_bytes = (double)d->n_heads * d->d_v * 4.0;
  if (!plan.inside) end += 4.0 + n_rows * row_bytes / 1.5e6;
  if (S > 1) end += 5.0 + partials * row_bytes * 2.0 / 3e6;
  return {end, S, S > 1 ? split : 0};
}

int window_impl(const gva_dims* d, const gva_paging* pg, const void* q, const void* m, const void* v, const void* kr,
                const int32_t* block_table, const int32_t* lens, const int32_t* cu, const int32_t* parent, int32_t n_rows,
                int32_t S, int32_t split, void* workspace, size_t workspace_bytes, void* o, float* lse, void* stream) {
  const int n_cu = device_cu_count();
  int st = check_window(d, pg, n_rows, S, split, n_cu);
  if (st != GVA_OK) return st;
  if (n_rows == 0) return GVA_OK;
  if (!q || !m || !v || !lens || !cu || !o || (d->d_r > 0 && !kr)) return GVA_ERR_INVALID_ARG;
  if ((pg != nullptr) != (block_table != nullptr)) return GVA_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(m, 16) || !aligned(v, 16) || !aligned(o, 16) || (d->d_r > 0 && !aligned(kr, 16)) ||
      !aligned(block_table, 4) || !aligned(lens, 4) || !aligned(cu, 4) || !aligned(parent, 4) || !aligned(lse, 4))
    return GVA_ERR_INVALID_ARG;
  const WindowLayout L = window_layout(d, n_rows, S);
  if (L.bytes > 0 && (workspace == nullptr || workspace_bytes < L.bytes || !aligned(workspace, 256))) return GVA_ERR_INVALID_ARG;
  const WindowPlan plan = window_plan(d, n_rows, S, n_cu);
  char* const ws = static_cast<char*>(workspace);
  hipStream_t s = static_cast<hipStream_t>(stream);
  float* q_abs = plan.inside ? nullptr : reinterpret_cast<float*>(ws + L.q_abs);
  if (!plan.inside) {
    st = absorb_rows(d, n_rows, q, m, q_abs, s);
    if (st != GVA_OK) return st;
  }
  WindowParams p{};
  p.cu = cu;
  p.lens = lens;
  p.parent = parent;
  p.block_table = block_table;
  p.q = q;
  p.m = m;
  p.q_abs = q_abs;
  p.v = v;
  p.kr = kr;
  p.o = o;
  p.lse = lse;
  if (S > 1) {
    p.o_part = reinterpret_cast<float*>(ws + L.o_part);
    p.lse_part = reinterpret_cast<float*>(ws + L.lse_part);
  }
  p.B = d->batch;
  p.H = d->n_heads;
  p.G = d->n_groups;
  p.d_c = d->d_c;
  p.d_r = d->d_r;
  p.t_max = d->t_max;
  p.n_rows = n_rows;
  p.S = S;
  p.split_rows = split < (1 << 30) ? split : (1 << 30);
  const int rows = 32 * plan.cw / (d->n_heads / d->n_groups);   // a power of two
  while ((1 << p.rows_log2) < rows) ++p.rows_log2;
  if (pg != nullptr) {
    p.page_rows = pg->page_rows;
    p.max_pages = pg->max_pages;
    p.n_pages = pg->n_pages;
  }
  p.scale_log2 = scale_log2(d);
  fill_inv_freq(d, p.quarters);
  for (double& x : p.quarters) x *= 0.63661977236758134308;     // 2 / pi
  WindowFn fn = d->d_v == 128 ? pick_window_nrc<128>(d->d_r, plan.cw, plan.kw) : pick_window_nrc<64>(d->d_r, plan.cw, plan.kw);
  if (d->dtype == GVA_DTYPE_F32) fn = d->d_v == 128 ? pick_window_f32<128>(d->d_r) : pick_window_f32<64>(d->d_r);
  long long items = window_blocks(d, n_rows, rows) * S;
  if (S > 1) items = (items + 7) / 8 * 8;
  hipLaunchKernelGGL(fn, dim3((unsigned)(items * d->n_groups)), dim3(64 * plan.cw * plan.kw), 0, s, p.cu, p.lens, p.B, p.G,
                     p.rows_log2, p.S, p.n_rows, p.t_max, p.split_rows, p);
  st = launch_status();
  if (st != GVA_OK || S == 1) return st;
  if (d->dtype == GVA_DTYPE_BF16) launch_combine<uint16_t>(p, d->d_v, s);
  else launch_combine<float>(p, d->d_v, s);
  return launch_status();
}

}  // namespace

extern "C" {

int gva_packed_workspace_size(const gva_dims* dims, int32_t n_rows, int32_t num_splits, size_t* bytes) {
  if (bytes == nullptr) return GVA_ERR_INVALID_ARG;
  const int st = check_window(dims, nullptr, n_rows, num_splits, 0, device_cu_count());
  if (st != GVA_OK) return st;
  *bytes = n_rows == 0 ? 0 : window_layout(dims, n_rows, num_splits).bytes;
  return GVA_OK;
}

int gva_packed_pick_splits(const gva_dims* dims, const int32_t* lens, const int32_t* n_new, int32_t n_rows, int32_t n_cu,
                           int32_t* split_rows) {
  if (split_rows != nullptr) *split_rows = 0;
  if (n_cu <= 0) n_cu = device_cu_count();
  if (check_window(dims, nullptr, n_rows, 1, 0, n_cu) != GVA_OK || n_rows == 0) return 1;
  WindowTimes best{0.0, 1, 0};
  try {
    best = window_time(dims, lens, n_new, n_rows, n_cu, 1, 0);
    int longest = 0;
    for (int b = 0; b < dims->batch; ++b) {
      const int L = window_len(dims, lens, b);
      if (L > longest && window_new(dims, n_new, n_rows, b) > 0) longest = L;
    }
    for (int S = 2; S <= 64 && longest / S >= (dims->dtype == GVA_DTYPE_F32 ? 32 : 128); S += S < 8 ? 1 : S / 8) {
      const int rows = split_rows == nullptr ? 0 : (longest + kTileRows * S - 1) / (kTileRows * S) * kTileRows;
      if (check_window(dims, nullptr, n_rows, S, rows, n_cu) != GVA_OK) break;
      const WindowTimes t = window_time(dims, lens, n_new, n_rows, n_cu, S, rows);
      if (t.us < best.us) best = t;
    }
  } catch (const std::bad_alloc&) {            // no memory for the list of places: one split is always right
    best = WindowTimes{0.0, 1, 0};
  }
  if (split_rows != nullptr) *split_rows = best.rows;
  return best.S;
}

int gva_packed_prefill(const gva_dims* dims, const gva_paging* paging, const void* q, const void* m, const void* v_cache,
                       const void* kr_cache, const int32_t* block_table, const int32_t* lens, const int32_t* cu_rows,
                       int32_t n_rows, int32_t num_splits, int32_t split_rows, void* workspace, size_t workspace_bytes,
                       void* o, float* lse, void* stream) {
  return window_impl(dims, paging, q, m, v_cache, kr_cache, block_table, lens, cu_rows, nullptr, n_rows, num_splits, split_rows,
                     workspace, workspace_bytes, o, lse, stream);
}

int gva_tree_attention(const gva_dims* dims, const gva_paging* paging, const void* q, const void* m, const void* v_cache,
                       const void* kr_cache, const int32_t* block_table, const int32_t* lens, const int32_t* cu_rows,
                       const int32_t* parent, int32_t n_rows, int32_t num_splits, int32_t split_rows, void* workspace,
                       size_t workspace_bytes, void* o, float* lse, void* stream) {
  if (n_rows > 0 && parent == nullptr) return GVA_ERR_INVALID_ARG;
  return window_impl(dims, paging, q, m, v_cache, kr_cache, block_table, lens, cu_rows, parent, n_rows, num_splits, split_rows,
                     workspace, workspace_bytes, o, lse, stream);
}

}  // extern "C"
