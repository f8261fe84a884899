// libgva.so -- many requests on one pool of pages: block tables and slot maps
// from the requests' lengths (gva_page_tables), and what of a drafted tree is
// kept (gva_tree_commit).

#include "gva_window.h"

namespace {

// ========================================================== tables and slots
// One launch, no workspace, no atomics.  Every workgroup adds up what all
// sequences give back, need and bring (three sums over B, each thread a run of
// sequences, then a scan over the threads), and then does its share: some a wave
// per sequence for the table and the stack, the others a thread per packed row for
// the maps.  A row's page, or a page that is handed out, is found from those sums
// alone, never read back from what another workgroup writes: entry i of the stack
// is free_pages[i] below the old n_free, where nothing is written, and above it a
// page of a sequence that shrinks, whose table row nothing is written to either.
// Bound by latency: the lengths' loads, the scan, the search, a dependent load, the
// stores.  Up to kKept sequences' lengths stay in LDS, and divisions by the page size
// go by its reciprocal: 5.6 us for 512 sequences and 49 K rows, 3.7 to 4.3 for 64 and
// 64 (8.2 and 4.9 with the lengths read again and the integer divisions).
constexpr int kKept = 2048;

struct TablesParams {
  const int32_t* lens;
  const int32_t* n_new;
  int32_t* table;
  int32_t* free_pages;
  const int32_t* n_free;
  int32_t* new_lens;
  int32_t* new_n_free;
  int32_t* cu;
  int32_t* seq;
  int32_t* row;
  int32_t* slot;
  int32_t B, t_max, page_rows, max_pages, n_pages, n_rows;
  int32_t row_blocks;           // workgroups of the maps, ahead of those of the tables
  float inv_units;              // 32 / page_rows
};

// x / page_rows of a row x >= 0: whole 32-row units by the reciprocal, whose
// quotient, of at most 4096 pages, is off by one at the most.
__device__ __forceinline__ int page_of(const TablesParams& p, int x) {
  const int units = x >> 5, per = p.page_rows >> 5;
  int q = (int)((float)units * p.inv_units);
  const int r = units - q * per;
  q += r >= per ? 1 : 0;
  q -= r < 0 ? 1 : 0;
  return q;
}
__device__ __forceinline__ int pages_of(const TablesParams& p, int rows) { return rows > 0 ? page_of(p, rows - 1) + 1 : 0; }

struct Request {
  int len, n;                   // cached rows, rows to come (or to go)
  int have, hold;               // pages before and after
  bool fits;
};

__device__ __forceinline__ Request request_of(const TablesParams& p, int len, int n) {
  Request r;
  r.len = len;
  r.n = n;
  r.fits = n <= p.t_max - len;
  r.have = pages_of(p, len);
  r.hold = r.fits ? pages_of(p, len + n) : r.have;
  return r;
}

// What sequences give back, need and bring.
struct Sums {
  int back, need;
  long long rows;
};
__device__ __forceinline__ void add_request(Sums& s, const Request& r) {
  s.back += r.n < 0 ? r.have - r.hold : 0;
  s.need += r.n > 0 ? r.hold - r.have : 0;
  s.rows += r.n > 0 ? r.n : 0;
}

__device__ __forceinline__ long long wave_incl_scan64(long long v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const long long u = __shfl_up(v, o, 64);
    if (lane >= o) v += u;
  }
  return v;
}

__global__ void __launch_bounds__(kThreads) page_tables_kernel(TablesParams p) {
  // of the sequences before each thread's run; at kThreads those of all
  __shared__ int s_back[kThreads + 1], s_need[kThreads + 1];
  __shared__ long long s_rows[kThreads + 1];
  __shared__ Sums s_wave[kWaves];
  __shared__ int2 s_kept[kKept];
  const int tid = threadIdx.x, lane = tid & 63, w = tid >> 6;
  const int run = (p.B + kThreads - 1) / kThreads;
  const bool kept = p.B <= kKept;
  const int old_free = min(max(p.n_free[0], 0), p.n_pages);
  auto read = [&](int b) {
    const int len = clamp_len(p.lens, b, p.t_max), n = p.n_new[b];
    return make_int2(len, n < -len ? -len : (n > p.t_max ? p.t_max : n));
  };
  auto request = [&](int b) {
    const int2 x = kept ? s_kept[b] : read(b);
    return request_of(p, x.x, x.y);
  };
  Sums mine{0, 0, 0};
  for (int j = 0; j < run; ++j) {
    const int b = tid * run + j;
    if (b < p.B) {
      const int2 x = read(b);
      if (kept) s_kept[b] = x;
      add_request(mine, request_of(p, x.x, x.y));
    }
  }
  Sums in{wave_incl_scan(mine.back), wave_incl_scan(mine.need), wave_incl_scan64(mine.rows)};
  if (lane == 63) s_wave[w] = in;
  __syncthreads();
  Sums before{0, 0, 0};
#pragma unroll
  for (int k = 0; k < kWaves; ++k)
    if (k < w) {
      before.back += s_wave[k].back;
      before.need += s_wave[k].need;
      before.rows += s_wave[k].rows;
    }
  s_back[tid + 1] = before.back + in.back;
  s_need[tid + 1] = before.need + in.need;
  s_rows[tid + 1] = before.rows + in.rows;
  if (tid == 0) {
    s_back[0] = s_need[0] = 0;
    s_rows[0] = 0;
  }
  __syncthreads();
  const int top = min(old_free + s_back[kThreads], p.n_pages);   // entries of the stack before it is taken from

  // entry i of the stack
  auto entry = [&](int i) {
    if (i < old_free) return p.free_pages[i];
    int k = i - old_free, lo = 0, hi = kThreads;         // s_back[lo] <= k < s_back[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2;
      if (s_back[mid] <= k) lo = mid;
      else hi = mid;
    }
    k -= s_back[lo];
    for (int b = lo * run; b < p.B; ++b) {
      const Request r = request(b);
      const int back = r.n < 0 ? r.have - r.hold : 0;
      if (k < back) return p.table[(long long)b * p.max_pages + r.hold + k];
      k -= back;
    }
    return -1;
  };
  auto granted = [&](const Request& r, const Sums& s) {
    const int need = r.n > 0 ? r.hold - r.have : 0;
    return r.fits && (need == 0 || s.need + need <= top);
  };

  if ((int)blockIdx.x < p.row_blocks) {        // the packed rows
    // (unsigned: a step behind the last of 2^31 - 1 rows is past 2^31)
    for (unsigned i = blockIdx.x * kThreads + tid; i < (unsigned)p.n_rows; i += p.row_blocks * kThreads) {
      int seq = -1, row = -1, slot = -1;
      if (i < s_rows[kThreads]) {
        int lo = 0, hi = kThreads;                         // s_rows[lo] <= i < s_rows[hi]
        while (hi - lo > 1) {
          const int mid = (lo + hi) / 2;
          if (s_rows[mid] <= i) lo = mid;
          else hi = mid;
        }
        Sums s{0, s_need[lo], s_rows[lo]};
        Request r = request(seq = min(lo * run, p.B - 1));
        while (i >= s.rows + max(r.n, 0) && seq < p.B - 1) {
          add_request(s, r);
          r = request(++seq);
        }
        if (granted(r, s)) {
          row = r.len + (int)(i - s.rows);
          const int pg = page_of(p, row);
          const int id = pg < r.have ? p.table[(long long)seq * p.max_pages + pg] : entry(top - 1 - s.need - (pg - r.have));
          if (id >= 0 && id < p.n_pages) slot = id * p.page_rows + row - pg * p.page_rows;
        }
      }
      if (p.seq != nullptr) p.seq[i] = seq;
      if (p.row != nullptr) p.row[i] = row;
      if (p.slot != nullptr) p.slot[i] = slot;
    }
    return;
  }
  const int x = blockIdx.x - p.row_blocks, blocks = gridDim.x - p.row_blocks;
  for (int b = x * kWaves + w; b < p.B; b += blocks * kWaves) {
    const Request r = request(b);
    const int t = b / run;
    Sums s{s_back[t], s_need[t], s_rows[t]};   // of the sequences before b
    for (int j = t * run; j < b; ++j) add_request(s, request(j));
    const bool ok = granted(r, s);
    if (lane == 0) {
      p.new_lens[b] = r.n > 0 && !ok ? r.len : r.len + r.n;
      p.cu[b] = (int)(s.rows < p.n_rows ? s.rows : p.n_rows);
    }
    int32_t* const entries = p.table + (long long)b * p.max_pages;
    if (r.n < 0)
      for (int j = lane; j < r.have - r.hold; j += 64) {
        const int to = old_free + s.back + j;
        if (to < p.n_pages) p.free_pages[to] = entries[r.hold + j];
      }
    if (r.n > 0 && ok)
      for (int j = lane; j < r.hold - r.have; j += 64) entries[r.have + j] = entry(top - 1 - s.need - j);
  }
  if (x > 0 || w > 0) return;
  if (lane == 0) p.cu[p.B] = (int)(s_rows[kThreads] < p.n_rows ? s_rows[kThreads] : p.n_rows);
  // All that is granted: those refused are the last that need any, so it is
  // the largest sum that fits.
  int given = 0;
  for (int t = lane; t < kThreads; t += 64) {
    if (s_need[t] > top) continue;
    if (s_need[t + 1] <= top) {
      given = max(given, s_need[t + 1]);
      continue;
    }
    int need = s_need[t];
    given = max(given, need);
    for (int b = t * run; b < min((t + 1) * run, p.B); ++b) {
      const Request r = request(b);
      need += r.n > 0 ? r.hold - r.have : 0;
      if (need <= top) given = max(given, need);
    }
  }
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) given = max(given, __shfl_xor(given, o, 64));
  if (lane == 0) p.new_n_free[0] = top - given;
}

// n int32 from p on.
struct Span {
  const int32_t* p;
  long long n;
};
bool overlap(const Span& a, const Span& b) {
  return a.p != nullptr && b.p != nullptr && a.n > 0 && b.n > 0 && a.p < b.p + b.n && b.p < a.p + a.n;
}

// ================================================================== commit
// A workgroup per sequence and group, and one more for the positional keys.
// Every wave holds the parents, four to a lane, walks from the leaf up by lane reads
// and has the path as 256 bits; a node's place on it is the number of bits below
// its own.  (Walked by one thread over parents in LDS, with two barriers, a commit
// of 32 trees of 64 took 4.9 us, now 4.4.)  Rows move toward the front: a_k
// >= k and the path rises, so row k of the path overwrites only rows that earlier
// rows of it were read from, or itself; kThreads pieces are read, then written, at
// a time, in order.  Bound by latency: the parents, the walk, a row's read and write.
struct CommitParams {
  void* v;
  void* kr;
  const int32_t* table;
  const int32_t* lens;
  const int32_t* cu;
  const int32_t* parent;
  const int32_t* leaf;
  int32_t* new_lens;
  int32_t* accepted;
  int32_t B, G, t_max, n_rows, v_pieces, kr_pieces;   // 16-byte pieces of a row
  int32_t page_rows, max_pages, n_pages;
};

__global__ void __launch_bounds__(kThreads) tree_commit_kernel(CommitParams p) {
  __shared__ int16_t node[kMaxTree];           // the k-th from the root
  static_assert(kMaxTree == 256, "four nodes a lane");
  const int b = blockIdx.x, g = blockIdx.y, tid = threadIdx.x, lane = tid & 63;
  const int first = min(max(p.cu[b], 0), p.n_rows);
  const int n = max(min(max(p.cu[b + 1], 0), p.n_rows) - first, 0);
  const int L = clamp_len(p.lens, b, p.t_max);
  const int leaf = p.leaf[b];
  const int P = L - n;
  const bool takes = n <= kMaxTree && P >= 0 && leaf >= 0 && leaf < n;
  int len = 0;
  if (takes) {
    int up[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int i = lane + 64 * k, a = i < n ? p.parent[first + i] : -1;
      up[k] = a >= 0 && a < i ? a : -1;
    }
    unsigned long long on[4] = {0ull, 0ull, 0ull, 0ull};
    if (n <= 64) {                             // from a node to one before it: it ends
      for (int i = leaf; i >= 0; i = __builtin_amdgcn_readlane(up[0], i)) on[0] |= 1ull << i;
    } else {
      for (int i = leaf; i >= 0;) {
        const int l = i & 63, k = i >> 6;
        const unsigned long long bit = 1ull << l;
        on[0] |= k == 0 ? bit : 0ull;
        on[1] |= k == 1 ? bit : 0ull;
        on[2] |= k == 2 ? bit : 0ull;
        on[3] |= k == 3 ? bit : 0ull;
        i = __builtin_amdgcn_readlane(k == 0 ? up[0] : k == 1 ? up[1] : k == 2 ? up[2] : up[3], l);
      }
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (on[k] >> lane & 1ull) node[len + __popcll(on[k] & ((1ull << lane) - 1ull))] = (int16_t)(lane + 64 * k);
      len += __popcll(on[k]);
    }
  }
  __syncthreads();                             // (all waves wrote the same)
  if (g == 0) {
    if (tid == 0) p.new_lens[b] = max(P, 0) + len;
    if (p.accepted != nullptr)
      for (int i = tid; i < n; i += kThreads) p.accepted[first + i] = i < len ? node[i] : -1;
  }
  // the pieces of a row of this stream, and where row t's piece c lies
  const bool keys = g == p.G;
  const int npc = keys ? p.kr_pieces : p.v_pieces;
  u32x4* const base = static_cast<u32x4*>(keys ? p.kr : p.v);
  const int rows = p.table != nullptr ? p.page_rows : p.t_max;
  auto place = [&](int t, int c, long long& at) {
    long long page = b;
    if (p.table != nullptr) {
      page = p.table[(long long)b * p.max_pages + t / rows];
      if (page < 0 || page >= p.n_pages) return false;
      t %= rows;
    }
    at = ((keys ? page : page * p.G + g) * rows + t / kLayoutRows * kLayoutRows) * npc + c * kLayoutRows + t % kLayoutRows;
    return true;
  };
  const long long total = (long long)len * npc;
  for (long long i0 = 0; i0 < total; i0 += kThreads) {
    const long long i = i0 + tid;
    const int k = (int)(i / npc), c = (int)(i % npc);
    long long from = 0, to = 0;
    const bool moves = i < total && node[k] != k && place(P + node[k], c, from) && place(P + k, c, to);
    u32x4 piece = {0u, 0u, 0u, 0u};
    if (moves) piece = base[from];
    __syncthreads();                           // all of these rows have been read
    if (moves) base[to] = piece;
    __syncthreads();
  }
}

}  // namespace

extern "C" {

int gva_page_tables(const gva_dims* dims, const gva_paging* paging, const int32_t* lens, const int32_t* n_new,
                    int32_t* block_table, int32_t* free_pages, const int32_t* n_free, int32_t n_rows, int32_t* new_lens,
                    int32_t* new_n_free, int32_t* cu_rows, int32_t* seq, int32_t* row, int32_t* slot, void* stream) {
  int st = check_dims(dims);
  if (st != GVA_OK) return st;
  st = check_pool(dims, paging);
  if (st != GVA_OK) return st;
  if (n_rows < 0) return GVA_ERR_INVALID_ARG;
  if (!lens || !n_new || !block_table || !free_pages || !n_free || !new_lens || !new_n_free || !cu_rows) return GVA_ERR_INVALID_ARG;
  for (const void* x : {(const void*)lens, (const void*)n_new, (const void*)block_table, (const void*)free_pages,
                        (const void*)n_free, (const void*)new_lens, (const void*)new_n_free, (const void*)cu_rows,
                        (const void*)seq, (const void*)row, (const void*)slot})
    if (!aligned(x, 4)) return GVA_ERR_INVALID_ARG;
  const int B = dims->batch;
  const Span small_in[] = {{lens, B}, {n_new, B}, {n_free, 1}}, small_out[] = {{new_lens, B}, {cu_rows, B + 1}, {new_n_free, 1}};
  for (const Span& in : small_in)
    for (const Span& out : small_out)
      if (overlap(in, out)) return GVA_ERR_INVALID_ARG;
  if (B > 65535 || (long long)paging->n_pages * paging->page_rows > 0x7FFFFFFFLL) return GVA_ERR_UNSUPPORTED;
  // workgroups read all lengths, and some entries of the table and the stack, while others write
  const Span large[] = {{block_table, (long long)B * paging->max_pages}, {free_pages, paging->n_pages}};
  const Span maps[] = {{seq, n_rows}, {row, n_rows}, {slot, n_rows}};
  if (overlap(large[0], large[1])) return GVA_ERR_INVALID_ARG;
  for (const Span& map : maps)
    for (const Span& in : small_in)
      if (overlap(in, map)) return GVA_ERR_INVALID_ARG;
  for (const Span& x : large) {
    for (const Span& map : maps)
      if (overlap(x, map)) return GVA_ERR_INVALID_ARG;
    for (const Span& in : small_in)
      if (overlap(x, in)) return GVA_ERR_INVALID_ARG;
    for (const Span& out : small_out)
      if (overlap(x, out)) return GVA_ERR_INVALID_ARG;
  }
  const long long most = device_cu_count();
  const auto capped = [&](long long n) { return (int)(n < most ? n : most); };
  TablesParams p{lens, n_new, block_table, free_pages, n_free, new_lens, new_n_free, cu_rows, seq, row, slot,
                 B, dims->t_max, paging->page_rows, paging->max_pages, paging->n_pages, n_rows, 0, 32.f / (float)paging->page_rows};
  if (seq || row || slot) p.row_blocks = capped(((long long)n_rows + kThreads - 1) / kThreads);
  const int grid = p.row_blocks + capped((B + kWaves - 1) / kWaves);
  hipLaunchKernelGGL(page_tables_kernel, dim3((unsigned)grid), dim3(kThreads), 0, static_cast<hipStream_t>(stream), p);
  return launch_status();
}

int gva_tree_commit(const gva_dims* dims, const gva_paging* paging, void* v_cache, void* kr_cache, const int32_t* block_table,
                    const int32_t* lens, const int32_t* cu_rows, const int32_t* parent, const int32_t* leaf, int32_t n_rows,
                    int32_t* new_lens, int32_t* accepted, void* stream) {
  int st = check_dims(dims);
  if (st != GVA_OK) return st;
  if (n_rows < 0 || (paging != nullptr) != (block_table != nullptr)) return GVA_ERR_INVALID_ARG;
  if (paging != nullptr) {
    st = check_pool(dims, paging);
    if (st != GVA_OK) return st;
  }
  if (!v_cache || !lens || !cu_rows || !leaf || !new_lens || (dims->d_r > 0 && !kr_cache) || (n_rows > 0 && !parent))
    return GVA_ERR_INVALID_ARG;
  if (!aligned(v_cache, 16) || (dims->d_r > 0 && !aligned(kr_cache, 16)) || !aligned(block_table, 4) || !aligned(lens, 4) ||
      !aligned(cu_rows, 4) || !aligned(parent, 4) || !aligned(leaf, 4) || !aligned(new_lens, 4) || !aligned(accepted, 4))
    return GVA_ERR_INVALID_ARG;
  const long long B = dims->batch;
  const Span in[] = {{lens, B}, {cu_rows, B + 1}, {leaf, B}, {parent, n_rows}};
  if (overlap(in[0], {new_lens, B})) return GVA_ERR_INVALID_ARG;
  st = check_cache_layout(dims);
  if (st != GVA_OK) return st;
  for (const Span& x : in)                     // a sequence's other workgroups may read them later
    if (overlap(x, {new_lens, B}) || overlap(x, {accepted, n_rows})) return GVA_ERR_INVALID_ARG;
  const int streams = dims->n_groups + (dims->d_r > 0 ? 1 : 0);
  if (streams > 65535) return GVA_ERR_UNSUPPORTED;
  const int piece = (int)(16 / elem_size(dims));
  CommitParams p{v_cache, kr_cache, block_table, lens, cu_rows, parent, leaf, new_lens, accepted, dims->batch, dims->n_groups,
                 dims->t_max, n_rows, dims->d_v / piece, dims->d_r / piece,
                 paging ? paging->page_rows : 0, paging ? paging->max_pages : 0, paging ? paging->n_pages : 0};
  hipLaunchKernelGGL(tree_commit_kernel, dim3(dims->batch, streams), dim3(kThreads), 0, static_cast<hipStream_t>(stream), p);
  return launch_status();
}

}  // extern "C"
