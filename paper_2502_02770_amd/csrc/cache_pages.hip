// Pages of the cache: handed out, shared, given back (table and counts, integers only), copied and compacted (one layer's
// pools, bits only).  The state of the pool is one count per page; a page is free when its count is 0, and pages are
// handed out from the lowest free one up in the order of the requests.  Counts change by integer atomics, whose order
// does not matter, and the order of handing out is a prefix sum, so tables and counts never depend on timing.
#include <algorithm>
#include "tw_common.h"

namespace {

constexpr int TAKE_THREADS = 1024, TAKE_WAVES = TAKE_THREADS / 64;
constexpr int TAKE_STEPS = 16;                   // counts per lane and pass of the search for free pages
constexpr int TAKE_PASS = TAKE_THREADS * TAKE_STEPS;

struct PagesArgs {
  int32_t* table;                                // kv->page_table
  const int32_t* seq_lens;
  int32_t* ref;
  uint32_t* status;
  int batch, max_pages;
  unsigned pool_pages;
  // reserve
  const int32_t* n_new;
  int max_new;
  // free
  const int32_t* first;
  const int32_t* end;
  // fork
  const int32_t* parent;
  int new_batch;
  int32_t* new_table;
  int32_t* new_lens;
  int32_t* copy_src;
  int32_t* copy_dst;
  // workspace of the hand-out: requests before each row, the pages found
  int32_t* ws_before;
  int32_t* ws_found;
};

__device__ __forceinline__ int row_len(const PagesArgs& a, int b) {
  return max(0, min(a.seq_lens[b], a.max_pages * TW_PAGE));
}

// Every entry of the range loses its page.  Bound by the atomics' trips to memory; one thread per entry, all rows at once.
__global__ __launch_bounds__(256) void pages_free_kernel(PagesArgs a) {
  const int b = blockIdx.y;
  const int lo = min(max(a.first[b], 0), a.max_pages), hi = min(a.end[b], a.max_pages);   // (both: what is added to lo stays in 32 bits)
  for (int p = lo + (int)(blockIdx.x * 256 + threadIdx.x); p < hi; p += (int)gridDim.x * 256) {
    int32_t* e = a.table + (long long)b * a.max_pages + p;
    const int id = *e;
    if ((unsigned)id >= a.pool_pages) continue;
    *e = -1;
    if (atomicAdd(a.ref + id, -1) <= 0) {        // more references given back than there were
      atomicAdd(a.ref + id, 1);
      atomicOr(a.status, TW_STATUS_PAGE_COUNT);
    }
  }
}

// Blocks y < new_batch write row y of the new table; the others settle the counts of old row y - new_batch: its full pages by
// the number of children, the pages that only a first child takes over by whether there is one.
__global__ __launch_bounds__(256) void pages_fork_kernel(PagesArgs a) {
  __shared__ int seen;
  const int tid = threadIdx.x;
  if (tid == 0) seen = 0;
  __syncthreads();
  if ((int)blockIdx.y < a.new_batch) {
    const int i = blockIdx.y, r = a.parent[i];
    int32_t* out = a.new_table + (long long)i * a.max_pages;
    if (r < 0 || r >= a.batch) {                 // an empty row
      for (int p = (int)blockIdx.x * 256 + tid; p < a.max_pages; p += (int)gridDim.x * 256) out[p] = -1;
      if (blockIdx.x == 0 && tid == 0) { a.new_lens[i] = 0; a.copy_src[i] = a.copy_dst[i] = -1; }
      return;
    }
    int earlier = 0;
    for (int j = tid; j < i; j += 256) earlier |= a.parent[j] == r;
    if (earlier) seen = 1;
    __syncthreads();
    const bool first = seen == 0;
    const int len = row_len(a, r), full = len / TW_PAGE;
    const int32_t* row = a.table + (long long)r * a.max_pages;
    for (int p = (int)blockIdx.x * 256 + tid; p < a.max_pages; p += (int)gridDim.x * 256) {
      const int id = row[p];
      out[p] = (unsigned)id < a.pool_pages && (p < full || first) ? id : -1;
    }
    if (blockIdx.x == 0 && tid == 0) {
      a.new_lens[i] = len;
      int src = -1;                              // a request for a page of its own
      if (!first && len % TW_PAGE) src = row[full];
      a.copy_src[i] = (unsigned)src < a.pool_pages ? src : -1;
      a.copy_dst[i] = -1;
    }
    return;
  }
  const int r = (int)blockIdx.y - a.new_batch;
  int mine = 0;
  for (int j = tid; j < a.new_batch; j += 256) mine += a.parent[j] == r;
  if (mine) atomicAdd(&seen, mine);
  __syncthreads();
  const int children = seen;
  if (children == 1) return;
  const int full = row_len(a, r) / TW_PAGE, last = children ? full : a.max_pages;
  const int32_t* row = a.table + (long long)r * a.max_pages;
  for (int p = (int)blockIdx.x * 256 + tid; p < last; p += (int)gridDim.x * 256) {
    const int id = row[p];
    if ((unsigned)id >= a.pool_pages) continue;
    if (children) atomicAdd(a.ref + id, children - 1);
    else if (atomicAdd(a.ref + id, -1) <= 0) {
      atomicAdd(a.ref + id, 1);
      atomicOr(a.status, TW_STATUS_PAGE_COUNT);
    }
  }
}

// Entries of row b that reserve looks at.
__device__ __forceinline__ void reserve_range(const PagesArgs& a, int b, int* lo, int* hi) {
  const int n = max(0, min(a.n_new[b], a.max_new)), len = row_len(a, b);
  *lo = len / TW_PAGE;
  *hi = n ? (int)min((long long)a.max_pages, ((long long)len + n + TW_PAGE - 1) / TW_PAGE) : *lo;
}

// Unmapped entries among [lo, hi) of row b; a lane has a row of its own, and ranges longer than SHORT are looked through by the
// whole wave, one after the other.
constexpr int SHORT = 2;
__device__ __forceinline__ int unmapped_in(const PagesArgs& a, int b, int lo, int hi, int lane) {
  int n = 0;
  if (hi - lo <= SHORT)
    for (int p = lo; p < hi; ++p) n += (unsigned)a.table[(long long)b * a.max_pages + p] >= a.pool_pages;
  for (unsigned long long rest = __ballot(hi - lo > SHORT); rest; rest &= rest - 1) {
    const int l = __builtin_ctzll(rest), bl = __builtin_amdgcn_readlane(b, l), from = __builtin_amdgcn_readlane(lo, l), to = __builtin_amdgcn_readlane(hi, l);
    int sum = 0;
    for (int p0 = from; p0 < to; p0 += 64) {
      const int p = p0 + lane;
      sum += __popcll(__ballot(p < to && (unsigned)a.table[(long long)bl * a.max_pages + min(p, to - 1)] >= a.pool_pages));
    }
    if (lane == l) n = sum;
  }
  return n;
}

// Hands out pages: one workgroup, since the order of the pages is one chain of prefix sums.  Requests are counted row by
// row, the counts searched from page 0 until there are as many free pages as requests, the pages dealt out by rank.
// FORK: request i is copy_src[i] >= 0, the entry that row i's partly filled page stands in.  Otherwise (reserve): the
// unmapped entries of a row's range.  Bound by the trips to memory one after the other and, in a large pool, by what one CU
// reads (a pass of the search reads 64 KiB, the next one's counts are asked for before a pass is looked at).  Rows go to
// the waves in turn, so that few long ranges are not one wave's; the requests before each row and the pages found stay in
// LDS while they fit.
constexpr int TAKE_LDS = 4096;
template <bool FORK>
__global__ __launch_bounds__(TAKE_THREADS) void pages_take_kernel(PagesArgs a) {
  __shared__ uint32_t wsum[16];
  __shared__ int s_before[TAKE_LDS], s_found[TAKE_LDS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int rows = FORK ? a.new_batch : a.batch;
  int* before = rows <= TAKE_LDS ? s_before : a.ws_before;
  auto counts_of = [&](unsigned base, int* c) {  // of page base + 64 * (16 * wave + k) + lane
    const unsigned p0 = base + (unsigned)wave * (64 * TAKE_STEPS) + (unsigned)lane;
#pragma unroll
    for (int k = 0; k < TAKE_STEPS; ++k) c[k] = p0 + 64u * k < a.pool_pages ? a.ref[p0 + 64u * k] : 1;
  };
  int c[TAKE_STEPS], next[TAKE_STEPS];
  counts_of(0, next);
  // ---- requests before each row; a thread's row in round j is TAKE_THREADS j + 16 * lane + wave
  if (!FORK) {
    for (int b0 = 0; b0 < rows; b0 += TAKE_THREADS) {
      const int b = b0 + lane * TAKE_WAVES + wave;
      int lo = 0, hi = 0;
      if (b < rows) reserve_range(a, b, &lo, &hi);
      const int n = unmapped_in(a, b, lo, hi, lane);
      if (b < rows) before[b] = n;
    }
    __syncthreads();
  }
  uint32_t total = 0;
  for (int b0 = 0; b0 < rows; b0 += TAKE_THREADS) {
    const int b = b0 + tid;
    const uint32_t n = b < rows ? (FORK ? (uint32_t)(a.copy_src[b] >= 0) : (uint32_t)before[b]) : 0u;
    uint32_t sum;
    const uint32_t upto = tw_block_scan_u32(n, wsum, &sum);
    if (b < rows) before[b] = (int)(total + upto - n);
    total += sum;
  }
  if (total == 0) return;
  int* list = total <= (uint32_t)TAKE_LDS ? s_found : a.ws_found;
  // ---- the lowest free pages
  uint32_t found = 0;
  for (unsigned base = 0; base < a.pool_pages && found < total; base += TAKE_PASS) {
#pragma unroll
    for (int k = 0; k < TAKE_STEPS; ++k) c[k] = next[k];
    counts_of(base + TAKE_PASS, next);
    uint32_t mine = 0;
#pragma unroll
    for (int k = 0; k < TAKE_STEPS; ++k) mine += (uint32_t)__popcll(__ballot(c[k] == 0));
    if (lane == 0) wsum[wave] = mine;
    __syncthreads();
    uint32_t rank = found, all = 0;
#pragma unroll
    for (int w = 0; w < TAKE_WAVES; ++w) { const uint32_t x = wsum[w]; rank += w < wave ? x : 0u; all += x; }
    __syncthreads();
    if (mine && rank < total) {
      const unsigned p0 = base + (unsigned)wave * (64 * TAKE_STEPS) + (unsigned)lane;
#pragma unroll
      for (int k = 0; k < TAKE_STEPS; ++k) {
        const unsigned long long f = __ballot(c[k] == 0);
        const uint32_t r = rank + tw_bits_below(f);
        if (c[k] == 0 && r < total) { list[r] = (int)(p0 + 64u * k); a.ref[p0 + 64u * k] = 1; }
        rank += (uint32_t)__popcll(f);
      }
    }
    found += all;
  }
  if (found < total && tid == 0) atomicOr(a.status, TW_STATUS_POOL_EXHAUSTED);
  __syncthreads();
  // ---- dealt out
  if (FORK) {
    for (int i = tid; i < rows; i += TAKE_THREADS) {
      if (a.copy_src[i] < 0) continue;
      const uint32_t r = (uint32_t)before[i];
      if (r < found) {
        const int id = list[r];
        a.copy_dst[i] = id;
        a.new_table[(long long)i * a.max_pages + a.new_lens[i] / TW_PAGE] = id;
      } else {
        a.copy_src[i] = -1;
      }
    }
    return;
  }
  for (int b0 = 0; b0 < rows; b0 += TAKE_THREADS) {
    const int b = b0 + lane * TAKE_WAVES + wave;
    int lo = 0, hi = 0;
    uint32_t r = 0;
    if (b < rows) { reserve_range(a, b, &lo, &hi); r = (uint32_t)before[b]; }
    if (hi - lo <= SHORT)
      for (int p = lo; p < hi; ++p) {
        int32_t* e = a.table + (long long)b * a.max_pages + p;
        if ((unsigned)*e >= a.pool_pages) { *e = r < found ? list[r] : -1; ++r; }
      }
    for (unsigned long long rest = __ballot(hi - lo > SHORT); rest; rest &= rest - 1) {
      const int l = __builtin_ctzll(rest), bl = __builtin_amdgcn_readlane(b, l), from = __builtin_amdgcn_readlane(lo, l), to = __builtin_amdgcn_readlane(hi, l);
      uint32_t at = (uint32_t)__builtin_amdgcn_readlane((int)r, l);
      for (int p0 = from; p0 < to; p0 += 64) {
        const int p = p0 + lane;
        int32_t* e = a.table + (long long)bl * a.max_pages + min(p, to - 1);
        const unsigned long long want = __ballot(p < to && (unsigned)*e >= a.pool_pages);
        const uint32_t k = at + tw_bits_below(want);
        if (want >> lane & 1ull) *e = k < found ? list[k] : -1;
        at += (uint32_t)__popcll(want);
      }
    }
  }
}

// ---------------------------------------------------------------- one layer's rows
struct RowsArgs {
  uint4* k;
  uint4* v;
  uint4* codes;
  uint4* meta;
  uint4* bounds;
  const int32_t* src;                            // copy: pairs
  const int32_t* dst;
  const int32_t* table;                          // compact
  const int32_t* to;
  const int32_t* seq_lens;
  const int32_t* keep;
  const int32_t* count;
  const int32_t* start;
  int batch, Hkv, bits, max_pages, stride, n_copy;
  unsigned pool_pages;
};

// A (pair, KV head): 4096 + 4096 + 256 * bits + 256 + 512 bytes by one workgroup, all loads before the stores.  HBM.
__device__ __forceinline__ void copy_page(const RowsArgs& a, int i, int h, int tid) {
  const int s = a.src[i], d = a.dst[i];
  if ((unsigned)s >= a.pool_pages || (unsigned)d >= a.pool_pages || s == d) return;
  const long long sp = (long long)s * a.Hkv + h, dp = (long long)d * a.Hkv + h;
  const int nc = 16 * a.bits;
  uint4 x = make_uint4(0u, 0u, 0u, 0u), y = x, z = x;
  uint4* to = nullptr;                           // codes, (scale, zero), bounds: at most 176 pieces
  if (a.k) x = tw_ld_stream(a.k + sp * 256 + tid);
  if (a.v) y = tw_ld_stream(a.v + sp * 256 + tid);
  const uint4* from = nullptr;
  if (tid < nc) { if (a.codes) { from = a.codes + sp * nc + tid; to = a.codes + dp * nc + tid; } }
  else if (tid < nc + 16) { if (a.meta) { from = a.meta + sp * 16 + (tid - nc); to = a.meta + dp * 16 + (tid - nc); } }
  else if (tid < nc + 48) { if (a.bounds) { from = a.bounds + sp * 32 + (tid - nc - 16); to = a.bounds + dp * 32 + (tid - nc - 16); } }
  if (to) z = *from;
  if (a.k) a.k[dp * 256 + tid] = x;
  if (a.v) a.v[dp * 256 + tid] = y;
  if (to) *to = z;
}
__global__ __launch_bounds__(256) void pages_copy_kernel(RowsArgs a) {
  const long long all = (long long)a.n_copy * a.Hkv;
  for (long long i = blockIdx.x; i < all; i += gridDim.x) copy_page(a, (int)(i / a.Hkv), (int)(i % a.Hkv), (int)threadIdx.x);
}

// Compaction.  A workgroup takes WAVES destination pages of a KV head at a time, a wave each: the 16 rows of K, V, codes and
// (scale, zero), all loads before the stores; which row moves where is looked up once per token, through LDS.  To another
// table every step is a workgroup of its own.  In place one workgroup walks all steps of a (sequence, KV head), reads a
// step's rows before it writes them (one barrier, behind the loads) - destinations lie at or before their sources, so no
// step overwrites what a later one reads - and looks up the next step's moves meanwhile.
// In place 8 waves where that is one step, else 16.  us, 8 / 16 waves: one draft of 97 positions 6.3 / 6.3, 32 of them 8.5 / 8.7; one
// of 160 8.2 / 7.1, 32 of them 13.5 / 11.5; 1000 32.3 / 25.4.  Half of 4 x 16384 tokens kept 377 / 262, into other pages 52: one
// workgroup per (sequence, KV head) walks them, bound by its trips to memory, one step after the other.
__device__ __forceinline__ void hold(uint4& x) { asm volatile("" : "+v"(x.x), "+v"(x.y), "+v"(x.z), "+v"(x.w)); }

// Source and destination row (page * 16 + slot, of the pools without their head index) of destination position t; -1: none.
struct Move { int src, dst; };
template <bool INPLACE>
__device__ __forceinline__ Move move_of(const RowsArgs& a, int b, long long t, int start, int end, int len) {
  Move m = {-1, -1};
  if (t >= end) return m;
  const long long row = (long long)b * a.max_pages;
  const int dp = (INPLACE ? a.table : a.to)[row + t / TW_PAGE];
  const int s = t >= start ? a.keep[(long long)b * a.stride + (t - start)] : -1;
  if ((unsigned)dp >= a.pool_pages) return m;
  m.dst = dp * TW_PAGE + (int)(t % TW_PAGE);
  if (s < 0 || s >= len) return m;
  const int sp = a.table[row + s / TW_PAGE];
  if ((unsigned)sp < a.pool_pages) m.src = sp * TW_PAGE + s % TW_PAGE;
  return m;
}

// The smaller (larger) of a lane's value and that of the lane 32 or 16 away.
template <int DIST>
__device__ __forceinline__ void fold_bounds(float& lo, float& hi) {
  if (DIST == 32) {
    const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(lo), __float_as_uint(lo), false, false);
    const auto y = __builtin_amdgcn_permlane32_swap(__float_as_uint(hi), __float_as_uint(hi), false, false);
    lo = fminf(__uint_as_float(x[0]), __uint_as_float(x[1])); hi = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
  } else {
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(lo), __float_as_uint(lo), false, false);
    const auto y = __builtin_amdgcn_permlane16_swap(__float_as_uint(hi), __float_as_uint(hi), false, false);
    lo = fminf(__uint_as_float(x[0]), __uint_as_float(x[1])); hi = fmaxf(__uint_as_float(y[0]), __uint_as_float(y[1]));
  }
}

template <bool INPLACE, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void compact_kernel(RowsArgs a) {
  constexpr int STEP = WAVES * TW_PAGE;
  __shared__ Move moves[2][STEP];
  const int h = blockIdx.y, b = blockIdx.z, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int start = a.start[b];
  if (start < 0) return;
  const int len = max(0, min(a.seq_lens[b], a.max_pages * TW_PAGE));
  const int end = (int)min((long long)start + max(0, min(a.count[b], a.stride)), (long long)a.max_pages * TW_PAGE);
  long long t0 = start & ~(TW_PAGE - 1);
  if (!INPLACE) t0 += (long long)blockIdx.x * STEP;
  if (t0 >= end) return;
  // row (page, slot) of head h in a pool of `pieces` 16-byte pieces per row
  auto at = [&](int r, int pieces) -> long long { return (((long long)(r / TW_PAGE) * a.Hkv + h) * TW_PAGE + r % TW_PAGE) * pieces; };
  // a whole cache packed into other pages does not stay in the caches: K and V marked non-temporal both ways (4 x 16384 tokens, half
  // kept, 8 KV heads: 61.0 -> 52.3 us); the few rows of a draft are read again by the next step
  auto load = [](const uint4* p) -> uint4 { return INPLACE ? *p : tw_ld_stream(p); };
  auto store = [](uint4* p, const uint4& x) { if (INPLACE) *p = x; else tw_st_stream(p, x); };
  if (tid < STEP) moves[0][tid] = move_of<INPLACE>(a, b, t0 + tid, start, end, len);
  __syncthreads();
  const int piece = lane & 15, sub = lane >> 4;  // K and V: load j takes rows 4 j + sub; codes and (scale, zero): row lane % 16
  for (int turn = 0;; turn ^= 1) {
    const Move* mv = moves[turn] + wave * TW_PAGE;
    Move m[4];
    uint4 k[4], v[4], c[2], z;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      m[j] = mv[4 * j + sub];
      const int r = m[j].src >= 0 ? m[j].src : a.bounds ? m[j].dst : -1;       // rows that stay count for the bounds
      k[j] = v[j] = make_uint4(0u, 0u, 0u, 0u);
      if (r >= 0) k[j] = load(a.k + at(r, 16) + piece);
      if (m[j].src >= 0 && a.v) v[j] = load(a.v + at(m[j].src, 16) + piece);
    }
    const Move mc = mv[piece];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      c[i] = make_uint4(0u, 0u, 0u, 0u);
      if (mc.src >= 0 && a.codes && sub + 4 * i < a.bits) c[i] = a.codes[at(mc.src, a.bits) + sub + 4 * i];
    }
    z = make_uint4(0u, 0u, 0u, 0u);
    if (mc.src >= 0 && a.meta && sub == 0) z = a.meta[at(mc.src, 1)];
    const bool more = INPLACE && t0 + STEP < end;
    if (INPLACE) {
      if (more && tid < STEP) moves[turn ^ 1][tid] = move_of<INPLACE>(a, b, t0 + STEP + tid, start, end, len);
#pragma unroll
      for (int j = 0; j < 4; ++j) { hold(k[j]); hold(v[j]); }                  // every load of the step has returned
      hold(c[0]); hold(c[1]); hold(z);
      __syncthreads();
    }
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (m[j].src >= 0) {
        store(a.k + at(m[j].dst, 16) + piece, k[j]);
        if (a.v) store(a.v + at(m[j].dst, 16) + piece, v[j]);
      }
    if (mc.src >= 0) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (a.codes && sub + 4 * i < a.bits) a.codes[at(mc.dst, a.bits) + sub + 4 * i] = c[i];
      if (a.meta && sub == 0) a.meta[at(mc.dst, 1)] = z;
    }
    // the wave's page: its first position is a token whenever any of it is
    const int first = __builtin_amdgcn_readfirstlane(m[0].dst);
    if (a.bounds && first >= 0) {
      float lo[8], hi[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) { lo[i] = __builtin_inff(); hi[i] = -__builtin_inff(); }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        float f[8];
        tw_unpack8(k[j], f);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          lo[i] = fminf(lo[i], m[j].dst >= 0 ? f[i] : __builtin_inff());
          hi[i] = fmaxf(hi[i], m[j].dst >= 0 ? f[i] : -__builtin_inff());
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) { fold_bounds<32>(lo[i], hi[i]); fold_bounds<16>(lo[i], hi[i]); }
      if (sub < 2) {                             // lanes 0..15 the lower bounds, 16..31 the upper ones
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t x = __float_as_uint(sub ? hi[2 * i] : lo[2 * i]), y = __float_as_uint(sub ? hi[2 * i + 1] : lo[2 * i + 1]);
          w[i] = x >> 16 | (y & 0xFFFF0000u);
        }
        a.bounds[((long long)(first / TW_PAGE) * a.Hkv + h) * 32 + lane] = make_uint4(w[0], w[1], w[2], w[3]);
      }
    }
    if (!more) return;
    t0 += STEP;
  }
}

// ---------------------------------------------------------------- host side
size_t align256p(size_t x) { return (x + 255) & ~(size_t)255; }

int check_pages(const twilight_kv_t* kv, TwDims* d) {
  if (int e = tw_check_kv(kv, d)) return e;
  return d->max_pages > TW_MAX_ROW_PAGES ? TW_EINVAL : TW_OK;
}

PagesArgs pages_args(const twilight_kv_t* kv, const TwDims& d, int32_t* ref, uint32_t* status) {
  PagesArgs a = {};
  a.table = const_cast<int32_t*>(kv->page_table); a.seq_lens = kv->seq_lens; a.ref = ref; a.status = status;
  a.batch = d.batch; a.max_pages = d.max_pages; a.pool_pages = (unsigned)d.pool_pages;
  return a;
}
unsigned row_blocks(int max_pages) { return (unsigned)std::min((max_pages + 255) / 256, 64); }

size_t take_rows_bytes(long long rows) { return align256p((size_t)rows * 4); }

}  // namespace

// entries that a reservation of max_new tokens per row looks at; counted in 32 bits
static long long reserve_entries(const TwDims& d, int max_new) {
  return d.batch * std::min((long long)d.max_pages, max_new > 0 ? ((long long)max_new + TW_PAGE - 1) / TW_PAGE + 1 : 0ll);
}

size_t tw_pages_workspace(const TwDims& d, int max_new, int new_batch) {
  if (max_new < 0 || new_batch < 0 || new_batch > 65535) return 0;
  const long long rows = d.batch > new_batch ? d.batch : new_batch;
  const long long most = std::min<long long>(std::max(reserve_entries(d, max_new), (long long)new_batch), d.pool_pages);
  return take_rows_bytes(rows) + align256p((size_t)most * 4);
}

extern "C" int twilight_pages_reserve(const twilight_kv_t* kv, const int32_t* n_new, int32_t max_new, int32_t* ref_count,
                                      uint32_t* status, void* ws, size_t ws_bytes, void* stream) {
  TwDims d;
  if (int e = check_pages(kv, &d)) return e;
  if (!n_new || max_new <= 0 || !ref_count || !status || reserve_entries(d, max_new) >= (1ll << 31)) return TW_EINVAL;
  if (!ws || ws_bytes < tw_pages_workspace(d, max_new, 0)) return TW_EWORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  PagesArgs a = pages_args(kv, d, ref_count, status);
  a.n_new = n_new; a.max_new = max_new;
  a.ws_before = (int32_t*)ws;
  a.ws_found = (int32_t*)((char*)ws + take_rows_bytes(d.batch));
  tw_prof_before(TW_K_PAGES_TAKE, s);
  TW_LAUNCH((pages_take_kernel<false>), dim3(1), dim3(TAKE_THREADS), 0, s, a);
  return tw_prof_after(s);
}

extern "C" int twilight_pages_free(const twilight_kv_t* kv, const int32_t* first_page, const int32_t* end_page, int32_t* ref_count,
                                   uint32_t* status, void* stream) {
  TwDims d;
  if (int e = check_pages(kv, &d)) return e;
  if (!first_page || !end_page || !ref_count || !status) return TW_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  PagesArgs a = pages_args(kv, d, ref_count, status);
  a.first = first_page; a.end = end_page;
  tw_prof_before(TW_K_PAGES_FREE, s);
  TW_LAUNCH(pages_free_kernel, dim3(row_blocks(d.max_pages), (unsigned)d.batch), dim3(256), 0, s, a);
  return tw_prof_after(s);
}

extern "C" int twilight_pages_fork(const twilight_kv_t* kv, const int32_t* parent, int32_t new_batch, int32_t* new_table, int32_t* new_lens,
                                   int32_t* ref_count, int32_t* copy_src, int32_t* copy_dst, uint32_t* status,
                                   void* ws, size_t ws_bytes, void* stream) {
  TwDims d;
  if (int e = check_pages(kv, &d)) return e;
  if (!parent || !new_table || !new_lens || !ref_count || !copy_src || !copy_dst || !status) return TW_EINVAL;
  if (new_batch <= 0 || new_batch > 65535 || d.batch + new_batch > 65535 || new_table == kv->page_table || new_lens == kv->seq_lens) return TW_EINVAL;
  if (!ws || ws_bytes < tw_pages_workspace(d, 0, new_batch)) return TW_EWORKSPACE;
  hipStream_t s = (hipStream_t)stream;
  PagesArgs a = pages_args(kv, d, ref_count, status);
  a.parent = parent; a.new_batch = new_batch; a.new_table = new_table; a.new_lens = new_lens; a.copy_src = copy_src; a.copy_dst = copy_dst;
  a.ws_before = (int32_t*)ws;
  a.ws_found = (int32_t*)((char*)ws + take_rows_bytes(new_batch));
  tw_prof_before(TW_K_PAGES_FORK, s);
  TW_LAUNCH(pages_fork_kernel, dim3(row_blocks(d.max_pages), (unsigned)(d.batch + new_batch)), dim3(256), 0, s, a);
  if (int e = tw_prof_after(s)) return e;
  tw_prof_before(TW_K_PAGES_TAKE, s);
  TW_LAUNCH((pages_take_kernel<true>), dim3(1), dim3(TAKE_THREADS), 0, s, a);
  return tw_prof_after(s);
}

static bool pools_aligned(const twilight_kv_t* kv) {           // rows move in pieces of 16 bytes
  return !(((uintptr_t)kv->k_pool | (uintptr_t)kv->v_pool | (uintptr_t)kv->kq_pool | (uintptr_t)kv->kq_meta | (uintptr_t)kv->page_minmax) & 15);
}

static RowsArgs rows_args(const twilight_kv_t* kv, const TwDims& d) {
  RowsArgs a = {};
  a.k = (uint4*)kv->k_pool; a.v = (uint4*)kv->v_pool; a.codes = (uint4*)kv->kq_pool; a.meta = (uint4*)kv->kq_meta; a.bounds = (uint4*)kv->page_minmax;
  a.batch = d.batch; a.Hkv = d.Hkv; a.bits = d.bits; a.max_pages = d.max_pages; a.pool_pages = (unsigned)d.pool_pages;
  return a;
}

extern "C" int twilight_pages_copy(const twilight_kv_t* kv, const int32_t* copy_src, const int32_t* copy_dst, int32_t n_copy, void* stream) {
  TwDims d;
  if (int e = check_pages(kv, &d)) return e;
  if (!copy_src || !copy_dst || n_copy < 0 || !pools_aligned(kv)) return TW_EINVAL;
  if (n_copy == 0) return TW_OK;
  hipStream_t s = (hipStream_t)stream;
  RowsArgs a = rows_args(kv, d);
  a.src = copy_src; a.dst = copy_dst; a.n_copy = n_copy;
  tw_prof_before(TW_K_PAGES_COPY, s);
  TW_LAUNCH(pages_copy_kernel, dim3((unsigned)std::min((long long)n_copy * d.Hkv, 1ll << 20)), dim3(256), 0, s, a);
  return tw_prof_after(s);
}

extern "C" int twilight_tokens_compact(const twilight_kv_t* kv, const int32_t* keep_idx, const int32_t* keep_count, int32_t keep_stride,
                                       const int32_t* dst_start, const int32_t* dst_table, void* stream) {
  TwDims d;
  if (int e = check_pages(kv, &d)) return e;
  if (!keep_idx || !keep_count || keep_stride <= 0 || !dst_start || !kv->k_pool || !pools_aligned(kv)) return TW_EINVAL;
  hipStream_t s = (hipStream_t)stream;
  RowsArgs a = rows_args(kv, d);
  a.table = kv->page_table; a.to = dst_table; a.seq_lens = kv->seq_lens;
  a.keep = keep_idx; a.count = keep_count; a.start = dst_start; a.stride = keep_stride;
  const long long most = std::min((long long)keep_stride, (long long)d.max_pages * TW_PAGE) + TW_PAGE - 1;   // positions from a page's start on
  const bool in_place = !dst_table || dst_table == kv->page_table;
  tw_prof_before(TW_K_COMPACT, s);
  if (!in_place) TW_LAUNCH((compact_kernel<false, 4>), dim3((unsigned)((most + 63) / 64), (unsigned)d.Hkv, (unsigned)d.batch), dim3(256), 0, s, a);
  else if (most <= 8 * TW_PAGE) TW_LAUNCH((compact_kernel<true, 8>), dim3(1, (unsigned)d.Hkv, (unsigned)d.batch), dim3(512), 0, s, a);
  else TW_LAUNCH((compact_kernel<true, 16>), dim3(1, (unsigned)d.Hkv, (unsigned)d.batch), dim3(1024), 0, s, a);
  return tw_prof_after(s);
}
