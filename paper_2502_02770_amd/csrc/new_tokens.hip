// Attention of a sequence's newest tokens over its paged cache: a drafted tree of tokens (twilight_tree_attention), or a
// chunk of consecutive tokens with a sliding window and sinks (twilight_window_attention).
//
// The rows of a KV head are its G query heads times the N new tokens, row r = token r / G, head r % G, so that every K/V
// tile is loaded once for all of them.  A workgroup takes M = 32 * WR rows and walks tiles of 64 cached tokens:
//
//   S^T = K Q^T     v_mfma_f32_32x32x16_bf16, A = 32 tokens of K, B = 32 rows of Q (held in registers throughout)
//   P^T = exp2(S^T * log2(e)/sqrt(128) - m), m = the row's running maximum, followed only where it is 2^8 behind
//   O^T += V^T P^T  A = V^T (transposed LDS reads), B = P^T
//
// In the result layout of the first product a lane holds 16 tokens of ONE row (its partner lane in the other half wave
// the other 16), so maximum, sum and rescaling are in-lane but for one exchange between the halves, and the lane's own P
// values are its B operand of the second product as they stand: the order of the 16 tokens within a contraction step is
// free as long as the V^T operand has the same (slot 8 * h + j of step k = token 16 k + 8 (j / 4) + 4 h + j % 4).
// Scores, maxima, sums, accumulators and the parts of cut lists are fp32, and the sum is of the unrounded weights.  For its product P
// is bf16: of up to 64 rows, which the memory bounds, a weight and what its rounding left (16 bits, 2^-16 of a weight at most), so
// that a single token is as exact as in twilight_sparse_decode; of 128 rows the weight alone (2^-8 of it at most), as
// the second product and the remainders cost 24 to 35 % there: 8 drafts of 32 over 32768 tokens 205 -> 255 us, two prompts of 8192
// 815 -> 1102, against 64 single tokens 137 -> 140, a draft of 8 over 4096 13.1 -> 13.3.  A weight
// may reach 2^8 before m follows (kGrowth): rescaling the accumulators for every new maximum, which some row of 32 has in most
// tiles, took 54 of 211 vector instructions per tile (prompts of 8192 tokens: 852 us, 811 us without).
//
// K and V rows go from HBM to LDS without passing registers, 16 bytes per lane, a page of (token, head) rows being 4 KiB
// contiguous; the 16-byte pieces of a row are stored in an order that depends on the row (XOR), so that neither the
// 32-row reads of K nor the transposed reads of V meet in a bank.  Two buffers: a tile's loads are issued before the
// tile ahead of it is computed.
//
// Bounds.  Few rows (32 or 64 to a workgroup, 2 or 4 waves that split a tile's tokens): HBM, 8 drafts of 32 over 32768 tokens
// 1.08 GB in 209 us (5.2 TB/s; a large copy reads and writes 4.9).  128 rows (4 waves of 32 rows, all tokens each): a wave's tile
// is 32 matrix instructions of 32 cycles, 16 of which keep the SIMD from issuing vector instructions, and 151 vector
// instructions of 4 cycles (8 for the 32 exponentials): 1024 cycles of the matrix unit against 1244 of issue.  Two prompts
// of 8192 tokens under a window of 4096: 828 us, 1.00 PFLOP/s of the pairs that are visible; an 8192^3 library product 1.21.
#include <algorithm>
#include "tw_common.h"

namespace {

typedef __bf16 tw_bf16x8 __attribute__((ext_vector_type(8)));
typedef short tw_s16x4 __attribute__((ext_vector_type(4)));
typedef float tw_f32x16 __attribute__((ext_vector_type(16)));
#define TW_LDS __attribute__((address_space(3)))
#define TW_GLB __attribute__((address_space(1)))

constexpr float kScaleLog2 = 0.08838834764831845f * 1.4426950408889634f;   // log2(e) / sqrt(128)
constexpr float kLn2n = 0.6931471805599453f;
constexpr float kLow = -3.4028234663852886e38f;  // running maximum before any visible token, the lowest number: exp2(-inf - kLow) = 0
constexpr float kFar = 1073741824.f;             // from an |m| of 2^30 on, a row's scores are told apart by their own steps, 64 and more
constexpr float kGrowth = 8.f;                   // by how much (in powers of 2) a row's scores may exceed its m before m follows
constexpr int TILE = 64, TILE_BYTES = TILE * 256;
enum { MODE_TREE = 0, MODE_WINDOW = 1 };
constexpr int PLAN_ROUNDS = 2;                   // items per resident workgroup at most, as planned
constexpr int PLAN_MIN_TILES = 2;                // shortest chunk of a list
constexpr int STREAM_TILES = (96 << 20) / (2 * TILE_BYTES);   // tiles of K and V from which on they pass by the last-level cache
constexpr long long COMBINE_FEW = 512;           // rows of a launch up to which a workgroup joins one row's parts

// rows of K and V that no token stands for (beyond the sequence's end, on an unmapped page) are read from here
__device__ const uint4 tw_zero_row[16] = {};

struct NewArgs {
  const uint4* q;
  const char* k_pool;
  const char* v_pool;
  const int32_t* page_table;
  const int32_t* seq_lens;
  const int32_t* n_new;        // or NULL: max_new each
  const int32_t* offsets;      // or NULL: b * max_new
  const uint32_t* mask;
  uint2* out;
  float* lse;
  int32_t* ws_plan;            // [batch][2]: chunks of the sequence's lists, first partial result
  float2* ws_ml;
  float* ws_acc;
  int batch, Hq, Hkv, G, lgG, max_pages, max_new, mask_words, window, sinks, rb_max, cus, stream;
  unsigned pool_pages;
};

// the lowest x of 64 bits
__device__ __forceinline__ unsigned long long low_bits(int x) {
  return x <= 0 ? 0ull : x >= 64 ? ~0ull : (1ull << x) - 1ull;
}

__device__ __forceinline__ int seq_len(const NewArgs& a, int b) {
  const int n = a.seq_lens[b];
  return max(0, min(n, a.max_pages * TW_PAGE));
}
__device__ __forceinline__ int seq_new(const NewArgs& a, int b) {
  return a.n_new ? max(0, min(a.n_new[b], a.max_new)) : a.max_new;
}

// The pages that rows of tokens at positions p_lo .. p_hi see: `sink` pages from the start, then those from `first` on; four of
// this list to a tile, so that a few sinks and a window that begins inside 64 tokens cost no tile of their own: five prompts of 882
// tokens, a window of 51 and one sink 35.1 us with tiles at multiples of 64, 32.3 so.  Where few tiles are saved, working out the
// places costs more than that: one token, a window of 1024 and 4 sinks 10.5 and 10.8 us.
struct Span {
  int sink, first, pages, tiles;
  int both, behind, shift;                       // the tile with pages of both parts, the first one of the second; positions between the parts
  __device__ __forceinline__ int page(int v) const { return v < sink ? v : first + (v - sink); }
  __device__ __forceinline__ int start(int u) const { return u * TILE + (u >= behind ? shift : 0); }   // position of tile u's first page
};
template <int MODE>
__device__ __forceinline__ Span span_of(const NewArgs& a, int len, int p_lo, int p_hi) {
  Span s;
  const int end = MODE == MODE_TREE ? len : min(len, p_hi + 1);
  if (end <= 0) { s.sink = s.first = s.pages = s.tiles = s.behind = s.shift = 0; s.both = -1; return s; }
  s.first = MODE == MODE_TREE ? 0 : max(0, p_lo - a.window + 1) / TW_PAGE;
  s.sink = MODE == MODE_TREE ? 0 : min((int)(((unsigned)a.sinks + TW_PAGE - 1) / TW_PAGE), s.first);
  s.pages = s.sink + (end - 1) / TW_PAGE - s.first + 1;
  s.tiles = (s.pages + 3) / 4;
  s.behind = (s.sink + 3) / 4;
  s.both = s.sink & 3 && s.sink < s.first ? s.sink / 4 : -1;
  s.shift = (s.first - s.sink) * TW_PAGE;
  return s;
}

// Which part of which list a workgroup takes.  A list is a (row block, KV head) of a sequence; a sequence's lists are cut
// into the same number of chunks.
struct Item {
  int b, n, len, off;                            // the sequence, as Seq
  int rb, h, chunk, chunks, slot;
  uint32_t items;                                // of the launch, where one wave's lanes hold all sequences (no need to look for a next one)
};

// A sequence: its new tokens, length and first row, its lists and the tiles of the longest of them.
struct Seq {
  int n, len, off, lists, tiles;
};
template <int MODE, int M>
__device__ __forceinline__ Seq seq_of(const NewArgs& a, int b) {
  Seq s = {0, 0, 0, 0, 0};
  if (b >= a.batch) return s;
  s.off = a.offsets ? a.offsets[b] : b * a.max_new;
  s.n = seq_new(a, b);
  s.len = seq_len(a, b);
  const int blocks = (s.n * a.G + M - 1) / M;
  s.lists = blocks * a.Hkv;
  s.tiles = blocks == 0 ? 0 : max(1, span_of<MODE>(a, s.len, s.len - min(s.n, M / a.G), s.len - 1).tiles);
  return s;
}

// x / d for quotients up to 2^22
__device__ __forceinline__ uint32_t quotient(uint32_t x, uint32_t d) {
  uint32_t q = (uint32_t)((float)x * __builtin_amdgcn_rcpf((float)d));
  const int r = (int)(x - q * d);
  q = r < 0 ? q - 1u : (uint32_t)r >= d ? q + 1u : q;
  return q;
}

// Sum over the 64 lanes, for all of them.
__device__ __forceinline__ float wave_sum_f(float v) {
  v = tw_row16_sum(v);
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), TW_DPP_BCAST15, 0xA, 0xF, false));
  v += __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), TW_DPP_BCAST31, 0xC, 0xF, false));
  return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 63));
}

// Chunk length in tiles, for W = 2 workgroups per CU: lists whole, or cut into lengths that give every workgroup one or two
// items, or, with far more lists than workgroups, cut down to a workgroup's share of the tiles.  The cheapest, counted in the
// time of a tile beside another workgroup on the CU (128 rows 1.7 us, 32 rows from HBM 2.8 us): per round the chunk (0.8 of
// it where no CU has two: 1.1 to 1.5 us a tile) and 2 for plan, queries and first rows; where lists are cut 1.5 more for the
// launch that joins the parts, and 2e-4 per item and row for parts of 528 bytes a row, written and read.  With c > total / (W r)
// there are fewer than W r + lists items, and fewer than 2 W r of lists that are cut: what the workspace is sized for.
// (Sums in fp32, a thousandth more than their errors added.)  Every workgroup does this before it knows its item, so in
// few and short steps: with exact quotients by integer division it took 3 us of the 10 us that a single chat's call runs.
// *seq: this lane's sequence where 64 lanes hold them all; *stream stays true where that many tiles are read.
template <int MODE, int M>
__device__ __forceinline__ int plan_chunk(const NewArgs& a, int lane, Seq* seq, bool* stream) {
  constexpr float kJoin = 1.5f, kPart = 2e-4f * M;
  float total = 0.f, lists_all = 0.f, longest = 0.f;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    *seq = seq_of<MODE, M>(a, b0 + lane);
    total += wave_sum_f((float)seq->lists * (float)seq->tiles);
    lists_all += wave_sum_f((float)seq->lists);
    longest = __builtin_fmaxf(longest, tw_wave_max_f((float)seq->tiles));
  }
  const float cus = (float)a.cus, W = 2.f * cus;
  *stream = *stream && total > (float)STREAM_TILES;
  total *= 1.001f;
  auto cost_of = [&](float items, float c) { return __builtin_ceilf(items / W - 1e-4f) * (c * (items <= cus ? 0.8f : 1.f) + 2.f); };
  float best = cost_of(lists_all, longest), chunk = longest;
  if (total <= W * PLAN_MIN_TILES) {             // little work: the length where chunk and parts cost the same, short of the shortest none
    // (parts at half their price: they do not fill the memory's time)
    const float c = __builtin_fmaxf((float)PLAN_MIN_TILES, __builtin_floorf(__builtin_amdgcn_sqrtf(0.5f * kPart * total) + 0.5f));
    const float items = total * __builtin_amdgcn_rcpf(c);
    if (cost_of(items, c) + kJoin + items * (0.5f * kPart) < best) chunk = c;
  } else {
    for (int k = 0; k < 3; ++k) {                // one item per workgroup, somewhat fewer, two
      const float room = W * (k == 2 ? 2.f : 1.f) - 0.5f * lists_all;
      float c;
      if (room < 1.f) {
        if (k) continue;
        c = __builtin_floorf(total * 1.001f / W) + 1.f;
      } else {
        c = __builtin_floorf(total * 1.001f * __builtin_amdgcn_rcpf(room)) + 1.f;
        if (k == 1) c = __builtin_ceilf(1.125f * c);
      }
      c = __builtin_fmaxf(c, (float)PLAN_MIN_TILES);
      if (c >= longest) continue;                // the same as whole lists
      const float inv = __builtin_amdgcn_rcpf(c);
      float items = 0.f;
      for (int b0 = 0; b0 < a.batch; b0 += 64) {
        if (a.batch > 64) *seq = seq_of<MODE, M>(a, b0 + lane);
        items += wave_sum_f((float)seq->lists * __builtin_ceilf((float)seq->tiles * inv - 1e-4f));
      }
      const float cost = cost_of(items, c) + kJoin + items * kPart;
      if (cost < best) { best = cost; chunk = c; }
    }
  }
  return (int)__builtin_fminf(__builtin_fmaxf(chunk, 1.f), (float)(1 << 26));
}

// Item `want` of a launch whose lists are cut into chunks of `chunk` tiles; false: there are fewer.
template <int MODE, int M>
__device__ __forceinline__ bool find_item(const NewArgs& a, int lane, int chunk, Seq seq, uint32_t want, Item* it) {
  uint32_t items = 0, slots = 0;
  bool found = false;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    if (a.batch > 64) seq = seq_of<MODE, M>(a, b0 + lane);
    const int chunks = (int)quotient((uint32_t)(seq.tiles + chunk - 1), (uint32_t)chunk);
    const int lists = (seq.n * a.G + M - 1) / M * a.Hkv;             // (again, as it would be a register of the whole walk)
    const uint32_t mine = (uint32_t)(lists * chunks), part = chunks > 1 ? mine : 0u;
    const uint32_t ie = tw_wave_scan_u32(mine), se = tw_wave_scan_u32(part);
    if (want == 0 && threadIdx.x < 64 && b0 + lane < a.batch) {         // for the combine kernel
      a.ws_plan[2 * (b0 + lane)] = chunks;
      a.ws_plan[2 * (b0 + lane) + 1] = (int)(slots + se - part);
    }
    const unsigned long long here = __ballot(items + ie > want);
    if (!found && here) {
      const int l = __builtin_ctzll(here);
      const uint32_t before = items + (uint32_t)__builtin_amdgcn_readlane((int)(ie - mine), l);
      const uint32_t k = want - before;          // ((chunk * blocks) + block) * Hkv + head: blocks of the same rows' chunk on one XCD
      it->b = b0 + l;
      it->n = __builtin_amdgcn_readlane(seq.n, l);
      it->len = __builtin_amdgcn_readlane(seq.len, l);
      it->off = __builtin_amdgcn_readlane(seq.off, l);
      it->chunks = __builtin_amdgcn_readlane(chunks, l);
      const uint32_t all = (uint32_t)__builtin_amdgcn_readlane(lists, l);
      it->chunk = (int)quotient(k, all);
      const uint32_t rest = k - (uint32_t)it->chunk * all;
      it->rb = (int)quotient(rest, (uint32_t)a.Hkv);
      it->h = (int)(rest - (uint32_t)it->rb * (uint32_t)a.Hkv);
      it->slot = (int)(slots + (uint32_t)__builtin_amdgcn_readlane((int)(se - part), l) + k);
      found = true;
      it->items = a.batch <= 64 ? (uint32_t)__builtin_amdgcn_readlane((int)ie, 63) : 0xFFFFFFFFu;
      if (want != 0) return true;
    }
    items += (uint32_t)__builtin_amdgcn_readlane((int)ie, 63);
    slots += (uint32_t)__builtin_amdgcn_readlane((int)se, 63);
  }
  return found;
}

// Item of a launch that cuts nothing: the row blocks of a (sequence, KV head) one after the other, as they read the same rows (64
// drafts of 128 tokens over 2048, four row blocks each: 433 us with all sequences' last blocks ahead of their others), from
// the last (longest under a causal mask) to the first.
template <int M>
__device__ __forceinline__ bool whole_item(const NewArgs& a, Item* it) {
  unsigned i = blockIdx.x;
  it->h = (int)(i % (unsigned)a.Hkv); i /= (unsigned)a.Hkv;
  it->rb = a.rb_max - 1 - (int)(i % (unsigned)a.rb_max);
  it->b = (int)(i / (unsigned)a.rb_max);
  it->chunk = 0; it->chunks = 1; it->slot = 0;
  it->n = seq_new(a, it->b);
  it->len = seq_len(a, it->b);
  it->off = a.offsets ? a.offsets[it->b] : it->b * a.max_new;
  return it->rb * M < it->n * a.G;
}

// log-sum-exp of a row; -inf where it saw nothing (l = 0 and no NaN: a row with one has to show it)
__device__ __forceinline__ float row_lse(float m, float l) { return l == 0.f ? -__builtin_inff() : (m + __log2f(l)) * kLn2n; }

// The 16 rows of a page's K and V for one head, 16 bytes per lane.  HINT 2: non-temporal.
template <int HINT>
__device__ __forceinline__ void page_to_lds(const char* kp, const char* vp, unsigned k_off, unsigned v_off, unsigned char* dst) {
#pragma unroll
  for (int j = 0; j < 4; ++j)
    __builtin_amdgcn_global_load_lds((const TW_GLB unsigned int*)(kp + ((k_off ^ (unsigned)(64 * j)) + 1024u * j)), (TW_LDS unsigned int*)(dst + 1024 * j), 16, 0, HINT);
#pragma unroll
  for (int j = 0; j < 4; ++j)
    __builtin_amdgcn_global_load_lds((const TW_GLB unsigned int*)(vp + ((v_off ^ (unsigned)(32 * (j & 1))) + 1024u * j)), (TW_LDS unsigned int*)(dst + TILE_BYTES + 1024 * j), 16, 0, HINT);
}

// One item: a chunk of a list.
template <int MODE, int WR, int WT, bool SPLIT>
__device__ __forceinline__ void attend_item(const NewArgs& a, const Item& it, unsigned char (&buf0)[2 * TILE_BYTES], unsigned char (&buf1)[2 * TILE_BYTES],
                                            int lane, int wave, bool stream) {
  constexpr int NW = WR * WT, M = 32 * WR, MT = 2 / WT, PPW = 4 / NW;
  const int wr = wave / WT, wt = wave % WT, half = lane >> 5;
  const int b = __builtin_amdgcn_readfirstlane(it.b), rb = __builtin_amdgcn_readfirstlane(it.rb), h = __builtin_amdgcn_readfirstlane(it.h);
  const int n = __builtin_amdgcn_readfirstlane(it.n), len = __builtin_amdgcn_readfirstlane(it.len), off = __builtin_amdgcn_readfirstlane(it.off);
  const int ctx = len - n;                       // position of new token 0 (negative: a draft longer than the sequence)

  // this lane's row; rows beyond the last repeat it and are not stored
  const int rows = n * a.G, row = rb * M + wr * 32 + (lane & 31);
  const bool live = row < rows;
  const int tok = min(row, rows - 1) >> a.lgG, head = h * a.G + (min(row, rows - 1) & (a.G - 1));
  const int pos = ctx + tok;
  const long long qrow = (long long)(off + tok) * a.Hq + head;

  // first and last position of the workgroup's and of the wave's rows
  const int p_lo = ctx + ((rb * M) >> a.lgG), p_hi = ctx + ((min(rb * M + M, rows) - 1) >> a.lgG);
  const int w_lo = ctx + (min(rb * M + wr * 32, rows - 1) >> a.lgG), w_hi = ctx + (min(rb * M + wr * 32 + 31, rows - 1) >> a.lgG);
  const bool idle_wave = rb * M + wr * 32 >= rows;
  const Span sp = span_of<MODE>(a, len, p_lo, p_hi);
  const int per = SPLIT ? __builtin_amdgcn_readfirstlane((int)quotient((uint32_t)(sp.tiles + it.chunks - 1), (uint32_t)it.chunks)) : sp.tiles;
  const int u0 = SPLIT ? min(sp.tiles, per * __builtin_amdgcn_readfirstlane(it.chunk)) : 0, u1 = min(sp.tiles, u0 + per);

  tw_bf16x8 qf[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) qf[s] = *(const tw_bf16x8*)(a.q + qrow * 16 + 2 * s + half);

  // ---- addresses.  Loads: instruction j of a page stores rows 4 j .. 4 j + 3; lane -> row 4 j + lane / 16, stored piece
  // lane % 16, which is piece (lane % 16) ^ order(row) of the row: K order = row % 16, V order = 4 (row % 4) + 2 (row / 4 % 2).
  const int r0 = lane >> 4;
  const unsigned k_off = (unsigned)(r0 * 256 + (((lane & 15) ^ r0) << 4));
  const unsigned v_off = (unsigned)(r0 * 256 + (((lane & 15) ^ (r0 << 2)) << 4));
  // reads of K: row lane % 32, piece 2 s + half
  unsigned k_rd[8];
#pragma unroll
  for (int s = 0; s < 8; ++s) k_rd[s] = (unsigned)((wt * (TILE / WT) + (lane & 31)) * 256 + (((2 * s + half) ^ (lane & 15)) << 4));
  // transposed reads of V: 16 lanes take 4 tokens x 16 dims
  unsigned v_rd[4];
  {
    const int i = lane & 15, dh = (lane >> 4) & 1;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const int piece = (4 * d + 2 * dh + ((i & 3) >> 1)) ^ ((i >> 2) << 2) ^ (half << 1);
      v_rd[d] = (unsigned)(TILE_BYTES + (wt * (TILE / WT) + 4 * half + (i >> 2)) * 256 + piece * 16 + (i & 1) * 8);
    }
  }

  // ---- page ids of 64 tiles at a time: lane k holds the pages of tile base + k
  const int32_t* table = a.page_table + (long long)b * a.max_pages;
  int mine[PPW];                                 // the pages that this wave loads
  unsigned long long mapped[4];                  // per page of a tile: the tiles (bits) where it is mapped
  auto refill = [&](int u) {
    const int v0 = 4 * min(u + lane, u1 - 1);
    int id[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) id[j] = table[min(sp.page(v0 + j), a.max_pages - 1)];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      mapped[j] = __ballot(v0 + j < sp.pages && (unsigned)id[j] < a.pool_pages);
    }
#pragma unroll
    for (int p = 0; p < PPW; ++p) {
      const int j = wave * PPW + p;
      mine[p] = j == 0 ? id[0] : j == 1 ? id[1] : j == 2 ? id[2] : id[3];
    }
  };
  const long long head_off = (long long)h * TW_PAGE * 256, page_stride = (long long)a.Hkv * TW_PAGE * 256;
  int base = 0;                                  // first tile of the page ids held
  auto issue = [&](unsigned char* buf, int u) {
    const int k = u - base, t0 = sp.start(u);
#pragma unroll
    for (int p = 0; p < PPW; ++p) {
      const int pg = wave * PPW + p;
      const int id = __builtin_amdgcn_readlane(mine[p], k);
      const int gap = MODE == MODE_WINDOW && ((u == sp.both) & (4 * u + pg >= sp.sink)) ? sp.shift : 0;
      const int left = (unsigned)id < a.pool_pages ? len - (t0 + pg * TW_PAGE + gap) : 0;    // rows of the page that are tokens
      unsigned char* dst = buf + pg * 4096;
      const char* kp = a.k_pool + (long long)id * page_stride + head_off;
      const char* vp = a.v_pool + (long long)id * page_stride + head_off;
      if (left >= TW_PAGE) {
        if (stream) page_to_lds<2>(kp, vp, k_off, v_off, dst);
        else page_to_lds<0>(kp, vp, k_off, v_off, dst);
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool in = 4 * j + r0 < left;
          const char* ks = in ? kp + ((k_off ^ (unsigned)(64 * j)) + 1024u * j) : (const char*)tw_zero_row + ((lane & 15) << 4);
          const char* vs = in ? vp + ((v_off ^ (unsigned)(32 * (j & 1))) + 1024u * j) : (const char*)tw_zero_row + ((lane & 15) << 4);
          __builtin_amdgcn_global_load_lds((const TW_GLB unsigned int*)ks, (TW_LDS unsigned int*)(dst + 1024 * j), 16, 0, 0);
          __builtin_amdgcn_global_load_lds((const TW_GLB unsigned int*)vs, (TW_LDS unsigned int*)(dst + TILE_BYTES + 1024 * j), 16, 0, 0);
        }
      }
    }
  };

  tw_f32x16 o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  float m = kLow, l = 0.f;                       // m: of the whole row; l: of this lane's tokens
  // A weight is exp2(fma(score, c, -m)) with c = log2(e)/sqrt(128).  The fma keeps what rounding took off m = score * c of the
  // largest score, 2^-24 of it: from 2^30 on, where that leaves an exponent's range, m is kept with c = 1/4, which rounds nothing
  // (and scores that differ at all differ by 64 powers of two).  Then |m| is more than 2^30 whatever the score, which tells.
  auto scale_of = [](float m) -> float { return __builtin_fabsf(m) < kFar ? kScaleLog2 : 0.25f; };
  auto m_log2 = [&]() -> float { return __builtin_fabsf(m) < kFar ? m : m * kScaleLog2 * 4.f; };

  // the mask words of this lane's row that a tile's positions stand in, asked for ahead of the next tile's rows, so that they
  // are not waited for behind those
  struct Words { uint32_t w[3]; };
  auto mask_words = [&](int u) -> Words {
    Words x = {{0u, 0u, 0u}};
    const int j0 = u * TILE - ctx;       // draft token of the tile's first position
    if (MODE == MODE_TREE && j0 > -TILE) {
      const uint32_t* mrow = a.mask + (long long)(off + tok) * a.mask_words;
      const int w0 = j0 >= 0 ? j0 >> 5 : 0;
#pragma unroll
      for (int k = 0; k < 3; ++k)
        if (w0 + k < a.mask_words) x.w[k] = mrow[w0 + k];
    }
    return x;
  };
  auto held_pages = [&](int u) -> unsigned {     // of a tile: which of its four pages are mapped
    const int k = u - base;
    return (unsigned)(mapped[0] >> k & 1) | (unsigned)(mapped[1] >> k & 1) << 1 | (unsigned)(mapped[2] >> k & 1) << 2 | (unsigned)(mapped[3] >> k & 1) << 3;
  };
  auto arrived = [&]() {
    __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0): this wave's rows are in LDS
    __syncthreads();
  };
  auto compute = [&](const unsigned char* buf, int u, unsigned held, const Words& x) {
    const int t0 = sp.start(u);
    const bool in_a_row = MODE == MODE_TREE || u != sp.both;
    bool none = idle_wave, all = (held == 15u) & (t0 + TILE <= len);     // does no row of the wave see the tile, does every row see all of it
    if (MODE == MODE_TREE) {                     // (no short cuts in these: as branches they made 826 us of the prompts of 8192 tokens 838)
      all = all & (t0 + TILE <= ctx);
    } else {
      none = none | (in_a_row & ((t0 > w_hi) | ((t0 + TILE - 1 <= w_lo - a.window) & (t0 >= a.sinks))));
      all = all & in_a_row & (t0 + TILE - 1 <= w_lo) & ((t0 > w_hi - a.window) | (t0 + TILE <= a.sinks));
    }
    if (none) return;
    // K of the whole slice, then the products, each later operand's read behind a product; the first V operands come with
    // the last products, so that they wait for nothing behind the softmax
    tw_f32x16 s[MT];
    tw_bf16x8 kf[MT][8];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int st = 0; st < 8; ++st) kf[mt][st] = *(const tw_bf16x8*)(buf + k_rd[st] + mt * 32 * 256);
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[mt][r] = 0.f;
#pragma unroll
      for (int st = 0; st < 8; ++st) s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[mt][st], qf[st], s[mt], 0, 0, 0);
    }
    union Frag { tw_s16x4 s[2]; tw_bf16x8 v; };
    Frag vf[2 * MT][4];
    auto read_v = [&](int ks) {
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        vf[ks][d].s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((TW_LDS tw_s16x4*)(buf + v_rd[d] + ks * 4096));
        vf[ks][d].s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((TW_LDS tw_s16x4*)(buf + v_rd[d] + ks * 4096 + 2048));
      }
    };
    read_v(0);
    read_v(1);
    __builtin_amdgcn_sched_group_barrier(0x100, 8, 0);
    if (MT == 2) {
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
    }
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
    }
    if (!all) {
      unsigned long long vis;
      if (MODE == MODE_TREE) {
        vis = low_bits(ctx - t0);
        const int j0 = t0 - ctx;
        if (j0 > -TILE) {
          const unsigned long long w = (unsigned long long)x.w[1] << 32 | x.w[0];
          const int sh = j0 & 31;
          vis |= j0 < 0 ? w << -j0 : sh ? w >> sh | (unsigned long long)x.w[2] << (64 - sh) : w;
        }
        vis &= low_bits(len - t0);
      } else {
        // (pos < len.)  In the tile in which the sinks' pages end, the first `lead` positions are those, and the others follow the
        // window's first page as if they had begun at t1
        const int lead = in_a_row ? 0 : (sp.sink - 4 * u) * TW_PAGE, t1 = in_a_row ? t0 : sp.first * TW_PAGE - lead;
        vis = low_bits(pos + 1 - t1) & (~low_bits(pos - a.window + 1 - t1) | low_bits(a.sinks - t1));
        if (!in_a_row) vis = (vis & ~low_bits(lead)) | (low_bits(min(a.sinks, pos + 1) - t0) & low_bits(lead));
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (!(held >> j & 1u)) vis &= ~(0xFFFFull << (16 * j));
      vis >>= wt * (TILE / WT) + 4 * half;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const uint32_t w = (uint32_t)(vis >> (32 * mt));
#pragma unroll
        for (int r = 0; r < 16; ++r) {           // the row's bit, spread over a word, chooses the score or -inf: two instructions
          const uint32_t keep = (uint32_t)__builtin_amdgcn_sbfe((int)w, 8 * (r / 4) + r % 4, 1);
          s[mt][r] = __uint_as_float((keep & __float_as_uint(s[mt][r])) | (~keep & 0xFF800000u));
        }
      }
    }
    float mx = s[0][0];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[mt][r]);
    {
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(mx), __float_as_uint(mx), false, false);
      mx = fmaxf(__uint_as_float(sw[0]), __uint_as_float(sw[1]));
    }
    float c = scale_of(m);
    if (__any(mx * c > m + kGrowth)) {
      const float was = m_log2(), mn = fmaxf(was, mx * kScaleLog2), al = __builtin_amdgcn_exp2f(was - mn);
      l *= al;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= al;
      if (mn > was) m = __builtin_fabsf(mn) < kFar ? mn : mx * 0.25f;
      c = scale_of(m);
    }
    constexpr bool REST = WT == 2;
    tw_bf16x8 p[2 * MT], rest[2 * MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][r], c, -m));
        l += w;
        const __bf16 near = (__bf16)w;
        p[2 * mt + r / 8][r % 8] = near;
        if constexpr (REST) rest[2 * mt + r / 8][r % 8] = (__bf16)(w - (float)near);
      }
#pragma unroll
    for (int ks = 2; ks < 2 * MT; ++ks) read_v(ks);
#pragma unroll
    for (int ks = 0; ks < 2 * MT; ++ks)
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[ks][d].v, p[ks], o[d], 0, 0, 0);
    if constexpr (REST)                          // (behind the others: next to them they would wait for their accumulators)
#pragma unroll
      for (int ks = 0; ks < 2 * MT; ++ks)
#pragma unroll
        for (int d = 0; d < 4; ++d) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[ks][d].v, rest[ks], o[d], 0, 0, 0);
  };

  if (u0 < u1) {
    base = u0;
    refill(u0);
    issue(buf0, u0);
    for (int u = u0; u < u1; u += 2) {
      arrived();                                 // the tile's rows, for every wave; nobody reads the other buffer any more
      unsigned held = held_pages(u);
      Words x = mask_words(u);
      if (u + 1 < u1) issue(buf1, u + 1);
      compute(buf0, u, held, x);
      if (u + 1 >= u1) break;
      arrived();
      held = held_pages(u + 1);
      x = mask_words(u + 1);
      if (u + 2 < u1) {
        if (u + 2 - base >= 64) { base = u + 2; refill(base); }
        issue(buf0, u + 2);
      }
      compute(buf1, u + 1, held, x);
    }
  }

  // ---- the waves' states of the same rows merged
  m = m_log2();
  {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  }
  if constexpr (WT > 1) {
    __syncthreads();                             // the tiles have been read
    float* part = (float*)buf0 + wr * 32 * 128;  // WR * 32 rows x 128 floats: 16 KiB per row wave, in both buffers together
    float2* ml = (float2*)(buf1 + 16384) + wr * 32;
    static_assert(WT <= 2 && WR * 32 * 512 <= 2 * TILE_BYTES, "one partial per row wave");
    if (wt == 1) {
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) part[(d * 16 + r) * 64 + lane] = o[d][r];
      if (half == 0) ml[lane] = make_float2(m, l);
    }
    __syncthreads();
    if (wt != 0) return;
    const float2 x = ml[lane & 31];
    const float mn = fmaxf(m, x.x), s0 = __builtin_amdgcn_exp2f(m - mn), s1 = __builtin_amdgcn_exp2f(x.x - mn);
    l = l * s0 + x.y * s1;
    m = mn;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = o[d][r] * s0 + part[(d * 16 + r) * 64 + lane] * s1;
  }
  if (!live) return;
  if (!SPLIT || it.chunks == 1) {
    const float inv = l == 0.f ? 0.f : 1.0f / l;
    uint2* orow = a.out + qrow * 32;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        union { __bf16 e[4]; uint2 v; } w;
#pragma unroll
        for (int i = 0; i < 4; ++i) w.e[i] = (__bf16)(o[d][4 * k + i] * inv);
        orow[8 * d + 2 * k + half] = w.v;
      }
    if (a.lse && half == 0) a.lse[qrow] = row_lse(m, l);
    return;
  }
  const long long prow = (long long)it.slot * M + wr * 32 + (lane & 31);
  float4* acc = (float4*)(a.ws_acc + prow * 128);
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[8 * d + 2 * k + half] = make_float4(o[d][4 * k], o[d][4 * k + 1], o[d][4 * k + 2], o[d][4 * k + 3]);
  if (half == 0) a.ws_ml[prow] = make_float2(m, l);
}

// (Bounds of 256 threads also where there are 128: told that LDS leaves one wave to a SIMD, the compiler keeps the accumulators apart from
// the registers that vector instructions reach, and moves them to and fro for every rescaling: 40 lists of up to 7 tiles 10.2 us, 8.9 without.)
// SPLIT: resident workgroups stride over the items (workgroups beyond those would wait for a slot to find out that there is
// nothing left for them); otherwise a workgroup per list.
template <int MODE, int WR, int WT, bool SPLIT>
__global__ __launch_bounds__(256, 2) void new_tokens_kernel(NewArgs a) {
  constexpr int M = 32 * WR;
  __shared__ __align__(1024) unsigned char buf0[2 * TILE_BYTES];
  __shared__ __align__(1024) unsigned char buf1[2 * TILE_BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  Item it;
  // K and V that one workgroup alone reads and that are more than 96 MB together (the last-level cache holds 256) pass by it: non-temporal
  // loads, tree of 16 over 4 x 8192 tokens of 32 KV heads 104 -> 91 us (5.9 TB/s), 64 tokens under windows of 4096 156 -> 139 (6.1).
  // Less would still lie there for the next call on the same cache (calls on three caches in turn: of 128 MB 40.2 us, non-temporal
  // 35.6, of 73 MB 23.4 and 24.1, of 60 MB 20.5 and 24.6), and row blocks that share their rows read them from the caches (two prompts
  // of 8192 tokens 806 us, 894).
  bool stream = a.stream != 0;
  if (!SPLIT) {
    if (stream) {                                // as the lists really are
      float total = 0.f;
      for (int b0 = 0; b0 < a.batch; b0 += 64) {
        const Seq q = seq_of<MODE, M>(a, b0 + lane);
        total += wave_sum_f((float)q.lists * (float)q.tiles);
      }
      stream = total > (float)STREAM_TILES;
    }
    if (whole_item<M>(a, &it)) attend_item<MODE, WR, WT, SPLIT>(a, it, buf0, buf1, lane, wave, stream);
    return;
  }
  Seq seq;
  const int chunk = __builtin_amdgcn_readfirstlane(plan_chunk<MODE, M>(a, lane, &seq, &stream));
  uint32_t want = blockIdx.x;
  while (find_item<MODE, M>(a, lane, chunk, seq, want, &it)) {
    attend_item<MODE, WR, WT, SPLIT>(a, it, buf0, buf1, lane, wave, stream);
    want += gridDim.x;
    if (want >= it.items) break;
    __syncthreads();                             // the buffers have been read
  }
}

// The parts of cut lists joined.  A row (new token, head) is folded by LANES half waves of 32 lanes x 4 dims: two (a wave; four
// rows to a workgroup) where there are many rows, eight (a workgroup) where few rows have many parts each and the wait
// for one part after the other is what counts: 256 rows of 32 parts 4.0 us with eight, 8.3 us with two.  Whole calls, two / eight:
//   one sequence of 4096     rows  32: 11.9 / 11.0  256: 14.0 / 13.4   512: 15.7 / 15.4  1024: 16.6 / 16.9  4096: 28.3 / 29.8
//   4 sequences of 8192      rows 512: 30.8 / 31.0 1024: 32.5 / 33.2  2048: 36.6 / 37.2  8192: 60 / 64     16384: 93 / 100
//   16 sequences of 4096     rows 512: 49.2 / 49.5 2048: 49.5 / 50.8  8192: 57.5 / 61   16384: 70 / 77
template <int M, int LANES>
__global__ __launch_bounds__(256) void new_tokens_combine_kernel(NewArgs a) {
  constexpr int ROWS = 8 / LANES;
  const int lane = threadIdx.x & 63, dl = lane & 31, part = (threadIdx.x >> 5) % LANES;
  const int b = blockIdx.y, idx = (int)(blockIdx.x * ROWS + threadIdx.x / (32 * LANES));
  const int n = seq_new(a, b);
  const int tok = idx / a.Hq, head = idx - tok * a.Hq;
  const int chunks = a.ws_plan[2 * b];
  if (chunks <= 1) return;                       // written by the attention kernel itself
  const bool live = tok < n;
  const int blocks = (n * a.G + M - 1) / M, row = min(tok, n - 1) * a.G + (head & (a.G - 1));
  const long long step = (long long)blocks * a.Hkv * M;
  long long at = ((long long)a.ws_plan[2 * b + 1] + (row / M) * a.Hkv + (head >> a.lgG)) * M + row % M + part * step;
  float m = kLow, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto join = [&](float m2, float l2, const float4& v) {
    const float mn = fmaxf(m, m2), so = __builtin_amdgcn_exp2f(m - mn), sn = __builtin_amdgcn_exp2f(m2 - mn);
    l = l * so + l2 * sn;
    o.x = o.x * so + v.x * sn; o.y = o.y * so + v.y * sn; o.z = o.z * so + v.z * sn; o.w = o.w * so + v.w * sn;
    m = mn;
  };
#pragma unroll 4
  for (int c = part; c < chunks; c += LANES, at += LANES * step) {
    const float2 ml = a.ws_ml[at];
    join(ml.x, ml.y, ((const float4*)a.ws_acc)[at * 32 + dl]);
  }
  join(__shfl_xor(m, 32), __shfl_xor(l, 32), make_float4(__shfl_xor(o.x, 32), __shfl_xor(o.y, 32), __shfl_xor(o.z, 32), __shfl_xor(o.w, 32)));
  if (LANES == 8) {
    __shared__ float4 so4[4][32];
    __shared__ float2 sml[4];
    const int wave = threadIdx.x >> 6;
    if (lane < 32) so4[wave][dl] = o;
    if (lane == 0) sml[wave] = make_float2(m, l);
    __syncthreads();
    if (wave != 0) return;
#pragma unroll
    for (int w = 1; w < 4; ++w) join(sml[w].x, sml[w].y, so4[w][dl]);
  }
  if (!live || (lane >> 5)) return;
  const long long qrow = (long long)((a.offsets ? a.offsets[b] : b * a.max_new) + tok) * a.Hq + head;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  union { __bf16 e[4]; uint2 v; } w;
  w.e[0] = (__bf16)(o.x * inv); w.e[1] = (__bf16)(o.y * inv); w.e[2] = (__bf16)(o.z * inv); w.e[3] = (__bf16)(o.w * inv);
  a.out[qrow * 32 + dl] = w.v;
  if (a.lse && lane == 0) a.lse[qrow] = row_lse(m, l);
}

// ---------------------------------------------------------------- host side
// Rows to a workgroup: as many as there are, up to 128, since another row block reads the same K and V again.  Fewer rows leave the
// waves a half of the tile's tokens each, instead of rows that nobody has.  us with 32 / 64 / 128 to a workgroup, 8 KV heads:
//   one sequence of 4096     16 rows 12.3 / 12.3 / 12.7   64 rows  15.5 /  15.3 /  14.5   128 rows  19.4 /  17.9 /  16.9
//   8 sequences of 4096       4 rows 30.5 / 29.8 / 31.6   64 rows  41.3 /  36.6 /  36.8   128 rows  67.2 /  48.5 /  43.6
//   8 sequences of 32768     32 rows  172 /  170 /  169   64 rows   262 /   180 /   173   128 rows   464 /   298 /   204
// (what 64 lose against 128 is the weights' second product, which 128 leave out.)
int rows_per_block(long long rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : 128; }

// Lists that cannot be long are not cut, which saves the launch that joins the parts and their way through memory: up to 6 tiles,
// one more for every 32 lists, at most 32.  Few lists run no faster whole than cut from there on; many would leave CUs idle
// only where few of them are as long as the longest may be.  us, cut / whole, by tiles of all lists:
//   32 rows    8 lists  4: 10.1 /  7.3  6: 10.2 /  8.9  8: 10.2 / 10.5     160 lists   8: 18.0 / 13.3  16: 23.3 / 21.8  26: 30.9 / 42.9
//   64        32        6: 13.4 / 10.4  8: 13.4 / 11.6 12: 14.4 / 17.6     160        12: 24.1 / 19.6  16: 29.1 / 25.1  26: 37.0 / 44.3
//   128        8        6: 12.4 / 11.7  8: 12.6 / 14.0                     160        12: 27.3 / 22.1  16: 36.3 / 31.2  26: 55.3 / 49.9
//   32       512       16: 47.2 / 43.6 24: 66.7 / 63.0 32: 85.2 / 81.9
// and with ragged lengths up to that, for which more would be too many:
//   32       160        8: 10.3 / 10.8 12: 11.0 / 12.5 16: 13.7 / 18.2     128 rows   12: 14.8 / 14.9  16: 16.9 / 22.4  26: 25.5 / 34.6
// Nor are the row blocks of chunks and prompts under a window that fill the chip by themselves: right for sequences that are alike,
// and for ragged prompts, whose longest blocks the dispatcher starts first and evens out.  The host knows no n_new, though, and
// beside a chunk single tokens have a workgroup walk each of their lists; so where n_new is given and a list can be of more tiles
// than 192 for every turn of the chip, they are cut.  us, whole / cut:
//   prompts  2 of 8192, window 4096: 840 / 954    1 of 8192, no window: 557 / 640    8 of 50 to 4000: 394 / 516    16 of 512: 72.6 / 72.5
//   chunks   3 of 1499 over 9001, window 2047, 8 heads a group: 330 / 352    4 of 512 over 4096: 140 / 150    8 of 512 over 512 to 32768: 650 / 625
//            4 of 512 over 32768: 1043 / 1074    2 of 1024 over 100000: 3195 / 3380
//   mixed    512 and 3 single tokens over 32768: 815 / 361    512 and 31 over 8192 (16 tiles a turn): 531 / 260
//            2048 and 15 over 16384, window 4096 (5): 254 / 270    8192 and 63 over 8192 (0.5): 1377 / 1767, with 900 for the launch that joins
constexpr long long LONG_TURN = 192;
constexpr long long JOIN_ROWS = 1ll << 26;       // rows from which on the launch that joins, four to a workgroup, would have 2^32 threads
bool cut_lists(bool window, bool counted, int blocks, long long lists, long long longest, long long rows) {
  if (longest <= std::min(32ll, 6 + lists / 32)) return false;
  const long long places = 2ll * tw_num_cus();
  if (!window || blocks < 8 || lists < places) return true;
  return counted && longest * places > LONG_TURN * lists && rows < JOIN_ROWS;
}

template <int MODE, int WR, int WT>
int launch_new(NewArgs a, hipStream_t s) {
  constexpr int M = 32 * WR;
  const long long lists = (long long)a.rb_max * a.batch * a.Hkv, rows = (long long)a.max_new * a.Hq;
  long long longest = ((long long)a.max_pages * TW_PAGE + TILE - 1) / TILE;      // tiles that a list can have
  if (MODE == MODE_WINDOW)
    longest = std::min(longest, (((long long)a.sinks + TW_PAGE - 1) / TW_PAGE + ((long long)a.window + M / a.G + TW_PAGE - 2) / TW_PAGE + 1 + 3) / 4);
  a.stream = a.rb_max == 1 && lists * longest > STREAM_TILES;
  tw_prof_before(TW_K_NEW_TOKENS, s);
  if (!cut_lists(MODE == MODE_WINDOW, a.n_new != nullptr, a.rb_max, lists, longest, rows)) {
    TW_LAUNCH((new_tokens_kernel<MODE, WR, WT, false>), dim3((unsigned)lists), dim3(64 * WR * WT), 0, s, a);
    return tw_prof_after(s);
  }
  // resident workgroups (64 KiB of LDS each, two to a CU), no more than the lists could make items
  const long long most = lists * ((longest + PLAN_MIN_TILES - 1) / PLAN_MIN_TILES);
  TW_LAUNCH((new_tokens_kernel<MODE, WR, WT, true>), dim3((unsigned)std::min(most, 2ll * a.cus)), dim3(64 * WR * WT), 0, s, a);
  if (int e = tw_prof_after(s)) return e;
  tw_prof_before(TW_K_NEW_COMBINE, s);
  if (rows * a.batch <= COMBINE_FEW) TW_LAUNCH((new_tokens_combine_kernel<M, 8>), dim3((unsigned)rows, (unsigned)a.batch), dim3(256), 0, s, a);
  else TW_LAUNCH((new_tokens_combine_kernel<M, 2>), dim3((unsigned)((rows + 3) / 4), (unsigned)a.batch), dim3(256), 0, s, a);
  return tw_prof_after(s);
}

// Parts that a plan can make: fewer than 2 W rounds (see plan_chunk), and of one row block per sequence and KV head no more than its
// list has chunks of the shortest length (8 lists of 4096 tokens: 256 parts of 128 rows, 17 MB; all that fit the chip: 136 MB).
size_t part_slots(const TwDims& d, long long rows) {
  const long long most = (long long)tw_num_cus() * 4 * PLAN_ROUNDS;
  if (rows > 128) return (size_t)most;
  const long long tiles = ((long long)d.max_pages + 3) / 4, chunks = (tiles + PLAN_MIN_TILES - 1) / PLAN_MIN_TILES;
  return (size_t)std::min(most, chunks * d.batch * d.Hkv);
}

size_t align256n(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

size_t tw_new_tokens_workspace(const TwDims& d, int max_new) {
  if (max_new <= 0 || max_new > TW_MAX_NEW) return 0;
  const long long rows = (long long)max_new * d.G;
  const int M = rows_per_block(rows);
  const size_t slots = part_slots(d, rows);
  return align256n((size_t)d.batch * 8) + align256n(slots * M * 8) + slots * M * 512;
}

static int new_tokens_impl(const twilight_kv_t* kv, const void* q, const int32_t* n_new, const int32_t* new_offsets, int32_t max_new,
                           const uint32_t* mask, int32_t mask_words, int32_t window, int32_t sinks, bool tree,
                           void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  TwDims d;
  if (int e = tw_check_kv(kv, &d)) return e;
  if (!q || !out || !kv->k_pool || !kv->v_pool) return TW_EINVAL;
  if (max_new <= 0 || max_new > TW_MAX_NEW || d.max_pages > TW_MAX_ROW_PAGES) return TW_EINVAL;
  if (((uintptr_t)q | (uintptr_t)out | (uintptr_t)kv->k_pool | (uintptr_t)kv->v_pool | (uintptr_t)ws) & 15) return TW_EINVAL;
  if (!ws || ws_bytes < tw_new_tokens_workspace(d, max_new)) return TW_EWORKSPACE;
  const int M = rows_per_block((long long)max_new * d.G);
  NewArgs a;
  a.q = (const uint4*)q; a.k_pool = (const char*)kv->k_pool; a.v_pool = (const char*)kv->v_pool;
  a.page_table = kv->page_table; a.seq_lens = kv->seq_lens; a.n_new = n_new; a.offsets = new_offsets; a.mask = mask;
  a.out = (uint2*)out; a.lse = lse;
  const size_t slots = part_slots(d, (long long)max_new * d.G);
  a.ws_plan = (int32_t*)ws;
  a.ws_ml = (float2*)((char*)ws + align256n((size_t)d.batch * 8));
  a.ws_acc = (float*)((char*)a.ws_ml + align256n(slots * M * 8));
  a.batch = d.batch; a.Hq = d.Hq; a.Hkv = d.Hkv; a.G = d.G; a.lgG = __builtin_ctz(d.G); a.max_pages = d.max_pages;
  a.max_new = max_new; a.mask_words = mask_words; a.window = window; a.sinks = sinks; a.pool_pages = (unsigned)d.pool_pages;
  a.rb_max = (int)(((long long)max_new * d.G + M - 1) / M); a.cus = tw_num_cus(); a.stream = 0;
  const long long lists = (long long)a.rb_max * d.batch * d.Hkv;
  if (lists >= (1ll << 24) || (long long)max_new * d.batch >= (1ll << 31)) return TW_EINVAL;      // (a launch has fewer than 2^32 threads)
  hipStream_t s = (hipStream_t)stream;
  if (tree) {
    switch (M) {
      case 32: return launch_new<MODE_TREE, 1, 2>(a, s);
      case 64: return launch_new<MODE_TREE, 2, 2>(a, s);
      default: return launch_new<MODE_TREE, 4, 1>(a, s);
    }
  }
  switch (M) {
    case 32: return launch_new<MODE_WINDOW, 1, 2>(a, s);
    case 64: return launch_new<MODE_WINDOW, 2, 2>(a, s);
    default: return launch_new<MODE_WINDOW, 4, 1>(a, s);
  }
}

extern "C" int twilight_tree_attention(const twilight_kv_t* kv, const void* q, const int32_t* n_new, const int32_t* new_offsets,
                                       int32_t max_new, const uint32_t* tree_mask, int32_t mask_words, void* out, float* lse,
                                       void* ws, size_t ws_bytes, void* stream) {
  if (!tree_mask || max_new > TW_MAX_TREE || mask_words <= 0 || (long long)mask_words * 32 < max_new) return TW_EINVAL;
  return new_tokens_impl(kv, q, n_new, new_offsets, max_new, tree_mask, mask_words, 0, 0, true, out, lse, ws, ws_bytes, stream);
}

extern "C" int twilight_window_attention(const twilight_kv_t* kv, const void* q, const int32_t* n_new, const int32_t* new_offsets,
                                         int32_t max_new, int32_t window, int32_t num_sinks, void* out, float* lse,
                                         void* ws, size_t ws_bytes, void* stream) {
  if (window < 1 || num_sinks < 0) return TW_EINVAL;
  const int32_t most = 1 << 30;                  // longer than any sequence; positions minus it stay in 32 bits
  return new_tokens_impl(kv, q, n_new, new_offsets, max_new, nullptr, 0, window < most ? window : most, num_sinks < most ? num_sinks : most, false,
                         out, lse, ws, ws_bytes, stream);
}
