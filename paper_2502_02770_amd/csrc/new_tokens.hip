// Attention of a sequence's newest tokens over its paged cache: a drafted tree of tokens (twilight_tree_attention), or a
// chunk of consecutive tokens with a sliding window and sinks (twilight_window_attention).
//
// The rows of a KV head are its G query heads times the N new tokens, row r = token r / G, head r % G, so that every K/V
// tile is loaded once for all of them.  A workgroup takes M = 32 * WR rows and walks tiles of 64 cached tokens:
//
//   S^T = K Q^T     v_mfma_f32_32x32x16_bf16, A = 32 tokens of K, B = 32 rows of Q (held in registers throughout)
//   P^T = exp2(S^T * log2(e)/sqrt(128) - m), m = running maximum of the row
//   O^T += V^T P^T  A = V^T (transposed LDS reads), B = P^T
//
// In the result layout of the first product a lane holds 16 tokens of ONE row (its partner lane in the other half wave
// the other 16), so maximum, sum and rescaling are in-lane but for one exchange between the halves, and the lane's own P
// values are its B operand of the second product as they stand: the order of the 16 tokens within a contraction step is
// free as long as the V^T operand has the same (slot 8 * h + j of step k = token 16 k + 8 (j / 4) + 4 h + j % 4).
// P is rounded to bf16 for the product (each weight by at most 2^-8 of itself, the largest of a row exactly 1 at its time;
// the output is bf16 anyway); scores, maxima, sums and accumulators are fp32, and the sum is of the unrounded weights.
//
// K and V rows go from HBM to LDS without passing registers, 16 bytes per lane, a page of (token, head) rows being 4 KiB
// contiguous; the 16-byte pieces of a row are stored in an order that depends on the row (XOR), so that neither the
// 32-row reads of K nor the transposed reads of V meet in a bank.  Two buffers: a tile's loads are issued before the
// tile ahead of it is computed.
#include "tw_common.h"

namespace {

typedef __bf16 tw_bf16x8 __attribute__((ext_vector_type(8)));
typedef short tw_s16x4 __attribute__((ext_vector_type(4)));
typedef float tw_f32x16 __attribute__((ext_vector_type(16)));
#define TW_LDS __attribute__((address_space(3)))
#define TW_GLB __attribute__((address_space(1)))

constexpr float kScaleLog2 = 0.08838834764831845f * 1.4426950408889634f;   // log2(e) / sqrt(128)
constexpr float kLn2n = 0.6931471805599453f;
constexpr float kLow = -1e30f;                   // running maximum before any visible token: exp2(-inf - kLow) = 0
constexpr int TILE = 64, TILE_BYTES = TILE * 256;
enum { MODE_TREE = 0, MODE_WINDOW = 1 };
constexpr int PLAN_ROUNDS = 2;                   // items per resident workgroup at most, as planned
constexpr int PLAN_MIN_TILES = 2;                // shortest chunk of a list
constexpr int PLAN_ITEM_TILES = 2;               // fixed cost of an item in tiles: its plan, page and query loads, its partial result

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
  int batch, Hq, Hkv, G, lgG, max_pages, max_new, mask_words, window, sinks, rb_max, grid;
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

// The tiles that rows of tokens at positions p_lo .. p_hi see: `sink` tiles from the start, then those from `first` on.
struct Span {
  int sink, first, tiles;
  __device__ __forceinline__ int tile(int u) const { return u < sink ? u : first + (u - sink); }
};
template <int MODE>
__device__ __forceinline__ Span span_of(const NewArgs& a, int len, int p_lo, int p_hi) {
  Span s;
  const int end = MODE == MODE_TREE ? len : min(len, p_hi + 1);
  if (end <= 0) { s.sink = s.first = s.tiles = 0; return s; }
  s.first = MODE == MODE_TREE ? 0 : max(0, p_lo - a.window + 1) / TILE;
  s.sink = MODE == MODE_TREE ? 0 : min((int)(((unsigned)a.sinks + TILE - 1) / TILE), s.first);
  s.tiles = s.sink + (end - 1) / TILE - s.first + 1;
  return s;
}

// Which part of which list a workgroup takes.  A list is a (row block, KV head) of a sequence; a sequence's lists are cut
// into the same number of chunks.
struct Item {
  int b, rb, h, chunk, chunks, slot;
};

template <int MODE, int M>
__device__ __forceinline__ void lists_of(const NewArgs& a, int b, int* lists, int* tiles) {
  const int n = seq_new(a, b), len = seq_len(a, b);
  const int blocks = (n * a.G + M - 1) / M;
  *lists = blocks * a.Hkv;
  *tiles = blocks == 0 ? 0 : max(1, span_of<MODE>(a, len, len - min(n, M / a.G), len - 1).tiles);
}

__device__ __forceinline__ uint32_t quotient(unsigned long long x, uint32_t y) {   // at most 2^26, more tiles than a list has
  const unsigned long long r = x >> 32 ? x / y : (unsigned long long)((uint32_t)x / y);
  return r < (1ull << 26) ? (uint32_t)r : 1u << 26;
}

// Chunk length in tiles for `grid` resident workgroups: of a few lengths that give every workgroup one or two items, the
// one whose rounds are cheapest by the items that it really makes.  With c > total / (W r) there are fewer than W r + lists
// items, and fewer than 2 W r of lists that are cut: what the launch's grid and the workspace are sized for.
template <int MODE, int M>
__device__ __forceinline__ int plan_chunk(const NewArgs& a, int lane) {
  unsigned long long total = 0;
  uint32_t lists_all = 0;
  int lists = 0, tiles = 0;                      // of this lane's sequence, where 64 lanes hold them all
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    lists = tiles = 0;
    if (b0 + lane < a.batch) lists_of<MODE, M>(a, b0 + lane, &lists, &tiles);
    total += tw_readlane_u64(tw_wave_scan_u64((unsigned long long)lists * (unsigned)tiles), 63);
    lists_all += (uint32_t)__builtin_amdgcn_readlane((int)tw_wave_scan_u32((uint32_t)lists), 63);
  }
  const uint32_t W = (uint32_t)a.grid;
  uint32_t best = 0xFFFFFFFFu, chunk = PLAN_MIN_TILES;
  for (uint32_t k = 0; k < 2u * PLAN_ROUNDS; ++k) {
    const uint32_t r = 1u + (k >> 1), room = W * r > lists_all / 2u ? W * r - lists_all / 2u : 0u;
    uint32_t c;
    if (room == 0u) {
      if (k + 1u < 2u * PLAN_ROUNDS || best != 0xFFFFFFFFu) continue;
      c = quotient(total, W) + 1u;               // far more lists than workgroups: only the longest are cut
    } else {
      c = quotient(total, room) + 1u;
      if (k & 1u) c += c / 8u + 1u;
    }
    c = max(c, (uint32_t)PLAN_MIN_TILES);
    uint32_t items = 0;
    for (int b0 = 0; b0 < a.batch; b0 += 64) {
      if (a.batch > 64) {
        lists = tiles = 0;
        if (b0 + lane < a.batch) lists_of<MODE, M>(a, b0 + lane, &lists, &tiles);
      }
      items += (uint32_t)__builtin_amdgcn_readlane((int)tw_wave_scan_u32((uint32_t)lists * (((uint32_t)tiles + c - 1u) / c)), 63);
    }
    const uint32_t cost = (items + W - 1u) / W * (c + PLAN_ITEM_TILES);
    if (cost < best) { best = cost; chunk = c; }
  }
  return (int)chunk;
}

// This workgroup's item; false: none.
template <int MODE, int M, bool SPLIT>
__device__ __forceinline__ bool find_item(const NewArgs& a, int lane, Item* it) {
  if (!SPLIT) {                                  // row blocks from the last (longest under a causal mask) to the first
    unsigned i = blockIdx.x;
    it->h = (int)(i % (unsigned)a.Hkv); i /= (unsigned)a.Hkv;
    it->b = (int)(i % (unsigned)a.batch);
    it->rb = a.rb_max - 1 - (int)(i / (unsigned)a.batch);
    it->chunk = 0; it->chunks = 1; it->slot = 0;
    return it->rb * M < seq_new(a, it->b) * a.G;
  }
  const int chunk = plan_chunk<MODE, M>(a, lane);
  uint32_t items = 0, slots = 0;
  const uint32_t want = blockIdx.x;
  bool found = false;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    int lists = 0, tiles = 0;
    if (b0 + lane < a.batch) lists_of<MODE, M>(a, b0 + lane, &lists, &tiles);
    const int chunks = (tiles + chunk - 1) / chunk;
    const uint32_t mine = (uint32_t)(lists * chunks), part = chunks > 1 ? mine : 0u;
    const uint32_t ie = tw_wave_scan_u32(mine), se = tw_wave_scan_u32(part);
    if (blockIdx.x == 0 && threadIdx.x < 64 && b0 + lane < a.batch) {   // for the combine kernel
      a.ws_plan[2 * (b0 + lane)] = chunks;
      a.ws_plan[2 * (b0 + lane) + 1] = (int)(slots + se - part);
    }
    const unsigned long long here = __ballot(items + ie > want);
    if (!found && here) {
      const int l = __builtin_ctzll(here);
      const uint32_t before = items + (uint32_t)__builtin_amdgcn_readlane((int)(ie - mine), l);
      const uint32_t k = want - before;          // ((chunk * blocks) + block) * Hkv + head: blocks of the same rows' chunk on one XCD
      it->b = b0 + l;
      it->chunks = __builtin_amdgcn_readlane(chunks, l);
      const uint32_t all = (uint32_t)__builtin_amdgcn_readlane(lists, l);
      it->chunk = (int)(k / all);
      const uint32_t rest = k - (uint32_t)it->chunk * all;
      it->rb = (int)(rest / (uint32_t)a.Hkv);
      it->h = (int)(rest - (uint32_t)it->rb * (uint32_t)a.Hkv);
      it->slot = (int)(slots + (uint32_t)__builtin_amdgcn_readlane((int)(se - part), l) + k);
      found = true;
      if (blockIdx.x != 0) return true;
    }
    items += (uint32_t)__builtin_amdgcn_readlane((int)ie, 63);
    slots += (uint32_t)__builtin_amdgcn_readlane((int)se, 63);
  }
  return found;
}

template <int MODE, int WR, int WT, bool SPLIT>
__global__ __launch_bounds__(64 * WR * WT, WR * WT >= 4 ? 2 : 1) void new_tokens_kernel(NewArgs a) {
  constexpr int NW = WR * WT, M = 32 * WR, MT = 2 / WT, PPW = 4 / NW;
  __shared__ __align__(1024) unsigned char buf0[2 * TILE_BYTES];
  __shared__ __align__(1024) unsigned char buf1[2 * TILE_BYTES];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int wr = wave / WT, wt = wave % WT, half = lane >> 5;

  Item it;
  if (!find_item<MODE, M, SPLIT>(a, lane, &it)) return;
  const int b = __builtin_amdgcn_readfirstlane(it.b), rb = __builtin_amdgcn_readfirstlane(it.rb), h = __builtin_amdgcn_readfirstlane(it.h);
  const int n = __builtin_amdgcn_readfirstlane(seq_new(a, b)), len = __builtin_amdgcn_readfirstlane(seq_len(a, b));
  const int off = __builtin_amdgcn_readfirstlane(a.offsets ? a.offsets[b] : b * a.max_new);
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
  const int u0 = (int)((long long)sp.tiles * it.chunk / it.chunks), u1 = (int)((long long)sp.tiles * (it.chunk + 1) / it.chunks);

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
    const int ul = min(u + lane, u1 - 1), pg0 = sp.tile(ul) * (TILE / TW_PAGE);
    int id[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) id[j] = table[min(pg0 + j, a.max_pages - 1)];
#pragma unroll
    for (int j = 0; j < 4; ++j) mapped[j] = __ballot((unsigned)id[j] < a.pool_pages && (pg0 + j) * TW_PAGE < len);
#pragma unroll
    for (int p = 0; p < PPW; ++p) {
      const int j = wave * PPW + p;
      mine[p] = j == 0 ? id[0] : j == 1 ? id[1] : j == 2 ? id[2] : id[3];
    }
  };
  const long long head_off = (long long)h * TW_PAGE * 256, page_stride = (long long)a.Hkv * TW_PAGE * 256;
  int base = 0;                                  // first tile of the page ids held
  auto issue = [&](unsigned char* buf, int u) {
    const int k = u - base, t0 = sp.tile(u) * TILE;
#pragma unroll
    for (int p = 0; p < PPW; ++p) {
      const int pg = wave * PPW + p;
      const int id = __builtin_amdgcn_readlane(mine[p], k);
      const int left = (unsigned)id < a.pool_pages ? len - (t0 + pg * TW_PAGE) : 0;    // rows of the page that are tokens
      unsigned char* dst = buf + pg * 4096;
      const char* kp = a.k_pool + (long long)id * page_stride + head_off;
      const char* vp = a.v_pool + (long long)id * page_stride + head_off;
      if (left >= TW_PAGE) {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          __builtin_amdgcn_global_load_lds((const TW_GLB unsigned int*)(kp + ((k_off ^ (unsigned)(64 * j)) + 1024u * j)), (TW_LDS unsigned int*)(dst + 1024 * j), 16, 0, 0);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          __builtin_amdgcn_global_load_lds((const TW_GLB unsigned int*)(vp + ((v_off ^ (unsigned)(32 * (j & 1))) + 1024u * j)), (TW_LDS unsigned int*)(dst + TILE_BYTES + 1024 * j), 16, 0, 0);
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

  auto held_pages = [&](int u) -> unsigned {     // of a tile: which of its four pages are mapped
    const int k = u - base;
    return (unsigned)(mapped[0] >> k & 1) | (unsigned)(mapped[1] >> k & 1) << 1 | (unsigned)(mapped[2] >> k & 1) << 2 | (unsigned)(mapped[3] >> k & 1) << 3;
  };
  auto arrived = [&]() {
    __builtin_amdgcn_s_waitcnt(0x0F70);          // vmcnt(0): this wave's rows are in LDS
    __syncthreads();
  };
  auto compute = [&](const unsigned char* buf, int u, unsigned held) {
    const int t0 = sp.tile(u) * TILE;
    bool all = held == 15u && t0 + TILE <= len;
    if (MODE == MODE_TREE) {
      all = all && t0 + TILE <= ctx;
      if (idle_wave) return;
    } else {
      if (idle_wave || t0 > w_hi || (t0 + TILE - 1 <= w_lo - a.window && t0 >= a.sinks)) return;    // no row of the wave sees the tile
      all = all && t0 + TILE - 1 <= w_lo && (t0 > w_hi - a.window || t0 + TILE <= a.sinks);
    }
    tw_f32x16 s[MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
#pragma unroll
      for (int r = 0; r < 16; ++r) s[mt][r] = 0.f;
#pragma unroll
      for (int st = 0; st < 8; ++st) {
        const tw_bf16x8 kf = *(const tw_bf16x8*)(buf + k_rd[st] + mt * 32 * 256);
        s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf, qf[st], s[mt], 0, 0, 0);
      }
    }
    if (!all) {
      unsigned long long vis;
      if (MODE == MODE_TREE) {
        vis = low_bits(ctx - t0);
        const int j0 = t0 - ctx;                 // draft token of the tile's first position
        if (j0 > -TILE) {
          const uint32_t* mrow = a.mask + (long long)(off + tok) * a.mask_words;
          const int w0 = j0 >= 0 ? j0 >> 5 : 0;
          const uint32_t m0 = w0 < a.mask_words ? mrow[w0] : 0u, m1 = w0 + 1 < a.mask_words ? mrow[w0 + 1] : 0u;
          const unsigned long long w = (unsigned long long)m1 << 32 | m0;
          if (j0 >= 0) {
            const int sh = j0 & 31;
            const uint32_t m2 = w0 + 2 < a.mask_words ? mrow[w0 + 2] : 0u;
            vis |= sh ? w >> sh | (unsigned long long)m2 << (64 - sh) : w;
          } else {
            vis |= w << -j0;
          }
        }
        vis &= low_bits(len - t0);
      } else {
        vis = low_bits(pos + 1 - t0) & (~low_bits(pos - a.window + 1 - t0) | low_bits(a.sinks - t0)) & low_bits(len - t0);
      }
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (!(held >> j & 1u)) vis &= ~(0xFFFFull << (16 * j));
      vis >>= wt * (TILE / WT) + 4 * half;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const uint32_t w = (uint32_t)(vis >> (32 * mt));
#pragma unroll
        for (int r = 0; r < 16; ++r) s[mt][r] = w >> (8 * (r / 4) + r % 4) & 1u ? s[mt][r] : -__builtin_inff();
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
    const float mn = fmaxf(m, mx * kScaleLog2);
    if (__any(mn > m)) {                         // some row's maximum grew
      const float al = __builtin_amdgcn_exp2f(m - mn);
      l *= al;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= al;
      m = mn;
    }
    tw_bf16x8 p[2 * MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][r], kScaleLog2, -m));
        l += w;
        p[2 * mt + r / 8][r % 8] = (__bf16)w;
      }
#pragma unroll
    for (int ks = 0; ks < 2 * MT; ++ks)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        const tw_s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((TW_LDS tw_s16x4*)(buf + v_rd[d] + ks * 4096));
        const tw_s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((TW_LDS tw_s16x4*)(buf + v_rd[d] + ks * 4096 + 2048));
        union { tw_s16x4 s[2]; tw_bf16x8 v; } f;
        f.s[0] = lo; f.s[1] = hi;
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(f.v, p[ks], o[d], 0, 0, 0);
      }
  };

  if (u0 < u1) {
    base = u0;
    refill(u0);
    issue(buf0, u0);
    for (int u = u0; u < u1; u += 2) {
      arrived();                                 // the tile's rows, for every wave; nobody reads the other buffer any more
      unsigned held = held_pages(u);
      if (u + 1 < u1) issue(buf1, u + 1);
      compute(buf0, u, held);
      if (u + 1 >= u1) break;
      arrived();
      held = held_pages(u + 1);
      if (u + 2 < u1) {
        if (u + 2 - base >= 64) { base = u + 2; refill(base); }
        issue(buf0, u + 2);
      }
      compute(buf1, u + 1, held);
    }
  }

  // ---- the waves' states of the same rows merged
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
    const float inv = l > 0.f ? 1.0f / l : 0.f;
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
    if (a.lse && half == 0) a.lse[qrow] = l > 0.f ? (m + __log2f(l)) * kLn2n : -__builtin_inff();
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

// One wave per (sequence, new token, query head) whose list was cut: two half waves of 32 lanes x 4 dims fold every other
// partial result.
template <int M>
__global__ __launch_bounds__(256) void new_tokens_combine_kernel(NewArgs a) {
  const int lane = threadIdx.x & 63, half = lane >> 5, dl = lane & 31;
  const int b = blockIdx.y, idx = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int tok = idx / a.Hq, head = idx - tok * a.Hq;
  if (tok >= seq_new(a, b)) return;
  const int chunks = a.ws_plan[2 * b];
  if (chunks <= 1) return;                       // written by the attention kernel itself
  const int n = seq_new(a, b), blocks = (n * a.G + M - 1) / M, h = head >> a.lgG;
  const int row = tok * a.G + (head & (a.G - 1)), rb = row / M;
  const long long step = (long long)blocks * a.Hkv * M;
  long long at = ((long long)a.ws_plan[2 * b + 1] + rb * a.Hkv + h) * M + row % M + half * step;
  float m = kLow, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int c = half; c < chunks; c += 2, at += 2 * step) {
    const float2 ml = a.ws_ml[at];
    const float4 v = ((const float4*)a.ws_acc)[at * 32 + dl];
    const float mn = fmaxf(m, ml.x), so = __builtin_amdgcn_exp2f(m - mn), sn = __builtin_amdgcn_exp2f(ml.x - mn);
    l = l * so + ml.y * sn;
    o.x = o.x * so + v.x * sn; o.y = o.y * so + v.y * sn; o.z = o.z * so + v.z * sn; o.w = o.w * so + v.w * sn;
    m = mn;
  }
  const float m2 = __shfl_xor(m, 32), l2 = __shfl_xor(l, 32), mn = fmaxf(m, m2);
  const float s0 = __builtin_amdgcn_exp2f(m - mn), s1 = __builtin_amdgcn_exp2f(m2 - mn);
  l = l * s0 + l2 * s1;
  o.x = o.x * s0 + __shfl_xor(o.x, 32) * s1; o.y = o.y * s0 + __shfl_xor(o.y, 32) * s1;
  o.z = o.z * s0 + __shfl_xor(o.z, 32) * s1; o.w = o.w * s0 + __shfl_xor(o.w, 32) * s1;
  const long long qrow = (long long)((a.offsets ? a.offsets[b] : b * a.max_new) + tok) * a.Hq + head;
  const float inv = l > 0.f ? 1.0f / l : 0.f;
  if (half == 0) {
    union { __bf16 e[4]; uint2 v; } w;
    w.e[0] = (__bf16)(o.x * inv); w.e[1] = (__bf16)(o.y * inv); w.e[2] = (__bf16)(o.z * inv); w.e[3] = (__bf16)(o.w * inv);
    a.out[qrow * 32 + dl] = w.v;
    if (a.lse && lane == 0) a.lse[qrow] = l > 0.f ? (mn + __log2f(l)) * kLn2n : -__builtin_inff();
  }
}

// ---------------------------------------------------------------- host side
int rows_per_block(long long rows) { return rows <= 32 ? 32 : rows <= 64 ? 64 : 128; }

// Workgroups that the plan counts on: 64 KiB of LDS each, two to a CU.
int plan_grid() { return 2 * tw_num_cus(); }

// Lists that fill the chip by themselves are not cut: the row blocks of a chunk or prompt under a window.
bool cut_lists(const TwDims& d, bool window, long long max_new, int M) {
  const long long blocks = (max_new * d.G + M - 1) / M;
  return !(window && blocks >= 8 && blocks * d.batch * d.Hkv >= 2ll * tw_num_cus());
}

template <int MODE, int WR, int WT>
int launch_new(NewArgs a, bool cut, long long lists, hipStream_t s) {
  constexpr int M = 32 * WR;
  tw_prof_before(TW_K_NEW_TOKENS, s);
  if (MODE == MODE_WINDOW && !cut) {
    TW_LAUNCH((new_tokens_kernel<MODE_WINDOW, WR, WT, false>), dim3((unsigned)lists), dim3(64 * WR * WT), 0, s, a);
    return tw_prof_after(s);
  }
  a.grid = plan_grid();
  TW_LAUNCH((new_tokens_kernel<MODE, WR, WT, true>), dim3((unsigned)(a.grid * PLAN_ROUNDS + lists)), dim3(64 * WR * WT), 0, s, a);
  if (int e = tw_prof_after(s)) return e;
  tw_prof_before(TW_K_NEW_COMBINE, s);
  TW_LAUNCH((new_tokens_combine_kernel<M>), dim3((unsigned)(((long long)a.max_new * a.Hq + 3) / 4), (unsigned)a.batch), dim3(256), 0, s, a);
  return tw_prof_after(s);
}

size_t align256n(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace

size_t tw_new_tokens_workspace(const TwDims& d, int max_new) {
  if (max_new <= 0 || max_new > TW_MAX_NEW) return 0;
  const int M = rows_per_block((long long)max_new * d.G);
  const size_t slots = (size_t)plan_grid() * 2 * PLAN_ROUNDS;
  return align256n((size_t)d.batch * 8) + align256n(slots * M * 8) + slots * M * 512;
}

static int new_tokens_impl(const twilight_kv_t* kv, const void* q, const int32_t* n_new, const int32_t* new_offsets, int32_t max_new,
                           const uint32_t* mask, int32_t mask_words, int32_t window, int32_t sinks, bool tree,
                           void* out, float* lse, void* ws, size_t ws_bytes, void* stream) {
  TwDims d;
  if (int e = tw_check_kv(kv, &d)) return e;
  if (!q || !out || !kv->k_pool || !kv->v_pool) return TW_EINVAL;
  if (max_new <= 0 || max_new > TW_MAX_NEW || d.max_pages > TW_MAX_ROW_PAGES) return TW_EINVAL;
  if (!ws || ws_bytes < tw_new_tokens_workspace(d, max_new)) return TW_EWORKSPACE;
  const int M = rows_per_block((long long)max_new * d.G);
  NewArgs a;
  a.q = (const uint4*)q; a.k_pool = (const char*)kv->k_pool; a.v_pool = (const char*)kv->v_pool;
  a.page_table = kv->page_table; a.seq_lens = kv->seq_lens; a.n_new = n_new; a.offsets = new_offsets; a.mask = mask;
  a.out = (uint2*)out; a.lse = lse;
  const size_t slots = (size_t)plan_grid() * 2 * PLAN_ROUNDS;
  a.ws_plan = (int32_t*)ws;
  a.ws_ml = (float2*)((char*)ws + align256n((size_t)d.batch * 8));
  a.ws_acc = (float*)((char*)a.ws_ml + align256n(slots * M * 8));
  a.batch = d.batch; a.Hq = d.Hq; a.Hkv = d.Hkv; a.G = d.G; a.lgG = __builtin_ctz(d.G); a.max_pages = d.max_pages;
  a.max_new = max_new; a.mask_words = mask_words; a.window = window; a.sinks = sinks; a.pool_pages = (unsigned)d.pool_pages;
  a.rb_max = (int)(((long long)max_new * d.G + M - 1) / M); a.grid = 0;
  const long long lists = (long long)a.rb_max * d.batch * d.Hkv;
  if (lists > (1ll << 30) || (long long)max_new * d.Hq >= (1ll << 31) || (long long)max_new * d.batch >= (1ll << 31)) return TW_EINVAL;
  const bool cut = cut_lists(d, !tree, max_new, M);
  hipStream_t s = (hipStream_t)stream;
  if (tree) {
    switch (M) {
      case 32: return launch_new<MODE_TREE, 1, 2>(a, cut, lists, s);
      case 64: return launch_new<MODE_TREE, 2, 2>(a, cut, lists, s);
      default: return launch_new<MODE_TREE, 4, 1>(a, cut, lists, s);
    }
  }
  switch (M) {
    case 32: return launch_new<MODE_WINDOW, 1, 2>(a, cut, lists, s);
    case 64: return launch_new<MODE_WINDOW, 2, 2>(a, cut, lists, s);
    default: return launch_new<MODE_WINDOW, 4, 1>(a, cut, lists, s);
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
