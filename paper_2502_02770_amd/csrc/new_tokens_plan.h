// What the kernels that attend a sequence's newest tokens share (bf16 pools, pools in 4 bits): which pages a row block sees, how the
// lists of a launch are cut and which part a workgroup takes, and the launch that joins the parts of cut lists.
//
// `A` is a kernel's argument struct: seq_lens, n_new, offsets, ws_plan, ws_ml, ws_acc, out, lse, batch, Hq, Hkv, G, lgG, max_pages,
// max_new, window, sinks, rb_max, cus, and the constants
//   TILE_PAGES    pages of a tile, the unit in which lists are cut (a power of 2)
//   MIN_TILES     shortest chunk of a list
//   STREAM_TILES  (plan_chunk) tiles of K and V from which on they pass by the last-level cache
//   PAD           (lists shared out evenly) what a piece of a list costs beside its tiles, in tiles
#pragma once
#include <algorithm>
#include "tw_common.h"
#include "new_tokens_span.h"

namespace {

constexpr float kLn2n = 0.6931471805599453f;
constexpr float kScaleLog2 = 0.08838834764831845f * 1.4426950408889634f;   // log2(e) / sqrt(128)
constexpr float kLow = -3.4028234663852886e38f;  // running maximum before any visible token, the lowest number: exp2(-inf - kLow) = 0
constexpr float kFar = 1073741824.f;             // from an |m| of 2^30 on, a row's scores are told apart by their own steps, 64 and more
constexpr int PLAN_ROUNDS = 2;                   // items per resident workgroup at most, as planned
constexpr long long COMBINE_FEW = 512;           // rows of a launch up to which a workgroup joins one row's parts

// the lowest x of 64 bits
__device__ __forceinline__ unsigned long long low_bits(int x) {
  return x <= 0 ? 0ull : x >= 64 ? ~0ull : (1ull << x) - 1ull;
}

template <class A>
__device__ __forceinline__ int seq_len(const A& a, int b) {
  const int n = a.seq_lens[b];
  return max(0, min(n, a.max_pages * TW_PAGE));
}
template <class A>
__device__ __forceinline__ int seq_new(const A& a, int b) {
  return a.n_new ? max(0, min(a.n_new[b], a.max_new)) : a.max_new;
}

// Which part of which list a workgroup takes.  A list is a (row block, KV head) of a sequence; a sequence's lists are cut
// into the same number of chunks.
struct Item {
  int b, n, len, off;                            // the sequence, as Seq
  int rb, h, chunk, chunks, slot;
  uint32_t items;                                // of the launch, where one wave's lanes hold all sequences (no need to look for a next one)
};

// A sequence: its new tokens, length and first row, its lists, and the tiles that its last tokens see.  Under a window another list can have one
// more: who cuts by this count takes a share of the tiles that the list has.  With MOST, no list has more (longest_span).
struct Seq {
  int n, len, off, lists, tiles;
};
template <int MODE, int M, bool MOST = false, class A>
__device__ __forceinline__ Seq seq_of(const A& a, int b) {
  Seq s = {0, 0, 0, 0, 0};
  if (b >= a.batch) return s;
  // (what is not given is read from another list and not used: the loads are on their way together)
  const int len = a.seq_lens[b], n = (a.n_new ? a.n_new : a.seq_lens)[b], off = (a.offsets ? a.offsets : a.seq_lens)[b];
  s.off = a.offsets ? off : b * a.max_new;
  s.n = a.n_new ? max(0, min(n, a.max_new)) : a.max_new;
  s.len = max(0, min(len, a.max_pages * TW_PAGE));
  const int blocks = (s.n * a.G + M - 1) / M;
  s.lists = blocks * a.Hkv;
  const int block = M / a.G;
  const auto sp = MOST ? longest_span(a, s.len, s.n, block) : span_of<MODE>(a, s.len, s.len - min(s.n, block), s.len - 1);
  s.tiles = blocks == 0 ? 0 : max(1, sp.tiles);
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
template <int MODE, int M, class A>
__device__ __forceinline__ int plan_chunk(const A& a, int lane, Seq* seq, bool* stream) {
  constexpr float kJoin = 1.5f, kPart = 2e-4f * M;
  float total = 0.f, lists_all = 0.f, longest = 0.f;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    *seq = seq_of<MODE, M>(a, b0 + lane);
    total += wave_sum_f((float)seq->lists * (float)seq->tiles);
    lists_all += wave_sum_f((float)seq->lists);
    longest = __builtin_fmaxf(longest, tw_wave_max_f((float)seq->tiles));
  }
  const float cus = (float)a.cus, W = 2.f * cus;
  *stream = *stream && total > (float)A::STREAM_TILES;
  total *= 1.001f;
  auto cost_of = [&](float items, float c) { return __builtin_ceilf(items / W - 1e-4f) * (c * (items <= cus ? 0.8f : 1.f) + 2.f); };
  float best = cost_of(lists_all, longest), chunk = longest;
  if (total <= W * A::MIN_TILES) {             // little work: the length where chunk and parts cost the same, short of the shortest none
    // (parts at half their price: they do not fill the memory's time)
    const float c = __builtin_fmaxf((float)A::MIN_TILES, __builtin_floorf(__builtin_amdgcn_sqrtf(0.5f * kPart * total) + 0.5f));
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
      c = __builtin_fmaxf(c, (float)A::MIN_TILES);
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
template <int MODE, int M, class A>
__device__ __forceinline__ bool find_item(const A& a, int lane, int chunk, Seq seq, uint32_t want, Item* it) {
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
template <int M, class A>
__device__ __forceinline__ bool whole_item(const A& a, Item* it) {
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
// `chunks` parts of a row, part c at row at(c) of the workspace, joined by this workgroup's LANES half waves, and the row written where it is live.
template <int LANES, class A, class F>
__device__ __forceinline__ void fold_parts(const A& a, int b, int tok, int head, bool live, int chunks, F at) {
  const int lane = threadIdx.x & 63, dl = lane & 31, part = (threadIdx.x >> 5) % LANES;
  float m = kLow, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  auto join = [&](float m2, float l2, const float4& v) {
    const float mn = fmaxf(m, m2), so = __builtin_amdgcn_exp2f(m - mn), sn = __builtin_amdgcn_exp2f(m2 - mn);
    l = l * so + l2 * sn;
    o.x = o.x * so + v.x * sn; o.y = o.y * so + v.y * sn; o.z = o.z * so + v.z * sn; o.w = o.w * so + v.w * sn;
    m = mn;
  };
#pragma unroll 4
  for (int c = part; c < chunks; c += LANES) {
    const long long r = at(c);
    const float2 ml = a.ws_ml[r];
    join(ml.x, ml.y, ((const float4*)a.ws_acc)[r * 32 + dl]);
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

// The parts of cut lists joined.  A row (new token, head) is folded by LANES half waves of 32 lanes x 4 dims: two (a wave; four
// rows to a workgroup) where there are many rows, eight (a workgroup) where few rows have many parts each and the wait
// for one part after the other is what counts: 256 rows of 32 parts 4.0 us with eight, 8.3 us with two.  Whole calls, two / eight:
//   one sequence of 4096     rows  32: 11.9 / 11.0  256: 14.0 / 13.4   512: 15.7 / 15.4  1024: 16.6 / 16.9  4096: 28.3 / 29.8
//   4 sequences of 8192      rows 512: 30.8 / 31.0 1024: 32.5 / 33.2  2048: 36.6 / 37.2  8192: 60 / 64     16384: 93 / 100
//   16 sequences of 4096     rows 512: 49.2 / 49.5 2048: 49.5 / 50.8  8192: 57.5 / 61   16384: 70 / 77
template <int M, int LANES, class A>
__device__ __forceinline__ void join_parts(const A& a) {
  constexpr int ROWS = 8 / LANES;
  const int b = blockIdx.y, idx = (int)(blockIdx.x * ROWS + threadIdx.x / (32 * LANES));
  const int n = seq_new(a, b);
  const int tok = idx / a.Hq, head = idx - tok * a.Hq;
  const int chunks = a.ws_plan[2 * b];
  if (chunks <= 1) return;                       // written by the attention kernel itself
  const int blocks = (n * a.G + M - 1) / M, row = min(tok, n - 1) * a.G + (head & (a.G - 1));
  const long long step = (long long)blocks * a.Hkv * M;
  const long long at = ((long long)a.ws_plan[2 * b + 1] + (row / M) * a.Hkv + (head >> a.lgG)) * M + row % M;
  fold_parts<LANES>(a, b, tok, head, tok < n, chunks, [=](int c) { return at + c * step; });
}

size_t align256n(size_t x) { return (x + 255) & ~(size_t)255; }

}  // namespace
