// Attention of a sequence's newest tokens over a cache that holds K and V in 4 bits (twilight_kv4_attention).
//
// K^ = c * s + z with one (s, z) per token and group of 32 dims, V^ alike.  The rows of a KV head are its G query heads times the
// N new tokens, as in new_tokens.hip; a workgroup takes M = 16 * RT of them, its four waves walk tiles of 64 tokens (4 pages)
// each on their own, and their states are merged at the end.
//
//   scores   S = sum_g s_g T_g + (z_g - 128 s_g) Q_g over the four groups g, T_g = sum_d q_d (128 + c_d), Q_g = sum_d q_d.  T_g is one
//            v_mfma_f32_16x16x32_bf16 (a group is its contraction): A = 16 tokens' codes, as bf16 128 + c (bits put in place: 8 bits hold
//            them exactly), B = 16 rows of q.  What the zeros and the 128 add is one more, for all groups: z - 128 s and Q_g in three bf16
//            parts each (24 bits), of whose products those that count in fp32 are six, 24 of the 32 terms.  Codes and q are exact, so a
//            score is as good as one of fp32 products (the 128 costs 4 of the 24 bits).
//   weights  P = exp2(S log2(e)/sqrt(128) - m), fp32; their sum is of the unrounded ones.  For the product with V they are fp16, with m
//            kept 11 below the row's maximum's logarithm: the largest is 2^11 to 2^15, and one of 2^-25 of it still has 11 bits.
//   output   O^T += V^T P^T, v_mfma_f32_16x16x32_f16 with V^ = fma(c, s, z) in fp16 (2^-11 of itself at most; c exact: 1024 + c or 64 + c
//            with the bits put in place, less that).
//
// The A operand of the scores takes its 16 tokens as four of each of the tile's four pages (token 4 n + i of page j in row 4 j + i of
// step n), so that the quarter wave j holds all scores of page j's tokens, a row of q in each lane: what the transposed read of V's
// codes (ds_read_b64_tr_b4: a lane gets 16 tokens of one dim) wants its weights to be.  K's codes go to registers, 16 bytes of a
// group to a lane, and are exchanged between the quarters (four permlane swaps; through LDS they cost as much); V's codes go to LDS without
// passing registers, both (s, z) through them, transposed.  The next tile's loads are issued while a tile is computed.
//
// Measured: 8 sequences of 32768, one token, 4 heads a group (M = 16) 75 us for 336 MB, 4.5 TB/s: what is left is issue beside the memory
// (vector 0.55, matrix 0.10 of the time).  64 sequences of 1000 to 32001, 7 tokens, 8 heads a group (two blocks of M = 32) 365 us for 856 MB:
// issue, some 490 vector instructions (0.65 of the time) and 72 matrix ones (0.19) to a tile and wave, half of which make codes and (s, z) into
// operands, and that twice; one block (4 tokens) 240 us, and 139 for every further one.  Operands from LDS asked for a step ahead: 389 -> 385 us
// and spills.  One sequence of 4096 11.2 us: two launches of 8 and 4, whose trips to memory follow each other.
#include "kv4_common.h"
#include "new_tokens_plan.h"

namespace {

typedef _Float16 tw_f16x8 __attribute__((ext_vector_type(8)));
typedef float tw_f32x16 __attribute__((ext_vector_type(16)));
typedef short tw_s16x4 __attribute__((ext_vector_type(4)));
typedef int tw_v2i __attribute__((ext_vector_type(2)));
#define TW_LDS __attribute__((address_space(3)))
#define TW_GLB __attribute__((address_space(1)))

constexpr int WAVES = 4;
// of a wave's LDS: V's codes of 64 tokens, twice; and what is made of their (s, z)
constexpr int BUF = 4096, MADE_Z = 1024, MADE_S = MADE_Z + 2048, MADE = MADE_S + 512;
constexpr float kLift = 11.f;                    // log2 of the weight of a row's maximum when m is set to it
constexpr float kGrowth4 = 4.f;                  // how far (in powers of 2) scores may pass it before m follows: weights stay below 2^16

struct Kv4Args {
  // a tile of the plan: the 16 pages that the four waves take together
  static constexpr int TILE_PAGES = 16, MIN_TILES = 1, PAD = 1;
  const uint4* q;
  const uint4* k_codes;
  const uint4* k_meta;
  const uint4* v_codes;
  const uint4* v_meta;
  const int32_t* page_table;
  const int32_t* seq_lens;
  const int32_t* n_new;        // or NULL: max_new each
  const int32_t* offsets;      // or NULL: b * max_new
  uint2* out;
  float* lse;
  int32_t* ws_plan;
  float2* ws_ml;
  float* ws_acc;
  int batch, Hq, Hkv, G, lgG, max_pages, max_new, window, sinks, rb_max, cus;
  unsigned pool_pages;
};

// How a launch that cuts its lists shares them out: all lists' tiles in one row, sequence by sequence, of which every workgroup takes as
// many as the others - the end of one list, whole ones, the start of another.  A list counts as many tiles as any of its sequence's may have
// (longest_span): what it has not is an empty part, what were not counted would not be read.  Chunks of a length and one after the other to the
// workgroups, as the bf16 kernel has them, left the chip idle for 38 % of the time where 64 sequences of 1000 to 32001 tokens make as
// many lists as there are workgroups.  Of a list that is cut, a workgroup w has a part with its first tile (place 2 w of the workspace) or
// one with its last (2 w + 1).
struct Piece {
  int b, n, len, off, rb, h;                     // the sequence, as Seq; row block and KV head
  int from, to, tiles;                           // of the list's tiles
  int slot;                                      // its place in the workspace, if the list is cut
};
// Where a workgroup has many tiles, a list counts PAD more than it has, for what a piece costs beside its tiles (queries, states merged): 64 ragged
// sequences 399 / 367 / 366 us with 0 / 1 / 2 of 256 tokens; blocks of 128 rows, three sequences' chunks, 168.5 / 168 / 170 with 2 / 3 / 4 of 64.
struct Shares {
  uint32_t each, more, pad, all;                 // tiles of a workgroup (the first `more` have one more), and together
  __device__ __forceinline__ uint32_t begin(uint32_t w) const { return w * each + min(w, more); }
  __device__ __forceinline__ uint32_t owner(uint32_t t) const {
    const uint32_t x = more * (each + 1u);
    return t < x ? quotient(t, each + 1u) : more + quotient(t - x, each);
  }
};
template <int M, class A>
__device__ __forceinline__ Shares shares_of(const A& a, int lane) {
  uint32_t total = 0, lists = 0;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    const Seq q = seq_of<MODE_WINDOW, M, true>(a, b0 + lane);
    total += (uint32_t)__builtin_amdgcn_readlane((int)tw_wave_scan_u32((uint32_t)q.lists * (uint32_t)q.tiles), 63);
    lists += (uint32_t)__builtin_amdgcn_readlane((int)tw_wave_scan_u32((uint32_t)q.lists), 63);
  }
  const uint32_t pad = total / 8u > gridDim.x * (uint32_t)A::MIN_TILES ? A::PAD : 0;
  const uint32_t wgs = max(1u, min(gridDim.x, total / (uint32_t)A::MIN_TILES));
  const uint32_t all = total + pad * lists, each = all / wgs;
  return {each, all - each * wgs, pad, all};
}
// The piece that begins with tile `pos`, the workgroup's first or a later one, of those before `end`; tells the launch that joins the parts where lists begin.
template <int M, class A>
__device__ __forceinline__ void piece_at(const A& a, int lane, uint32_t pad, bool first, uint32_t pos, uint32_t end, bool tell, Piece* it) {
  uint32_t tiles = 0;
  bool found = false;
  for (int b0 = 0; b0 < a.batch; b0 += 64) {
    Seq q = seq_of<MODE_WINDOW, M, true>(a, b0 + lane);
    q.tiles += (int)pad;
    const uint32_t mine = (uint32_t)q.lists * (uint32_t)q.tiles;
    const uint32_t te = tw_wave_scan_u32(mine);
    if (tell && b0 + lane < a.batch) ((int2*)a.ws_plan)[1 + b0 + lane] = make_int2((int)(tiles + te - mine), q.tiles);
    const unsigned long long here = __ballot(tiles + te > pos);
    if (!found && here) {
      const int l = __builtin_ctzll(here);
      it->b = b0 + l;
      it->n = __builtin_amdgcn_readlane(q.n, l);
      it->len = __builtin_amdgcn_readlane(q.len, l);
      it->off = __builtin_amdgcn_readlane(q.off, l);
      it->tiles = __builtin_amdgcn_readlane(q.tiles, l);
      const uint32_t in = pos - (tiles + (uint32_t)__builtin_amdgcn_readlane((int)(te - mine), l)), k = quotient(in, (uint32_t)it->tiles);
      it->from = (int)(in - k * (uint32_t)it->tiles);
      it->to = (int)min((uint32_t)it->tiles, (uint32_t)it->from + (end - pos));
      it->rb = (int)quotient(k, (uint32_t)a.Hkv);
      it->h = (int)(k - (uint32_t)it->rb * (uint32_t)a.Hkv);
      it->slot = 2 * (int)blockIdx.x + (first ? 0 : 1);
      found = true;
      if (!tell) return;
    }
    tiles += (uint32_t)__builtin_amdgcn_readlane((int)te, 63);
  }
}
template <int M, class A>
__device__ __forceinline__ bool whole_piece(const A& a, Piece* it) {
  Item x;
  if (!whole_item<M>(a, &x)) return false;
  it->b = x.b; it->n = x.n; it->len = x.len; it->off = x.off; it->rb = x.rb; it->h = x.h;
  it->from = 0; it->to = it->tiles = 1 << 30;    // all there are
  it->slot = 0;
  return true;
}
// The workgroup's pieces, one after the other.
template <int M, class A, class F>
__device__ __forceinline__ void for_pieces(const A& a, int lane, F attend) {
  const Shares s = shares_of<M>(a, lane);
  if (blockIdx.x == 0 && threadIdx.x == 0) *(int2*)a.ws_plan = make_int2((int)s.each, (int)s.more);
  Piece it;
  uint32_t pos = s.begin(blockIdx.x);
  const uint32_t end = min(s.all, s.begin(blockIdx.x + 1));    // (workgroups that are too many begin behind)
  for (bool first = true; pos < end; first = false) {
    piece_at<M>(a, lane, s.pad, first, pos, end, pos == 0 && threadIdx.x < 64, &it);
    int ln = lane;
    asm volatile("" : "+v"(ln));                 // what depends on the lane alone is worked out for every piece: held over them it would spill
    attend(it, ln);
    pos += (uint32_t)__builtin_amdgcn_readfirstlane(it.to - it.from);
    if (pos < end) __syncthreads();              // the buffers have been read
  }
}
// Rows of lists that were cut: their parts joined.
template <int M, int LANES, class A>
__device__ __forceinline__ void join_shares(const A& a) {
  constexpr int ROWS = 8 / LANES;
  const int b = blockIdx.y, idx = (int)(blockIdx.x * ROWS + threadIdx.x / (32 * LANES));
  const int n = seq_new(a, b), tok = idx / a.Hq, head = idx - tok * a.Hq;
  if (tok >= n) return;
  const Shares s = {(uint32_t)a.ws_plan[0], (uint32_t)a.ws_plan[1], 0u, 0u};
  const int2 p = ((const int2*)a.ws_plan)[1 + b];            // the sequence's first tile, tiles of a list
  const int row = tok * a.G + (head & (a.G - 1));
  const uint32_t k = (uint32_t)((row / M) * a.Hkv + (head >> a.lgG)), t0 = (uint32_t)p.x + k * (uint32_t)p.y;
  const uint32_t first = s.owner(t0), last = s.owner(t0 + (uint32_t)p.y - 1u);
  if (first == last) return;                     // written by the attention kernel itself
  const int late = t0 == s.begin(first) ? 0 : 1;    // the first part is its workgroup's last
  fold_parts<LANES>(a, b, tok, head, true, (int)(last - first + 1u), [=](int c) { return (long long)(2 * ((int)first + c) + (c ? 0 : late)) * M + row % M; });
}

// the lowest x of 16 bits
__device__ __forceinline__ uint32_t low16(int x) { return x <= 0 ? 0u : x >= 16 ? 0xFFFFu : (1u << x) - 1u; }

// x as the sum of three bf16 numbers.
struct Parts { float x, y, z; };
__device__ __forceinline__ Parts parts_of(float v) {
  const float x = (float)(__bf16)v, y = (float)(__bf16)(v - x);
  return {x, y, v - x - y};
}

// The 8 codes of a word times s plus z in fp16; element 2 e + i is nibble e + 4 i.
__device__ __forceinline__ tw_f16x8 codes_f16(uint32_t w, const uint4& s, const uint4& z) {
  union { uint32_t u; tw_f16x2 h; } c[4], sc, ze;
  union { tw_f16x2 h[4]; tw_f16x8 v; } x;
  const uint32_t up = w >> 8;
  c[0].u = tw_and_or(w, 0x000F000Fu, 0x64006400u);                            // 1024 + c
  c[1].u = tw_and_or(w, 0x00F000F0u, 0x54005400u);                            // 64 + c
  c[2].u = tw_and_or(up, 0x000F000Fu, 0x64006400u);
  c[3].u = tw_and_or(up, 0x00F000F0u, 0x54005400u);
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const tw_f16x2 lift = e & 1 ? tw_f16x2{(_Float16)64.f, (_Float16)64.f} : tw_f16x2{(_Float16)1024.f, (_Float16)1024.f};
    sc.u = e == 0 ? s.x : e == 1 ? s.y : e == 2 ? s.z : s.w;
    ze.u = e == 0 ? z.x : e == 1 ? z.y : e == 2 ? z.z : z.w;
    x.h[e] = __builtin_elementwise_fma(c[e].h - lift, sc.h, ze.h);
  }
  return x.v;
}

// One item: a chunk of a list.
template <int RT, bool SPLIT>
__device__ __forceinline__ void attend_item(const Kv4Args& a, const Piece& it, unsigned char (&buf0)[WAVES * BUF], unsigned char (&buf1)[WAVES * BUF],
                                            unsigned char (&made)[WAVES * MADE], int lane, int wave) {
  constexpr int M = 16 * RT;
  static_assert(RT <= 2, "64 rows to a wave are right, but 434 registers spilled: 64 ragged sequences 1274 us for 362");
  const int r16 = lane & 15, jq = lane >> 4;
  const int b = __builtin_amdgcn_readfirstlane(it.b), rb = __builtin_amdgcn_readfirstlane(it.rb), h = __builtin_amdgcn_readfirstlane(it.h);
  const int n = __builtin_amdgcn_readfirstlane(it.n), len = __builtin_amdgcn_readfirstlane(it.len), off = __builtin_amdgcn_readfirstlane(it.off);
  const int ctx = len - n;                       // position of new token 0 (negative: more new tokens than the sequence has)
  const int rows = n * a.G;
  // this lane's rows; those beyond the last repeat it and are not stored
  auto row_of = [&](int rt) { return min(rb * M + rt * 16 + r16, rows - 1); };
  auto qrow_of = [&](int rt) { return (long long)(off + (row_of(rt) >> a.lgG)) * a.Hq + h * a.G + (row_of(rt) & (a.G - 1)); };
  const int p_lo = ctx + ((rb * M) >> a.lgG), p_hi = ctx + ((min(rb * M + M, rows) - 1) >> a.lgG);
  const auto sp = span_of<MODE_WINDOW>(a, len, p_lo, p_hi);
  const int u0 = SPLIT ? min(sp.tiles, __builtin_amdgcn_readfirstlane(it.from)) : 0, u1 = SPLIT ? min(sp.tiles, __builtin_amdgcn_readfirstlane(it.to)) : sp.tiles;
  const bool whole = !SPLIT || it.to - it.from == it.tiles;

  // ---- pages of 16 tiles at a time: lane k holds page k % 4 of the wave's tile base + k / 4
  const int32_t* table = a.page_table + (long long)b * a.max_pages;
  int mine = 0, base = u0;
  unsigned long long mapped = 0;
  auto refill = [&](int u) {
    const int v = 16 * (u + (lane >> 2)) + 4 * wave + (lane & 3);
    const bool in = u + (lane >> 2) < u1 && v < sp.pages;
    const int id = table[min(sp.page(in ? v : 0), a.max_pages - 1)];
    const bool ok = in && (unsigned)id < a.pool_pages;
    mine = ok ? id : 0;                          // (page 0 is read for one that is not there, and not used)
    mapped = __ballot(ok);
  };
  const int tok4 = lane >> 2, piece4 = (lane & 3) ^ (lane >> 4);
  struct Slots { int s[4]; };                    // the first token's place of a tile's pages
  auto slots_of = [&](int u) -> Slots {
    if (u - base >= 16) { base = u; refill(u); }
    const int k = 4 * (u - base);
    Slots x;
#pragma unroll
    for (int p = 0; p < 4; ++p) x.s[p] = (__builtin_amdgcn_readlane(mine, k + p) * a.Hkv + h) * TW_PAGE;
    return x;
  };
  auto one_of = [](const Slots& x, int p) -> int {
    const int s0 = x.s[0], s1 = x.s[1], s2 = x.s[2], s3 = x.s[3], lo = p & 1 ? s1 : s0, hi = p & 1 ? s3 : s2;
    return p & 2 ? hi : lo;
  };
  auto issue_lds = [&](unsigned char* buf, const Slots& x) {
#pragma unroll
    for (int p = 0; p < 4; ++p)
      __builtin_amdgcn_global_load_lds((const TW_GLB unsigned int*)(a.v_codes + ((long long)(x.s[p] + tok4) * 4 + piece4)), (TW_LDS unsigned int*)(buf + 1024 * p), 16, 0, 0);
  };
  uint4 kc[4], km, vm;                           // K's codes and both (s, z) of a tile on its way
  auto issue_regs = [&](const Slots& x) {
    const uint4* kp = a.k_codes + ((long long)(one_of(x, r16 >> 2) + (r16 & 3)) * 4 + jq);
#pragma unroll
    for (int i = 0; i < 4; ++i) kc[i] = kp[16 * i];
    const int tok = one_of(x, jq) + r16;
    km = a.k_meta[tok];
    vm = a.v_meta[tok];
  };

  // Queries, page table and first tile are asked for before anything waits for the queries
  int pos[RT];
  uint4 qr[RT][4];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    pos[rt] = ctx + (row_of(rt) >> a.lgG);
    const uint4* qp = a.q + qrow_of(rt) * 16 + jq;
#pragma unroll
    for (int g = 0; g < 4; ++g) qr[rt][g] = qp[4 * g];
  }
  unsigned char *const mine0 = buf0 + wave * BUF, *const mine1 = buf1 + wave * BUF;
  Slots x = {};
  if (u0 < u1) {
    refill(u0);
    x = slots_of(u0);
    issue_lds(mine0, x);
    issue_regs(x);
  }
  const uint32_t take[3] = {0u - (uint32_t)(jq == 0), 0u - (uint32_t)(jq == 1), 0u - (uint32_t)(jq == 2)};      // (masks: choices would be branches)
  tw_bf16x8 qf[RT][4], qz[RT];                   // qz: Q_g's parts; quarters 0 and 1 the first and second twice, 2 the third and the first, 3 none
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    uint32_t w[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float f[8], sum = 0.f;
      tw_unpack8(qr[rt][g], f);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += f[i];
      qf[rt][g] = tw_q_like_codes(qr[rt][g]);
      const Parts q = parts_of(tw_quarters_sum(sum));
      union { __bf16 e[2]; uint32_t u; } xx, yy, zx;
      xx.e[0] = xx.e[1] = zx.e[1] = (__bf16)q.x; yy.e[0] = yy.e[1] = (__bf16)q.y; zx.e[0] = (__bf16)q.z;
      w[g] = (xx.u & take[0]) | (yy.u & take[1]) | (zx.u & take[2]);
    }
    qz[rt] = tw_as_bf16(make_uint4(w[0], w[1], w[2], w[3]));
  }

  tw_v4f o[RT][8];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int d = 0; d < 8; ++d) o[rt][d] = tw_v4f{0.f, 0.f, 0.f, 0.f};
  float m[RT], l[RT];                            // m: of the whole row; l: of this lane's tokens
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) { m[rt] = kLow; l[rt] = 0.f; }
  // scores beyond 2^30 are told apart by their own steps: there m is kept with a factor of 1/4 instead of log2(e)/sqrt(128), as it
  // is in new_tokens.hip
  auto scale_of = [](float m) -> float { return __builtin_fabsf(m) < kFar ? kScaleLog2 : 0.25f; };
  auto m_log2 = [](float m) -> float { return __builtin_fabsf(m) < kFar ? m : m * kScaleLog2 * 4.f; };

  // What is made of a tile's (s, z), this lane's token r16 of its quarter's page.  V's: s and z of 8 tokens in the order of codes_f16, by
  // (page, group, 8 tokens).  K's: z - 128 s in parts, the first and second of all groups, then the first and third; the scales.
  unsigned char* const vm_lds = made + wave * MADE;
  const unsigned vm_wr = (unsigned)(jq * 256 + (r16 >> 3) * 32 + ((r16 & 3) * 2 + ((r16 >> 2) & 1)) * 2);
  // `here`: this quarter's page is mapped; `more`: tile u + 1, at x, follows, whose registers are asked for as soon as tile u's are free
  auto compute = [&](const unsigned char* buf, int u, bool here, bool more, const Slots& x) {
    const int v = 16 * u + 4 * wave + jq, t0 = sp.page(v) * TW_PAGE;      // this quarter's page
    uint32_t vis[RT], all = 0xFFFFu;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const uint32_t see = low16(pos[rt] + 1 - t0) & (~low16(pos[rt] - a.window + 1 - t0) | low16(a.sinks - t0));
      vis[rt] = here ? see : 0u;
      all &= vis[rt];
    }
    const bool full = __all(all == 0xFFFFu);
    {
      const bool token = here && t0 + r16 < len;             // (what is none: 0, whose weight is 0)
      const uint32_t w[4] = {vm.x, vm.y, vm.z, vm.w}, y[4] = {km.x, km.y, km.z, km.w};
      uint32_t z12[4], z13[4];
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const uint32_t sz = token ? w[g] : 0u;
        *(unsigned short*)(vm_lds + vm_wr + 64 * g) = (unsigned short)sz;
        *(unsigned short*)(vm_lds + vm_wr + 64 * g + 16) = (unsigned short)(sz >> 16);
        const uint32_t k = token ? y[g] : 0u;
        const Parts z = parts_of(__builtin_fmaf(tw_half_lo(k), -128.f, tw_half_hi(k)));
        union { __bf16 e[2]; uint32_t u; } a12, a13;
        a12.e[0] = a13.e[0] = (__bf16)z.x; a12.e[1] = (__bf16)z.y; a13.e[1] = (__bf16)z.z;
        z12[g] = a12.u; z13[g] = a13.u;
      }
      *(uint4*)(vm_lds + MADE_Z + lane * 32) = make_uint4(z12[0], z12[1], z12[2], z12[3]);
      *(uint4*)(vm_lds + MADE_Z + lane * 32 + 16) = make_uint4(z13[0], z13[1], z13[2], z13[3]);
      *(uint2*)(vm_lds + MADE_S + lane * 8) = make_uint2(__builtin_amdgcn_perm(y[1], y[0], 0x05040100u), __builtin_amdgcn_perm(y[3], y[2], 0x05040100u));
    }
    tw_v4f s[RT][4];
#pragma unroll
    for (int st = 0; st < 4; ++st) {
      __builtin_amdgcn_sched_barrier(0);         // (the compiler would gather all steps' operands, and spill)
      tw_transpose_quarters(kc[st]);
      const tw_bf16x8 kf[4] = {tw_codes_bf16(kc[st].x), tw_codes_bf16(kc[st].y), tw_codes_bf16(kc[st].z), tw_codes_bf16(kc[st].w)};
      const tw_bf16x8 zf = *(const tw_bf16x8*)(vm_lds + MADE_Z + ((r16 >> 2) * 16 + 4 * st + (r16 & 3)) * 32 + (jq == 2 ? 16 : 0));
      uint2 sc[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) sc[i] = *(const uint2*)(vm_lds + MADE_S + (jq * 16 + 4 * st + i) * 8);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        tw_v4f t[4], y = {0.f, 0.f, 0.f, 0.f};
        y = __builtin_amdgcn_mfma_f32_16x16x32_bf16(zf, qz[rt], y, 0, 0, 0);
#pragma unroll
        for (int g = 0; g < 4; ++g) t[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[g], qf[rt][g], tw_v4f{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t w = g & 2 ? sc[i].y : sc[i].x;
            y[i] = __builtin_fmaf(g & 1 ? tw_half_hi(w) : tw_half_lo(w), t[g][i], y[i]);
          }
        s[rt][st] = y;
        asm volatile("" : "+v"(s[rt][st]));      // here and now: sunk behind the branch below, all steps' products would wait in registers
      }
    }
    if (more) issue_regs(x);
    tw_f16x8 p[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      __builtin_amdgcn_sched_barrier(0);
      if (!full) {
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[rt][st][i] = vis[rt] >> (4 * st + i) & 1u ? s[rt][st][i] : -__builtin_inff();
      }
      float mx = s[rt][0][0];
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx = fmaxf(mx, s[rt][st][i]);
      mx = tw_quarters_max(mx);
      float c = scale_of(m[rt]);
      if (__any(mx * c > m[rt] + (kLift + kGrowth4))) {
        const float was = m_log2(m[rt]), mn = fmaxf(was, mx * kScaleLog2 - kLift), al = __builtin_amdgcn_exp2f(was - mn);
        l[rt] *= al;
#pragma unroll
        for (int d = 0; d < 8; ++d)
#pragma unroll
          for (int i = 0; i < 4; ++i) o[rt][d][i] *= al;
        if (mn > was) m[rt] = __builtin_fabsf(mn) < kFar ? mn : mx * 0.25f;
        c = scale_of(m[rt]);
      }
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[rt][st][i], c, -m[rt]));
          l[rt] += w;
          p[rt][st >> 1][2 * i + (st & 1)] = (_Float16)w;
        }
      asm volatile("" : "+v"(p[rt][0]), "+v"(p[rt][1]));
    }
    // (the second half's products come a group later, so that none follows the one whose sum it adds to)
    tw_f16x8 late[2];
    auto second = [&](int g) {
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[rt][2 * g + k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(late[k], p[rt][1], o[rt][2 * g + k], 0, 0, 0);
    };
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      __builtin_amdgcn_sched_barrier(0);
      if (g) second(g - 1);
      uint4 sc[2], ze[2];
#pragma unroll
      for (int kk = 0; kk < 2; ++kk) {
        sc[kk] = *(const uint4*)(vm_lds + jq * 256 + g * 64 + kk * 32);
        ze[kk] = *(const uint4*)(vm_lds + jq * 256 + g * 64 + kk * 32 + 16);
      }
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const tw_v2i w = __builtin_amdgcn_ds_read_tr4_b64_v2i32((TW_LDS tw_v2i*)(buf + jq * 1024 + r16 * 64 + ((g ^ (r16 >> 2)) << 4) + k * 8));
        const tw_f16x8 now = codes_f16((uint32_t)w.x, sc[0], ze[0]);
        late[k] = codes_f16((uint32_t)w.y, sc[1], ze[1]);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) o[rt][2 * g + k] = __builtin_amdgcn_mfma_f32_16x16x32_f16(now, p[rt][0], o[rt][2 * g + k], 0, 0, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    second(3);
  };
  auto arrived = [&]() {
    __builtin_amdgcn_s_waitcnt(0x0070);          // vmcnt(0), lgkmcnt(0): the tile is here, and the other buffer has been read
    asm volatile("" ::: "memory");
  };

  if (u0 < u1) {
    for (int u = u0; u < u1; u += 2) {           // (a wave's buffers are its own: nothing to wait for but its own loads)
      // the older of two workgroups on a CU would be served first, and leave the other alone at the end: they take turns
      if ((blockIdx.x >= gridDim.x / 2) == ((u - u0) % 4 < 2)) __builtin_amdgcn_s_setprio(1);
      else __builtin_amdgcn_s_setprio(0);
      arrived();
      bool here = mapped >> (4 * (u - base) + jq) & 1, more = u + 1 < u1;
      if (more) { x = slots_of(u + 1); issue_lds(mine1, x); }
      compute(mine0, u, here, more, x);
      if (!more) break;
      arrived();
      here = mapped >> (4 * (u + 1 - base) + jq) & 1;
      more = u + 2 < u1;
      if (more) { x = slots_of(u + 2); issue_lds(mine0, x); }
      compute(mine1, u + 1, here, more, x);
    }
  }

  // ---- the waves' states merged, a row tile at a time: every wave takes two of the eight blocks of 16 dims
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float mw = m_log2(m[rt]), lw = tw_quarters_sum(l[rt]);
    __syncthreads();                             // tiles, or the row tile before, have been read
    float* part = (float*)((wave & 2 ? buf1 : buf0) + (wave & 1) * 8192);
    static_assert(WAVES * BUF >= 2 * 8192, "two waves' parts to a buffer");
#pragma unroll
    for (int d = 0; d < 8; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) part[(d * 4 + i) * 64 + lane] = o[rt][d][i];
    if (jq == 0) ((float2*)made)[wave * 16 + r16] = make_float2(mw, lw);
    __syncthreads();
    float2 ml[WAVES];
    float mn = kLow, ls = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) { ml[w] = ((const float2*)made)[w * 16 + r16]; mn = fmaxf(mn, ml[w].x); }
    float al[WAVES], sum[2][4];
#pragma unroll
    for (int w = 0; w < WAVES; ++w) { al[w] = __builtin_amdgcn_exp2f(ml[w].x - mn); ls += ml[w].y * al[w]; }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        sum[k][i] = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) sum[k][i] += ((const float*)((w & 2 ? buf1 : buf0) + (w & 1) * 8192))[((2 * wave + k) * 4 + i) * 64 + lane] * al[w];
      }
    if (rb * M + rt * 16 + r16 >= rows) continue;
    // element i of block d: dim 16 d + 8 (jq / 2) + 2 (jq % 2) + {0, 4, 1, 5}[i]
    const int at = 16 * wave + 4 * (jq >> 1) + (jq & 1);                      // in pairs of dims
    if (whole) {
      const float inv = ls == 0.f ? 0.f : 1.0f / ls;
      const long long qrow = qrow_of(rt);
      uint32_t* orow = (uint32_t*)a.out + qrow * 64;
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          union { __bf16 e[2]; uint32_t u; } w;
          w.e[0] = (__bf16)(sum[k][i] * inv); w.e[1] = (__bf16)(sum[k][i + 2] * inv);
          orow[at + 8 * k + 2 * i] = w.u;
        }
      if (a.lse && jq == 0 && wave == 0) a.lse[qrow] = row_lse(mn, ls);
    } else {
      const long long prow = (long long)it.slot * M + rt * 16 + r16;
      float2* acc = (float2*)(a.ws_acc + prow * 128);
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i) acc[at + 8 * k + 2 * i] = make_float2(sum[k][i], sum[k][i + 2]);
      if (jq == 0 && wave == 0) a.ws_ml[prow] = make_float2(mn, ls);
    }
  }
}

// SPLIT: resident workgroups share the lists; otherwise a workgroup per list.
template <int RT, bool SPLIT>
__global__ __launch_bounds__(256, 2) void kv4_attention_kernel(Kv4Args a) {
  constexpr int M = 16 * RT;
  __shared__ __align__(1024) unsigned char buf0[WAVES * BUF];
  __shared__ __align__(1024) unsigned char buf1[WAVES * BUF];
  __shared__ __align__(1024) unsigned char made[WAVES * MADE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  if (!SPLIT) {
    Piece it;
    if (whole_piece<M>(a, &it)) attend_item<RT, SPLIT>(a, it, buf0, buf1, made, lane, wave);
    return;
  }
  for_pieces<M>(a, lane, [&](const Piece& it, int ln) { attend_item<RT, SPLIT>(a, it, buf0, buf1, made, ln, wave); });
}

// ------------------------------------------------------------------------------------------------------ many rows
// More than 256 rows: a workgroup takes 128 of them, 32 to a wave, and its waves share a tile of 64 tokens in LDS: each turns one page's
// codes into operands, K's to bf16 numbers 0 .. 15, V's to fp16 values, between the products of the tile before (rows of operands and
// their reads as in new_tokens.hip).  The scores' group products T_g = sum_d q_d c_d are two v_mfma_f32_32x32x16_bf16 each, scaled and
// summed by one fma per score and group; what the zeros add, sum_g z_g Q_g, is two more products for all groups: z (11 bits) in two
// bf16 parts, Q_g in three.
//
// Measured: 257 tokens of three sequences of 9001 under a window of 6001, 4 heads a group (1028 rows) 168 us, 0.45 PFLOP/s of the attention's
// own products: vector issue 0.46 of the time (an exponential, a maximum and five fmas to a score), matrix 0.23, waits at the barrier of a tile.
struct Kv4WideArgs : Kv4Args {
  static constexpr int TILE_PAGES = 4, MIN_TILES = 2, PAD = 3;
};
constexpr int WIDE_M = 128, WIDE_V = 64 * 256, WIDE_Z = 2 * WIDE_V, WIDE_S = WIDE_Z + 64 * 16, WIDE_BUF = WIDE_S + 64 * 8;

template <bool SPLIT>
__device__ __forceinline__ void attend_wide(const Kv4WideArgs& a, const Piece& it, unsigned char (&buf0)[WIDE_BUF], unsigned char (&buf1)[WIDE_BUF],
                                            int lane, int wave) {
  constexpr int M = WIDE_M, MT = 2;
  const int half = lane >> 5;
  const int b = __builtin_amdgcn_readfirstlane(it.b), rb = __builtin_amdgcn_readfirstlane(it.rb), h = __builtin_amdgcn_readfirstlane(it.h);
  const int n = __builtin_amdgcn_readfirstlane(it.n), len = __builtin_amdgcn_readfirstlane(it.len), off = __builtin_amdgcn_readfirstlane(it.off);
  const int ctx = len - n, rows = n * a.G, row = rb * M + wave * 32 + (lane & 31);
  const bool live = row < rows;
  const int tok = min(row, rows - 1) >> a.lgG, pos = ctx + tok;
  const long long qrow = (long long)(off + tok) * a.Hq + h * a.G + (min(row, rows - 1) & (a.G - 1));
  const int p_lo = ctx + ((rb * M) >> a.lgG), p_hi = ctx + ((min(rb * M + M, rows) - 1) >> a.lgG);
  const int w_lo = ctx + (min(rb * M + wave * 32, rows - 1) >> a.lgG), w_hi = ctx + (min(rb * M + wave * 32 + 31, rows - 1) >> a.lgG);
  const auto sp = span_of<MODE_WINDOW>(a, len, p_lo, p_hi);
  const int u0 = SPLIT ? min(sp.tiles, __builtin_amdgcn_readfirstlane(it.from)) : 0, u1 = SPLIT ? min(sp.tiles, __builtin_amdgcn_readfirstlane(it.to)) : sp.tiles;
  const bool whole = !SPLIT || it.to - it.from == it.tiles;

  tw_bf16x8 qf[8], qz[2];                        // qz: Q_g in parts, each for both parts of z; the third for the lower half's slots alone
#pragma unroll
  for (int k = 0; k < 8; ++k) qf[k] = tw_as_bf16(a.q[qrow * 16 + 2 * k + half]);
  auto sums_of_q = [&]() {
    float part[2][4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      float sum = 0.f;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        union { tw_bf16x8 v; uint4 u; } x;
        x.v = qf[2 * g + k];
        float f[8];
        tw_unpack8(x.u, f);
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += f[i];
      }
      const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(sum), __float_as_uint(sum), false, false);
      sum = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
      const float first = (float)(__bf16)sum, second = (float)(__bf16)(sum - first);
      part[0][g] = half ? second : first;
      part[1][g] = half ? 0.f : sum - first - second;
    }
#pragma unroll
    for (int k = 0; k < 2; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) qz[k][i] = (__bf16)part[k][i / 2];
  };

  // ---- LDS.  Rows of 16 pieces of 16 bytes, stored in an order that depends on the row, as in new_tokens.hip: K's piece ^ row % 16, V's
  // piece ^ (4 (row % 4) + 2 (row / 4 % 2)).  This lane stages token lane / 4 of its wave's page, group lane % 4.
  const int st = lane >> 2, sg = lane & 3, v_order = ((st & 3) << 2) | ((st >> 2 & 1) << 1);
  // of piece 2 s + half of K's row (32 s changes the bits of the piece), of the 4 tokens and 16 dims that 16 lanes take of V's (64 d)
  const unsigned k_at = (unsigned)((lane & 31) * 256 + ((half ^ (lane & 15)) << 4));
  const unsigned v_at = (unsigned)(WIDE_V + (4 * half + ((lane & 15) >> 2)) * 256 +
                                   (((2 * (lane >> 4 & 1) + ((lane & 3) >> 1)) ^ ((lane & 15) >> 2 << 2) ^ (half << 1)) << 4) + (lane & 1) * 8);

  // ---- page ids of 64 tiles at a time: lane k holds those of tile base + k
  const int32_t* table = a.page_table + (long long)b * a.max_pages;
  int mine = 0, base = u0;
  unsigned long long mapped[4];                  // per page of a tile: the tiles (bits) where it is mapped
  auto refill = [&](int u) {
    const int v0 = 4 * min(u + lane, u1 - 1);
    int id[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) id[j] = table[min(sp.page(v0 + j), a.max_pages - 1)];
#pragma unroll
    for (int j = 0; j < 4; ++j) mapped[j] = __ballot(v0 + j < sp.pages && (unsigned)id[j] < a.pool_pages);
    const int x = wave & 2 ? (wave & 1 ? id[3] : id[2]) : (wave & 1 ? id[1] : id[0]);
    mine = (unsigned)x < a.pool_pages ? x : 0;   // (page 0 is read for one that is not there, and not used)
  };
  auto held_pages = [&](int u) -> unsigned {
    const int k = u - base;
    return (unsigned)(mapped[0] >> k & 1) | (unsigned)(mapped[1] >> k & 1) << 1 | (unsigned)(mapped[2] >> k & 1) << 2 | (unsigned)(mapped[3] >> k & 1) << 3;
  };
  struct Codes { uint4 k, v; uint32_t km, vm; };
  auto fetch = [&](Codes& x, int u) {
    const int tk = (__builtin_amdgcn_readlane(mine, u - base) * a.Hkv + h) * TW_PAGE + st;
    x.k = a.k_codes[(long long)tk * 4 + sg];
    x.v = a.v_codes[(long long)tk * 4 + sg];
    x.km = ((const uint32_t*)a.k_meta)[(long long)tk * 4 + sg];
    x.vm = ((const uint32_t*)a.v_meta)[(long long)tk * 4 + sg];
  };
  // this lane's part of a tile's operands: (scale, zero) first, then four words of K's and V's codes
  const int stt = wave * TW_PAGE + st;           // of the tile
  struct Staged { tw_f16x2 s, z; };
  auto stage_meta = [&](unsigned char* buf, Codes& x, int u, unsigned held) -> Staged {
    const bool token = (held >> wave & 1u) && sp.page(4 * u + wave) * TW_PAGE + st < len;
    const uint32_t km = token ? x.km : 0u, vm = token ? x.vm : 0u;            // what is no token: 0, whose weight is 0
    const float z = tw_half_hi(km), z1 = (float)(__bf16)z;
    union { __bf16 e[2]; uint32_t u; } zz;
    zz.e[0] = (__bf16)z1; zz.e[1] = (__bf16)(z - z1);
    *(uint32_t*)(buf + WIDE_Z + stt * 16 + sg * 4) = zz.u;
    // scales by (group, 32 tokens, half wave): the 16 tokens of a lane's scores together
    const int t32 = stt & 31;
    *(unsigned short*)(buf + WIDE_S + ((sg * 2 + (stt >> 5)) * 2 + (t32 >> 2 & 1)) * 32 + (4 * (t32 >> 3) + (t32 & 3)) * 2) = (unsigned short)km;
    union { uint32_t u; tw_f16x2 h; } s2, z2;
    s2.u = __builtin_amdgcn_perm(vm, vm, 0x05040504u);
    z2.u = __builtin_amdgcn_perm(vm, vm, 0x07060706u);
    return {s2.h, z2.h};
  };
  auto stage_word = [&](unsigned char* buf, uint32_t kw, uint32_t vw, int i, const Staged& sz) {
    const uint32_t kn[2] = {kw & 0x0F0F0F0Fu, kw >> 4 & 0x0F0F0F0Fu}, vn[2] = {vw & 0x0F0F0F0Fu, vw >> 4 & 0x0F0F0F0Fu};
    uint32_t ko[4], vo[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t w = kn[j >> 1] >> (16 * (j & 1));
      ko[j] = __builtin_amdgcn_perm(__float_as_uint((float)(w >> 8 & 0xFFu)), __float_as_uint((float)(w & 0xFFu)), 0x07060302u);
      union { uint32_t u; tw_f16x2 h; } c, o;
      c.u = __builtin_amdgcn_perm(0x64646464u, vn[j >> 1], j & 1 ? 0x04030402u : 0x04010400u);        // 1024 + c
      o.h = __builtin_elementwise_fma(c.h - tw_f16x2{(_Float16)1024.f, (_Float16)1024.f}, sz.s, sz.z);
      vo[j] = o.u;
    }
    *(uint4*)(buf + stt * 256 + (((4 * sg + i) ^ st) << 4)) = make_uint4(ko[0], ko[1], ko[2], ko[3]);
    *(uint4*)(buf + WIDE_V + stt * 256 + (((4 * sg + i) ^ v_order) << 4)) = make_uint4(vo[0], vo[1], vo[2], vo[3]);
  };

  tw_f32x16 o[4];
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  float m = kLow, l = 0.f;
  auto scale_of = [](float m) -> float { return __builtin_fabsf(m) < kFar ? kScaleLog2 : 0.25f; };
  auto m_log2 = [&]() -> float { return __builtin_fabsf(m) < kFar ? m : m * kScaleLog2 * 4.f; };

  // The scores of tile u, and between their products the next tile's operands made (of whatever the registers hold where there is none)
  tw_f32x16 s[MT];
  auto scores = [&](const unsigned char* buf, unsigned char* then, Codes& x, int u, unsigned next) {
    unsigned k_rd = k_at;
    asm volatile("" : "+v"(k_rd));               // (the addresses made of it are worked out here: held, they would spill)
    const Staged sz = stage_meta(then, x, u + 1, next);
    const uint32_t kw[4] = {x.k.x, x.k.y, x.k.z, x.k.w}, vw[4] = {x.v.x, x.v.y, x.v.z, x.v.w};
#pragma unroll
    for (int mt = 0; mt < MT; ++mt) {
      const tw_bf16x8 z = *(const tw_bf16x8*)(buf + WIDE_Z + (mt * 32 + (lane & 31)) * 16);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[mt][r] = 0.f;
      s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(z, qz[0], s[mt], 0, 0, 0);
      s[mt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(z, qz[1], s[mt], 0, 0, 0);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        tw_f32x16 t;
#pragma unroll
        for (int r = 0; r < 16; ++r) t[r] = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k)
          t = __builtin_amdgcn_mfma_f32_32x32x16_bf16(*(const tw_bf16x8*)(buf + (k_rd ^ (unsigned)(32 * (2 * g + k))) + mt * 32 * 256), qf[2 * g + k], t, 0, 0, 0);
        if (g % 2 == 1) {
          const int i = 2 * mt + g / 2;
          stage_word(then, kw[i], vw[i], i, sz);
        }
        const unsigned char* sc = buf + WIDE_S + ((g * 2 + mt) * 2 + half) * 32;
        const uint4 x = *(const uint4*)sc, y = *(const uint4*)(sc + 16);
        const uint32_t w[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
        for (int r = 0; r < 16; ++r) s[mt][r] = __builtin_fmaf(r & 1 ? tw_half_hi(w[r / 2]) : tw_half_lo(w[r / 2]), t[r], s[mt][r]);
        asm volatile("" : "+v"(s[mt]));          // here and now: sunk behind the branches to come, all groups' products would wait in registers
      }
    }
  };
  auto weights = [&](const unsigned char* buf, int u, unsigned held) {
    bool all = held == 15u;                      // does every row see all of the tile
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int t = sp.page(4 * u + j) * TW_PAGE;
      all = all & (t + TW_PAGE - 1 <= w_lo) & ((t > w_hi - a.window) | (t + TW_PAGE <= a.sinks));
    }
    unsigned v_rd = v_at;
    asm volatile("" : "+v"(v_rd));
    if (!all) {
      unsigned long long vis = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int t = sp.page(4 * u + j) * TW_PAGE;
        const uint32_t see = low16(pos + 1 - t) & (~low16(pos - a.window + 1 - t) | low16(a.sinks - t));
        if (held >> j & 1u) vis |= (unsigned long long)see << (16 * j);
      }
      vis >>= 4 * half;
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const uint32_t w = (uint32_t)(vis >> (32 * mt));
#pragma unroll
        for (int r = 0; r < 16; ++r) {           // the row's bit, spread over a word, chooses the score or -inf
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
    if (__any(mx * c > m + (kLift + kGrowth4))) {
      const float was = m_log2(), mn = fmaxf(was, mx * kScaleLog2 - kLift), al = __builtin_amdgcn_exp2f(was - mn);
      l *= al;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= al;
      if (mn > was) m = __builtin_fabsf(mn) < kFar ? mn : mx * 0.25f;
      c = scale_of(m);
    }
    tw_f16x8 p[2 * MT];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float w = __builtin_amdgcn_exp2f(__builtin_fmaf(s[mt][r], c, -m));
        l += w;
        p[2 * mt + r / 8][r % 8] = (_Float16)w;
      }
    union Frag { tw_s16x4 s[2]; tw_f16x8 v; };
#pragma unroll
    for (int ks = 0; ks < 2 * MT; ++ks)
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        Frag f;
        f.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((TW_LDS tw_s16x4*)(buf + (v_rd ^ (unsigned)(64 * d)) + ks * 4096));
        f.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((TW_LDS tw_s16x4*)(buf + (v_rd ^ (unsigned)(64 * d)) + ks * 4096 + 2048));
        o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(f.v, p[ks], o[d], 0, 0, 0);
      }
  };

  if (u0 < u1) {
    // tile u is in its buffer, the codes of tiles u + 1 (asked for two turns ago) and u + 2 on their way to registers; pages[]: which of
    // their pages are there
    Codes ahead[2];
    unsigned pages[2] = {0u, 0u};
    auto ask = [&](int k, int u) {               // (`base` moves on only past tiles that have been asked for)
      if (u >= u1) return;
      if (u - base >= 64) { base = u; refill(u); }
      fetch(ahead[k], u);
      pages[k] = held_pages(u);
    };
    refill(u0);
    ask(0, u0);
    ahead[1] = Codes{};                          // (what follows a last tile is made of something: of the tile's own codes, this would wait for them)
    ask(1, u0 + 1);
    sums_of_q();
    unsigned held = pages[0];
    {
      const Staged sz = stage_meta(buf0, ahead[0], u0, held);
      const uint32_t kw[4] = {ahead[0].k.x, ahead[0].k.y, ahead[0].k.z, ahead[0].k.w}, vw[4] = {ahead[0].v.x, ahead[0].v.y, ahead[0].v.z, ahead[0].v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) stage_word(buf0, kw[i], vw[i], i, sz);
    }
    ask(0, u0 + 2);
    auto turn = [&](const unsigned char* now, unsigned char* then, int k, int u) {
      __syncthreads();                           // the tile is there for every wave, and nobody reads the other buffer any more
      scores(now, then, ahead[k], u, pages[k]);
      const unsigned here = held;
      held = pages[k];
      ask(k, u + 3);
      weights(now, u, here);
    };
    for (int u = u0; u < u1; u += 2) {
      turn(buf0, buf1, 1, u);
      if (u + 1 >= u1) break;
      turn(buf1, buf0, 0, u + 1);
    }
  }

  // ---- the row's sum, and the row
  m = m_log2();
  {
    const auto sw = __builtin_amdgcn_permlane32_swap(__float_as_uint(l), __float_as_uint(l), false, false);
    l = __uint_as_float(sw[0]) + __uint_as_float(sw[1]);
  }
  if (!live) return;
  if (whole) {
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
  const long long prow = (long long)it.slot * M + wave * 32 + (lane & 31);
  float4* acc = (float4*)(a.ws_acc + prow * 128);
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int k = 0; k < 4; ++k) acc[8 * d + 2 * k + half] = make_float4(o[d][4 * k], o[d][4 * k + 1], o[d][4 * k + 2], o[d][4 * k + 3]);
  if (half == 0) a.ws_ml[prow] = make_float2(m, l);
}

template <bool SPLIT>
__global__ __launch_bounds__(256, 2) void kv4_wide_kernel(Kv4WideArgs a) {
  constexpr int M = WIDE_M;
  __shared__ __align__(1024) unsigned char buf0[WIDE_BUF];
  __shared__ __align__(1024) unsigned char buf1[WIDE_BUF];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  if (!SPLIT) {
    Piece it;
    if (whole_piece<M>(a, &it)) attend_wide<SPLIT>(a, it, buf0, buf1, lane, wave);
    return;
  }
  for_pieces<M>(a, lane, [&](const Piece& it, int ln) { attend_wide<SPLIT>(a, it, buf0, buf1, ln, wave); });
}

template <int M, int LANES>
__global__ __launch_bounds__(256) void kv4_combine_kernel(Kv4Args a) { join_shares<M, LANES>(a); }

// ---------------------------------------------------------------- host side
// Rows to a workgroup.  us with blocks of 32 / 64 (as 128, two waves to 32 rows) / 128 rows, of a KV head's rows (these and the next figures are of
// before page table and first tile were asked for ahead of the queries: the cases at the head of the file are 2 to 6 % faster since):
//   8 sequences of 8192, 8 heads a group   24: 37 / 57 / 72    64: 51 / 61 / 74    128: 92 / 105 / 81   256: 135 / 185 / 140   1024: 501 / 554 / 413
//   one of 4096, 4 heads a group           24: 15.2 / 16.2 / 15.8                  128: 21.4 / 23.8 / 22.1                      512: 32.7 / 39.0 / 35.5
//   16 of 2048, 4 heads a group            24: 28 / 36 / 42    64: 35 / 40 / 46    128: 42 / 62 / 52    256: 78 / 82 / 81       512: 147 / 152 / 113
int rows_per_block4(long long rows) { return rows <= 16 ? 16 : rows <= 256 ? 32 : WIDE_M; }

// Lists that cannot be long are not cut, which saves the launch that joins the parts: up to 512 tokens, 256 more for every 24 lists; at
// most 2048, or 4096 where two lists come to a place of the chip, as ragged lengths would leave it idle with more.  Nor are the row blocks of
// prompts that fill the chip by themselves, but where single tokens may stand beside a chunk (as in new_tokens.hip).  us, whole / cut, 8 heads:
//   one new token each     1 sequence of 512: 8.9 / 12.3   1024: 12.4 / 12.0   2048: 20.5 / 12.0     8 of 1024: 12.5 / 13.3   2048: 22.9 / 15.8
//                          32 of 2048: 24.5 / 26.4         4096: 47.1 / 43.9
//   6, 4 heads a group     1 of 512: 11.4 / 14.7           1024: 16.7 / 15.2                         32 of 2048: 31.9 / 36.6  4096: 59.0 / 60.9
//   128, 4 heads a group   1 of 256: 15.3 / 17.9           512: 24.4 / 20.3    8 of 2048: 81.4 / 81.8   4096: 153 / 144       32 of 4096: 424 / 484
template <class A>
bool cut_lists4(bool counted, int blocks, long long lists, long long longest) {
  constexpr long long UNIT = 16 / A::TILE_PAGES;             // tiles of 256 tokens
  const long long places = 2ll * tw_num_cus();
  if (longest <= UNIT * std::min(lists >= 2 * places ? 16ll : 8ll, 2 + lists / 24)) return false;
  if (blocks < 8 || lists < places) return true;
  return counted && longest * places > 48 * UNIT * lists;
}

template <int M, class A, class Whole, class Cut>
int launch_kv4(const A& a, Whole whole, Cut cut, hipStream_t s) {
  const long long lists = (long long)a.rb_max * a.batch * a.Hkv, rows = (long long)a.max_new * a.Hq;
  const long long longest = std::min((a.max_pages + A::TILE_PAGES - 1) / A::TILE_PAGES, window_tiles(a, M / a.G));      // tiles that a list can have
  tw_prof_before(TW_K_KV4_ATTENTION, s);
  if (!cut_lists4<A>(a.n_new != nullptr, a.rb_max, lists, longest) || rows >= (1ll << 26) || lists * (longest + A::PAD) >= (1ll << 32)) {
    TW_LAUNCH(whole, dim3((unsigned)lists), dim3(256), 0, s, a);
    return tw_prof_after(s);
  }
  const long long most = lists * ((longest + A::MIN_TILES - 1) / A::MIN_TILES);
  TW_LAUNCH(cut, dim3((unsigned)std::min(most, 2ll * a.cus)), dim3(256), 0, s, a);
  if (int e = tw_prof_after(s)) return e;
  tw_prof_before(TW_K_KV4_COMBINE, s);
  if (rows * a.batch <= COMBINE_FEW) TW_LAUNCH((kv4_combine_kernel<M, 8>), dim3((unsigned)rows, (unsigned)a.batch), dim3(256), 0, s, a);
  else TW_LAUNCH((kv4_combine_kernel<M, 2>), dim3((unsigned)((rows + 3) / 4), (unsigned)a.batch), dim3(256), 0, s, a);
  return tw_prof_after(s);
}

// Places for parts: two of every workgroup that can have tiles.
size_t part_slots4(const TwDims& d, long long rows) {
  const int M = rows_per_block4(rows), chunk = M <= 32 ? Kv4Args::TILE_PAGES * Kv4Args::MIN_TILES : Kv4WideArgs::TILE_PAGES * Kv4WideArgs::MIN_TILES;
  const long long lists = (rows + M - 1) / M * d.batch * d.Hkv, places = 2ll * tw_num_cus();
  return (size_t)(2 * std::min(places, lists * ((d.max_pages + chunk - 1) / chunk)));
}

}  // namespace

size_t tw_kv4_workspace(const TwDims& d, int max_new) {
  if (max_new <= 0 || max_new > TW_MAX_NEW) return 0;
  const long long rows = (long long)max_new * d.G;
  const int M = rows_per_block4(rows);
  const size_t slots = part_slots4(d, rows);
  return align256n((size_t)(d.batch + 1) * 8) + align256n(slots * M * 8) + slots * M * 512;
}

extern "C" int twilight_kv4_attention(const twilight_kv_t* kv, const void* vq_pool, const void* vq_meta, const void* q, const int32_t* n_new,
                                      const int32_t* new_offsets, int32_t max_new, int32_t window, int32_t num_sinks, void* out, float* lse,
                                      void* ws, size_t ws_bytes, void* stream) {
  TwDims d;
  if (int e = tw_check_kv(kv, &d)) return e;
  if (!q || !out || !kv->kq_pool || !kv->kq_meta || !vq_pool || !vq_meta || d.bits != 4) return TW_EINVAL;
  if (window < 1 || num_sinks < 0 || max_new <= 0 || max_new > TW_MAX_NEW || d.max_pages > TW_MAX_ROW_PAGES) return TW_EINVAL;
  if (((uintptr_t)q | (uintptr_t)out | (uintptr_t)kv->kq_pool | (uintptr_t)kv->kq_meta | (uintptr_t)vq_pool | (uintptr_t)vq_meta | (uintptr_t)ws) & 15)
    return TW_EINVAL;
  if (!ws || ws_bytes < tw_kv4_workspace(d, max_new)) return TW_EWORKSPACE;
  const long long rows = (long long)max_new * d.G;
  const int M = rows_per_block4(rows);
  const int32_t most = 1 << 30;                  // longer than any sequence; positions minus it stay in 32 bits
  Kv4WideArgs a;
  a.q = (const uint4*)q;
  a.k_codes = (const uint4*)kv->kq_pool; a.k_meta = (const uint4*)kv->kq_meta; a.v_codes = (const uint4*)vq_pool; a.v_meta = (const uint4*)vq_meta;
  a.page_table = kv->page_table; a.seq_lens = kv->seq_lens; a.n_new = n_new; a.offsets = new_offsets;
  a.out = (uint2*)out; a.lse = lse;
  const size_t slots = part_slots4(d, rows);
  a.ws_plan = (int32_t*)ws;
  a.ws_ml = (float2*)((char*)ws + align256n((size_t)(d.batch + 1) * 8));
  a.ws_acc = (float*)((char*)a.ws_ml + align256n(slots * M * 8));
  a.batch = d.batch; a.Hq = d.Hq; a.Hkv = d.Hkv; a.G = d.G; a.lgG = __builtin_ctz(d.G); a.max_pages = d.max_pages; a.max_new = max_new;
  a.window = std::min(window, most); a.sinks = std::min(num_sinks, most); a.pool_pages = (unsigned)d.pool_pages;
  a.rb_max = (int)((rows + M - 1) / M); a.cus = tw_num_cus();
  const long long lists = (long long)a.rb_max * d.batch * d.Hkv;
  if (lists >= (1ll << 24) || (long long)max_new * d.batch >= (1ll << 31)) return TW_EINVAL;      // (a launch has fewer than 2^32 threads)
  hipStream_t s = (hipStream_t)stream;
  switch (M) {
    case 16: return launch_kv4<16>((const Kv4Args&)a, kv4_attention_kernel<1, false>, kv4_attention_kernel<1, true>, s);
    case 32: return launch_kv4<32>((const Kv4Args&)a, kv4_attention_kernel<2, false>, kv4_attention_kernel<2, true>, s);
    default: return launch_kv4<WIDE_M>(a, kv4_wide_kernel<false>, kv4_wide_kernel<true>, s);
  }
}
