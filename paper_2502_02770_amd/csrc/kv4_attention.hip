// Attention of a sequence's newest tokens over a cache that holds K and V in 4 bits (twilight_kv4_attention).
//
// K^ = c * s + z with one (s, z) per token and group of 32 dims, V^ alike.  The rows of a KV head are its G query heads times the
// N new tokens, as in new_tokens.hip; a workgroup takes M = 16 * RT of them, its four waves walk tiles of 64 tokens (4 pages)
// each on their own, and their states are merged at the end.
//
//   scores   S = sum_g s_g T_g + z_g Q_g over the four groups g, T_g = sum_d q_d c_d, Q_g = sum_d q_d.  T_g is one
//            v_mfma_f32_16x16x32_bf16 (a group is its contraction): A = 16 tokens' codes, as bf16 128 + c (one `and`, one `or` on two
//            codes of a word; 8 bits hold them exactly), B = 16 rows of q, C = -128 Q_g, which takes the 128 off again.  Codes and q are
//            exact, so a score is as good as one of fp32 products (the 128 costs 4 of the 24 bits).
//   weights  P = exp2(S log2(e)/sqrt(128) - m), fp32; their sum is of the unrounded ones.  For the product with V they are fp16, with m
//            kept 11 below the row's maximum's logarithm: the largest is 2^11 to 2^15, and one of 2^-25 of it still has 11 bits.
//   output   O^T += V^T P^T, v_mfma_f32_16x16x32_f16 with V^ = fma(c, s, z) in fp16 (2^-11 of itself at most; c exact: 1024 + c or 64 + c
//            with the bits put in place, less that).
//
// The A operand of the scores takes its 16 tokens as four of each of the tile's four pages (token 4 n + i of page j in row 4 j + i of
// step n), so that the quarter wave j holds all scores of page j's tokens, a row of q in each lane: what the transposed read of V's
// codes (ds_read_b64_tr_b4: a lane gets 16 tokens of one dim) wants its weights to be.  K's codes go to registers, 16 bytes of a
// group to a lane, and are exchanged between the quarters (four permlane swaps); V's codes and K's (s, z) go to LDS without passing
// registers, V's (s, z) through them, transposed.  The next tile's loads are issued before a tile is computed.
#include "kv4_common.h"
#include "new_tokens_plan.h"

namespace {

typedef _Float16 tw_f16x8 __attribute__((ext_vector_type(8)));
typedef int tw_v2i __attribute__((ext_vector_type(2)));
#define TW_LDS __attribute__((address_space(3)))
#define TW_GLB __attribute__((address_space(1)))

constexpr int WAVES = 4;
constexpr int BUF = 4096 + 1024;                 // of a wave: V's codes and K's (s, z) of 64 tokens
constexpr int TILE_BYTES4 = 64 * 160;            // what a wave's tile has in memory
constexpr float kLift = 11.f;                    // log2 of the weight of a row's maximum when m is set to it
constexpr float kGrowth4 = 4.f;                  // how far (in powers of 2) scores may pass it before m follows: weights stay below 2^16

struct Kv4Args {
  // a tile of the plan: the 16 pages that the four waves take together
  static constexpr int TILE_PAGES = 16, MIN_TILES = 1, STREAM_TILES = (96 << 20) / (WAVES * TILE_BYTES4);
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

// the lowest x of 16 bits
__device__ __forceinline__ uint32_t low16(int x) { return x <= 0 ? 0u : x >= 16 ? 0xFFFFu : (1u << x) - 1u; }

// The 8 codes of a word times s plus z in fp16; element 2 e + i is nibble e + 4 i.
__device__ __forceinline__ tw_f16x8 codes_f16(uint32_t w, const uint4& s, const uint4& z) {
  union { uint32_t u; tw_f16x2 h; } c[4], sc, ze;
  union { tw_f16x2 h[4]; tw_f16x8 v; } x;
  const uint32_t up = w >> 8;
  c[0].u = (w & 0x000F000Fu) | 0x64006400u;      // 1024 + c
  c[1].u = (w & 0x00F000F0u) | 0x54005400u;      // 64 + c
  c[2].u = (up & 0x000F000Fu) | 0x64006400u;
  c[3].u = (up & 0x00F000F0u) | 0x54005400u;
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
__device__ __forceinline__ void attend_item(const Kv4Args& a, const Item& it, unsigned char (&buf0)[WAVES * BUF], unsigned char (&buf1)[WAVES * BUF],
                                            unsigned char (&vms)[WAVES * 1024], int lane, int wave) {
  constexpr int M = 16 * RT;
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
  const int per = SPLIT ? __builtin_amdgcn_readfirstlane((int)quotient((uint32_t)(sp.tiles + it.chunks - 1), (uint32_t)it.chunks)) : sp.tiles;
  const int u0 = SPLIT ? min(sp.tiles, per * __builtin_amdgcn_readfirstlane(it.chunk)) : 0, u1 = min(sp.tiles, u0 + per);

  int pos[RT];
  tw_bf16x8 qf[RT][4];
  float qs[RT][4];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    pos[rt] = ctx + (row_of(rt) >> a.lgG);
    const uint4* qp = a.q + qrow_of(rt) * 16 + jq;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const uint4 x = qp[4 * g];
      float f[8], sum = 0.f;
      tw_unpack8(x, f);
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += f[i];
      qs[rt][g] = tw_quarters_sum(sum);
      qf[rt][g] = tw_q_like_codes(x);
    }
  }

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
    const int tok = one_of(x, jq) + r16;
    __builtin_amdgcn_global_load_lds((const TW_GLB unsigned int*)(a.k_meta + tok), (TW_LDS unsigned int*)(buf + 4096), 16, 0, 0);
#pragma unroll
    for (int p = 0; p < 4; ++p)
      __builtin_amdgcn_global_load_lds((const TW_GLB unsigned int*)(a.v_codes + ((long long)(x.s[p] + tok4) * 4 + piece4)), (TW_LDS unsigned int*)(buf + 1024 * p), 16, 0, 0);
  };
  uint4 kc[4], vm;                               // K's codes and V's (s, z) of a tile on its way
  auto issue_regs = [&](const Slots& x) {
    const uint4* kp = a.k_codes + ((long long)(one_of(x, r16 >> 2) + (r16 & 3)) * 4 + jq);
#pragma unroll
    for (int i = 0; i < 4; ++i) kc[i] = kp[16 * i];
    vm = a.v_meta[one_of(x, jq) + r16];
  };

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

  unsigned char* const vm_lds = vms + wave * 1024;
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
    {                                            // V's (s, z), 0 for what is no token, whose weight is 0
      const bool token = here && t0 + r16 < len;
      const uint32_t w[4] = {vm.x, vm.y, vm.z, vm.w};
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const uint32_t sz = token ? w[g] : 0u;
        *(unsigned short*)(vm_lds + vm_wr + 64 * g) = (unsigned short)sz;
        *(unsigned short*)(vm_lds + vm_wr + 64 * g + 16) = (unsigned short)(sz >> 16);
      }
    }
    tw_v4f s[RT][4];
#pragma unroll
    for (int st = 0; st < 4; ++st) {
      __builtin_amdgcn_sched_barrier(0);         // (the compiler would gather all steps' operands, and spill)
      tw_transpose_quarters(kc[st]);
      const tw_bf16x8 kf[4] = {tw_codes_bf16(kc[st].x), tw_codes_bf16(kc[st].y), tw_codes_bf16(kc[st].z), tw_codes_bf16(kc[st].w)};
      uint4 km[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) km[i] = *(const uint4*)(buf + 4096 + (jq * 16 + 4 * st + i) * 16);
      float zr[4][4];                            // z (RT = 1), or z - 128 s: with several row tiles there are no registers for their C operands
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t w[4] = {km[i].x, km[i].y, km[i].z, km[i].w};
#pragma unroll
        for (int g = 0; g < 4; ++g) zr[i][g] = RT == 1 ? tw_half_hi(w[g]) : __builtin_fmaf(tw_half_lo(w[g]), -128.f, tw_half_hi(w[g]));
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        tw_v4f t[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float c = RT == 1 ? -128.f * qs[rt][g] : 0.f;
          t[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[g], qf[rt][g], tw_v4f{c, c, c, c}, 0, 0, 0);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float y = zr[i][0] * qs[rt][0];
          y = __builtin_fmaf(zr[i][1], qs[rt][1], y);
          y = __builtin_fmaf(zr[i][2], qs[rt][2], y);
          y = __builtin_fmaf(zr[i][3], qs[rt][3], y);
          y = __builtin_fmaf(tw_half_lo(km[i].x), t[0][i], y);
          y = __builtin_fmaf(tw_half_lo(km[i].y), t[1][i], y);
          y = __builtin_fmaf(tw_half_lo(km[i].z), t[2][i], y);
          s[rt][st][i] = __builtin_fmaf(tw_half_lo(km[i].w), t[3][i], y);
        }
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
    unsigned char *const mine0 = buf0 + wave * BUF, *const mine1 = buf1 + wave * BUF;
    refill(u0);
    Slots x = slots_of(u0);
    issue_lds(mine0, x);
    issue_regs(x);
    for (int u = u0; u < u1; u += 2) {           // (a wave's buffers are its own: nothing to wait for but its own loads)
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
#pragma unroll
    for (int d = 0; d < 8; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) part[(d * 4 + i) * 64 + lane] = o[rt][d][i];
    if (jq == 0) ((float2*)vms)[wave * 16 + r16] = make_float2(mw, lw);
    __syncthreads();
    float2 ml[WAVES];
    float mn = kLow, ls = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) { ml[w] = ((const float2*)vms)[w * 16 + r16]; mn = fmaxf(mn, ml[w].x); }
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
    if (!SPLIT || it.chunks == 1) {
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

// SPLIT: resident workgroups stride over the items; otherwise a workgroup per list.
template <int RT, bool SPLIT>
__global__ __launch_bounds__(256, 2) void kv4_attention_kernel(Kv4Args a) {
  constexpr int M = 16 * RT;
  __shared__ __align__(1024) unsigned char buf0[WAVES * BUF];
  __shared__ __align__(1024) unsigned char buf1[WAVES * BUF];
  __shared__ __align__(1024) unsigned char vms[WAVES * 1024];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  Item it;
  if (!SPLIT) {
    if (whole_item<M>(a, &it)) attend_item<RT, SPLIT>(a, it, buf0, buf1, vms, lane, wave);
    return;
  }
  Seq seq;
  bool stream = false;
  const int chunk = __builtin_amdgcn_readfirstlane(plan_chunk<MODE_WINDOW, M>(a, lane, &seq, &stream));
  uint32_t want = blockIdx.x;
  while (find_item<MODE_WINDOW, M>(a, lane, chunk, seq, want, &it)) {
    int ln = lane;
    asm volatile("" : "+v"(ln));                 // what depends on the lane alone is worked out for every item: held over the items it would spill
    attend_item<RT, SPLIT>(a, it, buf0, buf1, vms, ln, wave);
    want += gridDim.x;
    if (want >= it.items) break;
    __syncthreads();                             // the buffers have been read
    if (a.batch <= 64) seq = seq_of<MODE_WINDOW, M>(a, lane);        // (again: held over the item it would cost registers that there are not)
  }
}

template <int M, int LANES>
__global__ __launch_bounds__(256) void kv4_combine_kernel(Kv4Args a) { join_parts<M, LANES>(a); }

// ---------------------------------------------------------------- host side
int rows_per_block4(long long rows) { return rows <= 16 ? 16 : 32; }

bool cut_lists4(bool counted, int blocks, long long lists, long long longest) {
  if (longest <= std::min(8ll, 1 + lists / 64)) return false;
  const long long places = 2ll * tw_num_cus();
  if (blocks < 8 || lists < places) return true;
  return counted && longest * places > 48 * lists;
}

template <int RT>
int launch_kv4(const Kv4Args& a, hipStream_t s) {
  constexpr int M = 16 * RT;
  const long long lists = (long long)a.rb_max * a.batch * a.Hkv, rows = (long long)a.max_new * a.Hq;
  long long longest = ((long long)a.max_pages + 15) / 16;                       // tiles that a list can have
  longest = std::min(longest, (((long long)a.sinks + TW_PAGE - 1) / TW_PAGE + ((long long)a.window + M / a.G + TW_PAGE - 2) / TW_PAGE + 1 + 15) / 16);
  tw_prof_before(TW_K_KV4_ATTENTION, s);
  if (!cut_lists4(a.n_new != nullptr, a.rb_max, lists, longest) || rows >= (1ll << 26)) {
    TW_LAUNCH((kv4_attention_kernel<RT, false>), dim3((unsigned)lists), dim3(256), 0, s, a);
    return tw_prof_after(s);
  }
  TW_LAUNCH((kv4_attention_kernel<RT, true>), dim3((unsigned)std::min(lists * longest, 2ll * a.cus)), dim3(256), 0, s, a);
  if (int e = tw_prof_after(s)) return e;
  tw_prof_before(TW_K_KV4_COMBINE, s);
  if (rows * a.batch <= COMBINE_FEW) TW_LAUNCH((kv4_combine_kernel<M, 8>), dim3((unsigned)rows, (unsigned)a.batch), dim3(256), 0, s, a);
  else TW_LAUNCH((kv4_combine_kernel<M, 2>), dim3((unsigned)((rows + 3) / 4), (unsigned)a.batch), dim3(256), 0, s, a);
  return tw_prof_after(s);
}

// Parts that a plan can make: fewer than 2 W rounds (plan_chunk); of one row block per sequence and KV head no more than its list has tiles.
size_t part_slots4(const TwDims& d, long long rows) {
  const long long most = (long long)tw_num_cus() * 4 * PLAN_ROUNDS;
  if (rows > 32) return (size_t)most;
  return (size_t)std::min(most, ((long long)d.max_pages + 15) / 16 * d.batch * d.Hkv);
}

}  // namespace

size_t tw_kv4_workspace(const TwDims& d, int max_new) {
  if (max_new <= 0 || max_new > TW_MAX_NEW) return 0;
  const long long rows = (long long)max_new * d.G;
  const int M = rows_per_block4(rows);
  const size_t slots = part_slots4(d, rows);
  return align256n((size_t)d.batch * 8) + align256n(slots * M * 8) + slots * M * 512;
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
  Kv4Args a;
  a.q = (const uint4*)q;
  a.k_codes = (const uint4*)kv->kq_pool; a.k_meta = (const uint4*)kv->kq_meta; a.v_codes = (const uint4*)vq_pool; a.v_meta = (const uint4*)vq_meta;
  a.page_table = kv->page_table; a.seq_lens = kv->seq_lens; a.n_new = n_new; a.offsets = new_offsets;
  a.out = (uint2*)out; a.lse = lse;
  const size_t slots = part_slots4(d, rows);
  a.ws_plan = (int32_t*)ws;
  a.ws_ml = (float2*)((char*)ws + align256n((size_t)d.batch * 8));
  a.ws_acc = (float*)((char*)a.ws_ml + align256n(slots * M * 8));
  a.batch = d.batch; a.Hq = d.Hq; a.Hkv = d.Hkv; a.G = d.G; a.lgG = __builtin_ctz(d.G); a.max_pages = d.max_pages; a.max_new = max_new;
  a.window = std::min(window, most); a.sinks = std::min(num_sinks, most); a.pool_pages = (unsigned)d.pool_pages;
  a.rb_max = (int)((rows + M - 1) / M); a.cus = tw_num_cus();
  const long long lists = (long long)a.rb_max * d.batch * d.Hkv;
  if (lists >= (1ll << 24) || (long long)max_new * d.batch >= (1ll << 31)) return TW_EINVAL;      // (a launch has fewer than 2^32 threads)
  hipStream_t s = (hipStream_t)stream;
  return M == 16 ? launch_kv4<1>(a, s) : launch_kv4<2>(a, s);
}
