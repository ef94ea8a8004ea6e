// Tokens given up by the attention they got: the weights accumulated per cached token (twilight_attention_mass), and the choice of
// the tokens to keep (twilight_keep_tokens).  twilight_tokens_compact then moves what is kept.
#include <algorithm>
#include <type_traits>
#include "kv4_common.h"

#define TW_GLB __attribute__((address_space(1)))
#define TW_LDS __attribute__((address_space(3)))

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kScaleLog2 = 0.08838834764831845f * 1.4426950408889634f;   // log2(e) / sqrt(128)

// ------------------------------------------------------------------------------------------------------- accumulated weights
// mass[t] = decay mass[t] + sum over new tokens i and query heads of exp(q.K_t / sqrt(128) - lse_i): K once, nothing else of the cache.
//
// A workgroup has PT pages of a sequence, its four waves the KV heads in turn; a wave holds its head's K of those pages and goes through
// the head's rows (query heads x new tokens) by 16, over bf16 and with many rows two times 16: S = Q K^T, v_mfma_f32_16x16x32_bf16 (codes as 128 + c in bf16, as in
// kv4_attention.hip), a lane has one token and four rows.  What comes next is asked for ahead: with up to 16 rows the next head's K and
// queries, with more (MANY) the next rows.  The waves' sums are added in their order, so that the result does not depend on timing.
//
// Measured, 32 heads over 8: one token of 8 x 32768 of codes 42 us for 170 MB, 4.1 TB/s, beside vector issue 0.75 of the time; 64 tokens of 2 x 16001
// of bf16 41 us for 17 GFLOP and 67 MB: a wave's way through 256 rows of two heads, of which queries on their way are 9 us (33 with the first ones kept) and
// exponentials 4, beside one other wave of its SIMD.  One token of 4096 4.5 us: page table, K and queries, sums one after the other.
struct MassArgs {
  const uint4* q;
  const float* lse;
  const uint4* k;                                // bf16 rows, or codes
  const uint4* meta;
  const int32_t* page_table;
  const int32_t* seq_lens;
  const int32_t* n_new;
  const int32_t* offsets;
  const float* mass_in;
  float* mass_out;
  int Hq, Hkv, G, lgG, max_pages, max_new, window, sinks;
  unsigned pool_pages;
  float decay;
};

template <bool CODES, int PT, bool MANY>
__global__ __launch_bounds__(256, 2) void attention_mass_kernel(MassArgs a) {
  constexpr int BUF = MANY ? 2 * 4096 : 16;      // a wave's two blocks of rows
  __shared__ __align__(16) unsigned char buf0[4 * BUF], buf1[4 * BUF];
  __shared__ float red[4][16 * PT];
  const int b = blockIdx.y, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6)), r16 = lane & 15, jq = lane >> 4;
  const int len = max(0, min(a.seq_lens[b], a.max_pages * TW_PAGE)), n = a.n_new ? max(0, min(a.n_new[b], a.max_new)) : a.max_new;
  const long long first = (long long)blockIdx.x * (16 * PT);
  if (first >= len) return;
  const int t0 = (int)first, ctx = len - n, off = a.offsets ? a.offsets[b] : b * a.max_new, rows = n * a.G;
  int slot[PT];                                  // of the pages' first token, head 0; -1: nobody sees them
  const int32_t* table = a.page_table + (long long)b * a.max_pages + t0 / TW_PAGE;
#pragma unroll
  for (int p = 0; p < PT; ++p) {
    const int id = t0 + 16 * p < len ? table[p] : -1;
    slot[p] = __builtin_amdgcn_readfirstlane((unsigned)id < a.pool_pages ? id * a.Hkv * TW_PAGE : -1);
  }
  float acc[PT];
#pragma unroll
  for (int p = 0; p < PT; ++p) acc[p] = 0.f;

  struct Keys { uint4 k[PT][CODES ? 1 : 4], m[CODES ? PT : 1]; };
  auto load_keys = [&](int h) -> Keys {
    Keys x;
#pragma unroll
    for (int p = 0; p < PT; ++p) {
      const int row = max(slot[p], 0) + h * TW_PAGE + r16;
      if constexpr (CODES) {
        x.k[p][0] = a.k[(long long)row * 4 + jq];
        x.m[p] = a.meta[row];
      } else {
#pragma unroll
        for (int g = 0; g < 4; ++g) x.k[p][g] = tw_ld_stream(a.k + (long long)row * 16 + 4 * g + jq);
      }
    }
    return x;
  };
  // Row r0 + k behind row r0, or row r0 again for those behind the last
  auto place = [&](int r0, int k) -> uint32_t { return r0 + k < rows ? (uint32_t)((k >> a.lgG) * a.Hq + (k & (a.G - 1))) : 0u; };
  auto row_at = [&](int h, int r0) -> long long { return (long long)(off + (r0 >> a.lgG)) * a.Hq + h * a.G; };
  struct Rows { uint4 q[4]; float lse; };        // of row r16; with many rows the lse of row (lane % 32), and q in LDS
  auto load_rows = [&](int h) -> Rows {
    Rows x;
    const long long row = row_at(h, 0) + place(0, r16);
#pragma unroll
    for (int g = 0; g < 4; ++g) x.q[g] = a.q[row * 16 + 4 * g + jq];
    x.lse = a.lse[row];
    return x;
  };
  // 32 of many rows go to LDS, consecutive lanes to consecutive bytes: read straight into operands, lanes beside each other are a row apart, and
  // each load costs 64 cycles instead of 16 (64 rows of two prompts 47.7 -> 41.6 us).  Piece p of row r stands at p ^ r.
  auto ask = [&](unsigned char* buf, int h, int r0) -> Rows {
    Rows x;
    const long long row = row_at(h, r0);
    const char* q = (const char*)a.q + row * 256;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int k = 4 * i + jq;
      __builtin_amdgcn_global_load_lds((const TW_GLB unsigned int*)(q + (place(r0, k) * 256u + 16u * (uint32_t)(r16 ^ (k & 15)))), (TW_LDS unsigned int*)(buf + 1024 * i), 16, 0, 0);
    }
    x.lse = a.lse[row + place(r0, lane & 31)];
    return x;
  };
  auto arrived = []() {
    __builtin_amdgcn_s_waitcnt(0x0070);          // vmcnt(0), lgkmcnt(0): the step's rows are here, and the other buffer has been read
    asm volatile("" ::: "memory");
  };
  auto operands = [&](const Keys& x, int p, tw_bf16x8 (&kf)[4]) {
    uint4 c = x.k[p][0];
    tw_transpose_quarters(c);
    kf[0] = tw_codes_bf16(c.x); kf[1] = tw_codes_bf16(c.y); kf[2] = tw_codes_bf16(c.z); kf[3] = tw_codes_bf16(c.w);
  };
  // Blocks of rows that see any of the pages: those at positions from the first page's start on, and not so far behind that no window reaches
  const int from = min(rows, max(0, t0 - ctx) * a.G) & ~15;
  const int to = t0 < a.sinks ? rows : (int)max(0ll, min((long long)rows, ((long long)t0 + 16 * PT - 1 + a.window - ctx) * a.G));
  // The weights of NB blocks of 16 rows from row r0 on, the first of them block `block` of a step's
  constexpr int NB = MANY && !CODES ? 2 : 1;
  auto add = [&](const Keys& x, const tw_bf16x8 (&held)[PT][4], const Rows& rs, const unsigned char* buf, int block, int r0) {
    const int p_lo = ctx + (r0 >> a.lgG), p_hi = ctx + ((min(r0 + 16 * NB, rows) - 1) >> a.lgG);
    const bool all = t0 + 16 * PT - 1 <= p_lo && (t0 > p_hi - a.window || t0 + 16 * PT <= a.sinks);
    tw_bf16x8 qf[NB][4];
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const uint4 y = MANY ? *(const uint4*)(buf + 4096 * (block + n) + 256 * r16 + 16 * ((4 * g + jq) ^ r16)) : rs.q[g];
        qf[n][g] = CODES ? tw_q_like_codes(y) : tw_as_bf16(y);
      }
    float l2[NB][4];                             // lse in powers of 2; infinite (weights of 0) where there is no row, or none with a weight
    int pos[NB][4];
    const float mine = r0 - 16 * block + (MANY ? lane & 31 : r16) < rows && __builtin_fabsf(rs.lse) < __builtin_inff() ? rs.lse * kLog2e : __builtin_inff();
#pragma unroll
    for (int n = 0; n < NB; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {              // (four loads of the rows' own lse took 9 of 55 us of two prompts' last 64 tokens)
        l2[n][i] = __int_as_float(__builtin_amdgcn_ds_bpermute((16 * (block + n) + 4 * jq + i) * 4, __float_as_int(mine)));
        pos[n][i] = ctx + ((r0 + 16 * n + 4 * jq + i) >> a.lgG);
      }
    tw_v4f s[NB][PT];
    if constexpr (CODES) {
      tw_v4f less[4];                            // -128 Q_g of the lane's rows: a product with a constant
      tw_bf16x8 c;
#pragma unroll
      for (int i = 0; i < 8; ++i) c[i] = (__bf16)-128.f;
#pragma unroll
      for (int g = 0; g < 4; ++g) less[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[0][g], c, tw_v4f{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
      for (int p = 0; p < PT; ++p) {
        tw_bf16x8 kf[4];
        if constexpr (MANY) {
#pragma unroll
          for (int g = 0; g < 4; ++g) kf[g] = held[p][g];
        } else {
          operands(x, p, kf);
        }
        const uint32_t w[4] = {x.m[p].x, x.m[p].y, x.m[p].z, x.m[p].w};
        tw_v4f t[4];
#pragma unroll
        for (int g = 0; g < 4; ++g) t[g] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[0][g], kf[g], less[g], 0, 0, 0);
        tw_v4f& sum = s[0][p];
        sum = tw_v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const float z = tw_half_hi(w[g]) * (-1.f / 128.f);
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i] = __builtin_fmaf(z, less[g][i], sum[i]);
        }
#pragma unroll
        for (int g = 0; g < 4; ++g)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i] = __builtin_fmaf(tw_half_lo(w[g]), t[g][i], sum[i]);
      }
    } else {                                     // (no product follows the one that it adds to)
      constexpr bool APART = PT == 1;
      tw_v4f u[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n) {
        u[n] = tw_v4f{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int p = 0; p < PT; ++p) s[n][p] = tw_v4f{0.f, 0.f, 0.f, 0.f};
      }
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        if (NB > 1) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int p = 0; p < PT; ++p) {
          const tw_bf16x8 k = tw_as_bf16(x.k[p][g]);
#pragma unroll
          for (int n = 0; n < NB; ++n) {
            if (APART && (g & 1)) u[n] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[n][g], k, u[n], 0, 0, 0);
            else s[n][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[n][g], k, s[n][p], 0, 0, 0);
          }
        }
      }
      if (APART)
#pragma unroll
        for (int n = 0; n < NB; ++n) s[n][0] += u[n];
    }
    auto weigh = [&](auto masked) {
#pragma unroll
      for (int p = 0; p < PT; ++p) {
        const int t = t0 + 16 * p + r16;
#pragma unroll
        for (int n = 0; n < NB; ++n) {
          float w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            // (the maximum makes 0 of what is no number: a row that sees such a token has an lse that says so)
            w[i] = fmaxf(__builtin_amdgcn_exp2f(__builtin_fmaf(s[n][p][i], kScaleLog2, -l2[n][i])), 0.f);
            if constexpr (decltype(masked)::value) w[i] = (t <= pos[n][i]) & ((t > pos[n][i] - a.window) | (t < a.sinks)) ? w[i] : 0.f;
          }
          acc[p] += (w[0] + w[1]) + (w[2] + w[3]);
        }
      }
    };
    if (all) weigh(std::false_type{});           // (a branch of its own: asked at every score it would be one per score)
    else weigh(std::true_type{});
  };

  if (wave < a.Hkv && from < to) {
    tw_bf16x8 held[PT][4];                       // (codes as operands, made once for all rows)
    if constexpr (MANY) {
      unsigned char *const mine0 = buf0 + wave * BUF, *const mine1 = buf1 + wave * BUF;
      for (int h = wave; h < a.Hkv; h += 4) {
        Rows y0 = ask(mine0, h, from), y1;
        const Keys x = load_keys(h);
#pragma unroll
        for (int p = 0; p < PT; ++p)
          if constexpr (CODES) operands(x, p, held[p]);
        for (int r0 = from; r0 < to; r0 += 64) {
          arrived();
          if (r0 + 32 < to) y1 = ask(mine1, h, r0 + 32);
          add(x, held, y0, mine0, 0, r0);
          if (NB == 1 && r0 + 16 < to) add(x, held, y0, mine0, 1, r0 + 16);
          if (r0 + 32 >= to) break;
          arrived();
          if (r0 + 64 < to) y0 = ask(mine0, h, r0 + 64);
          add(x, held, y1, mine1, 0, r0 + 32);
          if (NB == 1 && r0 + 48 < to) add(x, held, y1, mine1, 1, r0 + 48);
        }
        arrived();                               // (the last rows have been read before the next head's are asked for)
      }
    } else {
      Keys x = load_keys(wave);
      Rows y = load_rows(wave);
      for (int h = wave; h < a.Hkv; h += 4) {
        const int next = h + 4 < a.Hkv ? h + 4 : h;
        const Keys xn = load_keys(next);
        const Rows yn = load_rows(next);
        add(x, held, y, nullptr, 0, 0);
        x = xn;
        y = yn;
      }
    }
  }
#pragma unroll
  for (int p = 0; p < PT; ++p) {
    const float sum = tw_quarters_sum(slot[p] < 0 ? 0.f : acc[p]);
    if (jq == 0) red[wave][16 * p + r16] = sum;
  }
  __syncthreads();
  const int t = t0 + (int)threadIdx.x;
  if (threadIdx.x < 16 * PT && t < len) {
    const long long at = (long long)b * a.max_pages * TW_PAGE + t;
    const float had = t < ctx ? a.decay * a.mass_in[at] : 0.f;
    a.mass_out[at] = had + ((red[0][threadIdx.x] + red[1][threadIdx.x]) + (red[2][threadIdx.x] + red[3][threadIdx.x]));
  }
}

// -------------------------------------------------------------------------------------------------------------- what to keep
// The budget's share of a sequence's tokens: its first ones, its latest ones, and of those between the heaviest.  A weight's bits in
// the order of the numbers are a key; the key of the last token kept is found by three histograms (of 11, 11 and 10 bits), each of
// the tokens that share the bits found before, and equal keys go to the lowest positions.
//
// Up to 8192 tokens are one launch, a sequence to a workgroup, all in registers: 7.6 us for 2049, most of it three rounds of counting in LDS and
// finding a digit.  More are four launches of 4 to 9 us (16 x 32768 22 us, 3 x 200003 29 us): at so few bytes (4 a token) trips to memory, since every
// launch reads the counts of all of a row's chunks that the one before left.
struct KeepArgs {
  const float* mass;
  const int32_t* seq_lens;
  const int32_t* budget;
  int32_t* idx;
  int32_t* count;
  float* mass_out;                               // or nullptr
  uint32_t* ws;                                  // [batch][SEQ_WORDS], [batch][chunks][CHUNK_WORDS]
  int max_pages, sinks, recent, stride, chunks, blocks;   // blocks of SUB tokens to a chunk
};
constexpr int KEEP_THREADS = 1024, SUB = 8 * KEEP_THREADS;
constexpr int CHUNK_WORDS = 2048 + 2048 + 1024 + 2;     // three histograms, tokens above the first two's digits
constexpr int SEQ_WORDS = 4;                            // what is known of a sequence after each launch: (bits, tokens to find) twice

struct KeepSeq {
  int len, kept, first, last, want;              // tokens, of them kept; of those kept first and latest ones, and of those between
};
__device__ __forceinline__ KeepSeq keep_seq(const KeepArgs& a, int b) {
  KeepSeq s;
  s.len = max(0, min(a.seq_lens[b], a.max_pages * TW_PAGE));
  s.kept = max(0, min(min(a.budget[b], s.len), a.stride));
  s.first = min(a.sinks, s.kept);
  s.last = min(a.recent, s.kept - s.first);
  s.want = s.kept - s.first - s.last;
  return s;
}
// Larger weight, larger key; no number: 1, below all of them; 0: not to be chosen by its weight (a first or latest token, or none).
__device__ __forceinline__ uint32_t keep_key(float x) { return x == x ? tw_float_key(x + 0.0f) : 1u; }

// The bin of 2048, from the highest down, in which the want-th token lies, and how many are in those above it.  One wave does it, 32 bins
// to a lane and then one bin to a lane: two barriers for the others, where a scan over the workgroup has five.
struct Digit { uint32_t bin, above; };
__device__ __forceinline__ Digit find_digit(const uint32_t* hist, uint32_t want, uint32_t* scratch) {
  if (threadIdx.x < 64) {
    const int lane = threadIdx.x;
    uint32_t sum = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {                // (each lane begins at another of its pieces, so that they do not meet in a bank)
      const uint4 x = *(const uint4*)(hist + 2016 - 32 * lane + 4 * ((i + lane) & 7));
      sum += (x.x + x.y) + (x.z + x.w);
    }
    const uint32_t incl = tw_wave_scan_u32(sum);
    const int l = __builtin_ctzll(__ballot(incl >= want) | 1ull << 63);
    const uint32_t before = (uint32_t)__builtin_amdgcn_readlane((int)(incl - sum), l);
    const int top = 2047 - 32 * l;
    const uint32_t n = lane < 32 ? hist[top - lane] : 0u, here = before + tw_wave_scan_u32(n);
    const int k = __builtin_ctzll(__ballot(here >= want) | 1ull << 31);
    if (lane == k) { scratch[16] = (uint32_t)(top - k); scratch[17] = here - n; }
  }
  __syncthreads();
  return {scratch[16], scratch[17]};
}

// A wave's rows of 64 consecutive tokens: row i begins at t0 + 64 i, a lane has one token of each.  Their weights, and the keys.
template <int E>
__device__ __forceinline__ void load_rows64(const float* row, int t0, int len, float (&x)[E]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < E; ++i) x[i] = t0 + 64 * i + lane < len ? row[t0 + 64 * i + lane] : 0.f;
}
template <int E>
__device__ __forceinline__ void keys_of64(int t0, int lo, int hi, const float (&x)[E], uint32_t (&key)[E]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int t = t0 + 64 * i + lane;
    key[i] = t >= lo && t < hi ? keep_key(x[i]) : 0u;
  }
}
// Of rows: tokens kept for a larger key (low half) and those of the last key kept (high half), at most 2^15 each
template <int E>
__device__ __forceinline__ uint32_t count_rows64(const uint32_t (&key)[E], uint32_t last_key) {
  uint32_t n = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) n += (uint32_t)__popcll(__ballot(key[i] > last_key)) + ((uint32_t)__popcll(__ballot(key[i] == last_key)) << 16);
  return n;
}
// The rows' tokens written where they are kept.  above, ties: tokens kept for a larger key, and of the last one, before them; room: how many of
// the latter are kept.  A row's kept tokens stand side by side.
template <int E>
__device__ __forceinline__ void emit_rows64(const KeepArgs& a, int b, const KeepSeq& s, const float (&x)[E], const uint32_t (&key)[E], int t0, uint32_t last_key,
                                            uint32_t above, uint32_t ties, uint32_t room) {
  const long long out = (long long)b * a.stride;
  const int lane = threadIdx.x & 63, hi = s.len - s.last;
#pragma unroll
  for (int i = 0; i < E; ++i) {
    const int first = t0 + 64 * i, t = first + lane;
    if (first >= s.len) break;
    const bool more = key[i] > last_key, tie = key[i] == last_key;
    const unsigned long long mm = __ballot(more), mt = __ballot(tie);
    const uint32_t rank = ties + tw_bits_below(mt);
    int at = -1;
    if (more || (tie && rank < room)) at = s.first + (int)(above + tw_bits_below(mm) + min(rank, room));
    if (t < s.first) at = t;
    if (t >= hi && t < s.len) at = s.kept - (s.len - t);
    if (at >= 0) {
      a.idx[out + at] = t;
      if (a.mass_out) a.mass_out[out + at] = x[i];
    }
    above += (uint32_t)__popcll(mm);
    ties += (uint32_t)__popcll(mt);
  }
}
// A digit of the rows' tokens that share the bits found before, counted
template <int PASS, int E>
__device__ __forceinline__ void count_digit(uint32_t* hist, const uint32_t (&key)[E], uint32_t prefix) {
  constexpr int shift = PASS == 0 ? 21 : PASS == 1 ? 10 : 0, bits = PASS == 2 ? 10 : 11;
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (key[i] != 0u && (PASS == 0 || key[i] >> (shift + bits - 1) >> 1 == prefix)) atomicAdd(&hist[(key[i] >> shift) & ((1u << bits) - 1u)], 1u);
}

// A whole sequence per workgroup, E tokens per thread in registers.
template <int THREADS, int E>
__global__ __launch_bounds__(THREADS) void keep_whole_kernel(KeepArgs a) {
  __shared__ __align__(16) uint32_t hist[3][2048];
  __shared__ uint32_t scratch[20];
  const int b = blockIdx.x, tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const KeepSeq s = keep_seq(a, b);
  if (tid == 0) a.count[b] = s.kept;
  if (s.kept == 0) return;
  const int t0 = wave * 64 * E, lo = s.first, hi = s.len - s.last;
  float x[E];
  uint32_t key[E];
  load_rows64<E>(a.mass + (long long)b * a.max_pages * TW_PAGE, t0, s.len, x);
  keys_of64<E>(t0, lo, hi, x, key);
  uint32_t prefix = ~0u, want = (uint32_t)s.want;            // (no key is this large)
  if (s.want > 0) {
#pragma unroll
    for (int i = 0; i < 3 * 2048 / THREADS; ++i) (&hist[0][0])[tid + THREADS * i] = 0;
    __syncthreads();
    prefix = 0;
#pragma unroll
    for (int pass = 0; pass < 3; ++pass) {
      if (pass == 0) count_digit<0, E>(hist[0], key, prefix);
      else if (pass == 1) count_digit<1, E>(hist[1], key, prefix);
      else count_digit<2, E>(hist[2], key, prefix);          // (the upper half of the last stays empty)
      __syncthreads();
      const Digit d = find_digit(hist[pass], want, scratch);
      prefix = prefix << (pass == 2 ? 10 : 11) | d.bin;
      want -= d.above;
    }
  }
  // kept for a larger key, and of the last key, before this wave's tokens
  const uint32_t mine = count_rows64<E>(key, prefix);
  if ((tid & 63) == 0) scratch[wave] = mine;
  __syncthreads();
  uint32_t before = 0;
  for (int w = 0; w < wave; ++w) before += scratch[w];
  emit_rows64<E>(a, b, s, x, key, t0, prefix, before & 0xFFFFu, before >> 16, want);
}

// Long sequences: a workgroup per chunk of tokens, a launch per histogram and one that writes.  PASS 0 .. 2 make a chunk's histogram of
// that digit; 1 .. 3 first find the digit before from all chunks' histograms, and the first chunk leaves it for the launches to come.
template <int PASS>
__global__ __launch_bounds__(KEEP_THREADS) void keep_chunk_kernel(KeepArgs a) {
  __shared__ __align__(16) uint32_t hist[2048];
  __shared__ uint32_t scratch[20];
  const int b = blockIdx.y, c = blockIdx.x, tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const KeepSeq s = keep_seq(a, b);
  if (PASS == 3 && c == 0 && tid == 0) a.count[b] = s.kept;
  const long long span = (long long)a.blocks * SUB, begin = c * span;
  if (s.kept == 0 || begin >= s.len) return;
  const int t0 = (int)begin, chunks = (int)((s.len + span - 1) / span);        // chunks of this sequence
  uint32_t* const known = a.ws + (long long)b * SEQ_WORDS;
  uint32_t* const all = a.ws + (long long)gridDim.y * SEQ_WORDS + (long long)b * a.chunks * CHUNK_WORDS;
  uint32_t* const own = all + (long long)c * CHUNK_WORDS;
  const float* row = a.mass + (long long)b * a.max_pages * TW_PAGE;
  const int lo = s.first, hi = s.len - s.last;
  float x[8];
  uint32_t key[8];
  // (a chunk of one block, as those of up to 128 x 8192 tokens are, is asked for at once)
  if (a.blocks == 1) load_rows64<8>(row, t0 + wave * 512, s.len, x);
  uint32_t prefix = 0, want = (uint32_t)s.want, above = 0, ties = 0;
  if (PASS > 0 && s.want > 0) {
    constexpr int D = PASS > 0 ? PASS - 1 : 0;   // the digit to find
    if (PASS > 1) { prefix = known[2 * (PASS - 2)]; want = known[2 * (PASS - 2) + 1]; }
    const uint32_t* h = all + 2048 * D;
    uint32_t n0 = 0, n1 = 0, mine0 = 0, mine1 = 0;           // this thread's two bins, or the one of the last digit: of all chunks, and of this
    if (D < 2) {                                 // one, or of all before this one
      for (int k0 = 0; k0 < chunks; k0 += 16) {  // (16 at once, those behind the last not asked for: each is a trip past this XCD's L2)
        uint2 y[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) y[k] = k0 + k < chunks ? *(const uint2*)(h + (long long)(k0 + k) * CHUNK_WORDS + 2 * tid) : make_uint2(0u, 0u);
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          n0 += y[k].x; n1 += y[k].y;
          if (k0 + k == c) { mine0 = y[k].x; mine1 = y[k].y; }
        }
      }
      *(uint2*)(hist + 2 * tid) = make_uint2(n0, n1);
    } else {
      for (int k0 = 0; k0 < chunks; k0 += 16) {
        uint32_t y[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) y[k] = k0 + k < chunks ? h[(long long)(k0 + k) * CHUNK_WORDS + tid] : 0u;
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          n0 += y[k];
          mine0 += k0 + k < c ? y[k] : 0u;
        }
      }
      hist[tid] = n0;
      hist[tid + 1024] = 0;
    }
    if (tid == 0) scratch[18] = scratch[19] = 0;
    __syncthreads();
    const Digit d = find_digit(hist, want, scratch);
    // tokens above the digit: this chunk's, for those behind it, or those of all before it
    const uint32_t bin = D < 2 ? 2 * tid : tid;
    uint32_t more = (bin > d.bin ? mine0 : 0u) + (D < 2 && bin + 1u > d.bin ? mine1 : 0u);
    if (D == 2) {
      for (int k = tid; k < c; k += KEEP_THREADS) more += all[(long long)k * CHUNK_WORDS + 5120] + all[(long long)k * CHUNK_WORDS + 5121];
      if (bin == d.bin) scratch[19] = mine0;
    }
    more = (uint32_t)__builtin_amdgcn_readlane((int)tw_wave_scan_u32(more), 63);
    if ((tid & 63) == 0 && more) atomicAdd(&scratch[18], more);
    __syncthreads();
    if (D < 2) {
      if (tid == 0) own[5120 + D] = scratch[18];
    } else {
      above = scratch[18];
      ties = scratch[19];
    }
    prefix = prefix << (D == 2 ? 10 : 11) | d.bin;
    want -= d.above;
    if (PASS < 3 && c == 0 && tid == 0) { known[2 * D] = prefix; known[2 * D + 1] = want; }
  }
  if (PASS < 3) {
    if (s.want == 0) return;
    hist[tid] = 0; hist[tid + 1024] = 0;
    __syncthreads();
    for (int k = 0; k < a.blocks; ++k) {
      const int t = t0 + k * SUB + wave * 512;
      if (t >= hi) break;
      if (a.blocks > 1) load_rows64<8>(row, t, s.len, x);
      keys_of64<8>(t, lo, hi, x, key);
      count_digit<PASS, 8>(hist, key, prefix);
    }
    __syncthreads();
    own[2048 * PASS + tid] = hist[tid];
    if (PASS < 2) own[2048 * PASS + 1024 + tid] = hist[tid + 1024];
    return;
  }
  if (s.want == 0) prefix = ~0u;                 // (no key is this large)
  for (int k = 0; k < a.blocks; ++k) {
    const int at = t0 + k * SUB, t = at + wave * 512;
    if (at >= s.len) break;
    if (a.blocks > 1) load_rows64<8>(row, t, s.len, x);
    keys_of64<8>(t, lo, hi, x, key);
    const uint32_t mine = count_rows64<8>(key, prefix);
    if ((tid & 63) == 0) scratch[wave] = mine;
    __syncthreads();
    uint32_t before = 0, total = 0;
#pragma unroll
    for (int w = 0; w < KEEP_THREADS / 64; ++w) { const uint32_t n = scratch[w]; before += w < wave ? n : 0u; total += n; }
    emit_rows64<8>(a, b, s, x, key, t, prefix, above + (before & 0xFFFFu), ties + (before >> 16), want);
    above += total & 0xFFFFu;
    ties += total >> 16;
    __syncthreads();                             // the counts have been read
  }
}

constexpr int WHOLE_TOKENS = 8192, MOST_CHUNKS = 128;

// Chunks of a long row, and blocks of SUB tokens in each.
void keep_chunks(const TwDims& d, int* chunks, int* blocks) {
  const long long subs = ((long long)d.max_pages * TW_PAGE + SUB - 1) / SUB;
  *blocks = (int)((subs + MOST_CHUNKS - 1) / MOST_CHUNKS);
  *chunks = (int)((subs + *blocks - 1) / *blocks);
}

// Pages to a workgroup: few where that leaves CUs without one, more for the loads (and, with many rows, the queries) that they share.  us with 1 / 2 / 4 /
// 8 pages, 32 heads over 8, by all sequences' pages:
//                     256                    512                     1024                   2002                   4096 or 16384
//   1 token    bf16   6.0  6.8  8.1 13.3     7.8  7.5 10.8 17.4      12.2 11.3 11.5 18.0    21.6 20.0 19.9 19.5    155  143  140  139
//   1 token    codes  6.3  6.4  6.4  8.6     6.3  6.5  6.6  8.7       6.4  6.7  6.5  8.7    10.2  8.8  8.8  9.8    62.7 47.8 41.3 45.0
//   64 tokens  bf16  15.1 17.9 29.8 85.3    21.4 18.3 30.3 85.6      38.6 26.0 31.2 87.2    71.3 47.2 41.8 93.7    142  91.3 78.5 149
//   64 tokens  codes 16.8 22.0 34.8  110    22.0 22.3 35.9  111      41.8 30.5 36.8  115    77.1 55.3 50.3  118    148  106  95.1 188
template <bool CODES, bool MANY>
void launch_mass(const MassArgs& a, int batch, hipStream_t s) {
  const long long pages = (long long)a.max_pages * batch, cus = tw_num_cus();
  auto grid = [&](int n) { return dim3((unsigned)((a.max_pages + n - 1) / n), (unsigned)batch); };
  const dim3 wg(256);
  if (pages <= cus * 3 / 2) TW_LAUNCH((attention_mass_kernel<CODES, 1, MANY>), grid(1), wg, 0, s, a);
  else if (pages <= 4 * cus) TW_LAUNCH((attention_mass_kernel<CODES, 2, MANY>), grid(2), wg, 0, s, a);
  else TW_LAUNCH((attention_mass_kernel<CODES, 4, MANY>), grid(4), wg, 0, s, a);
}

}  // namespace

size_t tw_keep_workspace(const TwDims& d) {
  if ((long long)d.max_pages * TW_PAGE <= WHOLE_TOKENS) return 256;
  int chunks, blocks;
  keep_chunks(d, &chunks, &blocks);
  return ((size_t)d.batch * (SEQ_WORDS + (size_t)chunks * CHUNK_WORDS) * 4 + 255) & ~(size_t)255;
}

extern "C" int twilight_attention_mass(const twilight_kv_t* kv, const void* q, const float* lse, const int32_t* n_new, const int32_t* new_offsets,
                                       int32_t max_new, int32_t window, int32_t num_sinks, float decay, const float* mass_in, float* mass_out,
                                       void* stream) {
  TwDims d;
  if (int e = tw_check_kv(kv, &d)) return e;
  const bool codes = kv->k_pool == nullptr;
  if (!q || !lse || !mass_in || !mass_out) return TW_EINVAL;
  if (codes && (!kv->kq_pool || !kv->kq_meta || d.bits != 4)) return TW_EINVAL;
  if (window < 1 || num_sinks < 0 || max_new <= 0 || max_new > TW_MAX_NEW || d.max_pages > TW_MAX_ROW_PAGES / 4) return TW_EINVAL;
  if ((long long)max_new * d.batch >= (1ll << 31) || !(decay >= 0.f) || decay > 3.4e38f) return TW_EINVAL;
  const void* k = codes ? kv->kq_pool : kv->k_pool;
  if (((uintptr_t)q | (uintptr_t)k | (codes ? (uintptr_t)kv->kq_meta : 0)) & 15) return TW_EINVAL;
  const int32_t most = 1 << 30;                  // longer than any sequence
  MassArgs a;
  a.q = (const uint4*)q; a.lse = lse; a.k = (const uint4*)k; a.meta = (const uint4*)kv->kq_meta; a.page_table = kv->page_table;
  a.seq_lens = kv->seq_lens; a.n_new = n_new; a.offsets = new_offsets; a.mass_in = mass_in; a.mass_out = mass_out;
  a.Hq = d.Hq; a.Hkv = d.Hkv; a.G = d.G; a.lgG = __builtin_ctz(d.G); a.max_pages = d.max_pages; a.max_new = max_new;
  a.window = std::min(window, most); a.sinks = std::min(num_sinks, most); a.pool_pages = (unsigned)d.pool_pages; a.decay = decay;
  hipStream_t s = (hipStream_t)stream;
  const bool many = (long long)max_new * d.G > 16;
  tw_prof_before(TW_K_MASS, s);
  if (codes) many ? launch_mass<true, true>(a, d.batch, s) : launch_mass<true, false>(a, d.batch, s);
  else many ? launch_mass<false, true>(a, d.batch, s) : launch_mass<false, false>(a, d.batch, s);
  return tw_prof_after(s);
}

extern "C" int twilight_keep_tokens(const twilight_kv_t* kv, const float* mass, const int32_t* budget, int32_t num_sinks, int32_t num_recent,
                                    int32_t* keep_idx, int32_t* keep_count, int32_t keep_stride, float* mass_out, void* ws, size_t ws_bytes, void* stream) {
  TwDims d;
  if (int e = tw_check_kv(kv, &d)) return e;
  if (!mass || !budget || !keep_idx || !keep_count || keep_stride <= 0 || num_sinks < 0 || num_recent < 0 || d.max_pages > TW_MAX_ROW_PAGES) return TW_EINVAL;
  if (((uintptr_t)mass | (uintptr_t)ws) & 15) return TW_EINVAL;
  if (!ws || ws_bytes < tw_keep_workspace(d)) return TW_EWORKSPACE;
  KeepArgs a = {};
  a.mass = mass; a.seq_lens = kv->seq_lens; a.budget = budget; a.idx = keep_idx; a.count = keep_count; a.mass_out = mass_out; a.ws = (uint32_t*)ws;
  a.max_pages = d.max_pages; a.sinks = num_sinks; a.recent = num_recent; a.stride = keep_stride;
  hipStream_t s = (hipStream_t)stream;
  const long long tokens = (long long)d.max_pages * TW_PAGE;
  if (tokens <= WHOLE_TOKENS) {
    tw_prof_before(TW_K_KEEP, s);
    const dim3 grid((unsigned)d.batch);
    if (tokens <= 4096) TW_LAUNCH((keep_whole_kernel<256, 16>), grid, dim3(256), 0, s, a);
    else TW_LAUNCH((keep_whole_kernel<512, 16>), grid, dim3(512), 0, s, a);
    return tw_prof_after(s);
  }
  keep_chunks(d, &a.chunks, &a.blocks);
  const dim3 grid((unsigned)a.chunks, (unsigned)d.batch), block(KEEP_THREADS);
  for (int pass = 0; pass < 4; ++pass) {
    tw_prof_before(TW_K_KEEP, s);
    switch (pass) {
      case 0: TW_LAUNCH(keep_chunk_kernel<0>, grid, block, 0, s, a); break;
      case 1: TW_LAUNCH(keep_chunk_kernel<1>, grid, block, 0, s, a); break;
      case 2: TW_LAUNCH(keep_chunk_kernel<2>, grid, block, 0, s, a); break;
      default: TW_LAUNCH(keep_chunk_kernel<3>, grid, block, 0, s, a); break;
    }
    if (int e = tw_prof_after(s)) return e;
  }
  return TW_OK;
}
