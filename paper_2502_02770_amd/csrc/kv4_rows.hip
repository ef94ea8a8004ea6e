// Rows of a cache that holds K and V in 4 bits: written (twilight_kv4_append) and read back as bf16 (twilight_kv4_read).
//
// A row of 128 dims has a code of 4 bits per dim and an fp16 (scale, zero) per group of 32: 160 bytes for K and V where bf16 has 512.
// One workgroup = one (sequence, KV head, logical page): 16 token slots x 16 lanes, a lane has 8 consecutive dims of K and of V (one
// 16-byte piece, one word of codes each), a quad of lanes a group.
//
// Measured, 4 x 8192 tokens of 8 heads, 176 MB each way: append with bounds 40 us (4.4 TB/s; vector issue, most of it the quantisation step that
// every copy of K shares), read 27 us (6.6 TB/s, codes partly from the last-level cache).  64 single tokens: 4.5 and 2.9 us, trips to memory
// (counts, page, row, bounds) one after the other.
#include "tw_common.h"
#include "kquant_common.h"

namespace {

struct RowArgs4 {
  const uint4* k_new;                            // append: rows in; read: rows out
  const uint4* v_new;
  uint4* k_out;
  uint4* v_out;
  const int32_t* start;
  const int32_t* n_rows;
  const int32_t* offsets;
  const int32_t* page_table;
  const int32_t* seq_lens;
  uint32_t* k_codes;
  uint32_t* k_meta;
  uint32_t* v_codes;
  uint32_t* v_meta;
  uint4* bounds;                                 // or nullptr
  int Hkv, max_pages, most;                      // most: bound of n_rows
  unsigned pool_pages;
};

// The workgroup's page of the rows start .. start + n - 1 of its sequence, and this thread's position in it; false: none.
__device__ __forceinline__ bool page_of(const RowArgs4& a, int b, long long start, long long end, long long* page, long long* tok) {
  if (start < 0 || end <= start) return false;
  const long long lp = start / TW_PAGE + blockIdx.x;
  if (lp * TW_PAGE >= end || lp >= a.max_pages) return false;
  *page = a.page_table[(long long)b * a.max_pages + lp];
  *tok = lp * TW_PAGE + (threadIdx.x >> 4);
  return true;
}

// Two bf16 numbers as two 16-bit integers of the same order, and back: minima and maxima are those of integers, two dims to an instruction,
// and a maximum is the complement of the complements' minimum, so that both go the same way.  (As floats, each operand made a quiet number
// first, and a lane's value from another by way of LDS: 51.5 us for 40, 64 single tokens 6.1 for 4.5.)
typedef short tw_s16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ tw_s16x2 pair_of(uint32_t w) { union { uint32_t u; tw_s16x2 s; } x; x.u = w; return x.s; }
__device__ __forceinline__ uint32_t word_of(tw_s16x2 s) { union { uint32_t u; tw_s16x2 s; } x; x.s = s; return x.u; }
__device__ __forceinline__ uint32_t in_order(uint32_t w) { return w ^ (word_of(pair_of(w) >> 15) & 0x7FFF7FFFu); }
__device__ __forceinline__ uint32_t least(uint32_t x, uint32_t y) { return word_of(__builtin_elementwise_min(pair_of(x), pair_of(y))); }
__device__ __forceinline__ uint32_t largest(uint32_t x, uint32_t y) { return word_of(__builtin_elementwise_max(pair_of(x), pair_of(y))); }
struct Range { float lo, hi; };
// Of a quad's 32 values, eight to a lane
__device__ __forceinline__ Range range_of(const uint32_t (&k)[4]) {
  const uint32_t m = least(least(k[0], k[1]), least(k[2], k[3])), n = ~largest(largest(k[0], k[1]), largest(k[2], k[3]));
  uint32_t w = least(__builtin_amdgcn_perm(n, m, 0x05040100u), __builtin_amdgcn_perm(n, m, 0x07060302u));    // the least; above it the complement of the largest
  w = least(w, (uint32_t)tw_dpp_i<TW_DPP_XOR1>((int)w));
  w = least(w, (uint32_t)tw_dpp_i<TW_DPP_XOR2>((int)w));
  w = in_order(w ^ 0xFFFF0000u);
  return {__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u)};
}

__global__ __launch_bounds__(256) void kv4_append_kernel(RowArgs4 a) {
  const int b = blockIdx.z, h = blockIdx.y, ts = threadIdx.x >> 4, seg = threadIdx.x & 15;
  const long long start = a.start[b], end = start + min(a.n_rows[b], a.most);
  long long page, tok;
  if (!page_of(a, b, start, end, &page, &tok)) return;
  const bool is_new = tok >= start && tok < end;
  // rows, then the page's bounds, on their way before anything waits: a step's few rows are all trips to memory
  uint4 rk = make_uint4(0u, 0u, 0u, 0u), rv = rk, ob = rk;
  if (is_new) {
    const long long row = ((long long)a.offsets[b] + (tok - start)) * a.Hkv + h;
    rk = tw_ld_stream(a.k_new + row * 16 + seg);
    rv = tw_ld_stream(a.v_new + row * 16 + seg);
  }
  if (page < 0 || page >= a.pool_pages) return;
  const long long slot = (page * a.Hkv + h) * TW_PAGE + ts;
  const int which = threadIdx.x >> 4;            // of the threads that write bounds: 0 the lower ones, 1 the upper ones
  uint4* const bounds = a.bounds + (page * a.Hkv + h) * 32 + which * 16 + seg;
  const bool begun = (tok - ts) < start;         // the page has tokens before the new ones
  if (a.bounds && threadIdx.x < 32 && begun) ob = *bounds;
  float x[8], y[8];
  tw_unpack8(rk, x);
  tw_unpack8(rv, y);
  uint32_t wk, wv, none, mk, mv;
  const uint32_t k[4] = {in_order(rk.x), in_order(rk.y), in_order(rk.z), in_order(rk.w)};
  const uint32_t v[4] = {in_order(rv.x), in_order(rv.y), in_order(rv.z), in_order(rv.w)};
  const Range rx = range_of(k), ry = range_of(v);
  tw_quantize_lane8_in<4>(x, rx.lo, rx.hi, seg, &wk, &none, &mk);
  tw_quantize_lane8_in<4>(y, ry.lo, ry.hi, seg, &wv, &none, &mv);
  if (is_new) {
    a.k_codes[slot * 16 + seg] = wk;
    a.v_codes[slot * 16 + seg] = wv;
    if ((seg & 3) == 0) { a.k_meta[slot * 4 + (seg >> 2)] = mk; a.v_meta[slot * 4 + (seg >> 2)] = mv; }
  }
  if (!a.bounds) return;

  // element-wise bounds of K over the page's tokens, of which those before `start` have theirs there
  __shared__ __align__(16) uint32_t red[4][2][16][4];
  const int wave = threadIdx.x >> 6, quarter = (threadIdx.x >> 4) & 3;
  uint32_t w[4];                                 // over the 4 token slots of this wave: the lower half gets the least, the upper one the complement of the largest
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const auto s = __builtin_amdgcn_permlane32_swap(is_new ? k[i] : 0x7FFF7FFFu, is_new ? ~k[i] : 0x7FFF7FFFu, false, false);
    w[i] = least(s[0], s[1]);
  }
#pragma unroll
  for (int i = 0; i < 4; i += 2) {               // of two words, the first to the even quarters
    const auto s = __builtin_amdgcn_permlane16_swap(w[i], w[i + 1], false, false);
    red[wave][quarter >> 1][seg][i + (quarter & 1)] = least(s[0], s[1]);
  }
  __syncthreads();
  if (threadIdx.x >= 32) return;
  auto join = [](const uint4& p, const uint4& q) { return make_uint4(least(p.x, q.x), least(p.y, q.y), least(p.z, q.z), least(p.w, q.w)); };
  auto part = [&](int i) { return *(const uint4*)red[i][which][seg]; };
  const uint32_t turn = which ? ~0u : 0u;
  uint4 x4 = join(join(part(0), part(1)), join(part(2), part(3)));
  if (begun) x4 = join(x4, make_uint4(in_order(ob.x) ^ turn, in_order(ob.y) ^ turn, in_order(ob.z) ^ turn, in_order(ob.w) ^ turn));
  *bounds = make_uint4(in_order(x4.x ^ turn), in_order(x4.y ^ turn), in_order(x4.z ^ turn), in_order(x4.w ^ turn));
}

// 8 codes times scale plus zero, rounded to bf16 (code * scale is exact in fp32, so there is one rounding before that).
__device__ __forceinline__ uint4 values_of(uint32_t w, uint32_t meta) {
  const float s = __half2float(__ushort_as_half((unsigned short)meta)), z = __half2float(__ushort_as_half((unsigned short)(meta >> 16)));
  union { __bf16 e[8]; uint4 v; } x;
#pragma unroll
  for (int i = 0; i < 8; ++i) x.e[i] = (__bf16)__builtin_fmaf((float)((w >> (8 * (i & 3) + 4 * (i >> 2))) & 15u), s, z);
  return x.v;
}

__global__ __launch_bounds__(256) void kv4_read_kernel(RowArgs4 a) {
  const int b = blockIdx.z, h = blockIdx.y, ts = threadIdx.x >> 4, seg = threadIdx.x & 15;
  const long long start = a.start[b], end = min(start + min(a.n_rows[b], a.most), (long long)min(a.seq_lens[b], a.max_pages * TW_PAGE));
  long long page, tok;
  if (!page_of(a, b, start, end, &page, &tok) || tok < start || tok >= end) return;
  const long long row = (((long long)a.offsets[b] + (tok - start)) * a.Hkv + h) * 16 + seg;
  uint4 k = make_uint4(0u, 0u, 0u, 0u), v = k;
  if (page >= 0 && page < a.pool_pages) {
    const long long slot = (page * a.Hkv + h) * TW_PAGE + ts;
    k = values_of(a.k_codes[slot * 16 + seg], a.k_meta[slot * 4 + (seg >> 2)]);
    v = values_of(a.v_codes[slot * 16 + seg], a.v_meta[slot * 4 + (seg >> 2)]);
  }
  tw_st_stream(a.k_out + row, k);
  tw_st_stream(a.v_out + row, v);
}

constexpr int MOST_ROWS = 1 << 27;                // rows of a sequence: a launch has fewer than 2^32 threads along its pages

int rows_args4(const twilight_kv_t* kv, const void* vq_pool, const void* vq_meta, const int32_t* start, const int32_t* n, const int32_t* offsets,
               int32_t most, TwDims* d, RowArgs4* a) {
  if (int e = tw_check_kv(kv, d)) return e;
  if (!kv->kq_pool || !kv->kq_meta || !vq_pool || !vq_meta || !start || !n || !offsets || most < 0 || most > MOST_ROWS || d->bits != 4) return TW_EINVAL;
  if (d->max_pages > TW_MAX_ROW_PAGES) return TW_EINVAL;
  if (((uintptr_t)kv->kq_pool | (uintptr_t)kv->kq_meta | (uintptr_t)vq_pool | (uintptr_t)vq_meta | (uintptr_t)kv->page_minmax) & 15) return TW_EINVAL;
  *a = RowArgs4{};
  a->start = start; a->n_rows = n; a->offsets = offsets; a->page_table = kv->page_table; a->seq_lens = kv->seq_lens;
  a->k_codes = (uint32_t*)kv->kq_pool; a->k_meta = (uint32_t*)kv->kq_meta; a->v_codes = (uint32_t*)vq_pool; a->v_meta = (uint32_t*)vq_meta;
  a->Hkv = d->Hkv; a->max_pages = d->max_pages; a->most = most; a->pool_pages = (unsigned)d->pool_pages;
  return TW_OK;
}

// pages that `most` rows starting anywhere inside a page touch
unsigned pages_touched(const TwDims& d, int most) {
  const long long n = ((long long)most + TW_PAGE - 1) / TW_PAGE + 1;
  return (unsigned)(n < d.max_pages ? n : d.max_pages);
}

}  // namespace

extern "C" int twilight_kv4_append(const twilight_kv_t* kv, void* vq_pool, void* vq_meta, const void* k_new, const void* v_new,
                                   const int32_t* start_pos, const int32_t* n_new, const int32_t* new_offsets, int32_t max_new, void* stream) {
  TwDims d;
  RowArgs4 a;
  if (int e = rows_args4(kv, vq_pool, vq_meta, start_pos, n_new, new_offsets, max_new, &d, &a)) return e;
  if (!k_new || !v_new || (((uintptr_t)k_new | (uintptr_t)v_new) & 15)) return TW_EINVAL;
  if (max_new == 0) return TW_OK;
  a.k_new = (const uint4*)k_new; a.v_new = (const uint4*)v_new; a.bounds = (uint4*)kv->page_minmax;
  hipStream_t s = (hipStream_t)stream;
  tw_prof_before(TW_K_KV4_APPEND, s);
  TW_LAUNCH(kv4_append_kernel, dim3(pages_touched(d, max_new), (unsigned)d.Hkv, (unsigned)d.batch), dim3(256), 0, s, a);
  return tw_prof_after(s);
}

extern "C" int twilight_kv4_read(const twilight_kv_t* kv, const void* vq_pool, const void* vq_meta, const int32_t* start_pos, const int32_t* n_rows,
                                 const int32_t* row_offsets, int32_t max_rows, void* k_out, void* v_out, void* stream) {
  TwDims d;
  RowArgs4 a;
  if (int e = rows_args4(kv, vq_pool, vq_meta, start_pos, n_rows, row_offsets, max_rows, &d, &a)) return e;
  if (!k_out || !v_out || (((uintptr_t)k_out | (uintptr_t)v_out) & 15)) return TW_EINVAL;
  if (max_rows == 0) return TW_OK;
  a.k_out = (uint4*)k_out; a.v_out = (uint4*)v_out;
  hipStream_t s = (hipStream_t)stream;
  tw_prof_before(TW_K_KV4_READ, s);
  TW_LAUNCH(kv4_read_kernel, dim3(pages_touched(d, max_rows), (unsigned)d.Hkv, (unsigned)d.batch), dim3(256), 0, s, a);
  return tw_prof_after(s);
}
