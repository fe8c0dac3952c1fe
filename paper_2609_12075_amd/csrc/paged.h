// Kernel arguments and launchers of the paged key/value cache.
#pragma once
#include "common.h"

// The pool and the batch as the kernels see them (include/vla_paged.h).
struct PagedKV {
  const void *k, *v;
  long page_stride, head_stride, tok_stride;   // elements
  int n_kv, hd, n_pages, page_shift;           // page_tokens = 1 << page_shift
};
struct RaggedBatch {
  const int32_t *start, *kv_len, *pages;
  int n_req, n_tok, max_new, max_len, pages_stride;
};

struct AppendArgs {
  PagedKV kv;
  RaggedBatch bt;
  const void *kin, *vin, *q;
  void* qo;
  long k_ts, k_hs, v_ts, v_hs, q_ts, q_hs, qo_ts, qo_hs;
  int n_q, n_axes, s1, s2;                     // pairs of axis 0 end at s1, of axis 1 at s2
  int half;                                    // pairs (0: no rotation)
  const int32_t* pos;
  double step;                                 // -log2(rope_base) / half
};
void launch_append(const AppendArgs& a, int et, hipStream_t s);

struct PagedAttnArgs {
  PagedKV kv;
  RaggedBatch bt;
  const void* q;
  void* o;
  long q_ts, q_hs, o_ts, o_hs;
  float* lse;
  int n_q, G;                                  // G = n_q / n_kv
  float scale, cap;
  int causal, window;
  const int32_t* prefix;
  int shared_len;                              // keys below it lie on the pages of request 0
  // Scratch: unnormalised outputs [n_tok][n_q][slots][hd], then (reference of
  // the weights in log2 units, sum) pairs [n_tok][n_q][slots], fp32. A sum of -1 in slot 0: the
  // row's output is written already.
  float* ws;
  // set by the launcher, per launch
  int klo, khi;                                // keys [klo, khi) only
  int tiles;                                   // row tiles of the grid
  int chunk;                                   // key tiles per range
  int ranges, slot0, slots;                    // ranges of this launch, its first slot, slots of a row
  int direct;                                  // rows whose keys fit one range are written at once
  unsigned mul_g, mul_kv, mul_blocks;          // ceil(2^32 / d) for d = G, n_kv and tiles * n_kv (0: d = 1)
};

// How an attention is computed. PAGED_KEYS: a block owns 16 rows (token, query
// head of the group), its waves split the keys; PAGED_ROWS: its waves split 128
// rows; PAGED_ROWS2: so do two groups of waves, which split the keys;
// PAGED_ROWS8: eight waves split 256 rows; PAGED_F32: fp32, 16 rows, waves
// split the keys, PAGED_F32R: 64 rows (32 at head dim 128). One part over the cache, or two: the common context (all rows
// of the batch in one sequence of tiles) and what follows it.
enum PagedKernel { PAGED_KEYS = 0, PAGED_ROWS = 1, PAGED_F32 = 2, PAGED_ROWS2 = 3, PAGED_ROWS8 = 4, PAGED_F32R = 5 };
struct PagedPart { int kernel, tiles, chunk, ranges; };
struct PagedPlan { int n_parts, hdp, slots; PagedPart part[2]; };
PagedPlan paged_plan(const PagedAttnArgs& a, int et);
size_t paged_attention_ws(const PagedAttnArgs& a, const PagedPlan& p);
void launch_paged_attention(const PagedAttnArgs& a, const PagedPlan& p, int et, hipStream_t s);

// ---------------------------------------------------------------- device side
struct ReqSpan { int first, n, len; };         // first row, new tokens, tokens in the cache

// n / d for mul = ceil(2^32 / d) and n < 2^31: the product's high word is the
// quotient or one more.
__device__ __forceinline__ int div_by(int n, int d, unsigned mul) {
  if (mul == 0) return n;
  const int q = (int)__umulhi((unsigned)n, mul);
  return q - (q * d > n);
}

// A request's rows and lengths from start[r], start[r + 1] and kv_len[r], cut to
// the stated bounds.
__device__ __forceinline__ ReqSpan span_of(const RaggedBatch& b, int s0, int s1, int len, int page_shift) {
  ReqSpan p;
  p.first = s0 < 0 ? 0 : (s0 > b.n_tok ? b.n_tok : s0);
  const int e = s1 > b.n_tok ? b.n_tok : s1;
  p.n = e - p.first;
  if (p.n > b.max_new) p.n = b.max_new;
  if (p.n < 0) p.n = 0;
  const long cap = (long)b.pages_stride << page_shift;
  if (len > b.max_len) len = b.max_len;
  if (len > cap) len = (int)cap;
  p.len = len < 0 ? 0 : len;
  return p;
}

__device__ __forceinline__ ReqSpan span_of(const RaggedBatch& b, int r, int page_shift) {
  return span_of(b, b.start[r], b.start[r + 1], b.kv_len[r], page_shift);
}

// The request of a token: the last r with start[r] <= tok (requests without
// tokens share their start with the next one); n_req when tok lies behind the
// last. A wavefront looks at 64 starts at a time, so up to 4095 requests take
// two rounds of loads. Wave-uniform tok; all lanes of the wave call it.
__device__ __forceinline__ int request_of(const RaggedBatch& b, int tok) {
  const int lane = threadIdx.x & 63;
  int lo = 0, n = b.n_req + 1;                 // start[lo] <= tok is known or assumed
  while (n > 1) {
    const int step = (n + 63) / 64, i = lo + lane * step;
    const bool le = i < lo + n && b.start[i] <= tok;
    const unsigned long long m = __ballot(le);
    if (m == 0) return b.n_req;                // (starts that do not begin at 0)
    const int last = 63 - __builtin_clzll(m);
    const int end = lo + n;
    lo += last * step;
    n = end - lo < step ? end - lo : step;
  }
  return lo;
}

// The same for a token of each lane's own.
__device__ __forceinline__ int lane_request_of(const RaggedBatch& b, int tok) {
  // one token a request is the usual batch
  if (tok < b.n_req && b.start[tok] <= tok && tok < b.start[tok + 1]) return tok;
  int lo = 0, hi = b.n_req;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (b.start[mid] <= tok) lo = mid;
    else hi = mid;
  }
  return lo;
}
