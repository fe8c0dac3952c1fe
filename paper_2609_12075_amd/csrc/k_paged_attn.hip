// Attention over a paged key/value cache on gfx950.
//
// Rows are (token, query head of a KV head's group) pairs in token-major
// order, so the query heads that share a KV head read its keys once and a tile
// of rows spans few places. Both products run on the matrix cores (bf16: 16 x 16
// tiles where rows are few, 32 x 32 in prompts). The scores are computed transposed
// (S^T = K Q^T): a lane holds keys of one row only, so the row statistics need
// one exchange between the lane halves, and the probabilities are the second
// product's operand as they are (its key order inside 16 keys permuted alike
// on the V side). Softmax is online in fp32, in log2 units.
//
// A key range of a row tile is a list of key tiles: those below the prefix,
// then those of the window and the causal part; tiles that no row of a block
// sees are not in it. Only tiles at a border of some row's keys are masked
// element by element. Ranges of one tile of rows go to different blocks where
// the rows alone would not fill the chip, and are merged by a second kernel.
#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <type_traits>

#include "paged.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.69314718055994531f;

// 16 zero bytes: what 16-byte pieces behind the last key or head_dim read
static __device__ __align__(16) unsigned char zero_piece[16];

// ---------------------------------------------------------------- rows and their keys
// Row r of a tile sees key j (of the launch's [klo, khi)) when j < pre or lo <= j < hi.
struct Limits { int pre, lo, hi; };

// What a block computes: rows row0 .. of the nrows rows of request r (or of the
// batch), the list of key tiles [ubeg, uend) of them, and where results go.
struct Item {
  int g, r, row0, nrows, first, place0, len, prefix;
  int klim;                                    // keys from here on are not read
  int n1, t2, ntiles;                          // tile list: 0 .. n1 - 1, then t2 ..
  int ubeg, uend, slot;
  const int32_t* pages;
};

__device__ __forceinline__ Limits limits(const PagedAttnArgs& a, int p, int len, int prefix) {
  Limits m;
  if (!a.causal) {
    m.pre = min(len, a.khi);
    m.lo = m.hi = 0;
    return m;
  }
  m.pre = min(min(prefix, len), a.khi);
  m.lo = max(a.klo, a.window ? p - a.window + 1 : 0);
  m.hi = min(min(p + 1, len), a.khi);
  return m;
}

// Uniform reads of the batch's description: through the scalar cache, several
// at a time (nobody writes them while a kernel runs).
__device__ __forceinline__ int fetch(const int32_t* p, long i) {
  typedef const __attribute__((address_space(4))) int32_t* C;
  return *(C)(uintptr_t)(p + i);
}

// What block L (KV heads fastest: with eight of them, one on each die) and key
// range `range` compute; false: nothing. KT keys a tile; lists of keys below
// the prefix are padded to PAD tiles, so that PAD neighbours of a list are
// neighbours in the cache. FLAT: the rows of the whole batch in one sequence of
// tiles, over pages of request 0.
template <int BR, int KT, int PAD, bool FLAT>
__device__ __forceinline__ bool find_item(const PagedAttnArgs& a, int L, int range, Item& it) {
  const RaggedBatch& bt = a.bt;
  const int v = div_by(L, a.kv.n_kv, a.mul_kv);
  it.g = L - v * a.kv.n_kv;
  it.slot = a.slot0 + range;
  if constexpr (FLAT) {
    const int s0 = max(0, fetch(bt.start, 0)), s1 = min(bt.n_tok, fetch(bt.start, bt.n_req));
    it.r = 0;
    it.first = s0;
    it.nrows = (s1 - s0) * a.G;
    it.row0 = v * BR;
    it.len = it.klim = a.khi;
    it.place0 = it.prefix = 0;
    it.pages = bt.pages;
    if (it.row0 >= it.nrows) return false;
    it.n1 = it.ntiles = (unsigned)(a.khi - a.klo + KT - 1) / KT;
    it.t2 = it.n1;
  } else {
    // causal row tiles get longer: the long ones first
    const int tile = a.causal ? a.tiles - 1 - v : v;
    int t = 0;
    if (bt.max_new * a.G <= BR) {
      it.r = tile;
    } else {
      // request r's tiles begin at start[r] G / BR + r, which leaves room for all of them; the last that begins
      // at or before `tile`
      const int lane = threadIdx.x & 63;
      int lo = 0, n = bt.n_req;
      while (n > 1) {
        const int step = (n + 63) / 64, i = lo + lane * step;
        const bool le = i < lo + n && (int)((long)bt.start[i] * a.G / BR) + i <= tile;
        const unsigned long long m = __ballot(le);
        if (m == 0) break;
        const int last = 63 - __builtin_clzll(m), end = lo + n;
        lo += last * step;
        n = min(step, end - lo);
      }
      it.r = __builtin_amdgcn_readfirstlane(lo);
    }
    const int s0 = fetch(bt.start, it.r), s1 = fetch(bt.start, it.r + 1), kl = fetch(bt.kv_len, it.r);
    const int pf = fetch(a.prefix ? a.prefix : bt.kv_len, it.r);
    it.prefix = a.prefix ? pf : 0;
    if (bt.max_new * a.G > BR) t = tile - ((int)((long)s0 * a.G / BR) + it.r);
    const ReqSpan sp = span_of(bt, s0, s1, kl, a.kv.page_shift);
    it.first = sp.first;
    it.nrows = sp.n * a.G;
    it.row0 = t * BR;
    if (t < 0 || it.row0 >= it.nrows) return false;
    it.len = sp.len;
    it.place0 = sp.len - sp.n;
    it.klim = min(sp.len, a.khi);
    it.pages = bt.pages + (long)it.r * bt.pages_stride;
    const int last = min(it.row0 + BR, it.nrows) - 1;
    const Limits m0 = limits(a, it.place0 + div_by(it.row0, a.G, a.mul_g), it.len, it.prefix);
    const Limits m1 = limits(a, it.place0 + div_by(last, a.G, a.mul_g), it.len, it.prefix);
    it.n1 = (unsigned)(max(0, m0.pre - a.klo) + KT * PAD - 1) / (KT * PAD) * PAD;
    it.t2 = max(it.n1, (int)((unsigned)max(0, m0.lo - a.klo) / KT));
    const int t2e = (unsigned)(max(0, m1.hi - a.klo) + KT - 1) / KT;
    it.ntiles = it.n1 + max(0, t2e - it.t2);
  }
  it.ubeg = range * a.chunk;
  it.uend = min(it.ntiles, it.ubeg + a.chunk);
  return true;
}

struct Row { int tok, head; Limits lim; };

// Row `row` of the item (rows behind the last one stand for the last one).
template <bool FLAT>
__device__ __forceinline__ Row row_of(const PagedAttnArgs& a, const Item& it, int row) {
  Row w;
  const int rc = min(row, it.nrows - 1), t = div_by(rc, a.G, a.mul_g);
  w.tok = it.first + t;
  w.head = it.g * a.G + rc - t * a.G;
  if constexpr (FLAT) {
    const int r = lane_request_of(a.bt, w.tok);
    const ReqSpan sp = span_of(a.bt, r, a.kv.page_shift);
    w.lim = limits(a, sp.len - sp.n + w.tok - sp.first, sp.len, a.prefix ? a.prefix[r] : 0);
  } else {
    w.lim = limits(a, it.place0 + t, it.len, it.prefix);
  }
  return w;
}

__device__ __forceinline__ bool sees(const Limits& m, int j) {
  return (j < m.pre) | ((unsigned)(j - m.lo) < (unsigned)max(0, m.hi - m.lo));
}

// The least and largest limits of a wave's rows, for the test of whole tiles.
struct WaveLimits { int pre0, pre1, lo0, lo1, hi0, hi1; };

template <int ROWS, bool FLAT>
__device__ __forceinline__ WaveLimits wave_limits(const PagedAttnArgs& a, const Limits& m) {
  WaveLimits w;
  if constexpr (FLAT) {
    w = {m.pre, m.pre, m.lo, m.lo, m.hi, m.hi};
#pragma unroll
    for (int o = ROWS / 2; o > 0; o >>= 1) {
      w.pre0 = min(w.pre0, __shfl_xor(w.pre0, o)); w.pre1 = max(w.pre1, __shfl_xor(w.pre1, o));
      w.lo0 = min(w.lo0, __shfl_xor(w.lo0, o)); w.lo1 = max(w.lo1, __shfl_xor(w.lo1, o));
      w.hi0 = min(w.hi0, __shfl_xor(w.hi0, o)); w.hi1 = max(w.hi1, __shfl_xor(w.hi1, o));
    }
    w = {__builtin_amdgcn_readfirstlane(w.pre0), __builtin_amdgcn_readfirstlane(w.pre1),
         __builtin_amdgcn_readfirstlane(w.lo0), __builtin_amdgcn_readfirstlane(w.lo1),
         __builtin_amdgcn_readfirstlane(w.hi0), __builtin_amdgcn_readfirstlane(w.hi1)};
  } else {                                     // limits ascend with the row
    w.pre0 = w.pre1 = __builtin_amdgcn_readfirstlane(m.pre);
    w.lo0 = __builtin_amdgcn_readfirstlane(m.lo);
    w.hi0 = __builtin_amdgcn_readfirstlane(m.hi);
    w.lo1 = __builtin_amdgcn_readlane(m.lo, ROWS - 1);
    w.hi1 = __builtin_amdgcn_readlane(m.hi, ROWS - 1);
  }
  return w;
}
__device__ __forceinline__ bool tile_full(const WaveLimits& w, int k0, int k1) {
  return k1 <= w.pre0 || (k0 >= w.lo1 && k1 <= w.hi0);
}
__device__ __forceinline__ bool tile_unseen(const WaveLimits& w, int k0, int k1) {
  return k0 >= w.pre1 && (k0 >= w.hi1 || k1 <= w.lo0);
}

// ---------------------------------------------------------------- small pieces
// The maximum that passes a NaN on, in one instruction.
__device__ __forceinline__ float vmax(float a, float b) { return __builtin_elementwise_maximum(a, b); }
__device__ __forceinline__ float other_half(float v, float& mine) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  mine = __uint_as_float(r[0]);
  return __uint_as_float(r[1]);
}
__device__ __forceinline__ float max_x32(float v) { float m; const float o = other_half(v, m); return vmax(m, o); }
__device__ __forceinline__ float sum_x32(float v) { float m; const float o = other_half(v, m); return m + o; }

// The capped score in log2 units: cap tanh(s scale / cap) log2 e, with
// tanh(x) = 1 - 2 / (1 + e^2x); c1 = 2 scale log2 e / cap, c2 = cap log2 e.
// (hardware exp2 and reciprocal: off by a few 2^-24 of the cap)
__device__ __forceinline__ float capped(float s, float c1, float c2) {
  return c2 - 2.f * c2 * __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(s * c1));
}

// The element offset of a page for this KV head, or -1 where it is not there.
__device__ __forceinline__ long page_offset(const PagedAttnArgs& a, int id, int g) {
  return (unsigned)id < (unsigned)a.kv.n_pages ? (long)id * a.kv.page_stride + (long)g * a.kv.head_stride : -1;
}

__device__ __forceinline__ void store_stats(const PagedAttnArgs& a, long row, int slot, float m, float l) {
  float* st = a.ws + (long)a.bt.n_tok * a.n_q * a.slots * a.kv.hd + (row * a.slots + slot) * 2;
  st[0] = m;
  st[1] = l;
}
__device__ __forceinline__ float* part_of(const PagedAttnArgs& a, long row, int slot) {
  return a.ws + (row * a.slots + slot) * a.kv.hd;
}

// A range without keys: its statistics say so. (Whole blocks; rows split over the block's threads.)
template <int BR>
__device__ __forceinline__ void empty_range(const PagedAttnArgs& a, const Item& it) {
  for (int i = threadIdx.x; i < BR; i += blockDim.x) {
    const int row = it.row0 + i;
    if (row >= it.nrows) break;
    const int t = div_by(row, a.G, a.mul_g);
    store_stats(a, (long)(it.first + t) * a.n_q + it.g * a.G + row - t * a.G, it.slot, -INFINITY, 0.f);
  }
}

// ---------------------------------------------------------------- bf16 tiles in LDS
// Tiles of K and V are key-major rows of HDP elements; the 16-byte piece c of
// row r sits in slot c ^ swz(r). LDS answers 256 bytes a cycle where they lie in
// different banks: one piece of 16 rows (the scores' operand), 64 bytes of four
// rows or 32 of eight (the transposing reads of 32 or 16 dims). The row's number
// with its bits reversed spreads all three: the lowest bit moves a row by half
// of the banks, the next by a quarter. (Unreversed, the transposing reads took
// four times as long and LDS was busy for half of a long prompt's time.)
// Tiles move global -> LDS with the direct loads (lane l's 16 bytes at LDS base + 16 l).
template <int HDP>
struct Lay {
  static constexpr int CR = HDP / 8, ROWB = HDP * 2, SW = CR >= 16 ? 0 : 1;   // (two rows of 64 dims are as wide as the banks)
  __device__ static constexpr unsigned swz(unsigned r) { return __builtin_bitreverse32(r >> SW << (28 + SW)) & (15u >> SW); }
};

__device__ __forceinline__ unsigned lds_addr(const void* p) {
  return (unsigned)(uintptr_t)(const __attribute__((address_space(3))) char*)(p);
}

// 16 bytes a lane, global -> LDS (wave-uniform dst + 16 lane). Written out: the
// compiler, which cannot tell the slots of a ring apart, waits for all of its
// own direct loads before each LDS read; these loads' waits are in the loops.
__device__ __forceinline__ void dma16(const void* src, unsigned dst) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(src), "s"(dst) : "memory", "m0");
}

// The same from a wave-uniform base and 32-bit offsets of the lanes.
__device__ __forceinline__ void dma16(const char* base, unsigned off, unsigned dst) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(dst) : "memory", "m0");
}

// V^T fragments of a 16-key group: subtile u (32 dims) holds, of lane l, dim
// l % 32 of keys 4 (l / 32) + 0..3 and + 8..11: two transposing reads of four
// keys each. at: the lane's byte address of subtile 0's first read; off: bytes
// to the group.
typedef short v4s __attribute__((ext_vector_type(4)));
__device__ __forceinline__ bf16x4 read_tr(unsigned at) {
  typedef __attribute__((address_space(3))) v4s* P;
  return __builtin_bit_cast(bf16x4, __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)at));
}
template <int HDP>
__device__ __forceinline__ bf16x8 read_vt(unsigned at, int u, int off) {
  // (eight rows further the swizzle differs in its lowest bit)
  const bf16x4 l = read_tr((at ^ (u % 4 << 6)) + off + u / 4 * 256),
               h = read_tr((at ^ (u % 4 << 6) ^ 16) + off + u / 4 * 256 + 8 * Lay<HDP>::ROWB);
  return __builtin_shufflevector(l, h, 0, 1, 2, 3, 4, 5, 6, 7);
}
// The lane's first byte for read_vt within a tile.
template <int HDP>
__device__ __forceinline__ unsigned vt_address() {
  const int lane = threadIdx.x & 63, s = lane & 15, r = 4 * (lane >> 5) + (s >> 2);
  const int c = 2 * ((lane >> 4) & 1) + ((s & 3) >> 1);
  return r * Lay<HDP>::ROWB + ((c ^ Lay<HDP>::swz(r)) << 4) + ((s & 1) << 3);
}
// 16 bytes of a key row: 8 dims from 16 c on (and 8 of the lane half).
__device__ __forceinline__ bf16x8 read_k(unsigned at, int c, int off) {
  typedef const __attribute__((address_space(3))) bf16x8* P;
  return *(P)(uintptr_t)((at ^ (c % 8 << 5)) + off + c / 8 * 256);
}

// The window of page offsets a block keeps in LDS (bytes from the pool's bases
// of this KV head's rows; -1: not there), entries w0 .. w0 + PW - 1.
constexpr int PW = 256;

// Fills the window of page offsets from entry e0 on; true where one of its pages
// below the item's last key is not there, whether some row sees its keys or not
// (the block then looks the pages of its keys up one by one, in all tiles from
// there on: 8000 keys behind a window of 1024, one token of 32 heads of 128,
// 13.4 us with the pages before the window given back, 11.7 with all there).
// (all threads of the block, at least PW, call it, and none reads the window or the flags
// of an earlier call any more; ends with a barrier; `guessed`: this
// thread's entry of the window from entry `guess` on, requested earlier)
struct Window { long off[PW]; int flag[8]; };

template <int THREADS>
__device__ __forceinline__ bool fill_window(const PagedAttnArgs& a, const Item& it, Window& win, int e0, int guess = -1,
                                            int guessed = 0) {
  const int n = (it.klim + (1 << a.kv.page_shift) - 1) >> a.kv.page_shift, i = threadIdx.x;
  bool bad = false;
  if (THREADS == PW || i < PW) {
    long off = -1;
    if (e0 + i < n) {
      off = page_offset(a, e0 == guess ? guessed : it.pages[e0 + i], it.g);
      bad = off < 0;
      off = off < 0 ? -1 : off * 2;
    }
    win.off[i] = off;
  }
  const bool any = __ballot(bad) != 0;
  if ((threadIdx.x & 63) == 0) win.flag[threadIdx.x >> 6] = any;
  __syncthreads();
  int f = 0;
#pragma unroll
  for (int w = 0; w < PW / 64; ++w) f |= win.flag[w];
  return f != 0;
}

// Moves a wave's share of a tile of KT key rows into LDS: NWV waves share a
// tile, load j of the tile (RS rows) belongs to wave j % NWV.
template <int HDP, int KT, int NWV>
struct Mover {
  using Y = Lay<HDP>;
  static constexpr int RS = 64 / Y::CR, N = KT / RS / NWV, ROWS = N * RS;
  unsigned lrow, piece, wave, ts2, smask;
  int shift, hd;
  const Window* win;
  // where the row of each lane begins (lane l: row l % ROWS of the wave's), and whether it is there
  long at;
  bool ok;

  __device__ __forceinline__ Mover(const PagedAttnArgs& a, const Window& w, int wv) {
    const unsigned lane = threadIdx.x & 63;
    lrow = lane / Y::CR;
    piece = ((lane % Y::CR) ^ Y::swz(lrow)) << 4;
    wave = wv;
    ts2 = (unsigned)(a.kv.tok_stride * 2);
    shift = a.kv.page_shift;
    smask = (1u << shift) - 1;
    hd = a.kv.hd;
    win = &w;
  }
  // the rows of the tile at key k0 (window from entry w0; keys from klim on are zeros)
  __device__ __forceinline__ void rows(int k0, int w0, int klim) {
    const int l = (threadIdx.x & 63) % ROWS, kk = k0 + (l / RS * NWV + (int)wave) * RS + l % RS;
    const long off = win->off[max(0, (min(kk, klim - 1) >> shift) - w0)];
    at = off + (unsigned long)(kk & smask) * ts2;
    ok = (kk < klim) & (off >= 0);
  }
  template <bool BOTH>
  __device__ __forceinline__ void load(const char* kb, const char* vb, unsigned dst_k, unsigned dst_v) const {
    // all rows there, each load's rows in one page: bases are scalars
    if (__ballot(ok) == ~0ull && shift >= __builtin_ctz(RS) && hd == HDP) {
      const int lo = (int)at, hi = (int)(at >> 32);
      const unsigned row = lrow * ts2;
      // (long unrolled code is read from memory in each launch: at a few
      // cycles an instruction a loop of four is faster than 16 in a row)
#pragma unroll 4
      for (int i = 0; i < N; ++i) {
        const unsigned j = i * NWV + wave, off = row + (piece ^ (Y::swz(j * RS) << 4));
        const long b = (long)((unsigned long)(unsigned)__builtin_amdgcn_readlane(hi, i * RS) << 32 |
                              (unsigned)__builtin_amdgcn_readlane(lo, i * RS));
        dma16(kb + b, off, dst_k + j * 1024);
        if constexpr (BOTH) dma16(vb + b, off, dst_v + j * 1024);
      }
    } else {
#pragma unroll 1
      for (int i = 0; i < N; ++i) {
        const unsigned j = i * NWV + wave, c = piece ^ (Y::swz(j * RS) << 4);
        const int src = i * RS + lrow;
        const long b = __shfl(at, src) + c;
        const bool there = __shfl((int)ok, src) & (c < 2u * hd);
        const char* z = reinterpret_cast<const char*>(zero_piece);
        dma16(there ? kb + b : z, dst_k + j * 1024);
        if constexpr (BOTH) dma16(there ? vb + b : z, dst_v + j * 1024);
      }
    }
  }
};

// ---------------------------------------------------------------- bf16, common
// State of a wave: 32 rows, all dims.
template <int HDP>
struct Acc {
  f32x16 o[HDP / 32];
  float m, l;                                  // m: reference of the exponents (log2); l: this lane's keys
};

// One tile of 16 N keys' scores into weights: cap, mask, running maximum, sum.
// sc[st][i] is key 32 st + 8 (i / 4) + 4 (lane / 32) + i % 4 of the tile.
template <int HDP, int NS, bool CAP>
__device__ __forceinline__ void softmax_tile(Acc<HDP>& s, f32x16 (&sc)[NS], float sl2, float c1, float c2, bool full,
                                             const Limits& lim, int k0, const PagedAttnArgs& a, const Item& it,
                                             bool holes) {
  const int h4 = (threadIdx.x & 32) >> 3;
  if constexpr (CAP) {
#pragma unroll
    for (int st = 0; st < NS; ++st)
#pragma unroll
      for (int i = 0; i < 16; ++i) sc[st][i] = capped(sc[st][i], c1, c2);
  }
  if (!full) {
#pragma unroll
    for (int st = 0; st < NS; ++st)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (!sees(lim, k0 + st * 32 + (i / 4) * 8 + h4 + i % 4)) sc[st][i] = -INFINITY;
    if (holes) {
      unsigned gone = 0;
#pragma unroll 1
      for (int i = 0; i < 16 * NS; ++i) {
        const int j = min(k0 + (i / 4) * 8 + h4 + i % 4, it.klim - 1);
        gone |= (unsigned)((unsigned)it.pages[j >> a.kv.page_shift] >= (unsigned)a.kv.n_pages) << i;
      }
#pragma unroll
      for (int i = 0; i < 16 * NS; ++i)
        if (gone >> i & 1) sc[i / 16][i % 16] = -INFINITY;
    }
  }
  float mx = sc[0][0];
#pragma unroll
  for (int i = 1; i < 16 * NS; ++i) mx = vmax(mx, sc[i / 16][i % 16]);
  mx = max_x32(mx);
  if constexpr (!CAP) mx *= sl2;
  // The reference is put 2^8 above a row's maximum and moves only where a score
  // passes it (or the row saw its first key): the outputs are rescaled rarely
  // then, no weight is above 1 (weights of 2^8 would let values overflow that
  // a sum of weights of at most 1 holds), and a row's largest weight, 2^-8 or
  // more, loses nothing in fp32 or, rounded, in bf16. Rows that have seen
  // nothing take a reference of 0: no -inf - -inf.
  if (__ballot(mx > s.m)) {
    const float mn = vmax(s.m, mx + 8.f), alpha = __builtin_amdgcn_exp2f(s.m - (mn == -INFINITY ? 0.f : mn));
    s.m = mn;
    s.l *= alpha;
#pragma unroll
    for (int u = 0; u < HDP / 32; ++u) s.o[u] *= alpha;
  }
  const float ref = s.m == -INFINITY ? 0.f : s.m;
  float ps[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int st = 0; st < NS; ++st)
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const float x = CAP ? sc[st][i] - ref : __builtin_fmaf(sc[st][i], sl2, -ref);
      const float p = __builtin_amdgcn_exp2f(x);
      sc[st][i] = p;
      ps[i % 4] += p;
    }
  // (the sum takes the weights before their rounding to bf16: one rounding less)
  s.l += (ps[0] + ps[1]) + (ps[2] + ps[3]);
}

__device__ __forceinline__ bf16x8 weights_of(const f32x16& s, int c) {
  bf16x8 p;
#pragma unroll
  for (int e = 0; e < 8; ++e) p[e] = (bf16)s[8 * c + e];
  return p;
}

// A wave whose outputs are not all finite adds its rows again key by key: a
// weight of zero times an infinite (or NaN) value that the row does not see is
// a NaN in the products above. `tile(n)`: first key of the wave's n-th tile.
template <int HDP, bool CAP, typename Tile>
__device__ __forceinline__ void repair(const PagedAttnArgs& a, const Item& it, Acc<HDP>& s, const bf16x8 (&qf)[HDP / 16],
                                       const Limits& lim, float sl2, float c1, float c2, int ntiles, int kt, Tile tile) {
  float z = 0.f;
#pragma unroll
  for (int u = 0; u < HDP / 32; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) z = __builtin_fmaf(s.o[u][i], 0.f, z);
  if (__ballot(z != z) == 0) return;
  const int h = (threadIdx.x & 32) >> 5, hd = a.kv.hd;
  const float ref = s.m == -INFINITY ? 0.f : s.m;
#pragma unroll
  for (int u = 0; u < HDP / 32; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) s.o[u][i] = 0.f;
#pragma unroll 1
  for (int n = 0; n < ntiles; ++n) {
    const int k0 = tile(n);
#pragma unroll 1
    for (int j = k0; j < min(k0 + kt, it.klim); ++j) {
      const bool vis = sees(lim, j);
      if (__ballot(vis) == 0) continue;
      const long off = page_offset(a, it.pages[j >> a.kv.page_shift], it.g);
      if (off < 0) continue;
      const long at = off + (long)(j & ((1 << a.kv.page_shift) - 1)) * a.kv.tok_stride;
      const bf16 *kp = reinterpret_cast<const bf16*>(a.kv.k) + at, *vp = reinterpret_cast<const bf16*>(a.kv.v) + at;
      float d = 0.f;
#pragma unroll
      for (int c = 0; c < HDP / 16; ++c)
        if (16 * c + 8 * h < hd) {
          const bf16x8 x = *reinterpret_cast<const bf16x8*>(kp + 16 * c + 8 * h);
#pragma unroll
          for (int e = 0; e < 8; ++e) d = __builtin_fmaf((float)x[e], (float)qf[c][e], d);
        }
      d = sum_x32(d);
      const float p = __builtin_amdgcn_exp2f((CAP ? capped(d, c1, c2) : d * sl2) - ref);
#pragma unroll
      for (int u = 0; u < HDP / 32; ++u)
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int dim = 32 * u + 8 * q + 4 * h;
          if (dim < hd && vis) {
            const bf16x4 x = *reinterpret_cast<const bf16x4*>(vp + dim);
#pragma unroll
            for (int e = 0; e < 4; ++e) s.o[u][4 * q + e] = __builtin_fmaf(p, (float)x[e], s.o[u][4 * q + e]);
          }
        }
    }
  }
}

// A lane's pieces of a query row: 8 dims every STEP; pieces from `end` dims on
// are not there (their loads read the row's first piece).
template <int N, int STEP>
__device__ __forceinline__ void load_q(const bf16* row, int first, int end, bf16x8 (&q)[N]) {
#pragma unroll
  for (int c = 0; c < N; ++c) {
    const int d = first + STEP * c;
    q[c] = *reinterpret_cast<const bf16x8*>(row + (d < end ? d : 0));
  }
}
// The queries are in registers from here on (else the compiler, which does not
// know the waits of the loop, waits for all loads before each use of them), and
// pieces that are not there are zeros.
template <int N, int STEP>
__device__ __forceinline__ void hold(int first, int end, bool whole, bf16x8 (&q)[N]) {
#pragma unroll
  for (int c = 0; c < N; ++c) asm volatile("" : "+v"(q[c]));
  if (!whole) {
#pragma unroll
    for (int c = 0; c < N; ++c)
      if (first + STEP * c >= end) q[c] = bf16x8{};
  }
}
// The kernel's arguments that are needed late are requested with the first.
__device__ __forceinline__ void touch(const PagedAttnArgs& a) {
  asm volatile("" ::"s"(a.q), "s"(a.q_ts), "s"(a.q_hs), "s"(a.kv.k), "s"(a.kv.v), "s"(a.kv.page_stride),
               "s"(a.kv.head_stride), "s"(a.kv.tok_stride));
  asm volatile("" ::"s"(a.scale), "s"(a.cap), "s"(a.window), "s"(a.ws), "s"(a.slots), "s"(a.o), "s"(a.o_ts), "s"(a.o_hs));
}

__device__ __forceinline__ float inverse(float l) { return l == 0.f ? 0.f : 1.f / l; }

// N times four dims of a row, at dim(i) and of the value val(i): to the output,
// or to the range's slot.
template <int HDP, int N, typename Dim, typename Val>
__device__ __forceinline__ void put(const PagedAttnArgs& a, const Item& it, const Row& w, bool direct, float inv, Dim dim,
                                    Val val) {
  const bool whole = a.kv.hd == HDP;
  if (direct) {
    bf16* op = reinterpret_cast<bf16*>(a.o) + (long)w.tok * a.o_ts + (long)w.head * a.o_hs;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const f32x4 v = val(i) * inv;
      if (whole || dim(i) < a.kv.hd)
        *reinterpret_cast<bf16x4*>(op + dim(i)) = bf16x4{(bf16)v[0], (bf16)v[1], (bf16)v[2], (bf16)v[3]};
    }
  } else {
    float* pp = part_of(a, (long)w.tok * a.n_q + w.head, it.slot);
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const f32x4 v = val(i);
      if (whole || dim(i) < a.kv.hd) *reinterpret_cast<f32x4*>(pp + dim(i)) = v;
    }
  }
}
// The statistics of a row (one lane of it calls this). direct: the row's log-sum-exp.
__device__ __forceinline__ void put_stats(const PagedAttnArgs& a, const Item& it, const Row& w, bool direct, float m, float l) {
  const long row = (long)w.tok * a.n_q + w.head;
  if (!direct) {
    store_stats(a, row, it.slot, m, l);
    return;
  }
  if (a.lse) a.lse[row] = (m + __builtin_amdgcn_logf(l)) * LN2;
  if (a.slots > 1) store_stats(a, row, 0, 0.f, -1.f);
}

// ---------------------------------------------------------------- bf16, waves split the rows
// 32 rows a wave, 32 NWR a block. KS groups of NWR waves take every KS-th SUB
// key tiles, which a group's waves load together, through a ring of two rounds.
// (64 keys a tile; 32 at head dim 256.) Eight waves of rows and two tiles a
// round where there are rows enough: half the loads and round overhead of four.
// Two groups of four where the blocks are few: their results meet in LDS.
// A prompt of 8191 of 32 heads of 128, causal: 529-569 us, 1.03 PFLOP/s at the
// 1.9 GHz to which the chip throttles (a product of 8192^3 reaches 1.42): the
// matrix pipe is busy for 46 % of the time, the vector pipe for 44 % (a wave's
// softmax of a tile takes as long as its products). Measured slower: the scores of
// the next tile between the weights of this one (700 us), the two waves of a
// SIMD a barrier apart, one in its products and one in its softmax (711).
template <int HDP, int KS, int NWR>
struct RowsShared {
  static constexpr int KT = HDP == 256 ? 32 : 64, SUB = NWR / 4, RING = 2 * KS * SUB * 2 * KT * Lay<HDP>::ROWB;
  static constexpr int MERGE = KS > 1 ? 256 * HDP * 2 : 0;       // half of each group's outputs
  __attribute__((aligned(1024))) char mem[RING > MERGE ? RING : MERGE];
  Window win;
  float stats[KS][KS > 1 ? 128 : 1][2];
};

template <int HDP, bool CAP, int KS, int NWR, bool FLAT>
__device__ __forceinline__ void rows_body(const PagedAttnArgs& a, RowsShared<HDP, KS, NWR>& sh, int L, int range) {
  using Y = Lay<HDP>;
  constexpr int KT = RowsShared<HDP, KS, NWR>::KT, SUB = RowsShared<HDP, KS, NWR>::SUB, NS = KT / 32, NC = HDP / 16, ND = HDP / 32;
  constexpr int TILE = SUB * KT * Y::ROWB, ROUND = KS * 2 * TILE, BR = 32 * NWR, RTL = KS * SUB;   // RTL: tiles of a round
  char* smem = sh.mem;
  Window& win = sh.win;
  auto& stats = sh.stats;
  touch(a);
  Item it;
  if (!find_item<BR, KT, RTL, FLAT>(a, L, range, it)) return;
  const bool direct = a.direct && it.ntiles <= a.chunk;
  if (it.ubeg >= it.uend && !(direct && it.ubeg == 0)) {
    if (!direct) empty_range<BR>(a, it);
    return;
  }
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kg = wave / NWR, wr = wave % NWR;
  const int lq = lane & 31, h = lane >> 5, hd = a.kv.hd, shift = a.kv.page_shift;
  // (the window's first page numbers go out ahead of the queries: loads return in order)
  auto first_key = [&](int u) { return a.klo + (u < it.n1 ? u : u - it.n1 + it.t2) * KT; };
  const int nrounds = (it.uend - it.ubeg + RTL - 1) / RTL;
  int w0 = nrounds > 0 ? first_key(it.ubeg) >> shift : 0, guessed = 0;
  if (nrounds > 0 && tid < PW) guessed = it.pages[min(w0 + tid, (it.klim - 1) >> shift)];
  const int wrow = it.row0 + wr * 32;
  const bool active = wrow < it.nrows;
  const Row w = row_of<FLAT>(a, it, wrow + lq);
  const WaveLimits wl = wave_limits<32, FLAT>(a, w.lim);
  bf16x8 qf[NC];
  {
    const bf16* qp = reinterpret_cast<const bf16*>(a.q) + (long)w.tok * a.q_ts + (long)w.head * a.q_hs;
    load_q<NC, 16>(qp, 8 * h, hd, qf);
  }
  Acc<HDP> s;
#pragma unroll
  for (int u = 0; u < ND; ++u)
#pragma unroll
    for (int i = 0; i < 16; ++i) s.o[u][i] = 0.f;
  s.m = -INFINITY;
  s.l = 0.f;
  const float sl2 = a.scale * LOG2E, c1 = CAP ? 2.f * sl2 / a.cap : 0.f, c2 = a.cap * LOG2E;

  const char *kb = reinterpret_cast<const char*>(a.kv.k), *vb = reinterpret_cast<const char*>(a.kv.v);
  const unsigned ring = lds_addr(smem);
  bool holes = false;
  Mover<HDP, SUB * KT, NWR> mv(a, win, wr);
  auto issue = [&](int p) {                    // round p
    const int u = it.ubeg + p * RTL + kg * SUB;
    if (u >= it.uend) return;
    const unsigned dst = ring + (p & 1) * ROUND + kg * 2 * TILE;
    mv.rows(first_key(u), w0, it.klim);
    mv.template load<true>(kb, vb, dst, dst + TILE);
  };
  if (nrounds > 0) {
    holes = fill_window<64 * NWR * KS>(a, it, win, w0, w0, guessed);
    issue(0);
  }
  hold<NC, 16>(8 * h, hd, hd == HDP, qf);
  // where the lane's K and V fragments begin; the swizzled pieces of a row
  // differ in address bits only, which costs an instruction a read and no
  // registers (held for all pieces they spill at head dim 256)
  const unsigned ka = lq * Y::ROWB + ((h ^ Y::swz(lq)) << 4), va = vt_address<HDP>();
  for (int p = 0; p < nrounds; ++p) {
    // this round has landed, and every wave is done with the round before
    asm volatile("s_waitcnt vmcnt(0)\n\ts_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (p + 1 < nrounds) {
      const int n0 = first_key(it.ubeg + (p + 1) * RTL), e0 = n0 >> shift, e1 = (min(n0 + RTL * KT, it.klim) - 1) >> shift;
      if (e0 < w0 || e1 >= w0 + PW) {          // (block-uniform; the barrier was the window's last use)
        w0 = e0;
        holes |= fill_window<64 * NWR * KS>(a, it, win, w0);
      }
      issue(p + 1);
    }
#pragma unroll 1
    for (int sub = 0; sub < SUB; ++sub) {
      const int u = it.ubeg + p * RTL + kg * SUB + sub, k0 = first_key(u);
      if (!active || u >= it.uend || tile_unseen(wl, k0, k0 + KT)) continue;
      unsigned kt = ring + (p & 1) * ROUND + kg * 2 * TILE + sub * (KT * Y::ROWB) + ka, vt = kt - ka + TILE + va;
      asm volatile("" : "+v"(kt), "+v"(vt));
      // fragments are requested well ahead of their products (LDS answers after
      // a few of these): all keys' first, two groups of the values' before the
      // softmax. Head dim 256 has registers for two fragments ahead of a product
      // (one: five capped prompts of 866 tokens 52.8 -> 50.2 us, two of 1500 of 16 heads
      // 62.4 -> 57.3 on one host; four, or parts of the queries in LDS for them: no faster)
      f32x16 sc[NS];
      constexpr bool AHEAD = HDP <= 128;
      bf16x8 kf[AHEAD ? NS : 1][AHEAD ? NC : 2];
      if constexpr (AHEAD) {
#pragma unroll
        for (int st = 0; st < NS; ++st)
#pragma unroll
          for (int c = 0; c < NC; ++c) kf[st][c] = read_k(kt, c, st * 32 * Y::ROWB);
        __builtin_amdgcn_sched_barrier(0);
      } else {
#pragma unroll
        for (int c = 0; c < 2; ++c) kf[0][c] = read_k(kt, c, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
      // (at head dim 256 the products go first: five capped prompts of 866 tokens 48.4 -> 47.0 us; at 64 and 128,
      // where the softmax is the longer part, the other way round)
      if constexpr (HDP == 256) __builtin_amdgcn_s_setprio(1);
#pragma unroll
      for (int st = 0; st < NS; ++st) {
#pragma unroll
        for (int i = 0; i < 16; ++i) sc[st][i] = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          sc[st] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[AHEAD ? st : 0][AHEAD ? c : c % 2], qf[c], sc[st], 0, 0, 0);
          if constexpr (!AHEAD) {
            if (c + 2 < NC) kf[0][c % 2] = read_k(kt, c + 2, 0);
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
      if constexpr (HDP == 256) __builtin_amdgcn_s_setprio(0);
      bf16x8 vf[2][ND];
      auto values = [&](int c) {
#pragma unroll
        for (int u2 = 0; u2 < ND; ++u2) vf[c % 2][u2] = read_vt<HDP>(vt, u2, c * 16 * Y::ROWB);
      };
      if constexpr (AHEAD) {
        values(0);
        values(1);
        __builtin_amdgcn_sched_barrier(0);
      }
      softmax_tile<HDP, NS, CAP>(s, sc, sl2, c1, c2, !holes && tile_full(wl, k0, k0 + KT), w.lim, k0, a, it, holes);
      if constexpr (HDP == 256) __builtin_amdgcn_s_setprio(1);
      if constexpr (AHEAD) {
#pragma unroll
        for (int c = 0; c < KT / 16; ++c) {
          const bf16x8 pf = weights_of(sc[c / 2], c % 2);
#pragma unroll
          for (int u2 = 0; u2 < ND; ++u2)
            s.o[u2] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[c % 2][u2], pf, s.o[u2], 0, 0, 0);
          if (c + 2 < KT / 16) values(c + 2);
        }
      } else {
        constexpr int N = KT / 16 * ND;
        bf16x8 vr[2];
#pragma unroll
        for (int n = 0; n < 2; ++n) vr[n] = read_vt<HDP>(vt, n % ND, n / ND * 16 * Y::ROWB);
        const bf16x8 pf[2] = {weights_of(sc[0], 0), weights_of(sc[0], 1)};
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int n = 0; n < N; ++n) {
          s.o[n % ND] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vr[n % 2], pf[n / ND], s.o[n % ND], 0, 0, 0);
          if (n + 2 < N) vr[n % 2] = read_vt<HDP>(vt, (n + 2) % ND, (n + 2) / ND * 16 * Y::ROWB);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if constexpr (HDP == 256) __builtin_amdgcn_s_setprio(0);
    }
  }
  s.l = sum_x32(s.l);
  if (active) {
    // (SUB is 1 where there are two groups)
    const int mine = it.uend - it.ubeg - kg;
    repair<HDP, CAP>(a, it, s, qf, w.lim, sl2, c1, c2, mine > 0 ? (mine + KS - 1) / KS : 0, KT,
                     [&](int n) { return first_key(it.ubeg + n * KS + kg); });
  }
  if constexpr (KS == 2) {
    // each group keeps half of the dims and hands the other half over
    __syncthreads();                           // the ring is free
    f32x4* mo = reinterpret_cast<f32x4*>(smem);
    auto slot = [&](int g, int j) { return ((g * 4 + wr) * (ND * 2) + j) * 64 + lane; };
    if (h == 0) {
      stats[kg][wr * 32 + lq][0] = s.m;
      stats[kg][wr * 32 + lq][1] = s.l;
    }
    auto hand = [&](auto from) {
      constexpr int U = decltype(from)::value;
#pragma unroll
      for (int j = 0; j < ND * 2; ++j) {
        const f32x16& x = s.o[U + j / 4];
        mo[slot(kg, j)] = f32x4{x[4 * (j % 4)], x[4 * (j % 4) + 1], x[4 * (j % 4) + 2], x[4 * (j % 4) + 3]};
      }
    };
    if (kg == 0) hand(std::integral_constant<int, ND / 2>{});
    else hand(std::integral_constant<int, 0>{});
    __syncthreads();
    if (wrow + lq >= it.nrows) return;
    const float m2 = stats[1 - kg][wr * 32 + lq][0], l2 = stats[1 - kg][wr * 32 + lq][1], m = vmax(s.m, m2);
    // (a group without keys weighs nothing)
    const float w1 = s.m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(s.m - m);
    const float w2 = m2 == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m2 - m);
    const float l = kg == 0 ? s.l * w1 + l2 * w2 : l2 * w2 + s.l * w1, inv = inverse(l);
    auto finish = [&](auto from) {
      constexpr int U = decltype(from)::value;
      put<HDP, ND * 2>(a, it, w, direct, inv, [&](int j) { return 32 * (U + j / 4) + 8 * (j % 4) + 4 * h; },
                       [&](int j) {
                         const f32x16& x = s.o[U + j / 4];
                         // (a group without keys has handed over zeros)
                         return f32x4{x[4 * (j % 4)], x[4 * (j % 4) + 1], x[4 * (j % 4) + 2], x[4 * (j % 4) + 3]} * w1 +
                                mo[slot(1 - kg, j)] * w2;
                       });
    };
    if (kg == 0) finish(std::integral_constant<int, 0>{});
    else finish(std::integral_constant<int, ND / 2>{});
    if (kg == 0 && h == 0) put_stats(a, it, w, direct, m, l);
    return;
  }
  if (wrow + lq >= it.nrows) return;
  const float inv = inverse(s.l);
  put<HDP, ND * 4>(a, it, w, direct, inv, [&](int j) { return 32 * (j / 4) + 8 * (j % 4) + 4 * h; }, [&](int j) {
    const f32x16& x = s.o[j / 4];
    return f32x4{x[4 * (j % 4)], x[4 * (j % 4) + 1], x[4 * (j % 4) + 2], x[4 * (j % 4) + 3]};
  });
  if (h == 0) put_stats(a, it, w, direct, s.m, s.l);
}

// ---------------------------------------------------------------- bf16, waves split the keys
// 16 rows a block; wave w takes every fourth tile of 32 keys (16 at head dim 256) into a K and a
// V slot of its own and waits for its own loads only: no barrier in the loop,
// and a slot is loaded again as soon as its fragments are in registers. The
// waves' (max, sum, output) meet in LDS at the end. For single tokens, whose
// time is that of the keys' and values' bytes (64 tokens over 5060 keys of 8
// heads of 128 on average: 1.42 GB in 259 us, 5.5 TB/s, where a copy of 4 GB
// moves 4.8), or where those are few, of the chain of memory round trips and of
// the instructions (cold in each launch; one token over 881 keys of 8 heads of
// 256: 8 us and 3.5 for the merge): hence 16-row products
// (v_mfma_f32_16x16x32), which for the usual few query heads a KV head leave
// half the registers and code of the 32-row ones.
// Lane l holds of S^T the keys 16 st + 4 (l / 16) + 0..3 of row l % 16, which
// is key slot order 4 (l / 16) + 0..3, 16 + 4 (l / 16) + 0..3 of the second product.
__device__ __forceinline__ float max_x16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return vmax(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float sum_x16(float v) {
  const auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// o += V^T P^T over the 32 or 16 keys of two fragments
__device__ __forceinline__ f32x4 pv_mma(bf16x8 v, bf16x8 p, f32x4 o) {
  return __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, p, o, 0, 0, 0);
}
__device__ __forceinline__ f32x4 pv_mma(bf16x4 v, bf16x4 p, f32x4 o) {
  return __builtin_amdgcn_mfma_f32_16x16x16bf16_1k(__builtin_bit_cast(v4s, v), __builtin_bit_cast(v4s, p), o, 0, 0, 0);
}

template <int HDP>
struct KeysShared {
  static constexpr int KT = HDP == 256 ? 16 : 32, NW = 4;
  static constexpr int SLOTS = NW * 2 * KT * Lay<HDP>::ROWB, MERGE = NW * HDP / 16 * 1024;
  __attribute__((aligned(1024))) char mem[SLOTS > MERGE ? SLOTS : MERGE];
  Window win;
  float stats[NW][16][2];
};

template <int HDP, bool CAP, bool FLAT>
__device__ __forceinline__ void keys_body(const PagedAttnArgs& a, KeysShared<HDP>& sh, int L, int range) {
  using Y = Lay<HDP>;
  constexpr int KT = KeysShared<HDP>::KT, NST = KT / 16, NW = 4, NC = HDP / 32, ND = HDP / 16;
  constexpr int TILE = KT * Y::ROWB, LK = TILE / 1024;
  char* smem = sh.mem;
  Window& win = sh.win;
  auto& stats = sh.stats;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), shift = a.kv.page_shift;
  touch(a);
  // the page numbers that the range needs if no window moves it: requested with the batch's lengths
  // (where a request is one tile of rows, the block knows which)
  const int guess = FLAT || a.bt.max_new * a.G <= 16 ? (a.klo + range * a.chunk * KT) >> shift : -1;
  int guessed = 0;
  if (guess >= 0 && a.bt.pages_stride > 0) {
    const int tile = div_by(L, a.kv.n_kv, a.mul_kv), r = FLAT ? 0 : (a.causal ? a.tiles - 1 - tile : tile);
    guessed = a.bt.pages[(long)r * a.bt.pages_stride + min(guess + tid, a.bt.pages_stride - 1)];
  }
  Item it;
  if (!find_item<16, KT, NW, FLAT>(a, L, range, it)) return;
  const bool direct = a.direct && it.ntiles <= a.chunk;
  if (it.ubeg >= it.uend && !(direct && it.ubeg == 0)) {
    if (!direct) empty_range<16>(a, it);
    return;
  }
  const int lq = lane & 15, grp = lane >> 4, hd = a.kv.hd;
  const Row w = row_of<FLAT>(a, it, it.row0 + lq);
  const WaveLimits wl = wave_limits<16, FLAT>(a, w.lim);
  bf16x8 qf[NC];
  f32x4 o[ND];
  float m = -INFINITY, l = 0.f;
  load_q<NC, 32>(reinterpret_cast<const bf16*>(a.q) + (long)w.tok * a.q_ts + (long)w.head * a.q_hs, 8 * grp, hd, qf);
  const float sl2 = a.scale * LOG2E, c1 = CAP ? 2.f * sl2 / a.cap : 0.f, c2 = a.cap * LOG2E;
  auto first_key = [&](int u) { return a.klo + (u < it.n1 ? u : u - it.n1 + it.t2) * KT; };
  const char *kb = reinterpret_cast<const char*>(a.kv.k), *vb = reinterpret_cast<const char*>(a.kv.v);
  int w0 = 0;
  bool holes = false;
  const unsigned slot_k = lds_addr(smem) + wave * 2 * TILE, slot_v = slot_k + TILE;
  Mover<HDP, KT, 1> mv(a, win, 0);
  const int nrounds = (it.uend - it.ubeg + NW - 1) / NW;
  if (nrounds > 0) {
    w0 = first_key(it.ubeg) >> shift;
    holes = fill_window<256>(a, it, win, w0, guess, guessed);
    if (it.ubeg + wave < it.uend) {
      mv.rows(first_key(it.ubeg + wave), w0, it.klim);
      mv.template load<false>(kb, nullptr, slot_k, 0);
      mv.template load<false>(vb, nullptr, slot_v, 0);
    }
  }
  // (zeros while the loads are under way)
  float zero = 0.f;
  asm volatile("" : "+v"(zero));
#pragma unroll
  for (int u = 0; u < ND; ++u) o[u] = f32x4{zero, zero, zero, zero};
  hold<NC, 32>(8 * grp, hd, hd == HDP, qf);
  const unsigned ka = slot_k + lq * Y::ROWB + ((grp ^ Y::swz(lq)) << 4);
  const int vr = 4 * grp + (lq >> 2);
  const unsigned va = slot_v + vr * Y::ROWB + ((((lq & 3) >> 1) ^ Y::swz(vr)) << 4) + ((lq & 1) << 3);
#pragma unroll 1
  for (int p = 0; p < nrounds; ++p) {
    const int u = it.ubeg + p * NW + wave, k0 = first_key(u);
    const bool next = u + NW < it.uend;
    if (p + 1 < nrounds) {                     // the next round's pages (block-uniform)
      const int n0 = first_key(it.ubeg + (p + 1) * NW), e0 = n0 >> shift,
                e1 = max(n0, min(n0 + NW * KT, it.klim) - 1) >> shift;
      if (e0 < w0 || e1 >= w0 + PW) {
        __syncthreads();
        w0 = e0;
        holes |= fill_window<256>(a, it, win, w0);
      }
    }
    if (u >= it.uend) continue;
    // this tile's keys have landed once only its values' loads are pending
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LK) : "memory");
    bf16x8 kf[NST][NC];
#pragma unroll
    for (int st = 0; st < NST; ++st)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        typedef const __attribute__((address_space(3))) bf16x8* P;
        kf[st][c] = *(P)(uintptr_t)((ka ^ (c % 4 << 6)) + st * 16 * Y::ROWB + c / 4 * 256);
      }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (next) {
      mv.rows(first_key(u + NW), w0, it.klim);
      mv.template load<false>(kb, nullptr, slot_k, 0);
    }
    const bool full = !holes && tile_full(wl, k0, k0 + KT);
    typedef __attribute__((ext_vector_type(4 * NST))) __bf16 frag;   // the keys of a lane
    frag pf;
    f32x4 sc[NST];
#pragma unroll
    for (int st = 0; st < NST; ++st) {
      f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;         // two chains
#pragma unroll
      for (int c = 0; c < NC; c += 2) {
        s0 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[st][c], qf[c], s0, 0, 0, 0);
        s1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[st][c + 1], qf[c + 1], s1, 0, 0, 0);
      }
      sc[st] = s0 + s1;
    }
    float mx = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4 * NST; ++i) {
      float x = sc[i / 4][i % 4];
      x = CAP ? capped(x, c1, c2) : x * sl2;
      if (!full) {
        const int j = k0 + i / 4 * 16 + 4 * grp + i % 4;
        if (!sees(w.lim, j)) x = -INFINITY;
        if (holes && (unsigned)it.pages[min(j, it.klim - 1) >> shift] >= (unsigned)a.kv.n_pages) x = -INFINITY;
      }
      sc[i / 4][i % 4] = x;
      mx = vmax(mx, x);
    }
    mx = max_x32(max_x16(mx));
    // (the reference lies 2^8 above the maximum that it was taken at, as in softmax_tile)
    if (__ballot(mx > m)) {
      const float mn = vmax(m, mx + 8.f), alpha = __builtin_amdgcn_exp2f(m - (mn == -INFINITY ? 0.f : mn));
      const bool some = __ballot(m != -INFINITY) != 0;      // (else there is nothing yet to rescale)
      m = mn;
      l *= alpha;
      if (some) {
#pragma unroll
        for (int u2 = 0; u2 < ND; ++u2) o[u2] *= alpha;
      }
    }
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int i = 0; i < 4 * NST; ++i) {
      const float x = __builtin_amdgcn_exp2f(sc[i / 4][i % 4] - ref);
      l += x;
      pf[i] = (bf16)x;
    }
    // the values have landed once only the next keys' loads are pending
    if (next) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LK) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    frag vf[ND];
#pragma unroll
    for (int u2 = 0; u2 < ND; ++u2) {
      const unsigned at = (va ^ (u2 % 8 << 5)) + u2 / 8 * 256;
      if constexpr (NST == 2) vf[u2] = __builtin_shufflevector(read_tr(at), read_tr(at + 16 * Y::ROWB), 0, 1, 2, 3, 4, 5, 6, 7);
      else vf[u2] = read_tr(at);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
    if (next) mv.template load<false>(vb, nullptr, slot_v, 0);
#pragma unroll
    for (int u2 = 0; u2 < ND; ++u2) o[u2] = pv_mma(vf[u2], pf, o[u2]);
  }
  float z = 0.f;
  l = sum_x32(sum_x16(l));
#pragma unroll
  for (int u = 0; u < ND; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) z = __builtin_fmaf(o[u][e], 0.f, z);
  // rows with an output that is not finite: again, key by key (as `repair`)
  if (__ballot(z != z) != 0) {
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int u = 0; u < ND; ++u) o[u] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
    for (int u = it.ubeg + wave; u < it.uend; u += NW) {
      const int k0 = first_key(u);
#pragma unroll 1
      for (int j = k0; j < min(k0 + KT, it.klim); ++j) {
        const bool vis = sees(w.lim, j);
        if (__ballot(vis) == 0) continue;
        const long off = page_offset(a, it.pages[j >> shift], it.g);
        if (off < 0) continue;
        const long at = off + (long)(j & ((1 << shift) - 1)) * a.kv.tok_stride;
        float d = 0.f;
#pragma unroll
        for (int c = 0; c < NC; ++c)
          if (32 * c + 8 * grp < hd) {
            const bf16x8 x = *reinterpret_cast<const bf16x8*>(reinterpret_cast<const bf16*>(a.kv.k) + at + 32 * c + 8 * grp);
#pragma unroll
            for (int e = 0; e < 8; ++e) d = __builtin_fmaf((float)x[e], (float)qf[c][e], d);
          }
        d = sum_x32(sum_x16(d));
        const float pj = __builtin_amdgcn_exp2f((CAP ? capped(d, c1, c2) : d * sl2) - ref);
#pragma unroll
        for (int u2 = 0; u2 < ND; ++u2)
          if (vis && 16 * u2 + 4 * grp < hd) {
            const bf16x4 x = *reinterpret_cast<const bf16x4*>(reinterpret_cast<const bf16*>(a.kv.v) + at + 16 * u2 + 4 * grp);
#pragma unroll
            for (int e = 0; e < 4; ++e) o[u2][e] = __builtin_fmaf(pj, (float)x[e], o[u2][e]);
          }
      }
    }
  }
  // the waves store outputs and statistics, then each adds a quarter of the dims in wave order
  __syncthreads();
  f32x4* mo = reinterpret_cast<f32x4*>(smem);
#pragma unroll
  for (int u = 0; u < ND; ++u) mo[(wave * ND + u) * 64 + lane] = o[u];
  if (grp == 0) {
    stats[wave][lq][0] = m;
    stats[wave][lq][1] = l;
  }
  __syncthreads();
  float mm = -INFINITY, ll = 0.f, wt[NW];
#pragma unroll
  for (int q = 0; q < NW; ++q) mm = vmax(mm, stats[q][lq][0]);
#pragma unroll
  for (int q = 0; q < NW; ++q) {
    // (a wave without keys weighs nothing)
    wt[q] = stats[q][lq][0] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(stats[q][lq][0] - mm);
    ll += stats[q][lq][1] * wt[q];
  }
  if (it.row0 + lq >= it.nrows) return;
  const float inv = inverse(ll);
  // (a wave, or a row of it, without keys has stored zeros)
  const f32x4* mine = mo + wave * (ND / NW) * 64 + lane;
  put<HDP, ND / NW>(a, it, w, direct, inv, [&](int i) { return 16 * (wave * (ND / NW) + i) + 4 * grp; }, [&](int i) {
    f32x4 acc = mine[i * 64] * wt[0];
#pragma unroll
    for (int q = 1; q < NW; ++q) acc += mine[(q * ND + i) * 64] * wt[q];
    return acc;
  });
  if (wave == 0 && grp == 0) put_stats(a, it, w, direct, mm, ll);
}

// ---------------------------------------------------------------- bf16 kernels
template <int HDP, bool CAP, int KIND>
__global__ void __launch_bounds__(KIND == PAGED_KEYS ? 256 : 512, 2) paged_kernel(PagedAttnArgs a) {
  if constexpr (KIND == PAGED_ROWS8) {
    __shared__ RowsShared<HDP, 1, 8> sh;
    rows_body<HDP, CAP, 1, 8, false>(a, sh, blockIdx.x, blockIdx.y);
  } else if constexpr (KIND == PAGED_ROWS2) {
    __shared__ RowsShared<HDP, 2, 4> sh;
    rows_body<HDP, CAP, 2, 4, false>(a, sh, blockIdx.x, blockIdx.y);
  } else {
    __shared__ KeysShared<HDP> sh;
    keys_body<HDP, CAP, false>(a, sh, blockIdx.x, blockIdx.y);
  }
}

// A batch with a common context: that by KIND (all rows in one sequence of
// tiles, the grid's first blocks: they take longest; as the last ones 64 tokens
// over 8192 common keys of 8 heads of 128 took 50 us, not 42), what follows it
// in tiles of 16 rows: the two do not wait for each other.
template <int HDP, bool CAP, int KIND>
__global__ void __launch_bounds__(256, 2) paged_pair_kernel(PagedAttnArgs a, PagedAttnArgs b) {
  union Shared {
    RowsShared<HDP, 1, 4> rows;
    KeysShared<HDP> keys;
  };
  __shared__ __attribute__((aligned(1024))) char mem[KIND == PAGED_ROWS ? sizeof(Shared) : sizeof(KeysShared<HDP>)];
  Shared& sh = *reinterpret_cast<Shared*>(mem);
  const int per_a = a.tiles * a.kv.n_kv, na = per_a * a.ranges;
  int L = blockIdx.x;
  if (L < na) {
    const int range = div_by(L, per_a, a.mul_blocks);
    L -= range * per_a;
    if constexpr (KIND == PAGED_ROWS) rows_body<HDP, CAP, 1, 4, true>(a, sh.rows, L, range);
    else keys_body<HDP, CAP, true>(a, sh.keys, L, range);
  } else {
    const int per_b = b.tiles * b.kv.n_kv;
    L -= na;
    const int range = div_by(L, per_b, b.mul_blocks);
    L -= range * per_b;
    keys_body<HDP, CAP, false>(b, sh.keys, L, range);
  }
}

// ---------------------------------------------------------------- fp32
// 16 RT rows a block, eight waves split the tiles of 16 keys; both products on
// v_mfma_f32_16x16x4_f32 with operands straight from global memory. A tile's
// page numbers are requested while the tile before is computed. RT is 1 for few
// rows; for prompts 4 at head dim 64 and 2 at 128 (what the registers hold), which
// read the keys and values that much less often.
template <int HDP>
struct F32Shared {
  static constexpr int REC = HDP / 4 + 4;
  __attribute__((aligned(16))) float mg[4][64 * REC];
};
static constexpr int f32_row_tiles(int hdp) { return hdp == 64 ? 4 : hdp == 128 ? 2 : 1; }

template <int HDP, bool CAP, int RT, bool FLAT>
__device__ __forceinline__ void f32_body(const PagedAttnArgs& a, F32Shared<HDP>& sh, int L, int range) {
  constexpr int NW = 8, KT = 16, NC = HDP / 16, REC = F32Shared<HDP>::REC;
  auto& mg = sh.mg;
  Item it;
  if (!find_item<16 * RT, KT, 1, FLAT>(a, L, range, it)) return;
  const bool direct = a.direct && it.ntiles <= a.chunk;
  if (it.ubeg >= it.uend && !(direct && it.ubeg == 0)) {
    if (!direct) empty_range<16 * RT>(a, it);
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int lr = lane & 15, lk = lane >> 4, hd = a.kv.hd, shift = a.kv.page_shift, smask = (1 << shift) - 1;
  const f32x4 zero = {0.f, 0.f, 0.f, 0.f};
  Row w[RT];
  f32x4 qf[RT][NC], o[RT][NC];
  float m[RT], l[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    w[t] = row_of<FLAT>(a, it, it.row0 + t * 16 + lr);
    const float* qp = reinterpret_cast<const float*>(a.q) + (long)w[t].tok * a.q_ts + (long)w[t].head * a.q_hs;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      qf[t][c] = c * 16 + lk * 4 < hd ? *reinterpret_cast<const f32x4*>(qp + c * 16 + lk * 4) : zero;
      o[t][c] = zero;
    }
    m[t] = -INFINITY;
    l[t] = 0.f;
  }
  auto first_key = [&](int u) { return a.klo + (u < it.n1 ? u : u - it.n1 + it.t2) * KT; };
  auto page_at = [&](int j) { return it.pages[min(j, it.klim - 1) >> shift]; };
  const float *kb = reinterpret_cast<const float*>(a.kv.k), *vb = reinterpret_cast<const float*>(a.kv.v);
  // the score of a dot product; exact functions, the sums' errors are of their size
  auto score = [&](float d) { return CAP ? a.cap * tanhf(d * a.scale / a.cap) : d * a.scale; };
  // one tile's scores of row tile t into weights, and its values added
  auto add = [&](int t, f32x4 sc, int k0, const bool (&vok)[4], const f32x4 (&vf)[NC]) {
    float mx = -INFINITY;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sc[e] = vok[e] && sees(w[t].lim, k0 + 4 * lk + e) ? score(sc[e]) : -INFINITY;
      mx = vmax(mx, sc[e]);
    }
    mx = vmax(mx, __shfl_xor(mx, 16));
    mx = vmax(mx, __shfl_xor(mx, 32));
    const float mn = vmax(m[t], mx), ref = mn == -INFINITY ? 0.f : mn, alpha = __expf(m[t] - ref);
    float ps = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sc[e] = __expf(sc[e] - ref);
      ps += sc[e];
    }
    l[t] = l[t] * alpha + ps;
    m[t] = mn;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      o[t][c] *= alpha;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[t][c] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[c][e], sc[e], o[t][c], 0, 0, 0);
    }
  };
  int pk = 0, pv[4] = {0, 0, 0, 0};
  auto request = [&](int u) {
    const int k0 = first_key(u);
    pk = page_at(k0 + lr);
#pragma unroll
    for (int e = 0; e < 4; ++e) pv[e] = page_at(k0 + 4 * lk + e);
  };
  if (it.ubeg + wave < it.uend) request(it.ubeg + wave);
#pragma unroll 1
  for (int u = it.ubeg + wave; u < it.uend; u += NW) {
    const int k0 = first_key(u);
    const long ko = page_offset(a, pk, it.g) + (long)((k0 + lr) & smask) * a.kv.tok_stride;
    const bool kok = (unsigned)pk < (unsigned)a.kv.n_pages && k0 + lr < it.klim;
    long vo[4];
    bool vok[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = k0 + 4 * lk + e;
      vok[e] = (unsigned)pv[e] < (unsigned)a.kv.n_pages && j < it.klim;
      vo[e] = page_offset(a, pv[e], it.g) + (long)(j & smask) * a.kv.tok_stride;
    }
    f32x4 kf[NC], vf[NC];                      // vf[c][e]: V[key 4 lk + e][16 c + lr]
#pragma unroll
    for (int c = 0; c < NC; ++c)
      kf[c] = kok && c * 16 + lk * 4 < hd ? *reinterpret_cast<const f32x4*>(kb + ko + c * 16 + lk * 4) : zero;
    auto load_v = [&]() {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int c = 0; c < NC; ++c) vf[c][e] = vok[e] && c * 16 + lr < hd ? vb[vo[e] + c * 16 + lr] : 0.f;
    };
    if constexpr (HDP <= 128) load_v();        // (at 256 both would not fit the registers)
    if (u + NW < it.uend) request(u + NW);
    if constexpr (HDP > 128) {
      // (one row tile: values after the scores)
      f32x4 sc = zero;
#pragma unroll
      for (int c = 0; c < NC; ++c)
#pragma unroll
        for (int e = 0; e < 4; ++e) sc = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[c][e], qf[0][c][e], sc, 0, 0, 0);
      load_v();
      add(0, sc, k0, vok, vf);
    } else {
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        f32x4 sc = zero;
#pragma unroll
        for (int c = 0; c < NC; ++c)
#pragma unroll
          for (int e = 0; e < 4; ++e) sc = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[c][e], qf[t][c][e], sc, 0, 0, 0);
        add(t, sc, k0, vok, vf);
      }
    }
  }
  // rows with an output that is not finite: again, key by key (as `repair`)
  float z = 0.f;
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    l[t] += __shfl_xor(l[t], 16);
    l[t] += __shfl_xor(l[t], 32);
#pragma unroll
    for (int c = 0; c < NC; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) z = __builtin_fmaf(o[t][c][e], 0.f, z);
  }
  if (__ballot(z != z) != 0) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const float ref = m[t] == -INFINITY ? 0.f : m[t];
#pragma unroll
      for (int c = 0; c < NC; ++c) o[t][c] = zero;
#pragma unroll 1
      for (int u = it.ubeg + wave; u < it.uend; u += NW) {
        const int k0 = first_key(u);
#pragma unroll 1
        for (int j = k0; j < min(k0 + KT, it.klim); ++j) {
          const bool vis = sees(w[t].lim, j);
          if (__ballot(vis) == 0) continue;
          const long off = page_offset(a, it.pages[j >> shift], it.g);
          if (off < 0) continue;
          const long at = off + (long)(j & smask) * a.kv.tok_stride;
          float d = 0.f;
#pragma unroll
          for (int c = 0; c < NC; ++c)
            if (c * 16 + lk * 4 < hd) {
              const f32x4 x = *reinterpret_cast<const f32x4*>(kb + at + c * 16 + lk * 4);
#pragma unroll
              for (int e = 0; e < 4; ++e) d = __builtin_fmaf(x[e], qf[t][c][e], d);
            }
          d += __shfl_xor(d, 16);
          d += __shfl_xor(d, 32);
          const float p = __expf(score(d) - ref);
#pragma unroll
          for (int c = 0; c < NC; ++c)
            if (vis && c * 16 + lk * 4 < hd) {
              const f32x4 x = *reinterpret_cast<const f32x4*>(vb + at + c * 16 + lk * 4);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[t][c][e] = __builtin_fmaf(p, x[e], o[t][c][e]);
            }
        }
      }
    }
  }
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    // merge the waves, the upper half into the lower until wave 0 holds all
    for (int n = NW / 2; n > 0; n /= 2) {
      if (wave >= n && wave < 2 * n) {
        float* dst = mg[wave - n] + lane * REC;
#pragma unroll
        for (int c = 0; c < NC; ++c) *reinterpret_cast<f32x4*>(dst + 4 * c) = o[t][c];
        dst[HDP / 4] = m[t];
        dst[HDP / 4 + 1] = l[t];
      }
      __syncthreads();
      if (wave < n) {
        const float* src = mg[wave] + lane * REC;
        const float m2 = src[HDP / 4], l2 = src[HDP / 4 + 1], mm = vmax(m[t], m2);
        // (a wave without keys weighs nothing)
        const float w1 = m[t] == -INFINITY ? 0.f : __expf(m[t] - mm), w2 = m2 == -INFINITY ? 0.f : __expf(m2 - mm);
#pragma unroll
        for (int c = 0; c < NC; ++c) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(src + 4 * c);
          // (0 times a NaN value that the row sees stays a NaN; a wave without keys has zeros)
          if (w1 != 1.f) o[t][c] *= w1;
          o[t][c] += x * w2;
        }
        l[t] = l[t] * w1 + l2 * w2;
        m[t] = mm;
      }
      __syncthreads();
    }
    if (wave == 0 && it.row0 + t * 16 + lr < it.nrows) {
      const float inv = inverse(l[t]);
      const long row = (long)w[t].tok * a.n_q + w[t].head;
      float* op = direct ? reinterpret_cast<float*>(a.o) + (long)w[t].tok * a.o_ts + (long)w[t].head * a.o_hs : part_of(a, row, it.slot);
#pragma unroll
      for (int c = 0; c < NC; ++c)
        if (c * 16 + lk * 4 < hd) *reinterpret_cast<f32x4*>(op + c * 16 + lk * 4) = direct ? o[t][c] * inv : o[t][c];
      if (lk == 0) {
        if (!direct) {
          store_stats(a, row, it.slot, m[t] * LOG2E, l[t]);
        } else {
          if (a.lse) a.lse[row] = m[t] + logf(l[t]);
          if (a.slots > 1) store_stats(a, row, 0, 0.f, -1.f);
        }
      }
    }
  }
}

template <int HDP, bool CAP, int RT>
__global__ void __launch_bounds__(512) paged_f32_kernel(PagedAttnArgs a) {
  __shared__ F32Shared<HDP> sh;
  f32_body<HDP, CAP, RT, false>(a, sh, blockIdx.x, blockIdx.y);
}

// As paged_pair_kernel.
template <int HDP, bool CAP>
__global__ void __launch_bounds__(512) paged_f32_pair_kernel(PagedAttnArgs a, PagedAttnArgs b) {
  __shared__ F32Shared<HDP> sh;
  const int per_a = a.tiles * a.kv.n_kv, na = per_a * a.ranges;
  int L = blockIdx.x;
  if (L < na) {
    const int range = div_by(L, per_a, a.mul_blocks);
    f32_body<HDP, CAP, 1, true>(a, sh, L - range * per_a, range);
  } else {
    const int per_b = b.tiles * b.kv.n_kv;
    L -= na;
    const int range = div_by(L, per_b, b.mul_blocks);
    f32_body<HDP, CAP, 1, false>(b, sh, L - range * per_b, range);
  }
}

// ---------------------------------------------------------------- merge of ranges
// LPR lanes own a row, four dims each, and WPR such groups share its slots,
// eight at a time (their statistics and outputs in one round trip), merged in
// order; the groups' sums meet in LDS in group order.
template <typename T, int LPR, int WPR>
__global__ void __launch_bounds__(256) paged_merge_kernel(PagedAttnArgs a) {
  constexpr int RB = 256 / (LPR * WPR), N = 8;
  const int tid = threadIdx.x, sub = tid % LPR, grp = tid / LPR % WPR, S = a.slots, hd = a.kv.hd;
  const long row = blockIdx.x * (long)RB + tid / (LPR * WPR);
  const int tok = (int)(row / a.n_q), head = (int)(row - (long)tok * a.n_q);
  const float* stat = a.ws + (long)a.bt.n_tok * a.n_q * S * hd + row * S * 2;
  const bool in_rows = tok < a.bt.n_tok;
  // rows of no request, and those that are written already (what their slots hold is read, and not used)
  const bool live = in_rows && tok >= a.bt.start[0] && tok < a.bt.start[a.bt.n_req] && !(stat[1] < 0.f);
  const bool dok = sub * 4 < hd;
  float m = -INFINITY, l = 0.f;
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
  for (int b = grp * N; in_rows && b < S; b += WPR * N) {
    float ms[N], ls[N];
    f32x4 pt[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const bool in = b + k < S;
      ms[k] = in ? stat[2 * (b + k)] : 0.f;
      ls[k] = in ? stat[2 * (b + k) + 1] : 0.f;
      pt[k] = in && dok ? *reinterpret_cast<const f32x4*>(part_of(a, row, b + k) + sub * 4) : f32x4{0.f, 0.f, 0.f, 0.f};
    }
    // (a range without keys has a sum of 0 and no output; a NaN sum is not 0)
    float mb = m;
#pragma unroll
    for (int k = 0; k < N; ++k) mb = ls[k] == 0.f ? mb : vmax(mb, ms[k]);
    const float w0 = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mb);
    l *= w0;
    s *= w0;
    m = mb;
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const float w = __builtin_amdgcn_exp2f(ms[k] - mb);
      if (ls[k] == 0.f) continue;
      l += ls[k] * w;
      s += pt[k] * w;
    }
  }
  if constexpr (WPR > 1) {
    __shared__ float st[256][2];
    __shared__ __attribute__((aligned(16))) f32x4 acc[256];
    st[tid][0] = m;
    st[tid][1] = l;
    acc[tid] = s;
    __syncthreads();
    if (grp != 0) return;
    float mm = m;
#pragma unroll
    for (int g = 1; g < WPR; ++g) mm = vmax(mm, st[tid + g * LPR][0]);
    const float w0 = m == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m - mm);
    l *= w0;
    s *= w0;
#pragma unroll
    for (int g = 1; g < WPR; ++g) {
      // (as above: a group without keys goes by its sum, as one whose first scores are NaN has no maximum either)
      const float lg = st[tid + g * LPR][1];
      if (lg == 0.f) continue;
      const float w = __builtin_amdgcn_exp2f(st[tid + g * LPR][0] - mm);
      l += lg * w;
      s += acc[tid + g * LPR] * w;
    }
    m = mm;
  }
  if (!live) return;
  const float inv = inverse(l);
  if (dok) {
    T* op = reinterpret_cast<T*>(a.o) + (long)tok * a.o_ts + (long)head * a.o_hs + sub * 4;
    if constexpr (sizeof(T) == 2) *reinterpret_cast<bf16x4*>(op) = bf16x4{(bf16)(s[0] * inv), (bf16)(s[1] * inv), (bf16)(s[2] * inv), (bf16)(s[3] * inv)};
    else *reinterpret_cast<f32x4*>(op) = s * inv;
  }
  if (a.lse && sub == 0) a.lse[row] = m * LN2 + logf(l);
}

}  // namespace

// ---------------------------------------------------------------- host
// Rows of a tile, keys of a key tile and key tiles of a round of kernel k at
// padded head dim hdp.
static int tile_rows(int k, int hdp) {
  return k == PAGED_ROWS8 ? 256 : k == PAGED_ROWS || k == PAGED_ROWS2 ? 128 : k == PAGED_F32R ? 16 * f32_row_tiles(hdp) : 16;
}
static int tile_keys(int k, int hdp) {
  const int wide = hdp == 256 ? 1 : 2;
  return k == PAGED_F32 || k == PAGED_F32R ? 16 : k == PAGED_KEYS ? 16 * wide : 32 * wide;
}
static int round_tiles(int k) { return k == PAGED_KEYS ? 4 : k == PAGED_ROWS2 || k == PAGED_ROWS8 ? 2 : k == PAGED_F32 || k == PAGED_F32R ? 2 : 1; }

// How long a part would take with kernel p.kernel (us) by a simple model, and
// the number of key ranges that makes it least: the blocks' start, as many
// rounds of tiles at a time as blocks are resident, each at a round's latency,
// a block's bytes at what one CU takes in, or all bytes at the memory's rate
// (requests' keys differ) or the L2's; a part of a last block's rounds, as
// lengths differ and it runs alone; and, where a row has several ranges, the merge's
// launch and their outputs. Ranges are counted over all keys up to max_len, those
// before a window too, which no tile's list holds (a prefix may lie there). Starts and rounds are measured; the model
// need only be right where the kernels' times differ much. (One request's token
// over 881 keys of 8 heads of 256: ranges of 64 keys 10.5 us, 128 11.9, 256
// 13.8. 64 tokens over up to 8101 keys of 8 heads of 128: one range 272 us, four
// 262, eight 259, sixteen 270. Twelve prompts of 64 over 864 keys of 8 heads of
// 256: in tiles of 16 rows and two ranges 24.1 us, of 128 and one range 39.6,
// four 29.7; five of 866, capped: 110 against 48. One prompt of 4000 of 15 heads of 64:
// tiles of 16 rows 97 us, 128 55, 256 77; of 8191 of 32 heads of 128: 128 rows 636, 256 580.)
struct PartShape {
  int hdp, hd, keys, seen, n_kv, n_req;        // seen: keys that a tile of rows sees at most
  long rows;
  double share;                                // of `seen` that the tiles see on average
  bool cap, beside;
};

static double cut(PagedPart& p, const PartShape& q) {
  const int w = q.hdp == 64 ? 0 : q.hdp == 128 ? 1 : 2, kt = tile_keys(p.kernel, q.hdp), unit = round_tiles(p.kernel);
  const bool f32 = p.kernel == PAGED_F32 || p.kernel == PAGED_F32R;
  const int es = f32 ? 4 : 2;
  // by PagedKernel and padded head dim
  static const double START[6][3] = {{4, 5, 5}, {5, 7.5, 12}, {4, 4, 4}, {5, 7.5, 12}, {0, 5.5, 0}, {4.5, 4.5, 4.5}};
  static const double ROUND[6][3] = {{1, 1, 1.3}, {1, 1.2, 1.7}, {1, 1, 1}, {1.55, 1.8, 1.9}, {0, 3.1, 0}, {2.5, 2.5, 2.5}};
  static const int RESIDENT[6][3] = {{1024, 512, 512}, {512, 512, 256}, {512, 512, 512}, {256, 256, 256}, {0, 256, 0}, {256, 256, 256}};
  const long full = std::max(1, (q.keys + kt * unit - 1) / (kt * unit));     // rounds of all keys
  const long total = std::max(1, (q.seen + kt * unit - 1) / (kt * unit));
  const long blocks = (long)p.tiles * q.n_kv, resident = RESIDENT[p.kernel][w];
  const bool small = p.kernel == PAGED_KEYS;   // (two blocks and more a CU slow each other down)
  const double bytes = 2.0 * es * kt * unit * q.hd, differ = std::min(1.0, (double)q.n_req / p.tiles);
  double best = 1e30;
  long best_per = full;
  // (the parts of a batch with a common context run side by side)
  const long most = std::min<long>(256, std::max<long>(1, (q.beside ? 512 : 4 * resident) / blocks));
  for (long s = 1; s <= std::min(total, most); ++s) {
    const long per = (total + s - 1) / s, n = s > 1 ? (full + per - 1) / per : 1;
    if ((total + per - 1) / per != s) continue;
    const double on = (double)std::min(blocks * s, resident), per_cu = blocks * s / 256.0, passes = blocks * s / (double)resident;
    const double uneven = per_cu > 1.0 && per_cu <= resident / 256 ? std::ceil(per_cu) / per_cu : 1.0;
    const double rounds = f32 ? (per + 3) / 4 : per;         // (eight waves, a tile each)
    const double slow = (small && passes > 1.0 ? 1.25 : 1.0) * (small && q.cap ? 1.3 : 1.0);
    const double busy = std::max(rounds * ROUND[p.kernel][w] * slow,
                                 per * bytes * std::max({1e-5, on * differ * uneven / 5e6, on / (f32 ? 15e6 : 20e6)}));
    const double t = START[p.kernel][w] + std::ceil(passes) +
                     busy * (q.share < 0.95 ? std::max(1.0, passes * q.share + 0.3) : std::ceil(passes)) +
                     (small || f32 ? 0.5 * rounds : 0.0) +
                     (n > 1 ? 4.0 + q.rows * (double)n * q.hd * 8 / 2e6 : 0.0);
    if (t < best) { best = t; best_per = s > 1 ? per : full; }
  }
  best_per = std::max<long>(best_per, (full + 65534) / 65535);                // (the grid's second extent)
  p.chunk = (int)(best_per * unit);
  p.ranges = (int)((full + best_per - 1) / best_per);
  return best;
}

PagedPlan paged_plan(const PagedAttnArgs& a, int et) {
  PagedPlan p{};
  p.hdp = a.kv.hd <= 64 ? 64 : a.kv.hd <= 128 ? 128 : 256;
  const long all = (long)a.bt.n_tok * a.G, rows_req = (long)a.bt.max_new * a.G;
  // a part by kernel k: flat: the rows of the batch in one sequence of tiles
  auto part = [&](int k, bool flat, int keys, PagedPart& q) {
    const int br = tile_rows(k, p.hdp);
    q.kernel = k;
    q.tiles = (int)(flat ? std::max<long>(1, (all + br - 1) / br) : rows_req <= br ? a.bt.n_req : all / br + a.bt.n_req);
    const int seen = a.causal && a.window && !flat ? (int)std::min<long>(keys, (long)a.window + br / a.G + 1) : keys;
    const double share = a.causal && !a.window && !a.prefix && !flat && keys > 0 ? 1.0 - 0.5 * std::min(a.bt.max_new, keys) / keys : 1.0;
    return cut(q, PartShape{p.hdp, a.kv.hd, keys, seen, a.kv.n_kv, flat ? 1 : a.bt.n_req, (long)a.bt.n_tok * a.n_q, share, a.cap > 0.f, a.shared_len > 0});
  };
  auto least = [&](std::initializer_list<int> kernels, bool flat, int keys) {
    PagedPart best{};
    double t = 1e30;
    for (int k : kernels) {
      PagedPart q{};
      const double tk = part(k, flat, keys, q);
      if (tk < t) { t = tk; best = q; }
    }
    return best;
  };
  const int rest = a.bt.max_len - a.shared_len;
  p.n_parts = a.shared_len > 0 ? 2 : 1;
  if (et == ET_F32) {
    // (more rows a block: two prompts of 2000 of 32 heads of 128 1113 -> 883 us, of 3000 of 15 heads of 64 410 -> 349, six
    // of 700 of 4 heads of 64 30 -> 43; for a common context never faster)
    if (a.shared_len > 0) p.part[0] = least({PAGED_F32}, true, a.shared_len);
    PagedPart& last = p.part[p.n_parts - 1];
    if (a.shared_len == 0 && p.hdp < 256 && rows_req > 16) last = least({PAGED_F32, PAGED_F32R}, false, rest);
    else last = least({PAGED_F32}, false, rest);
  } else if (a.shared_len > 0) {
    // Up to 32 tiles of 16 rows (128 at head dim 256, where a block of 128 rows takes long to begin and end) the
    // common context goes in those, beyond in tiles of 128: 16 rows x 2 x 8 heads of 128 over 4096 keys 15.7 and 16.9 us,
    // x 6 x 8 21.5 and 20.8, x 16 x 2 16.3 and 18.6; of 256 x 32 over 832 13.9 and 20.5, x 128 over 2048 31.5 and
    // 36.5, x 192 over 4096 65 and 43. What follows is a few keys of many requests: tiles of 16 (or as fast).
    const long tiles16 = (all + 15) / 16 * a.kv.n_kv;
    p.part[0] = least({tiles16 <= (p.hdp == 256 ? 128 : 32) ? PAGED_KEYS : PAGED_ROWS}, true, a.shared_len);
    p.part[1] = least({PAGED_KEYS}, false, rest);
  } else if (rows_req <= 16) {
    p.part[0] = least({PAGED_KEYS}, false, rest);
  } else if (p.hdp == 128) {
    // (256 rows a block pay off here only: two prompts of 4000 of 32 heads of 128 303 -> 270 us, four of 1500 of 8 heads of
    // 64 23 -> 34, two of 1500 of 16 heads of 256 63 -> 91)
    p.part[0] = least({PAGED_KEYS, PAGED_ROWS2, PAGED_ROWS8}, false, rest);
  } else {
    p.part[0] = least({PAGED_KEYS, PAGED_ROWS2}, false, rest);
  }
  // (a launch has less than 2^32 threads in x; a merge's rows have up to 256 each)
  long blocks = 0;
  for (int i = 0; i < p.n_parts; ++i) {
    const PagedPart& q = p.part[i];
    p.slots += q.ranges;
    blocks += (long)q.tiles * a.kv.n_kv * (p.n_parts == 2 ? q.ranges : 1);
  }
  VLA_REQUIRE(blocks < 1 << 23 && (p.slots == 1 || (long)a.bt.n_tok * a.n_q < 1 << 24),
              "too many rows for one call: " + std::to_string(a.bt.n_tok) + " tokens of " + std::to_string(a.n_q) + " heads");
  return p;
}

size_t paged_attention_ws(const PagedAttnArgs& a, const PagedPlan& p) {
  return p.slots > 1 ? (size_t)a.bt.n_tok * a.n_q * p.slots * (a.kv.hd + 2) * 4 : 0;
}

// The kernels that the launches below know, of a part of n: another one in the
// plan is an error, not a launch that reads bf16 as fp32.
static bool has_kernel(int et, int k, int hdp, int part, int n) {
  if (et == ET_F32) return k == PAGED_F32 || (k == PAGED_F32R && n == 1 && hdp < 256);
  if (n == 2) return k == PAGED_KEYS || (k == PAGED_ROWS && part == 0);
  return k == PAGED_KEYS || k == PAGED_ROWS2 || (k == PAGED_ROWS8 && hdp == 128);
}

template <int HDP, bool CAP>
static void launch_one(const PagedAttnArgs& a, int kernel, hipStream_t s) {
  const dim3 grid((unsigned)a.tiles * a.kv.n_kv, a.ranges);
  if (kernel == PAGED_KEYS) hipLaunchKernelGGL((paged_kernel<HDP, CAP, PAGED_KEYS>), grid, dim3(256), 0, s, a);
  else if (HDP == 128 && kernel == PAGED_ROWS8) hipLaunchKernelGGL((paged_kernel<HDP, CAP, HDP == 128 ? PAGED_ROWS8 : PAGED_KEYS>), grid, dim3(512), 0, s, a);
  else if (kernel == PAGED_ROWS2) hipLaunchKernelGGL((paged_kernel<HDP, CAP, PAGED_ROWS2>), grid, dim3(512), 0, s, a);
  else if (HDP < 256 && kernel == PAGED_F32R) hipLaunchKernelGGL((paged_f32_kernel<HDP, CAP, f32_row_tiles(HDP)>), grid, dim3(512), 0, s, a);
  else hipLaunchKernelGGL((paged_f32_kernel<HDP, CAP, 1>), grid, dim3(512), 0, s, a);
}

// The two parts of a batch with a common context.
template <int HDP, bool CAP>
static void launch_pair(const PagedAttnArgs& a, const PagedAttnArgs& b, int ka, hipStream_t s) {
  const dim3 grid((unsigned)(a.tiles * a.kv.n_kv * a.ranges + b.tiles * b.kv.n_kv * b.ranges));
  if (ka == PAGED_ROWS) hipLaunchKernelGGL((paged_pair_kernel<HDP, CAP, PAGED_ROWS>), grid, dim3(256), 0, s, a, b);
  else if (ka == PAGED_KEYS) hipLaunchKernelGGL((paged_pair_kernel<HDP, CAP, PAGED_KEYS>), grid, dim3(256), 0, s, a, b);
  else hipLaunchKernelGGL((paged_f32_pair_kernel<HDP, CAP>), grid, dim3(512), 0, s, a, b);
}

template <int HDP, bool CAP>
static void launch_parts(const PagedAttnArgs (&a)[2], const PagedPlan& p, hipStream_t s) {
  if (p.n_parts == 2) launch_pair<HDP, CAP>(a[0], a[1], p.part[0].kernel, s);
  else launch_one<HDP, CAP>(a[0], p.part[0].kernel, s);
}

template <typename T, int LPR>
static void launch_merge(const PagedAttnArgs& a, long rows, hipStream_t s) {
  const int wpr = a.slots > 8 ? 4 : 1, rb = 256 / (LPR * wpr);
  const dim3 grid((unsigned)((rows + rb - 1) / rb));
  if (wpr == 4) hipLaunchKernelGGL((paged_merge_kernel<T, LPR, 4>), grid, dim3(256), 0, s, a);
  else hipLaunchKernelGGL((paged_merge_kernel<T, LPR, 1>), grid, dim3(256), 0, s, a);
}
template <typename T>
static void launch_merge(const PagedAttnArgs& a, int hdp, long rows, hipStream_t s) {
  if (hdp == 64) launch_merge<T, 16>(a, rows, s);
  else if (hdp == 128) launch_merge<T, 32>(a, rows, s);
  else launch_merge<T, 64>(a, rows, s);
}

void launch_paged_attention(const PagedAttnArgs& a, const PagedPlan& p, int et, hipStream_t s) {
  if (a.bt.n_tok <= 0 || a.bt.max_new <= 0) return;
  auto mul = [](long d) { return d == 1 ? 0u : (unsigned)(((1ull << 32) + d - 1) / d); };
  PagedAttnArgs part[2] = {a, a};
  int slot = 0;
  for (int i = 0; i < p.n_parts; ++i) {
    const PagedPart& q = p.part[i];
    VLA_REQUIRE(has_kernel(et, q.kernel, p.hdp, i, p.n_parts),
                "no paged attention kernel " + std::to_string(q.kernel) + " for head dim " + std::to_string(p.hdp));
    PagedAttnArgs& b = part[i];
    const bool flat = p.n_parts == 2 && i == 0;
    b.klo = p.n_parts == 2 && i == 1 ? a.shared_len : 0;
    b.khi = flat ? a.shared_len : 1 << 30;
    b.tiles = q.tiles; b.chunk = q.chunk; b.ranges = q.ranges;
    b.slot0 = slot; b.slots = p.slots;
    b.direct = p.n_parts == 1;
    b.mul_g = mul(a.G); b.mul_kv = mul(a.kv.n_kv); b.mul_blocks = mul((long)q.tiles * a.kv.n_kv);
    slot += q.ranges;
  }
  const bool cap = a.cap > 0.f;
  if (p.hdp == 64) cap ? launch_parts<64, true>(part, p, s) : launch_parts<64, false>(part, p, s);
  else if (p.hdp == 128) cap ? launch_parts<128, true>(part, p, s) : launch_parts<128, false>(part, p, s);
  else cap ? launch_parts<256, true>(part, p, s) : launch_parts<256, false>(part, p, s);
  if (p.slots > 1) {
    PagedAttnArgs b = a;
    b.slots = p.slots;
    const long rows = (long)a.bt.n_tok * a.n_q;
    if (et == ET_BF16) launch_merge<bf16>(b, p.hdp, rows, s);
    else launch_merge<float>(b, p.hdp, rows, s);
  }
}
