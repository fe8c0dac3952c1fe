// Paged key/value cache on gfx950: appending to it, with the rotation applied
// on the way.
#include <algorithm>

#include "paged.h"

namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) float f32x4;

template <typename T>
__device__ __forceinline__ void load8(const void* p, long i, float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    const bf16x8 v = *reinterpret_cast<const bf16x8*>(reinterpret_cast<const bf16*>(p) + i);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = (float)v[e];
  } else {
    const f32x4* v = reinterpret_cast<const f32x4*>(reinterpret_cast<const float*>(p) + i);
#pragma unroll
    for (int e = 0; e < 8; ++e) x[e] = v[e / 4][e % 4];
  }
}
template <typename T>
__device__ __forceinline__ void store8(void* p, long i, const float (&x)[8]) {
  if constexpr (sizeof(T) == 2) {
    bf16x8 v;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (bf16)x[e];
    *reinterpret_cast<bf16x8*>(reinterpret_cast<bf16*>(p) + i) = v;
  } else {
    f32x4* v = reinterpret_cast<f32x4*>(reinterpret_cast<float*>(p) + i);
    v[0] = f32x4{x[0], x[1], x[2], x[3]};
    v[1] = f32x4{x[4], x[5], x[6], x[7]};
  }
}

// ---------------------------------------------------------------- append
// One block per token. Pair f turns by pos * base^(-f / half): the angle in
// turns is formed and reduced in fp64, so that far positions keep their
// fraction (pos 2^31 leaves 2^-22 of a turn), and its sine and cosine are
// fp32. They are the same for all heads: computed once into LDS. Bound by the
// rows read and written once (7261 tokens of 48 heads of 128: 178.5 MB in 36.6
// us, 4.9 TB/s, what a large copy moves), single tokens by the launch and two round trips
// (3.7 us a call that is waited for, 2.6 at least).
template <typename T>
__global__ void __launch_bounds__(256) append_kernel(AppendArgs a) {
  __shared__ float cs[128], sn[128];
  const int tok = blockIdx.x, tid = threadIdx.x;
  const int r = request_of(a.bt, tok);
  if (r >= a.bt.n_req) return;                 // a row behind the last request
  const ReqSpan sp = span_of(a.bt, r, a.kv.page_shift);
  if (tok - sp.first >= sp.n) return;
  const int place = sp.len - sp.n + tok - sp.first;
  int page = -1;
  if (place >= 0) page = a.bt.pages[(long)r * a.bt.pages_stride + (place >> a.kv.page_shift)];
  const bool there = (unsigned)page < (unsigned)a.kv.n_pages;
  if (tid < a.half) {
    const int ax = tid < a.s1 ? 0 : (tid < a.s2 ? 1 : 2);
    const int pos = a.pos ? a.pos[(long)tok * a.n_axes + ax] : place;
    const double t = pos * (exp2(tid * a.step) * 0.15915494309189533577);   // turns
    sincospif(2.0f * (float)(t - rint(t)), &sn[tid], &cs[tid]);
  }
  __syncthreads();
  const int hd = a.kv.hd, half = a.half, pu = half / 8, U = pu + (hd - 2 * half) / 8, V = hd / 8;
  const int nq = a.n_q * U, nk = there ? a.kv.n_kv * U : 0, nv = there ? a.kv.n_kv * V : 0;
  const long slot = (long)page * a.kv.page_stride + (long)(place & ((1 << a.kv.page_shift) - 1)) * a.kv.tok_stride;
  for (int i = tid; i < nq + nk + nv; i += 256) {
    float x[8], y[8];
    if (i >= nq + nk) {
      const int h = (i - nq - nk) / V, d = (i - nq - nk) % V * 8;
      load8<T>(a.vin, (long)tok * a.v_ts + (long)h * a.v_hs + d, x);
      store8<T>(const_cast<void*>(a.kv.v), slot + (long)h * a.kv.head_stride + d, x);
      continue;
    }
    const bool is_q = i < nq;
    const int j = is_q ? i : i - nq, h = j / U, u = j % U;
    const void* src = is_q ? a.q : a.kin;
    void* dst = is_q ? a.qo : const_cast<void*>(a.kv.k);
    const long si = is_q ? (long)tok * a.q_ts + (long)h * a.q_hs : (long)tok * a.k_ts + (long)h * a.k_hs;
    const long di = is_q ? (long)tok * a.qo_ts + (long)h * a.qo_hs : slot + (long)h * a.kv.head_stride;
    if (u < pu) {
      const int f = u * 8;
      load8<T>(src, si + f, x);
      load8<T>(src, si + half + f, y);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float c = cs[f + e], s = sn[f + e], xa = x[e], xb = y[e];
        x[e] = xa * c - xb * s;
        y[e] = xb * c + xa * s;
      }
      store8<T>(dst, di + f, x);
      store8<T>(dst, di + half + f, y);
    } else {
      const int d = 2 * half + (u - pu) * 8;
      load8<T>(src, si + d, x);
      store8<T>(dst, di + d, x);
    }
  }
}

}  // namespace

void launch_append(const AppendArgs& a, int et, hipStream_t s) {
  if (a.bt.n_tok <= 0) return;
  if (et == ET_BF16) hipLaunchKernelGGL(append_kernel<bf16>, dim3(a.bt.n_tok), dim3(256), 0, s, a);
  else hipLaunchKernelGGL(append_kernel<float>, dim3(a.bt.n_tok), dim3(256), 0, s, a);
}
