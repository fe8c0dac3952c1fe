// C ABI of the paged key/value cache (include/vla_paged.h): argument checks,
// and the launches on the pool's device.
#include <algorithm>
#include <cmath>
#include <new>

#include "../../include/vla_paged.h"
#include "model.h"
#include "paged.h"

namespace {

template <typename F>
vla_status guarded(F&& f) {
  try {
    vla_clear_error();
    f();
    return VLA_OK;
  } catch (const VlaError& e) {
    vla_set_error(e.msg);
    return (vla_status)e.status;
  } catch (const std::bad_alloc&) {
    vla_set_error("host allocation failed");
    return VLA_ENOMEM;
  } catch (const std::exception& e) {
    vla_set_error(e.what());
    return VLA_EINVAL;
  }
}

bool aligned(const void* p, size_t n) { return reinterpret_cast<uintptr_t>(p) % n == 0; }

// A stride of rows that 16-byte accesses reach; not looked at where `extent` is 1. (`what` and `along` make the message)
void check_stride(int64_t st, int extent, int hd, int es, const char* what, const char* along) {
  if (extent <= 1) return;
  VLA_REQUIRE(st >= hd && st * es % 16 == 0,
              std::string(what) + along + " stride must be at least head_dim and a multiple of 16 bytes");
}

void check_rows(const void* p, int64_t ts, int64_t hs, int rows, int heads, int hd, int es, const char* what) {
  VLA_REQUIRE(p != nullptr || rows == 0, std::string("null ") + what);
  VLA_REQUIRE(aligned(p, 16), std::string(what) + " must be 16-byte aligned");
  check_stride(ts, rows, hd, es, what, " token");
  check_stride(hs, heads, hd, es, what, " head");
}

void fill(const vla_kv_pool* p, const vla_ragged* b, bool buffers, PagedKV& kv, RaggedBatch& bt) {
  VLA_REQUIRE(p && b, "null pool or batch");
  VLA_REQUIRE(p->dtype == VLA_F32 || p->dtype == VLA_BF16, "pool dtype must be VLA_F32 or VLA_BF16");
  VLA_REQUIRE(p->n_kv >= 1 && p->n_kv <= 4096, "n_kv must be in [1, 4096]");
  VLA_REQUIRE(p->head_dim >= 8 && p->head_dim <= 256 && p->head_dim % 8 == 0, "head_dim must be a multiple of 8 in [8, 256]");
  VLA_REQUIRE(p->page_tokens >= 1 && p->page_tokens <= 65536 && (p->page_tokens & (p->page_tokens - 1)) == 0,
              "page_tokens must be a power of two in [1, 65536]");
  VLA_REQUIRE(p->n_pages >= 1, "n_pages must be positive");
  VLA_REQUIRE(b->n_req >= 1 && b->n_req <= 65535, "n_req must be in [1, 65535]");
  VLA_REQUIRE(b->n_tok >= 0 && b->n_tok < (1 << 24), "n_tok must be in [0, 2^24)");
  VLA_REQUIRE(b->max_new >= 0 && b->max_len >= 0 && b->max_len <= (1 << 30), "max_new or max_len out of range");
  VLA_REQUIRE(b->pages_stride >= 0 && (int64_t)b->pages_stride * p->page_tokens >= b->max_len,
              "max_len tokens do not fit into pages_stride pages");
  const int es = (int)elem_size(p->dtype);
  check_stride(p->page_stride, p->n_pages, p->head_dim, es, "pool", " page");
  check_stride(p->head_stride, p->n_kv, p->head_dim, es, "pool", " head");
  check_stride(p->token_stride, p->page_tokens, p->head_dim, es, "pool", " token");
  VLA_REQUIRE(p->page_tokens == 1 || p->token_stride * es < (1LL << 28), "pool token stride must be below 2^28 bytes");
  if (buffers) {
    VLA_REQUIRE(p->k && p->v && aligned(p->k, 16) && aligned(p->v, 16), "pool k and v must be 16-byte aligned buffers");
    VLA_REQUIRE(b->start && b->kv_len && (b->pages || b->pages_stride == 0), "null start, kv_len or pages");
    VLA_REQUIRE(aligned(b->start, 4) && aligned(b->kv_len, 4) && aligned(b->pages, 4), "start, kv_len and pages must be 4-byte aligned");
    // (does not change while the process runs; first calls of several threads wait for one of them)
    static const int ndev = [] {
      int n = 0;
      VLA_HIP(hipGetDeviceCount(&n));
      return n;
    }();
    VLA_REQUIRE(p->device >= 0 && p->device < ndev, "device " + std::to_string(p->device) + " not present");
  }
  kv.k = p->k; kv.v = p->v;
  kv.page_stride = p->page_stride; kv.head_stride = p->head_stride; kv.tok_stride = p->token_stride;
  kv.n_kv = p->n_kv; kv.hd = p->head_dim; kv.n_pages = p->n_pages; kv.page_shift = __builtin_ctz(p->page_tokens);
  bt.start = b->start; bt.kv_len = b->kv_len; bt.pages = b->pages;
  // (no request brings more than all tokens; products with it stay below 2^30)
  bt.n_req = b->n_req; bt.n_tok = b->n_tok; bt.max_new = std::min(b->max_new, b->n_tok); bt.max_len = b->max_len;
  bt.pages_stride = b->pages_stride;
}

PagedAttnArgs attention_args(const vla_kv_pool* p, const vla_ragged* b, const vla_attention_args* t, bool shared,
                             int shared_len, bool buffers) {
  VLA_REQUIRE(t != nullptr, "null attention arguments");
  PagedAttnArgs a{};
  // (the host's own checks first, so that a refusal needs no GPU)
  fill(p, b, false, a.kv, a.bt);
  VLA_REQUIRE(t->n_q >= 1 && t->n_q <= 4096 && t->n_q % p->n_kv == 0, "n_q must be a multiple of n_kv in [1, 4096]");
  VLA_REQUIRE((long)b->n_tok * t->n_q < (1L << 30), "n_tok * n_q must be below 2^30");
  VLA_REQUIRE(t->scale >= 0.f && std::isfinite(t->scale), "scale must be positive, or 0 for 1 / sqrt(head_dim)");
  // (bf16: a capped score is off by a few 2^-24 of the cap, see `capped`)
  VLA_REQUIRE(t->cap >= 0.f && std::isfinite(t->cap), "cap must be >= 0");
  VLA_REQUIRE(t->cap == 0.f || (t->cap >= 1e-6f && (t->cap <= 1e4f || p->dtype == VLA_F32)),
              "cap must be 0, or at least 1e-6 and (bf16) at most 1e4");
  VLA_REQUIRE(t->causal == 0 || t->causal == 1, "causal must be 0 or 1");
  VLA_REQUIRE(t->window >= 0 && (t->window == 0 || t->causal), "window must be >= 0 and needs causal");
  VLA_REQUIRE(!t->prefix || t->causal, "prefix needs causal");
  if (shared)
    VLA_REQUIRE(shared_len > 0 && shared_len <= b->max_len && shared_len % p->page_tokens == 0,
                "shared_len must be a positive multiple of page_tokens, at most max_len");
  const int es = (int)elem_size(p->dtype);
  if (buffers) {
    check_rows(t->q, t->q_tok_stride, t->q_head_stride, b->n_tok, t->n_q, p->head_dim, es, "q");
    check_rows(t->o, t->o_tok_stride, t->o_head_stride, b->n_tok, t->n_q, p->head_dim, es, "o");
    VLA_REQUIRE(aligned(t->lse, 4) && aligned(t->prefix, 4), "lse and prefix must be 4-byte aligned");
    fill(p, b, true, a.kv, a.bt);
  }
  a.q = t->q; a.o = t->o;
  a.q_ts = t->q_tok_stride; a.q_hs = t->q_head_stride; a.o_ts = t->o_tok_stride; a.o_hs = t->o_head_stride;
  a.lse = t->lse; a.n_q = t->n_q; a.G = t->n_q / p->n_kv;
  a.scale = t->scale > 0.f ? t->scale : 1.0f / std::sqrt((float)p->head_dim);
  a.cap = t->cap; a.causal = t->causal; a.window = std::min(t->window, 1 << 30); a.prefix = t->prefix;
  a.shared_len = shared_len;
  a.ws = static_cast<float*>(t->ws);
  return a;
}

vla_status attend(const vla_kv_pool* p, const vla_ragged* b, const vla_attention_args* t, bool shared, int shared_len,
                  hipStream_t s) {
  return guarded([&] {
    const PagedAttnArgs a = attention_args(p, b, t, shared, shared_len, true);
    const PagedPlan plan = paged_plan(a, p->dtype);
    const size_t need = paged_attention_ws(a, plan);
    VLA_REQUIRE(need == 0 || (t->ws && t->ws_bytes >= need && aligned(t->ws, 16)),
                "this attention needs " + std::to_string(need) + " bytes of 16-byte aligned scratch");
    DeviceGuard g(p->device);
    launch_paged_attention(a, plan, p->dtype, s);
    VLA_HIP(hipGetLastError());
  });
}

}  // namespace

extern "C" {

vla_status vla_kv_append(const vla_kv_pool* p, const vla_ragged* b, const vla_append_args* t, hipStream_t s) {
  return guarded([&] {
    VLA_REQUIRE(t != nullptr, "null append arguments");
    AppendArgs a{};
    fill(p, b, false, a.kv, a.bt);
    const int es = (int)elem_size(p->dtype), rows = b->n_tok, hd = p->head_dim;
    check_rows(t->k, t->k_tok_stride, t->k_head_stride, rows, p->n_kv, hd, es, "k");
    check_rows(t->v, t->v_tok_stride, t->v_head_stride, rows, p->n_kv, hd, es, "v");
    VLA_REQUIRE(t->n_q >= 0 && t->n_q <= 4096, "n_q must be in [0, 4096]");
    if (t->n_q > 0) {
      check_rows(t->q, t->q_tok_stride, t->q_head_stride, rows, t->n_q, hd, es, "q");
      check_rows(t->q_out, t->qo_tok_stride, t->qo_head_stride, rows, t->n_q, hd, es, "q_out");
    }
    VLA_REQUIRE(t->n_axes >= 0 && t->n_axes <= 3, "n_axes must be in [0, 3]");
    int ends[3] = {0, 0, 0}, half = 0;
    for (int i = 0; i < t->n_axes; ++i) {
      VLA_REQUIRE(t->sections[i] >= 0 && t->sections[i] <= 128, "sections must be in [0, 128]");
      half += t->sections[i];
      ends[i] = half;
    }
    if (t->n_axes > 0) {
      VLA_REQUIRE(half > 0 && half % 8 == 0 && 2 * half <= hd,
                  "the sections' pairs must sum to a positive multiple of 8, at most head_dim / 2");
      VLA_REQUIRE(t->rope_base > 1.f && std::isfinite(t->rope_base), "rope_base must be above 1");
      VLA_REQUIRE(t->positions || t->n_axes == 1, "positions may be left out with one axis only");
      VLA_REQUIRE(aligned(t->positions, 4), "positions must be 4-byte aligned");
    }
    fill(p, b, true, a.kv, a.bt);
    a.kin = t->k; a.vin = t->v; a.q = t->q; a.qo = t->q_out;
    a.k_ts = t->k_tok_stride; a.k_hs = t->k_head_stride; a.v_ts = t->v_tok_stride; a.v_hs = t->v_head_stride;
    a.q_ts = t->q_tok_stride; a.q_hs = t->q_head_stride; a.qo_ts = t->qo_tok_stride; a.qo_hs = t->qo_head_stride;
    a.n_q = t->n_q; a.n_axes = t->n_axes;
    a.s1 = ends[0]; a.s2 = t->n_axes > 1 ? ends[1] : half;
    a.half = half; a.pos = t->positions;
    a.step = half ? -std::log2((double)t->rope_base) / half : 0.0;
    DeviceGuard g(p->device);
    launch_append(a, p->dtype, s);
    VLA_HIP(hipGetLastError());
  });
}

vla_status vla_attention_workspace(const vla_kv_pool* p, const vla_ragged* b, const vla_attention_args* t,
                                   int shared_len, size_t* bytes) {
  return guarded([&] {
    VLA_REQUIRE(bytes != nullptr, "null bytes");
    const PagedAttnArgs a = attention_args(p, b, t, shared_len != 0, shared_len, false);
    *bytes = paged_attention_ws(a, paged_plan(a, p->dtype));
  });
}

vla_status vla_debug_paged_plan(const vla_kv_pool* p, const vla_ragged* b, const vla_attention_args* t, int shared_len,
                                int* plan) {
  return guarded([&] {
    VLA_REQUIRE(plan != nullptr, "null plan");
    const PagedPlan q = paged_plan(attention_args(p, b, t, shared_len != 0, shared_len, false), p->dtype);
    plan[0] = q.hdp;
    for (int i = 0; i < 2; ++i) {
      const PagedPart r = i < q.n_parts ? q.part[i] : PagedPart{-1, 0, 0, 0};
      plan[1 + 4 * i] = r.kernel; plan[2 + 4 * i] = r.tiles; plan[3 + 4 * i] = r.chunk; plan[4 + 4 * i] = r.ranges;
    }
  });
}

vla_status vla_paged_attention(const vla_kv_pool* p, const vla_ragged* b, const vla_attention_args* t, hipStream_t s) {
  return attend(p, b, t, false, 0, s);
}

vla_status vla_shared_attention(const vla_kv_pool* p, const vla_ragged* b, const vla_attention_args* t, int shared_len,
                                hipStream_t s) {
  return attend(p, b, t, true, shared_len, s);
}

}  // extern "C"
