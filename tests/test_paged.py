"""Paged cache, host side: exported symbols, refusals before anything touches a
GPU, and the 64-bit definitions that the GPU tests compare with."""
import ctypes
import math
import os
import re

import pytest
import torch

import paged_util as U
from paper_2609_12075_amd import paged, vla

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_library_exports_every_declared_symbol():
    src = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "vla_paged.h")).read(), flags=re.S)
    declared = set(re.findall(r"\b(vla_\w+)\s*\(", src))
    assert declared == set(paged.EXPORTS)
    for name in declared:
        assert hasattr(vla.lib(), name), name


def good():
    pool = paged.KVPoolC(device=0, dtype=1, n_kv=2, head_dim=64, page_tokens=16, n_pages=8, k=4096, v=8192,
                         page_stride=2048, head_stride=1024, token_stride=64)
    batch = paged.RaggedC(n_req=3, n_tok=6, max_new=4, max_len=64, start=16, kv_len=32, pages=64, pages_stride=4)
    att = paged.AttentionArgsC(q=256, o=512, q_tok_stride=256, q_head_stride=64, o_tok_stride=256, o_head_stride=64,
                               n_q=4, causal=1)
    app = paged.AppendArgsC(k=256, v=512, k_tok_stride=128, k_head_stride=64, v_tok_stride=128, v_head_stride=64, n_q=4,
                            q=1024, q_out=2048, q_tok_stride=256, q_head_stride=64, qo_tok_stride=256,
                            qo_head_stride=64, n_axes=1, rope_base=1e4)
    app.sections[0] = 32
    return pool, batch, att, app


def refused(call, msg):
    assert call() == vla.VLA_EINVAL
    assert msg in vla.lib().vla_last_error().decode()


@pytest.mark.parametrize("which,field,value,msg", [
    ("pool", "dtype", 2, "dtype"),
    ("pool", "n_kv", 0, "n_kv"),
    ("pool", "head_dim", 60, "head_dim"),
    ("pool", "head_dim", 264, "head_dim"),
    ("pool", "page_tokens", 24, "power of two"),
    ("pool", "n_pages", 0, "n_pages"),
    ("pool", "page_stride", 2044, "pool page stride"),
    ("pool", "head_stride", 1, "pool head stride"),
    ("pool", "token_stride", 68, "pool token stride"),
    ("pool", "token_stride", -64, "pool token stride"),
    ("pool", "k", 4104, "16-byte aligned"),
    ("pool", "v", None, "16-byte aligned"),
    ("batch", "n_req", 0, "n_req"),
    ("batch", "n_tok", -1, "n_tok"),
    ("batch", "max_len", 65, "do not fit"),
    ("batch", "max_len", -1, "out of range"),
    ("batch", "max_new", -1, "out of range"),
    ("batch", "start", None, "null start"),
    ("batch", "kv_len", 34, "4-byte"),
    ("batch", "pages", None, "null start"),
    ("att", "q", None, "null q"),
    ("att", "o", 520, "o must be 16-byte"),
    ("att", "q_tok_stride", 60, "q token stride"),
    ("att", "o_head_stride", 32, "o head stride"),
    ("att", "n_q", 3, "multiple of n_kv"),
    ("att", "n_q", 0, "multiple of n_kv"),
    ("att", "scale", -1.0, "scale"),
    ("att", "scale", math.nan, "scale"),
    ("att", "cap", -1.0, "cap"),
    ("att", "cap", math.inf, "cap"),
    ("att", "causal", 2, "causal"),
    ("att", "window", -1, "window"),
    ("att", "lse", 2, "4-byte"),
    ("att", "prefix", 2, "4-byte"),
])
def test_attention_refusals(which, field, value, msg):
    pool, batch, att, _ = good()
    setattr({"pool": pool, "batch": batch, "att": att}[which], field, value)
    L = paged._lib()
    refused(lambda: L.vla_paged_attention(pool, batch, att, None), msg)
    if msg != "shared_len":
        refused(lambda: L.vla_shared_attention(pool, batch, att, 16, None), msg)


def test_masks_without_causal_refused():
    L = paged._lib()
    pool, batch, att, _ = good()
    att.causal, att.window = 0, 5
    refused(lambda: L.vla_paged_attention(pool, batch, att, None), "window")
    att.window, att.prefix = 0, 64
    refused(lambda: L.vla_paged_attention(pool, batch, att, None), "prefix")


@pytest.mark.parametrize("shared", [0, -16, 8, 80])
def test_shared_length_refusals(shared):
    L = paged._lib()
    pool, batch, att, _ = good()
    refused(lambda: L.vla_shared_attention(pool, batch, att, shared, None), "shared_len")


@pytest.mark.parametrize("field,value,msg", [
    ("k", None, "null k"),
    ("v", 516, "v must be 16-byte"),
    ("k_tok_stride", 68, "k token stride"),
    ("v_head_stride", 8, "v head stride"),
    ("q", None, "null q"),
    ("q_out", None, "null q_out"),
    ("qo_tok_stride", 0, "q_out token stride"),
    ("n_q", -1, "n_q"),
    ("n_axes", 4, "n_axes"),
    ("rope_base", 1.0, "rope_base"),
    ("rope_base", math.inf, "rope_base"),
    ("sections", (33, 0, 0), "sections"),
    ("sections", (4, 0, 0), "sections"),
    ("sections", (0, 0, 0), "sections"),
    ("sections", (-8, 0, 0), "sections"),
    ("positions", 2, "4-byte"),
])
def test_append_refusals(field, value, msg):
    L = paged._lib()
    pool, batch, _, app = good()
    if field == "sections":
        for i, s in enumerate(value):
            app.sections[i] = s
    else:
        setattr(app, field, value)
    refused(lambda: L.vla_kv_append(pool, batch, app, None), msg)


def test_positions_needed_for_several_axes():
    L = paged._lib()
    pool, batch, _, app = good()
    app.n_axes = 2
    app.sections[0], app.sections[1] = 16, 16
    refused(lambda: L.vla_kv_append(pool, batch, app, None), "positions")


def test_null_arguments_refused():
    L = paged._lib()
    pool, batch, att, app = good()
    need = ctypes.c_size_t()
    for args in ((None, batch, att), (pool, None, att), (pool, batch, None)):
        assert L.vla_paged_attention(*args, None) == vla.VLA_EINVAL
        assert L.vla_shared_attention(*args, 16, None) == vla.VLA_EINVAL
        assert L.vla_attention_workspace(*args, 0, ctypes.byref(need)) == vla.VLA_EINVAL
    assert L.vla_attention_workspace(pool, batch, att, 0, None) == vla.VLA_EINVAL
    assert L.vla_kv_append(None, batch, app, None) == vla.VLA_EINVAL
    assert L.vla_kv_append(pool, None, app, None) == vla.VLA_EINVAL
    assert L.vla_kv_append(pool, batch, None, None) == vla.VLA_EINVAL


def test_workspace_is_host_only_and_checked():
    L = paged._lib()
    pool, batch, att, _ = good()
    need = ctypes.c_size_t(123)
    assert L.vla_attention_workspace(pool, batch, att, 0, ctypes.byref(need)) == vla.VLA_OK
    assert L.vla_attention_workspace(pool, batch, att, 16, ctypes.byref(need)) == vla.VLA_OK
    att.n_q = 3
    assert L.vla_attention_workspace(pool, batch, att, 0, ctypes.byref(need)) == vla.VLA_EINVAL


def test_reference_matches_softmax_over_gathered_keys():
    c = U.Case([3, 1, 0, 5], [9, 40, 12, 5], 4, 2, 32, dtype="f32", page=8, seed=3)
    o, lse, bound, _ = U.attention_ref(c, causal=False)
    r = 1
    k = torch.stack([c.k[c.table[r][j // 8], :, j % 8] for j in range(40)]).double()
    v = torch.stack([c.v[c.table[r][j // 8], :, j % 8] for j in range(40)]).double()
    t = c.starts[1]
    for h in range(4):
        s = (k[:, h // 2] @ c.q[t, h].double()) * 32 ** -0.5
        assert torch.allclose(o[t, h], torch.softmax(s, 0) @ v[:, h // 2], atol=1e-12)
        assert abs(float(lse[t, h] - torch.logsumexp(s, 0))) < 1e-12
    # a planted mistake in the definition (scale, one key fewer) is outside the bound
    wrong, *_ = U.attention_ref(c, causal=False, scale=32 ** -0.5 * 1.01)
    assert float(((wrong - o).abs() / bound.clamp_min(1e-30))[:c.starts[-1]].max()) > 1.0


def test_reference_masks():
    c = U.Case([4], [4], 1, 1, 16, dtype="f32", page=4, seed=1)
    v = c.gathered(0, c.v)[0][0]
    o, lse, *_ = U.attention_ref(c, window=1)
    assert torch.allclose(o[:, 0], v)                       # each token sees itself alone
    o, *_ = U.attention_ref(c, window=1, prefix=[2])
    full, *_ = U.attention_ref(c, causal=False)
    assert torch.allclose(o[0], U.attention_ref(c, prefix=[2])[0][0])
    assert not torch.allclose(o[3], full[3])
    c.table[0] = [-1, -1]
    o, lse, *_ = U.attention_ref(c)
    assert (o == 0).all() and (lse == -math.inf).all()


def test_append_reference_rotates_like_complex_numbers():
    c = U.Case([2, 3], [10, 3], 2, 1, 32, dtype="f32", page=4, seed=2)
    g = torch.Generator().manual_seed(0)
    k, v = torch.randn(5, 1, 32, generator=g), torch.randn(5, 1, 32, generator=g)
    pos = [[7, 1, 2], [8, 3, 3], [0, 0, 0], [1, 5, 2], [2, 2, 9]]
    qo, kp, vp, touched = U.append_ref(c, k, v, c.q, pos, [4, 2, 2], 100.0)
    assert int(touched.sum()) == 5
    axis = [0] * 4 + [1] * 2 + [2] * 2
    for t in range(5):
        z = torch.complex(c.q[t, :, :8].double(), c.q[t, :, 8:16].double())
        th = torch.tensor([pos[t][axis[f]] * 100.0 ** (-f / 8) for f in range(8)], dtype=torch.float64)
        z = z * torch.polar(torch.ones_like(th), th)
        assert torch.allclose(qo[t, :, :8], z.real) and torch.allclose(qo[t, :, 8:16], z.imag)
        assert torch.equal(qo[t, :, 16:], c.q[t, :, 16:].double())
    assert torch.equal(vp[c.table[1][0], 0, 2], v[4, 0].double())


def test_plans_without_a_gpu_and_the_bounds_of_one_call():
    """The launch plan is host only; rows that no launch holds are refused before anything is enqueued."""
    p = paged.attention_plan(1, 1, 1, 881, 8, 1, 256, page=64)
    assert p["hdp"] == 256 and p["parts"][0][0] == "keys" and p["parts"][0][3] > 1
    assert [k[0] for k in paged.attention_plan(8, 8, 1, 900, 4, 4, 64, shared_len=512, bf16=False)["parts"]] == ["f32"] * 2
    # no request brings more than the batch's tokens
    assert paged.attention_plan(4, 16, 2 ** 31 - 1, 900, 8, 2, 64) == paged.attention_plan(4, 16, 16, 900, 8, 2, 64)
    for kw in (dict(bf16=True), dict(bf16=False)):
        with pytest.raises(vla.VlaError, match="too many rows"):
            paged.attention_plan(65535, 65535, 1, 64, 4096, 4096, 64, **kw)


@pytest.mark.parametrize("dtype,cap,ok", [(1, 1e4, True), (1, 1.1e4, False), (0, 1e8, True), (1, 1e-6, True), (1, 9e-7, False),
                                          (0, 1e-30, False), (0, -1.0, False), (1, float("nan"), False)])
def test_caps_that_the_scores_precision_does_not_carry(dtype, cap, ok):
    pool, batch, att, _ = good()
    pool.dtype, att.cap = dtype, cap
    need = ctypes.c_size_t()
    call = lambda: vla.lib().vla_attention_workspace(ctypes.byref(pool), ctypes.byref(batch), ctypes.byref(att), 0,   # noqa: E731
                                                     ctypes.byref(need))
    if ok:
        assert call() == vla.VLA_OK
    else:
        refused(call, "cap")
