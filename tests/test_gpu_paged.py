"""Paged cache on the GPU against the 64-bit definitions, at the sizes, masks
and layouts where it can go wrong."""
import math

import numpy as np
import pytest
import torch

import paged_util as U
from paper_2609_12075_amd import paged, synth, vla

pytestmark = pytest.mark.gpu


def run(c, cap=0.0, causal=True, window=0, prefix=None, scale=None, shared=None, lse=True, **kw):
    """The operator and its bound; checks every output row and the rows behind the last request."""
    pool, batch, q = c.device()
    out = torch.full_like(q, 7.0)
    ls = torch.full(q.shape[:2], 7.0, device="cuda") if lse else None
    pf = None if prefix is None else torch.tensor(prefix, dtype=torch.int32, device="cuda")
    a = dict(out=out, lse=ls, cap=cap, causal=causal, window=window, prefix=pf, scale=scale or 0.0, **kw)
    got = paged.attention(pool, batch, q, **a) if shared is None else paged.shared_attention(pool, batch, q, shared, **a)
    torch.cuda.synchronize()
    ref = U.attention_ref(c, cap, causal, window, prefix, scale)
    worst = U.check_attention(c, got, ref, ls)
    n = c.starts[-1]
    assert (got[n:] == 7).all() and (ls is None or (ls[n:] == 7).all()), "rows behind the last request"
    print(f"worst {worst:.3f} of the bound", flush=True)
    return got


HEADS = [(4, 4, 64), (15, 5, 64), (8, 1, 256), (8, 2, 128), (6, 2, 72), (5, 1, 80), (4, 2, 96), (3, 3, 8), (2, 1, 32),
         (40, 1, 64), (3, 1, 200)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_single_tokens(heads, dtype):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 200, 513, 1030]
    run(U.Case([1] * len(lens), lens, *heads, dtype=dtype, page=16, seed=1, extra_rows=3))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads", HEADS, ids=str)
def test_prompts(heads, dtype):
    run(U.Case([1, 33, 0, 70, 129, 5], [1, 33, 20, 200, 129, 300], *heads, dtype=dtype, page=32, seed=2, extra_rows=1))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("page", [1, 2, 8, 16, 64, 128, 1024])
def test_page_sizes(page, dtype):
    run(U.Case([1, 40, 3], [130, 170, 3], 4, 2, 64, dtype=dtype, page=page, seed=3))


MASKS = [dict(causal=False), dict(window=1), dict(window=17), dict(window=64, prefix=[5, 100, 0, 300]),
         dict(window=3, prefix=[200, 1, 65, 0]), dict(prefix=[200, 70, 64, 129]), dict(cap=30.0),
         dict(cap=5.0, window=100, prefix=[0, 64, 10, 3]), dict(causal=False, cap=50.0), dict(scale=0.3), dict(cap=0.5)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", MASKS, ids=str)
@pytest.mark.parametrize("new", [[1, 1, 1, 1], [130, 3, 64, 50]], ids=["tokens", "prompts"])
@pytest.mark.parametrize("heads", [(4, 2, 64), (8, 1, 128), (2, 1, 256)], ids=str)
def test_masks(heads, new, mask, dtype):
    run(U.Case(new, [200, 517, 64, 330], *heads, dtype=dtype, page=16, seed=4), **mask)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_see_nothing(dtype):
    # tokens before the first place (more brought than had), requests of length 0, pages that are not there
    c = U.Case([5, 2, 1, 3, 1], [3, 0, 70, 40, 33], 4, 2, 64, dtype=dtype, page=8, seed=5)
    c.table[2] = [-1] * len(c.table[2])                # no page at all
    c.table[3][1] = c.k.shape[0]                       # one past the pool
    c.table[3][2] = -2 ** 31
    c.table[4][0] = 2 ** 31 - 1
    got = run(c)
    assert (got[:2] == 0).all() and (got[5:8] == 0).all()
    run(c, causal=False)
    run(c, window=2, prefix=[1, 5, 9, 12, 0])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 40], ids=["tokens", "prompts"])
def test_unseen_values_do_not_reach_the_output(new, dtype):
    """Free slots, free pages and tokens that a row does not see hold infinities and NaN."""
    c = U.Case([new, new, new], [90, 300, 61], 4, 2, 128, dtype=dtype, page=16, seed=6, spare=4)
    used = torch.zeros(c.k.shape[0], c.page, dtype=torch.bool)
    for r, n in enumerate(c.length):
        for j in range(n):
            used[c.table[r][j // c.page], j % c.page] = True
    for pool, bad in ((c.k, math.nan), (c.v, math.inf)):
        pool.permute(0, 2, 1, 3)[~used] = bad
    run(c)
    run(c, causal=False)
    # the last token's value and key are infinite and NaN: only it sees them
    for r in (0, 2):
        j = c.length[r] - 1
        c.v[c.table[r][j // c.page], 1, j % c.page, ::3] = math.inf
        c.v[c.table[r][j // c.page], 0, j % c.page, 5] = math.nan
        c.v[c.table[r][j // c.page], 0, j % c.page, 7] = -math.inf
    run(c)
    j = c.length[1] - 1
    c.k[c.table[1][j // c.page], 0, j % c.page, 5] = math.nan
    run(c)
    # and values past the window
    c.v[c.table[1][0], :, 0] = math.nan
    run(c, window=40)


def test_scores_of_extreme_size():
    c = U.Case([1, 37], [100, 90], 4, 2, 64, page=16, seed=7, q_scale=300.0)
    run(c)
    run(c, cap=20.0)
    c = U.Case([1, 37], [100, 90], 4, 2, 64, dtype="f32", page=16, seed=7, q_scale=300.0)
    run(c, cap=20.0)
    # keys of the type's lowest value: scores of -inf weigh nothing
    c = U.Case([1], [70], 2, 1, 64, dtype="f32", page=16, seed=8)
    c.q.abs_()
    c.k[c.table[0][1]] = torch.finfo(torch.float32).min
    run(c)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new", [1, 50], ids=["tokens", "prompts"])
def test_layouts(new, dtype):
    """A token-major pool inside a larger one, queries as a slice of a fused row, outputs into wider rows."""
    c = U.Case([new, new, 2], [100, 140, 70], 6, 2, 64, dtype=dtype, page=16, seed=9)
    ref = U.attention_ref(c)
    n, h, p, d = c.k.shape
    big = torch.full((n, 2, p, h + 1, d + 16), math.nan, dtype=U.DT[dtype], device="cuda")   # [page][k|v][slot][head]
    k, v = (big[:, i, :, :h, 8:8 + d].permute(0, 2, 1, 3) for i in (0, 1))
    k.copy_(c.k)
    v.copy_(c.v)
    qkv = torch.randn(c.rows, 6 + 4, d, device="cuda").to(U.DT[dtype])
    qkv[:, 4:] = c.q.cuda()
    out = torch.full((c.rows, 6, 2 * d), 7.0, dtype=U.DT[dtype], device="cuda")
    got = paged.attention(paged.KVPool(k, v), c.batch(), qkv[:, 4:], out=out[:, :, d:])
    U.check_attention(c, got, ref)
    assert (out[:, :, :d] == 7).all()
    head_major = torch.empty(6, c.rows, d, dtype=U.DT[dtype], device="cuda").transpose(0, 1)
    U.check_attention(c, paged.attention(paged.KVPool(k, v), c.batch(), qkv[:, 4:], out=head_major), ref)


def test_offsets_past_32_bits():
    """Pages whose elements lie behind 2^32 (and bytes behind 2^33)."""
    c = U.Case([1, 40], [300, 200], 4, 2, 64, page=16, seed=10)
    n = c.k.shape[0]
    stride = (1 << 32) // (n - 2) // 8 * 8
    k, v = (torch.empty(stride * (n - 1) + 2048, dtype=torch.bfloat16, device="cuda").as_strided(
        c.k.shape, (stride, 1024, 64, 1)) for _ in range(2))
    assert (n - 1) * stride > 1 << 32
    k.copy_(c.k)
    v.copy_(c.v)
    U.check_attention(c, paged.attention(paged.KVPool(k, v), c.batch(), c.q.cuda()), U.attention_ref(c))
    new = torch.randn(c.rows, 2, 64).bfloat16()
    paged.append(paged.KVPool(k, v), c.batch(), new.cuda(), new.cuda())
    _, kp, vp, _ = U.append_ref(c, new, new, c.q, None, [], 1e4)
    assert torch.equal(k.cpu().double(), kp) and torch.equal(v.cpu().double(), vp)


SHARED = [
    dict(heads=(8, 1, 256), new=[1] * 16, tail=[1, 2, 63, 64, 65, 30, 5, 50, 17, 9, 40, 33, 1, 1, 100, 7], shared=832, page=64),
    dict(heads=(8, 2, 128), new=[1] * 5, tail=[1, 300, 17, 64, 2], shared=1024, page=16),
    dict(heads=(15, 5, 64), new=[7, 1, 0, 3, 12], tail=[7, 40, 0, 200, 12], shared=512, page=128),
    dict(heads=(4, 4, 64), new=[1, 1], tail=[3, 1], shared=16, page=16),
    dict(heads=(12, 12, 72), new=[1] * 3, tail=[1, 70, 5], shared=128, page=8),
    dict(heads=(2, 1, 64), new=[60, 50, 1], tail=[60, 80, 1], shared=256, page=32),
    dict(heads=(4, 2, 64), new=[1], tail=[40], shared=192, page=64),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("mask", [dict(), dict(cap=30.0), dict(window=40, prefix="some"), dict(causal=False)], ids=str)
@pytest.mark.parametrize("s", SHARED, ids=lambda s: str(s["heads"]))
def test_shared(s, mask, dtype):
    c = U.Case(s["new"], [s["shared"] + t for t in s["tail"]], *s["heads"], dtype=dtype, page=s["page"], seed=11,
               shared=s["shared"], extra_rows=2)
    mask = dict(mask)
    if mask.get("prefix"):
        mask["prefix"] = [(37 * r) % (s["shared"] + 9) for r in range(len(s["new"]))]
    run(c, shared=s["shared"], **mask)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shared_pages_of_row_0_and_short_requests(dtype):
    """Requests that end inside the common context see what their length leaves; the common entries are row 0's."""
    c = U.Case([1, 2, 1, 3, 1], [300, 256, 100, 17, 0], 4, 2, 64, dtype=dtype, page=16, seed=12, shared=256)
    run(c, shared=256)
    run(c, shared=256, causal=False)
    pool, batch, q = c.device()
    table = batch.pages.clone()
    table[1:, :256 // 16] = -1
    other = paged.Batch(batch.start, batch.kv_len, table, batch.n_tok, max(c.new), max(c.length))
    a = paged.shared_attention(pool, batch, q, 256)
    b = paged.shared_attention(pool, other, q, 256)
    assert torch.equal(a, b)


def test_shared_unseen_values_do_not_reach_the_output():
    c = U.Case([1, 4, 1], [130, 140, 128], 4, 2, 64, page=16, seed=13, shared=128)
    j = 127                                                    # the last common token, past a window of the others
    c.v[c.table[0][j // 16], 0, j % 16] = math.nan
    c.v[c.table[0][0], 1, 3] = math.inf
    run(c, shared=128, window=5)
    run(c, shared=128)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_do_not_depend_on_the_batch_and_repeat(dtype):
    c = U.Case([1, 100, 9], [700, 333, 50], 8, 2, 64, dtype=dtype, page=32, seed=14)
    pool, batch, q = c.device()
    a = paged.attention(pool, batch, q)
    for _ in range(3):
        assert torch.equal(a, paged.attention(pool, batch, q))
    loose = c.batch(max_new=150, max_len=len(c.table[0]) * c.page)
    U.check_attention(c, paged.attention(pool, loose, q), U.attention_ref(c))


def test_other_stream_and_given_workspace():
    c = U.Case([1, 100, 9], [700, 333, 50], 8, 2, 64, page=32, seed=15)
    pool, batch, q = c.device()
    ref = U.attention_ref(c)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    a = paged.attention(pool, batch, q, stream=s)
    need = paged.workspace_bytes(pool, batch, 8)
    b = paged.attention(pool, batch, q, ws=torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"), stream=s)
    s.synchronize()
    assert torch.equal(a, b)
    U.check_attention(c, a, ref)
    if need > 16:
        with pytest.raises(vla.VlaError, match="scratch"):
            paged.attention(pool, batch, q, ws=torch.empty(16, dtype=torch.uint8, device="cuda"))


def test_replayed_step_follows_changed_lengths():
    """A captured step (append, attention, shared attention) is replayed while the device tensors of the batch
    change within their bounds; every replay equals the eager call."""
    c = U.Case([1, 1, 1, 1], [140, 131, 200, 129], 8, 2, 64, page=16, seed=16, shared=128, spare=40)
    pool, _, q = c.device()
    free = [p for p in range(c.k.shape[0]) if all(p not in row for row in c.table)]
    for row in c.table:                                        # room for the tokens to come
        row[row.index(-1)] = free.pop()
    batch = c.batch(max_len=len(c.table[0]) * 16)
    kn, vn = (torch.randn(4, 2, 64, device="cuda").bfloat16() for _ in range(2))
    qo, o1, o2 = (torch.zeros_like(q) for _ in range(3))
    ws = [torch.empty(max(16, paged.workspace_bytes(pool, batch, 8, s)), dtype=torch.uint8, device="cuda") for s in (0, 128)]

    def step():
        paged.append(pool, batch, kn, vn, q=q, q_out=qo, sections=[32])
        paged.attention(pool, batch, qo, out=o1, ws=ws[0])
        paged.shared_attention(pool, batch, qo, 128, out=o2, ws=ws[1])

    step()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for i in range(5):
        batch.kv_len += 1
        q.copy_(torch.randn_like(q))
        kn.copy_(torch.randn_like(kn))
        step()
        want = [x.clone() for x in (qo, o1, o2, pool.k, pool.v)]
        for x in (qo, o1, o2):
            x.zero_()
        pool.k[batch.pages[:, 8:].long().clamp_min(0).flatten()] *= 1      # eager work between the replays
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip((qo, o1, o2, pool.k, pool.v), want):
            assert torch.equal(x, y), i
        c.length = [n + 1 for n in c.length]
        c.k, c.v, c.q = pool.k.cpu(), pool.v.cpu(), qo.cpu()
        ref = U.attention_ref(c)
        U.check_attention(c, o1, ref)
        U.check_attention(c, o2, ref)


# ------------------------------------------------------------------ append
APPENDS = [
    dict(heads=(8, 1, 256), sections=[128], new=[1], length=[900], page=64),
    dict(heads=(15, 5, 64), sections=[16, 8, 8], new=[1, 40, 0, 7], length=[5, 60, 3, 7], page=16),
    dict(heads=(4, 4, 64), sections=[32], new=[3, 1], length=[17, 1], page=1),
    dict(heads=(2, 1, 72), sections=[8, 12, 12], new=[20, 20], length=[30, 20], page=8),
    dict(heads=(3, 3, 8), sections=[], new=[5], length=[9], page=2),
    dict(heads=(4, 2, 128), sections=[0, 8], new=[33, 2], length=[40, 70], page=32),
    dict(heads=(2, 2, 40), sections=[8], new=[9], length=[2 ** 20 + 3], page=65536),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("with_q", [True, False])
@pytest.mark.parametrize("s", APPENDS, ids=lambda s: str(s["heads"]))
def test_append(s, with_q, dtype):
    n_q, n_kv, hd = s["heads"]
    c = U.Case(s["new"], s["length"], n_q, n_kv, hd, dtype=dtype, page=s["page"], seed=17, extra_rows=3, spare=2)
    dt, half, axes = U.DT[dtype], sum(s["sections"]), len(s["sections"])
    g = torch.Generator().manual_seed(1)
    fused = torch.randn(c.rows, 2 * n_kv + 1, hd, generator=g).to(dt)
    k, v = fused[:, :n_kv], fused[:, n_kv:2 * n_kv]
    pos = None
    if axes:
        pos = torch.randint(0, 1 << 20, (c.rows, axes), generator=g, dtype=torch.int32)
        pos[0] = 2 ** 31 - 1
        pos[-1] = -5
    pool, batch, q = c.device()
    fd = fused.cuda()
    q_out = torch.full_like(q, 7.0) if with_q else None
    for positions in ([pos, None] if axes == 1 else [pos]):
        got = paged.append(pool, batch, fd[:, :n_kv], fd[:, n_kv:2 * n_kv], q=q if with_q else None, q_out=q_out,
                           positions=None if positions is None else positions.cuda(), sections=s["sections"])
        torch.cuda.synchronize()
        qo, kp, vp, touched = U.append_ref(c, k, v, c.q, None if positions is None else positions.tolist(),
                                           s["sections"], 10000.0)
        n = c.starts[-1]
        assert torch.equal(pool.v.cpu().double(), vp)
        kd = pool.k.cpu()
        assert torch.equal(kd[~touched], c.k[~touched]), "slots of other tokens"
        err = (kd.double() - kp).abs()[touched]
        assert (err <= U.rotation_bound(kp, dtype)[touched]).all(), float(err.max())
        if not half:
            assert torch.equal(kd.double(), kp)
        if with_q:
            gq = got.cpu()
            assert (gq[n:] == 7).all(), "rows behind the last request"
            assert ((gq[:n].double() - qo[:n]).abs() <= U.rotation_bound(qo[:n], dtype)).all()


def test_append_in_place_and_pages_that_are_not_there():
    c = U.Case([6, 4, 2], [20, 4, 1], 4, 2, 64, page=4, seed=18, spare=3)
    c.table[0][4] = -1                                          # places 16 .. 19 of request 0 have no page
    c.table[1][0] = c.k.shape[0]
    pool, batch, q = c.device()
    k, v = (torch.randn(c.rows, 2, 64).bfloat16() for _ in range(2))
    back = paged.append(pool, batch, k.cuda(), v.cuda(), q=q, q_out=q, sections=[32])
    assert back is q
    qo, kp, vp, touched = U.append_ref(c, k, v, c.q, None, [32], 10000.0)
    assert int(touched[:, 0].sum()) == 2 + 0 + 1
    assert torch.equal(pool.v.cpu().double(), vp)
    assert ((pool.k.cpu().double() - kp).abs() <= U.rotation_bound(kp, "bf16")).all()
    assert ((q.cpu().double() - qo).abs() <= U.rotation_bound(qo, "bf16")).all()


def test_lengths_out_of_their_bounds_stay_inside_the_buffers():
    """start and kv_len past the stated bounds: results of those requests are unspecified, the others' are right
    and nothing else is written."""
    c = U.Case([1, 1, 1], [40, 30, 20], 4, 2, 64, page=16, seed=19, extra_rows=2)
    pool, batch, q = c.device()
    ref = U.attention_ref(c)
    batch.kv_len[1] = 10 ** 6
    batch.pages[1, 2:] = 0
    out = paged.attention(pool, batch, q, out=torch.full_like(q, 7.0))
    want = paged.attention(pool, c.batch(), q)
    assert torch.equal(out[0], want[0]) and torch.equal(out[2], want[2]) and (out[3:] == 7).all()
    assert ref[0].shape == out.shape
    batch.kv_len[1] = -7
    out = paged.attention(pool, batch, q, out=torch.full_like(q, 7.0))
    assert torch.equal(out[0], want[0]) and torch.equal(out[2], want[2]) and (out[1] == 0).all()


# ------------------------------------------------------------------ bindings' refusals
def test_binding_refusals():
    c = U.Case([1, 2], [10, 20], 4, 2, 64, page=16, seed=20)
    pool, batch, q = c.device()
    k = torch.zeros(c.rows, 2, 64, device="cuda", dtype=torch.bfloat16)
    for bad in (q[:2], q[:, :, :32], q.float(), q.cpu(), q[0], q.transpose(1, 2).contiguous().transpose(1, 2)):
        with pytest.raises((ValueError, TypeError)):
            paged.attention(pool, batch, bad)
    with pytest.raises(vla.VlaError, match="multiple of n_kv"):
        paged.attention(pool, batch, q[:, :3])
    with pytest.raises(ValueError, match="lse"):
        paged.attention(pool, batch, q, lse=torch.zeros(c.rows, 3, device="cuda"))
    with pytest.raises(ValueError, match="prefix"):
        paged.attention(pool, batch, q, prefix=torch.zeros(2, device="cuda", dtype=torch.int64))
    with pytest.raises(ValueError, match="prefix"):
        paged.attention(pool, batch, q, prefix=torch.zeros(3, device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError, match="positions"):
        paged.append(pool, batch, k, k, positions=torch.zeros(c.rows, 1, device="cuda", dtype=torch.int32), sections=[8, 8])
    with pytest.raises(ValueError, match="three axes"):
        paged.append(pool, batch, k, k, sections=[8, 8, 8, 8])
    with pytest.raises(ValueError):
        paged.append(pool, batch, k[:, :1], k)
    with pytest.raises(ValueError):
        paged.append(pool, batch, k, k, q=q, q_out=q[:, :3], sections=[8])
    with pytest.raises(vla.VlaError, match="page_tokens"):
        paged.attention(paged.KVPool(pool.k[:, :, :15], pool.v[:, :, :15]), batch, q)
    with pytest.raises(vla.VlaError, match="shared_len"):
        paged.shared_attention(pool, batch, q, 8)
    with pytest.raises(ValueError):
        paged.KVPool(pool.k, pool.v[:1])
    with pytest.raises(ValueError):
        paged.KVPool(pool.k.cpu(), pool.v.cpu())
    with pytest.raises(TypeError):
        paged.KVPool(pool.k.half(), pool.v.half())
    with pytest.raises(ValueError, match="kv_len|start"):
        paged.Batch(batch.start.long(), batch.kv_len, batch.pages, c.rows, 2, 20)
    with pytest.raises(vla.VlaError, match="do not fit"):
        paged.attention(pool, paged.Batch(batch.start, batch.kv_len, batch.pages, c.rows, 2, 10 ** 6), q)


# ------------------------------------------------------------------ together, behind the VLM stage
@pytest.mark.parametrize("name", ["tiny", "smolvla", "pi0"])
def test_tokens_decoded_behind_a_prefill(name):
    """The VLM stage's prefix state goes into the pages (no rotation: its keys are rotated), then tokens follow one
    by one: appended with rotation and attended, alone and with the first request's prefix shared by two answers."""
    base = synth.CONFIGS[name]
    cfg = synth.reduced(base, max_batch=2) if name != "tiny" else base
    m = vla.Model(cfg, synth.make_weights(cfg))
    B, P, nq, nk, hd = 2, cfg.prefix_len, cfg.n_q, cfg.n_kv, cfg.head_dim
    inp = {k: torch.from_numpy(np.ascontiguousarray(x)).cuda() for k, x in synth.make_inputs(cfg, B).items()}
    kv = m.alloc_kv(B)
    m.prefill(B, inp["pixels"], inp["text_ids"], kv)
    dt = torch.float32 if cfg.dtype == synth.DTYPE_F32 else torch.bfloat16
    d = "f32" if dt == torch.float32 else "bf16"
    hand = kv.view(dt).view(cfg.llm_layers, 2, B, nk, P, hd)
    page, layer, steps = 16, cfg.llm_layers - 1, 5
    c = U.Case([1, 1], [P + steps] * 2, nq, nk, hd, dtype=d, page=page, seed=21)
    pool, _, _ = c.device()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    pages = i32(c.table)
    for b in range(B):                                          # the hand-off is head-major: tokens are its rows
        one = paged.Batch(i32([0, P]), i32([P]), pages[b:b + 1].contiguous(), P, P, P)
        paged.append(pool, one, hand[layer, 0, b].transpose(0, 1), hand[layer, 1, b].transpose(0, 1))
    c.k, c.v = pool.k.cpu(), pool.v.cpu()
    c.length = [P, P]
    for b in range(B):
        assert torch.equal(c.gathered(b, c.k)[0], hand[layer, 0, b].cpu().double())
        assert torch.equal(c.gathered(b, c.v)[0], hand[layer, 1, b].cpu().double())
    # the framework's attention over the contiguous hand-off and the paged one see the same keys
    g = torch.Generator().manual_seed(3)
    q = torch.randn(B, nq, hd, generator=g).to(dt)
    c.q = q
    ref = U.attention_ref(c)
    batch = c.batch(max_len=P + steps)
    U.check_attention(c, paged.attention(pool, batch, q.cuda()), ref)
    U.check_attention(c, vla.debug_attention(q.cuda()[:, :, None].contiguous(), hand[layer, 0].contiguous(),
                                             hand[layer, 1].contiguous()).view(B, nq, hd), ref)
    for s in range(steps):
        batch.kv_len += 1
        c.length = [n + 1 for n in c.length]
        fused = torch.randn(B, nq + 2 * nk, hd, generator=g).to(dt).cuda()
        qr = paged.append(pool, batch, fused[:, nq:nq + nk], fused[:, nq + nk:], q=fused[:, :nq], sections=[hd // 2],
                          rope_base=cfg.rope_base)
        qo, kp, vp, touched = U.append_ref(c, fused[:, nq:nq + nk].cpu(), fused[:, nq + nk:].cpu(),
                                           fused[:, :nq].cpu(), None, [hd // 2], cfg.rope_base)
        assert int(touched[:, 0].sum()) == B
        assert ((pool.k.cpu().double() - kp).abs() <= U.rotation_bound(kp, d)).all()
        c.k, c.v, c.q = pool.k.cpu(), pool.v.cpu(), qr.cpu()
        ref = U.attention_ref(c, cap=30.0)
        U.check_attention(c, paged.attention(pool, batch, qr, cap=30.0), ref)
    # two answers over the first request's prefix
    whole = P // page * page
    row = pages[0].clone()
    two = torch.stack([row, row])
    two[1, whole // page:] = pages[1, whole // page:]
    c.table = two.tolist()
    batch = paged.Batch(batch.start, batch.kv_len, two, B, 1, P + steps)
    ref = U.attention_ref(c)
    U.check_attention(c, paged.shared_attention(pool, batch, qr, whole), ref)
    U.check_attention(c, paged.attention(pool, batch, qr), ref)
    m.close()
