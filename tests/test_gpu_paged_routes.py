"""Every way in which a paged attention is launched, at shapes that state the way they are there for, so that a
change of the choice cannot leave one untested: ragged rows and keys, pages that a block's window of them does not
hold at once, pages that are not there, and each mask."""
import pytest
import torch

import paged_util as U
from paper_2609_12075_amd import paged

pytestmark = pytest.mark.gpu

# (new, length, heads, page), kernel, ranges
ROUTES = [
    # tiles of 16 rows: a request a tile, several tiles a request, one range and more
    (([1] * 5, [40, 900, 1, 333, 70], (8, 1, 256), 16), "keys", "split"),
    (([20, 3, 17], [600, 333, 17], (8, 2, 64), 2), "keys", "split"),
    (([20, 3, 17], [600, 333, 17], (8, 2, 256), 4), "keys", "split"),
    (([500, 1, 99], [900, 700, 99], (8, 2, 64), 16), "keys", 1),
    (([12, 1, 30], [200, 180, 30], (12, 12, 72), 1), "keys", 1),
    # 128 rows and two key groups: one range and more
    (([470, 30], [1500, 700], (8, 2, 64), 4), "rows2", "split"),
    (([300, 30], [2500, 2100], (8, 2, 128), 8), "rows2", "split"),
    (([300, 30], [2500, 1900], (8, 2, 256), 16), "rows2", "split"),
    (([900, 77, 523], [1200, 300, 600], (16, 8, 64), 1), "rows2", 1),
    # fp32: 16 rows a block, 64 or 32
    (([20, 3, 17], [600, 333, 17], (8, 2, 72), 2), "f32", "split"),
    (([300, 222], [320, 400], (32, 8, 128), 4), "f32_rows", 1),
    (([400, 222], [1620, 1400], (15, 5, 64), 16), "f32_rows", "split"),
    # 256 rows
    (([300, 290, 280, 299, 271, 300], [300, 310, 280, 299, 271, 333], (32, 32, 128), 1), "rows8", 1),
    (([250, 249, 250, 240, 233, 250], [250, 349, 250, 310, 233, 350], (32, 32, 72), 64), "rows8", 1),
    (([250, 249, 250, 240, 233, 250], [250, 349, 250, 310, 233, 350], (32, 32, 104), 2), "rows8", 1),
]
MASKS = [dict(), dict(cap=20.0), dict(causal=False), dict(window=70, prefix="some"), dict(window=33, cap=5.0)]


@pytest.mark.parametrize("mask", MASKS, ids=str)
@pytest.mark.parametrize("shape,kernel,ranges", ROUTES, ids=lambda x: str(x))
def test_routes(shape, kernel, ranges, mask):
    new, length, (n_q, n_kv, hd), page = shape
    f32 = kernel.startswith("f32")
    c = U.Case(new, length, n_q, n_kv, hd, dtype="f32" if f32 else "bf16", page=page, seed=31, extra_rows=2)
    if not mask:                                       # (a mask can change the choice)
        p = paged.attention_plan(len(new), c.rows, max(new), max(length), n_q, n_kv, hd, page, bf16=not f32)
        k = p["parts"][0]
        assert len(p["parts"]) == 1 and (k[0], "split" if k[3] > 1 else 1) == (kernel, ranges), p
        c.table[0][len(c.table[0]) // 3] = -1          # a page that is not there
        c.table[-1][0] = c.k.shape[0]
    mask = dict(mask)
    if mask.get("prefix"):
        mask["prefix"] = [(n * 5) // 8 for n in length]
    pf = torch.tensor(mask["prefix"], dtype=torch.int32, device="cuda") if "prefix" in mask else None
    pool, batch, q = c.device()
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    got = paged.attention(pool, batch, q, out=out, lse=lse, **{**mask, "prefix": pf})
    U.check_attention(c, got, U.attention_ref(c, **mask), lse)
    n = c.starts[-1]
    assert (out[n:] == 7).all() and (lse[n:] == 7).all()
    for _ in range(2):
        again = paged.attention(pool, batch, q, out=torch.full_like(q, 7.0), **{**mask, "prefix": pf})
        assert torch.equal(got, again)


# (new, tails, heads, page, shared), kernel of the common context
SHARED = [
    (([8, 1, 5] * 10, [9, 300, 40] * 10, (8, 4, 64), 4, 1024), "rows"),
    (([8, 1, 5] * 10, [9, 300, 40] * 10, (8, 4, 72), 1, 512), "rows"),
    (([16, 3, 9, 20] * 6, [30, 3, 150, 20] * 6, (8, 2, 256), 16, 512), "rows"),
    (([20, 3, 1], [300, 90, 1], (8, 1, 256), 2, 512), "keys"),
    (([1, 2, 1], [300, 90, 1], (8, 2, 128), 16, 2048), "keys"),
]


@pytest.mark.parametrize("mask", MASKS, ids=str)
@pytest.mark.parametrize("shape,kernel", SHARED, ids=lambda x: str(x)[:60])
def test_shared_routes(shape, kernel, mask):
    new, tails, (n_q, n_kv, hd), page, shared = shape
    length = [shared + t for t in tails]
    c = U.Case(new, length, n_q, n_kv, hd, page=page, seed=32, shared=shared, extra_rows=1)
    p = paged.attention_plan(len(new), c.rows, max(new), max(length), n_q, n_kv, hd, page, shared)
    assert [k[0] for k in p["parts"]] == [kernel, "keys"], p
    if not mask:
        for row in c.table:                            # a page of the common context that is not there
            row[shared // page // 2] = -1
        c.table[1][-2] = -7
    mask = dict(mask)
    if mask.get("prefix"):
        mask["prefix"] = [(n * 5) // 8 for n in length]
    pf = torch.tensor(mask["prefix"], dtype=torch.int32, device="cuda") if "prefix" in mask else None
    pool, batch, q = c.device()
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device="cuda")
    got = paged.shared_attention(pool, batch, q, shared, out=out, lse=lse, **{**mask, "prefix": pf})
    U.check_attention(c, got, U.attention_ref(c, **mask), lse)
    n = c.starts[-1]
    assert (out[n:] == 7).all() and (lse[n:] == 7).all()


@pytest.mark.parametrize("hd", [72, 128])
def test_unseen_values_do_not_reach_long_prompts(hd):
    """Infinite values that a causal row does not see, in the kernel of 256 rows."""
    new, length = ([250, 249, 250, 240, 233, 250], [250, 349, 250, 310, 233, 350])
    c = U.Case(new, length, 32, 32, hd, page=16, seed=33)
    p = paged.attention_plan(6, c.rows, 250, 350, 32, 32, hd)
    assert p["parts"][0][0] == "rows8", p
    j = c.length[0] - 5
    c.v[c.table[0][j // 16], 1, j % 16, 3] = float("inf")
    c.v[c.table[0][j // 16], 2, j % 16, 4] = float("nan")
    pool, batch, q = c.device()
    U.check_attention(c, paged.attention(pool, batch, q), U.attention_ref(c))


def test_two_streams_and_threads_of_calls():
    """Calls on two streams that overlap, each with tensors of its own, give what they give alone; tensors made for a
    call come from that stream's memory."""
    cs = [U.Case([1] * 7, [700 + 13 * i] * 7, 8, 2, 128, page=16, seed=40 + i) for i in range(2)]
    dev = [c.device() for c in cs]
    want = [paged.attention(*d) for d in dev]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for s in streams:
        s.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            got[i].append(paged.attention(*dev[i], stream=s))
            junk = torch.empty(1 << 20, device="cuda").fill_(float("nan"))       # freed at once, on the current stream
            del junk
    torch.cuda.synchronize()
    for i in range(2):
        for x in got[i]:
            assert torch.equal(x, want[i])



@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_loose_bounds_and_empty_batches(dtype):
    """max_new far over what any request can bring; a batch without tokens; caches without a page."""
    c = U.Case([3, 1, 40], [30, 200, 77], 8, 2, 64, dtype=dtype, page=16, seed=50)
    pool, _, q = c.device()
    ref = U.attention_ref(c)
    U.check_attention(c, paged.attention(pool, c.batch(max_new=2 ** 31 - 1), q), ref)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    none = paged.Batch(i32([0, 0]), i32([20]), i32([c.table[0]]), 0, 0, 20)
    empty = q[:0]
    assert paged.attention(pool, none, empty).shape == empty.shape
    assert paged.shared_attention(pool, none, empty, 16).shape == empty.shape
    k = torch.zeros(0, 2, 64, dtype=q.dtype, device="cuda")
    before = pool.k.clone()
    assert paged.append(pool, none, k, k, q=empty, sections=[32]).shape == empty.shape
    no_pages = paged.Batch(i32([0, 2]), i32([0]), torch.zeros(1, 0, dtype=torch.int32, device="cuda"), 2, 2, 0)
    lse = torch.zeros(2, 8, device="cuda")
    out = paged.attention(pool, no_pages, q[:2], lse=lse)
    assert (out == 0).all() and (lse == -float("inf")).all()
    out = paged.attention(pool, no_pages, q[:2], causal=False)
    assert (out == 0).all()
    paged.append(pool, no_pages, k.new_ones(2, 2, 64), k.new_ones(2, 2, 64))
    torch.cuda.synchronize()
    assert torch.equal(before, pool.k)


@pytest.mark.parametrize("dtype,cap", [("bf16", 1e4), ("bf16", 1e-6), ("f32", 1e6), ("f32", 1e-6)])
def test_caps_at_their_limits(dtype, cap):
    c = U.Case([1, 40, 3], [130, 170, 3], 8, 1, 256, dtype=dtype, page=16, seed=51)
    pool, batch, q = c.device()
    U.check_attention(c, paged.attention(pool, batch, q, cap=cap), U.attention_ref(c, cap=cap))
