"""Scratch of a paged attention as paged.workspace_bytes tells it, against what the call itself asks for (host only)."""
import ctypes
import itertools
import random
import types

import pytest

from paper_2609_12075_amd import paged, vla


def of_sizes(req, tok, max_new, max_len, n_kv, hd, page, dtype):
    """Stand-ins for a pool and a batch of such sizes (their memory is not looked at)."""
    pool = paged.KVPoolC(0, dtype, n_kv, hd, page, 4, None, None, page * n_kv * hd, page * hd, hd)
    batch = paged.RaggedC(req, tok, max_new, max_len, None, None, None, -(-max_len // page))
    return tuple(types.SimpleNamespace(c=x, ref=ctypes.byref(x)) for x in (pool, batch))


def asked(pool, batch, n_q, shared, causal, window, cap, prefix):
    """What vla_paged_attention and vla_shared_attention compare ws_bytes with."""
    a = paged.AttentionArgsC(n_q=n_q, causal=int(causal), window=window, cap=cap, prefix=64 if prefix else None)
    need = ctypes.c_size_t()
    vla._check(paged._lib().vla_attention_workspace(pool.ref, batch.ref, ctypes.byref(a), shared, ctypes.byref(need)))
    return need.value


def masks():
    for causal, window, cap, prefix in itertools.product((True, False), (0, 200), (0.0, 1e-3, 30.0), (False, True)):
        if causal or not (window or prefix):
            yield causal, window, cap, prefix


# shapes where a capped call, or one with a prefix, is launched in another way
SHAPES = [((16, 16, 1, 401), (16, 2, 128), 16), ((16, 16, 1, 1956), (8, 1, 256), 64), ((64, 64, 1, 900), (15, 5, 64), 16),
          ((3, 599, 500, 900), (8, 2, 64), 16), ((12, 768, 64, 864), (8, 1, 256), 64), ((5, 4330, 866, 866), (8, 1, 256), 64)]


@pytest.mark.parametrize("dtype", [1, 0], ids=["bf16", "f32"])
@pytest.mark.parametrize("sizes,heads,page", SHAPES, ids=str)
@pytest.mark.parametrize("common", [0, 256])
def test_told_bytes_are_what_the_call_needs(sizes, heads, page, common, dtype):
    pool, batch = of_sizes(*sizes, heads[1], heads[2], page, dtype)
    for causal, window, cap, prefix in masks():
        need = asked(pool, batch, heads[0], common, causal, window, cap, prefix)
        kw = dict(shared_len=common, causal=causal, window=window)
        # cap and prefix left out: enough for every call
        assert paged.workspace_bytes(pool, batch, heads[0], **kw) >= need, (causal, window, cap, prefix)
        assert paged.workspace_bytes(pool, batch, heads[0], cap=cap, **kw) >= need
        assert paged.workspace_bytes(pool, batch, heads[0], prefix=prefix, **kw) >= need
        assert paged.workspace_bytes(pool, batch, heads[0], cap=cap, prefix=prefix, **kw) == need


def test_shapes_where_a_cap_or_a_prefix_needs_more():
    pool, batch = of_sizes(16, 16, 1, 401, 2, 128, 16, 1)
    assert asked(pool, batch, 16, 0, True, 0, 0.0, False) == 0 < asked(pool, batch, 16, 0, True, 0, 30.0, False)
    assert paged.workspace_bytes(pool, batch, 16) == paged.workspace_bytes(pool, batch, 16, cap=30.0) > 0
    assert paged.workspace_bytes(pool, batch, 16, cap=0.0, prefix=False) == 0


def test_told_bytes_over_drawn_sizes():
    rng = random.Random(7)
    more = 0
    for _ in range(1500):
        req, new = rng.randint(1, 64), rng.choice([1, 1, rng.randint(2, 600)])
        n_q, n_kv, hd = rng.choice([(15, 5, 64), (8, 1, 256), (4, 4, 64), (32, 8, 128), (16, 2, 128), (12, 12, 72)])
        page, tok = rng.choice([1, 16, 64]), req * new
        max_len = new + rng.randint(0, 4000)
        shared = rng.choice([0, rng.randint(0, max_len) // page * page])
        pool, batch = of_sizes(req, tok, new, max_len, n_kv, hd, page, rng.randint(0, 1))
        causal, window, cap, prefix = rng.choice(list(masks()))
        need = asked(pool, batch, n_q, shared, causal, window, cap, prefix)
        assert paged.workspace_bytes(pool, batch, n_q, shared, causal, window) >= need
        more += need > asked(pool, batch, n_q, shared, causal, window, 0.0, False)
    assert more > 0


@pytest.mark.parametrize("kw,msg", [(dict(cap=-1.0), "cap"), (dict(cap=float("nan")), "cap"),
                                    (dict(causal=False, prefix=True), "prefix"), (dict(causal=False, window=3), "window"),
                                    (dict(shared_len=8), "shared_len")])
def test_refusals_of_the_call_are_told(kw, msg):
    pool, batch = of_sizes(2, 2, 1, 64, 2, 64, 16, 1)
    with pytest.raises(vla.VlaError, match=msg):
        paged.workspace_bytes(pool, batch, 4, **kw)
