"""Paged attentions with scratch of their own of the told size, caps and prefixes among them, eager and captured."""
import pytest
import torch

import paged_util as U
from paper_2609_12075_amd import paged

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("mask", [dict(), dict(cap=30.0), dict(prefix=True), dict(cap=30.0, prefix=True, window=100)], ids=str)
@pytest.mark.parametrize("new,length,heads,shared", [([1] * 16, [401] * 16, (16, 2, 128), 0), ([1] * 5, [301] * 5, (8, 1, 256), 128),
                                                     ([90, 3], [700, 500], (8, 2, 64), 0)], ids=lambda x: str(x)[-20:])
@pytest.mark.parametrize("stated", [True, False])
def test_attention_with_the_told_scratch(new, length, heads, shared, mask, stated):
    c = U.Case(new, length, *heads, page=16, seed=70, shared=shared)
    pool, batch, q = c.device()
    mask = dict(mask)
    if mask.get("prefix"):
        mask["prefix"] = [n // 2 for n in length]
    pf = torch.tensor(mask["prefix"], dtype=torch.int32, device="cuda") if "prefix" in mask else None
    kw = dict(cap=mask.get("cap", 0.0), prefix=pf is not None) if stated else {}
    need = paged.workspace_bytes(pool, batch, heads[0], shared, window=mask.get("window", 0), **kw)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda") if need else None
    out = torch.zeros_like(q)

    def step():
        args = dict(out=out, ws=ws, **{**mask, "prefix": pf})
        return paged.shared_attention(pool, batch, q, shared, **args) if shared else paged.attention(pool, batch, q, **args)

    step()
    torch.cuda.synchronize()
    ref = U.attention_ref(c, **mask)
    U.check_attention(c, out, ref)
    want = out.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for _ in range(3):
        out.fill_(7.0)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
