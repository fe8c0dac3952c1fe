"""Paged attention where NaN and the largest finite values meet the joins of an attention's parts: key ranges, the waves
of a block, a tile and the tiles before it. Bounds are those of paged_util."""
import math

import pytest
import torch

import paged_util as U
from paper_2609_12075_amd import paged

pytestmark = pytest.mark.gpu


def plan_of(c, shared=0, max_len=None, **kw):
    return paged.attention_plan(len(c.new), c.rows, max(c.new), max_len or max(c.length), c.n_q, c.n_kv, c.hd, c.page,
                                shared, bf16=c.dtype == "bf16", **kw)["parts"]


def check_nan(c, got, lse, head):
    """Every output of the query heads of KV head `head` in the last request is NaN, its log-sum-exp too; and all
    outputs are the definition's."""
    U.check_attention(c, got, U.attention_ref(c), lse)
    grp = c.n_q // c.n_kv
    t = c.starts[-2]
    mine = slice(head * grp, (head + 1) * grp)
    assert torch.isnan(got[t:c.starts[-1], mine]).all() and torch.isnan(lse[t:c.starts[-1], mine]).all()
    assert torch.isfinite(got[:t]).all() and torch.isfinite(lse[:t]).all()


# heads, type, length of the last request, bound on the lengths, ranges: its last keys are alone in the ranges
# 8 to 15, or 16 to 23, which the merge of more than eight takes together
RANGES = [
    ((8, 1, 256), "bf16", 520, 881, 14), ((32, 8, 128), "bf16", 1030, 1056, 9), ((4, 4, 64), "bf16", 1025, 1056, 9),
    ((8, 1, 256), "bf16", 1030, 1088, 17), ((32, 8, 128), "bf16", 2050, 2100, 17), ((4, 4, 64), "bf16", 2070, 2080, 17),
    ((4, 4, 64), "f32", 1030, 1056, 9), ((4, 4, 64), "f32", 2050, 2080, 17),
]


@pytest.mark.parametrize("heads,dtype,length,max_len,ranges", RANGES, ids=str)
@pytest.mark.parametrize("at", ["last", "first"])
def test_nan_key_in_a_range_of_its_own(heads, dtype, length, max_len, ranges, at):
    """A NaN in the newest key, the only keys of a group of ranges, or in the first key."""
    c = U.Case([1], [length], *heads, dtype=dtype, page=16, seed=60)
    assert plan_of(c, max_len=max_len)[0][3] == ranges
    j, head = length - 1 if at == "last" else 0, c.n_kv - 1
    c.k[c.table[0][j // 16], head, j % 16, 5] = math.nan
    c.table[0] += [-1] * (max_len // 16 + 1 - len(c.table[0]))
    pool, _, q = c.device()
    lse = torch.zeros(q.shape[:2], device="cuda")
    check_nan(c, paged.attention(pool, c.batch(max_len=max_len), q, lse=lse), lse, head)


@pytest.mark.parametrize("shared,heads,dtype,ranges", [
    (1024, (8, 2, 128), "bf16", 8), (1024, (4, 2, 64), "bf16", 8), (1024, (8, 1, 256), "bf16", 16),
    (2048, (8, 2, 128), "bf16", 16), (1024, (4, 2, 64), "f32", 8), (2048, (4, 2, 64), "f32", 16)], ids=str)
def test_nan_key_behind_a_common_context(shared, heads, dtype, ranges):
    """The range of what follows the common context is the only one of its group of eight."""
    c = U.Case([1] * 5, [shared + t for t in (32, 1, 9, 17, 30)], *heads, dtype=dtype, page=16, seed=61, shared=shared)
    p = plan_of(c, shared)
    assert [x[3] for x in p] == [ranges, 1], p
    j = c.length[-1] - 1
    c.k[c.table[-1][j // 16], 0, j % 16, 0] = math.nan
    pool, batch, q = c.device()
    lse = torch.zeros(q.shape[:2], device="cuda")
    check_nan(c, paged.shared_attention(pool, batch, q, shared, lse=lse), lse, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,length,heads", [([1], [250], (4, 2, 64)), ([1], [250], (2, 2, 256)),
                                              ([20, 3], [250, 128], (4, 2, 64)),
                                              ([300, 222], [320, 400], (32, 8, 128))], ids=str)
@pytest.mark.parametrize("nan_at,top_at", [(3, 20), (20, 3), (85, 3), (3, 85), (40, 120)])
def test_nan_value_of_a_weight_that_underflows(nan_at, top_at, new, length, heads, dtype):
    """A token sees a NaN value with a weight of e^-200, which fp32 holds as 0: 0 times NaN is NaN, in whichever wave
    of a block the two keys lie (tiles of 16 or 32 keys go to the waves in turn)."""
    c = U.Case(new, length, *heads, dtype=dtype, page=16, seed=62)
    c.q.zero_()
    c.q[..., 0] = 1.0
    c.k[..., 0] = 0.0
    page = c.table[0]
    c.k[page[top_at // 16], 0, top_at % 16, 0] = 200.0
    c.v[page[nan_at // 16], 0, nan_at % 16, ::5] = math.nan
    pool, batch, q = c.device()
    got = paged.attention(pool, batch, q, scale=1.0)
    U.check_attention(c, got, U.attention_ref(c, scale=1.0))
    assert torch.isnan(got[c.starts[1] - 1, 0, ::5]).all() and torch.isfinite(got[c.starts[1] - 1, 0, 1::5]).all()
