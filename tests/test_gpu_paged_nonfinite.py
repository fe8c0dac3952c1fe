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


# (new, length, heads, page, common context), the kernels and key tiles a range of the parts, and a key that is
# neither in the first tile that its wave takes of a range nor in the last request's own part
LARGE = [
    (([500, 1, 99], [900, 700, 99], (8, 2, 64), 16, 0), [("keys", 32)], 300),
    (([1] * 64, [600] * 64, (32, 8, 128), 16, 0), [("keys", 20)], 300),
    (([1] * 48, [600] * 48, (8, 8, 256), 16, 0), [("keys", 8)], 326),
    (([900, 77, 523], [1200, 300, 600], (16, 8, 64), 1, 0), [("rows2", 20)], 270),
    (([300, 30], [2500, 1900], (8, 2, 256), 16, 0), [("rows2", 16)], 1224),
    (([300, 290, 280, 299, 271, 300], [300, 310, 280, 299, 271, 333], (32, 32, 128), 1, 0), [("rows8", 6)], 200),
    (([16, 3, 9, 20] * 6, [1054, 1027, 1174, 1044] * 6, (8, 2, 256), 16, 1024), [("rows", 8), ("keys", 12)], 356),
    (([1] * 64, [2088] * 64, (32, 8, 128), 16, 2048), [("rows", 4), ("keys", 4)], 356),
    (([1] * 40, [2078] * 40, (8, 8, 128), 16, 2048), [("keys", 8), ("keys", 4)], 396),
]


@pytest.mark.parametrize("shape,parts,at", LARGE, ids=lambda x: str(x)[-60:])
def test_values_near_the_largest_one(shape, parts, at):
    """Values of 2^123: a weighted sum of them holds as long as no weight is above 1. The scores are 0 but for one key,
    of e^5 (2^7.2) times the weight of the keys before it."""
    new, length, heads, page, shared = shape
    c = U.Case(new, length, *heads, page=page, seed=63, shared=shared)
    p = plan_of(c, shared)
    assert [(x[0], x[2]) for x in p] == parts, p
    c.q.zero_()
    c.q[..., 0] = 1.0
    c.k[..., 0] = 0.0
    for r, n in enumerate(length):
        if at < n:
            c.k[c.table[r][at // page], :, at % page, 0] = 5.0
    c.v = (c.v.float() * 2.0 ** 123).bfloat16()
    pool, batch, q = c.device()
    lse = torch.zeros(q.shape[:2], device="cuda")
    kw = dict(lse=lse, scale=1.0)
    got = paged.shared_attention(pool, batch, q, shared, **kw) if shared else paged.attention(pool, batch, q, **kw)
    ref = U.attention_ref(c, scale=1.0)
    assert torch.isfinite(got).all()
    U.check_attention(c, got, ref, lse)
