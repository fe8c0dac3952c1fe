"""A request's rows in different company: alone, in other orders, beside others."""
import pytest
import torch

import paged_util as U
from paper_2609_12075_amd import paged

pytestmark = pytest.mark.gpu


def of(c, order):
    """The requests of c in another order (or some of them): pool, batch, q and the rows of c that they are."""
    rows = [t for r in order for t in range(c.starts[r], c.starts[r + 1])]
    start = [0]
    for r in order:
        start.append(start[-1] + c.new[r])
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")   # noqa: E731
    batch = paged.Batch(i32(start), i32([c.length[r] for r in order]), i32([c.table[r] for r in order]), n_tok=len(rows),
                        max_new=max(c.new), max_len=max(c.length))
    return batch, c.q[rows].cuda(), rows


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("new,length,heads", [([1] * 6, [700, 1, 33, 1500, 64, 200], (8, 2, 64)),
                                              ([1, 100, 9, 33], [700, 333, 50, 33], (8, 2, 64)),
                                              ([270, 3, 300], [900, 50, 301], (32, 8, 128)),
                                              ([40, 1, 77], [600, 350, 90], (8, 1, 256))], ids=str)
def test_a_request_in_other_batches(new, length, heads, dtype):
    """Another order of the same requests (launched alike: the same bounds and rows): the same bits. Alone, and beside
    fewer: the definition's value (the keys may be cut into other ranges)."""
    c = U.Case(new, length, *heads, dtype=dtype, page=16, seed=80)
    ref = U.attention_ref(c, cap=30.0, window=300, prefix=[40] * len(new))
    pool = paged.KVPool(c.k.cuda(), c.v.cuda())
    n = len(new)

    def call(order):
        batch, q, rows = of(c, order)
        pf = torch.full((len(order),), 40, dtype=torch.int32, device="cuda")
        got = paged.attention(pool, batch, q, cap=30.0, window=300, prefix=pf)
        whole = torch.zeros(c.rows, *got.shape[1:], dtype=got.dtype, device="cuda")
        whole[rows] = got
        return whole, rows

    want, _ = call(range(n))
    U.check_attention(c, want, ref)
    for order in (list(range(n))[::-1], list(range(1, n)) + [0]):
        got, _ = call(order)
        assert torch.equal(got, want), order
    for order in [[r] for r in range(n)] + [[0, n - 1], list(range(n - 1))]:
        got, rows = call(order)
        filled = want.clone()
        filled[rows] = got[rows]
        U.check_attention(c, filled, ref)
