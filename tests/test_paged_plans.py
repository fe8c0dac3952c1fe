"""What the choice of paged attention launches gives: only kernels that there are, in launches that hold every key (host
only)."""
import random

import pytest

from paper_2609_12075_amd import paged

HEADS = [(15, 5, 64), (8, 1, 256), (4, 4, 64), (32, 8, 128), (16, 2, 128), (12, 12, 72), (10, 2, 96), (7, 1, 80), (3, 3, 8)]


@pytest.mark.parametrize("bf16", [True, False])
def test_every_plan_names_a_kernel_of_its_type(bf16):
    rng = random.Random(11)
    seen = set()
    for _ in range(3000):
        n_q, n_kv, hd = rng.choice(HEADS)
        req, new = rng.randint(1, 64), rng.choice([1, rng.randint(2, 40), rng.randint(2, 3000)])
        page = rng.choice([1, 16, 64])
        max_len = new + rng.randint(0, 9000)
        shared = rng.choice([0, 0, max_len // 2 // page * page])
        causal = rng.random() < 0.8
        kw = dict(cap=rng.choice([0.0, 30.0]), causal=causal, window=rng.choice([0, 500]) if causal else 0,
                  prefix=causal and rng.random() < 0.3)
        p = paged.attention_plan(req, req * new, new, max_len, n_q, n_kv, hd, page, shared, bf16=bf16, **kw)
        names = [k[0] for k in p["parts"]]
        hdp = 64 if hd <= 64 else 128 if hd <= 128 else 256
        assert p["hdp"] == hdp and len(names) == (2 if shared else 1)
        if not bf16:
            assert all(n == "f32" or (n == "f32_rows" and not shared and hdp < 256) for n in names), (p, kw)
        elif shared:
            assert names[0] in ("keys", "rows") and names[1] == "keys", (p, kw)
        else:
            assert names[0] in ("keys", "rows2") or (names[0] == "rows8" and hdp == 128), (p, kw)
        seen.update(names)
        # ranges of all parts hold the keys of the part, in tiles of the kernel
        for (name, _, chunk, ranges), keys in zip(p["parts"], [shared, max_len - shared] if shared else [max_len]):
            wide = 1 if hdp == 256 else 2
            kt = 16 if name.startswith("f32") else 16 * wide if name == "keys" else 32 * wide
            assert chunk * ranges * kt >= keys, (p, kw)
    assert seen == ({"keys", "rows", "rows2", "rows8"} if bf16 else {"f32", "f32_rows"})
