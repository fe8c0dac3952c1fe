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


def test_first_calls_of_several_threads_answer_alike():
    """Each thread's first call counts the devices: the same answer for all of them (an error: device 99 is not
    there, or there is no GPU)."""
    import subprocess
    import sys
    code = """
import ctypes, threading
from paper_2609_12075_amd import paged
L = paged._lib()
pool = paged.KVPoolC(99, 1, 2, 64, 16, 8, 4096, 8192, 2048, 1024, 64)
batch = paged.RaggedC(3, 6, 4, 64, 16, 32, 64, 4)
att = paged.AttentionArgsC(q=256, o=512, q_tok_stride=256, q_head_stride=64, o_tok_stride=256, o_head_stride=64, n_q=4, causal=1)
go, got = threading.Barrier(16), []
def call():
    go.wait()
    for _ in range(20):
        got.append((L.vla_paged_attention(ctypes.byref(pool), ctypes.byref(batch), ctypes.byref(att), None), L.vla_last_error()))
ts = [threading.Thread(target=call) for _ in range(16)]
[t.start() for t in ts]
[t.join() for t in ts]
assert len(got) == 320 and len(set(got)) == 1 and got[0][0] != 0 and got[0][1], set(got)
"""
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300,
                       cwd=__file__.rsplit("/", 2)[0])
    assert r.returncode == 0, r.stderr[-2000:]
