"""The operators of a paged key/value cache: appending to it and attending over it.

A server that answers token by token (action tokens, text) keeps the keys and values of each robot's context in
pages of a shared pool. For every layer of every step it appends the step's keys and values, rotating queries and
keys by their positions on the way, and attends over what the cache then holds: whole prompts when a request
arrives, one token per request afterwards, both in one batch when they are mixed, and, where all requests begin
with the same long context (robots of one cell with one scene and instruction, several answers sampled for one
observation), with that context read once for the batch. The cases are these three calls; head layouts are those
of the configurations in `paper_2609_12075_amd/synth.py` and generic ones.

A batch is ragged: request r brings `new[r]` tokens, which are the last of the `length[r]` tokens it then has. Its
lengths are drawn from the case's own numbers, so that they belong to the case and not to the seed.
"""
import math
import random

import torch

own = False

BASE = 10000.0
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


# ------------------------------------------------------------------ cases


def _append(n_q, n_kv, hd, **kw):
    return {"kind": "append", "dtype": "bf16", "n_q": n_q, "n_kv": n_kv, "hd": hd, "rot": hd, "page": 64, "req": 1,
            "new": 1, "past": 0, "axes": 1, **kw}


def _attend(n_q, n_kv, hd, **kw):
    return {"kind": "attention", "dtype": "bf16", "n_q": n_q, "n_kv": n_kv, "hd": hd, "page": 64, "req": 1, "new": 1,
            "past": 0, "mixed": False, "causal": True, "cap": 0.0, "window": 0, "prefix": 0, **kw}


def _shared(n_q, n_kv, hd, **kw):
    return {"kind": "shared", "dtype": "bf16", "n_q": n_q, "n_kv": n_kv, "hd": hd, "page": 64, "req": 8, "new": 1,
            "past": 0, "shared": 1024, "cap": 0.0, **kw}


def listed():
    return [
        # one robot's next token, one layer: latency
        {"name": "append_token_b1", **_append(8, 1, 256, past=880)},
        # prompts of eleven robots whose image tokens have (time, row, column) positions: ragged, 3 axes
        {"name": "append_prompts_axes_b11", **_append(32, 8, 128, req=11, new=870, past=100, axes=3, page=16)},
        # the small fp32 model: a ragged batch of short prompts
        {"name": "append_f32_b4", **_append(4, 4, 64, dtype="f32", req=4, new=80, past=7)},
        # one robot's next token over its camera frames and instruction: latency
        {"name": "token_b1", **_attend(8, 1, 256, past=880)},
        # next tokens of a full batch over long histories of frames: bound by the keys and values
        {"name": "tokens_b64", **_attend(32, 8, 128, req=64, past=8100, page=16)},
        # prompts of five robots: everybody sees the images and the instruction, the answer is causal; capped scores
        {"name": "prompts_prefix_cap_b5", **_attend(8, 1, 256, req=5, new=866, cap=50.0, prefix=816)},
        # one prompt of many frames, causal: bound by the matrix products
        {"name": "prompt_long", **_attend(32, 8, 128, new=8191)},
        # a chunk of one prompt beside the next tokens of 23 others, with a window past the instruction
        {"name": "mixed_window_b24", **_attend(15, 5, 64, req=24, new=515, past=3000, mixed=True, window=1024, prefix=48,
                                               page=32)},
        # the small fp32 model
        {"name": "prompts_f32_b4", **_attend(4, 4, 64, dtype="f32", req=4, new=88, past=3)},
        # sixteen answers sampled for one observation
        {"name": "shared_samples_b16", **_shared(8, 1, 256, req=16, shared=832, past=50)},
        # next tokens of 64 robots of one cell with a long common context
        {"name": "shared_cell_b64", **_shared(32, 8, 128, req=64, shared=8192, past=400, page=16)},
        # a few tokens of each request, checked at once, over a common context
        {"name": "shared_chunk_b12", **_shared(15, 5, 64, req=12, new=7, shared=4096, past=1100, page=128, cap=30.0)},
    ]


HEADS = [(15, 5, 64), (8, 1, 256), (4, 4, 64), (32, 8, 128), (16, 2, 128), (12, 12, 72), (10, 2, 96), (7, 1, 80)]


def draw(rng):
    def log(lo, hi):
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))

    n_q, n_kv, hd = rng.choice(HEADS)
    heads = {"dtype": "f32" if rng.random() < 0.2 else "bf16", "page": rng.choice([16, 32, 64, 128])}
    kind = rng.choice(["append", "append", "attention", "attention", "attention", "attention", "shared", "shared"])
    if kind == "append":
        rot = rng.choice([hd, hd // 32 * 16]) // 16 * 16
        req = log(1, 64)
        c = _append(n_q, n_kv, hd, rot=rot, req=req, new=rng.choice([1, log(1, max(1, 9000 // req))]),
                    past=log(1, 8000), axes=rng.choice([1, 3]), **heads)
    elif kind == "attention":
        mode = rng.choice(["tokens", "tokens", "prompts", "mixed"])
        cap = rng.choice([0.0, 0.0, 30.0, 50.0])
        window = rng.choice([0, 0, log(16, 4096)])
        prefix = rng.choice([0, log(1, 900)])
        if mode == "tokens":
            c = _attend(n_q, n_kv, hd, req=log(1, 64), past=log(1, 8100), cap=cap, window=window, prefix=prefix, **heads)
        elif mode == "prompts":
            req = log(1, 12)
            c = _attend(n_q, n_kv, hd, req=req, new=log(2, 8000 // req), past=rng.choice([0, log(1, 2000)]), cap=cap,
                        window=window, prefix=prefix, **heads)
            if rng.random() < 0.2:
                c.update(causal=False, window=0, prefix=0)
        else:
            c = _attend(n_q, n_kv, hd, req=log(2, 40), new=log(16, 2000), past=log(1, 4000), mixed=True, cap=cap,
                        window=window, prefix=prefix, **heads)
    else:
        c = _shared(n_q, n_kv, hd, req=log(2, 64), new=rng.choice([1, 1, log(2, 16)]), past=log(1, 600),
                    shared=128 * log(1, 64), cap=rng.choice([0.0, 0.0, 30.0]), **heads)
    # no dearer than the largest listed call (in fp32 the matrix rate is a sixteenth)
    most = {"bytes": 2.0e9, "flops": 5.4e11 / (16 if c["dtype"] == "f32" else 1)}
    while any(work(c)[k] > most[k] for k in most):
        c["req"] = max(1, c["req"] * 3 // 4)
        c["past"] = c["past"] * 3 // 4
        c["new"] = max(1, c["new"] * 3 // 4)
    return c


def _lens(c):
    """The tokens that each request brings, and those that it then has."""
    rng = random.Random(",".join(f"{k}={c[k]}" for k in sorted(c) if k != "name"))
    new, length = [], []
    for r in range(c["req"]):
        n = c["new"]
        if c.get("mixed") and r > 0:
            n = 1
        elif r > 0 and n > 1:
            n = rng.randint(max(1, n // 4), n)
        past = c["past"] if r == 0 else rng.randint(c["past"] // 4, c["past"])
        new.append(n)
        length.append(c.get("shared", 0) + past + n)
    return new, length


def _seen(c, p, length):
    """How many keys the token at position p of a request sees."""
    if not c.get("causal", True):
        return length
    first = max(0, p - c["window"] + 1) if c.get("window") else 0
    prefix = min(c.get("prefix", 0), length)
    return prefix + max(0, p + 1 - max(first, prefix))


def work(c):
    new, length = _lens(c)
    es = DTYPES[c["dtype"]].itemsize
    row = c["hd"] * es
    n = sum(new)
    if c["kind"] == "append":
        # queries, keys and values read and written once, and the positions
        return {"bytes": 2 * n * (c["n_q"] + 2 * c["n_kv"]) * row + 4 * n * c["axes"],
                "flops": 3 * n * (c["n_q"] + c["n_kv"]) * c["rot"]}
    # keys and values that some token of the request sees (a common context once), queries and outputs
    shared = c.get("shared", 0)
    keys, pairs = shared, 0
    for n_r, len_r in zip(new, length):
        seen = [_seen(c, p, len_r) for p in range(len_r - n_r, len_r)]
        pairs += sum(seen)
        if c.get("window") and c.get("causal", True):
            prefix = min(c.get("prefix", 0), len_r)
            keys += prefix + max(0, len_r - max(prefix, len_r - n_r - c["window"] + 1, 0))
        else:
            keys += len_r - shared
    return {"bytes": 2 * keys * c["n_kv"] * row + 2 * n * c["n_q"] * row, "flops": 4 * c["hd"] * c["n_q"] * pairs}


# ------------------------------------------------------------------ inputs


def prepare(case, seed):
    c = case
    dt, dev = DTYPES[c["dtype"]], "cuda"
    g = torch.Generator(device=dev).manual_seed(7919 * seed + 13)
    rng = random.Random(seed)
    new, length = _lens(c)
    page, shared = c["page"], c.get("shared", 0)

    # the pool: pages in any order, some of them nobody's; a common context lies on the same pages for all
    need = [-(-n // page) for n in length]
    common = shared // page
    total = common + sum(n - common for n in need)
    ids = list(range(total + 5))
    rng.shuffle(ids)
    head, rest = ids[:common], ids[common:]
    stride = max(need) + 2
    table = []
    for n in need:
        own_pages, rest = rest[:n - common], rest[n - common:]
        row = head + own_pages
        table.append(row + [-1] * (stride - len(row)))
    shape = (total + 5, c["n_kv"], page, c["hd"])
    st = {"case": c, "new": new, "length": length,
          "k_pool": torch.randn(shape, generator=g, device=dev, dtype=dt),
          "v_pool": torch.randn(shape, generator=g, device=dev, dtype=dt),
          "pages": torch.tensor(table, dtype=torch.int32, device=dev),
          "kv_len": torch.tensor(length, dtype=torch.int32, device=dev)}
    start = [0]
    for n in new:
        start.append(start[-1] + n)
    st["starts"] = start
    st["start"] = torch.tensor(start, dtype=torch.int32, device=dev)
    # token buffers come in steps of eight rows; the rows behind the last request stay as they are
    rows = -(-start[-1] // 8) * 8 if start[-1] > 1 else 1
    st["q"] = 2.0 * torch.randn(rows, c["n_q"], c["hd"], generator=g, device=dev)
    st["q"] = st["q"].to(dt)
    st["out"] = torch.zeros(rows, c["n_q"], c["hd"], device=dev, dtype=dt)
    if c["kind"] == "append":
        # keys and values as a fused projection leaves them: slices of one row
        kv = torch.randn(rows, 2 * c["n_kv"], c["hd"], generator=g, device=dev).to(dt)
        st["k"], st["v"] = kv[:, :c["n_kv"]], kv[:, c["n_kv"]:]
        st["positions"] = torch.tensor(_positions(c, new, length, rows), dtype=torch.int32, device=dev)
        half = c["rot"] // 2
        st["sections"] = [half] if c["axes"] == 1 else [half - 2 * (half * 3 // 8), half * 3 // 8, half * 3 // 8]
    elif c.get("prefix"):
        st["prefix"] = torch.tensor([min(c["prefix"], n) for n in length], dtype=torch.int32, device=dev)
    if own:
        # what a server keeps: the pool for good, the batch's description for all layers of a step
        from paper_2609_12075_amd import paged
        st["pool"] = paged.KVPool(st["k_pool"], st["v_pool"])
        st["batch"] = paged.Batch(st["start"], st["kv_len"], st["pages"], n_tok=rows, max_new=max(new),
                                  max_len=max(length))
    return st


def _positions(c, new, length, rows):
    """One axis: the token's place. Three: a request begins with frames of 16 x 16 image tokens, which share a time
    and have a row and a column each, and goes on with text, whose three positions are equal."""
    out = []
    for n, end in zip(new, length):
        for p in range(end - n, end):
            if c["axes"] == 1:
                out.append([p])
            elif p < 768:
                f, i = divmod(p, 256)
                out.append([16 * f, 16 * f + i // 16, 16 * f + i % 16])
            else:
                out.append([48 + p - 768] * 3)
    return out + [[0] * c["axes"]] * (rows - len(out))


# ------------------------------------------------------------------ one pass


def run(st):
    c = st["case"]
    if own:
        from paper_2609_12075_amd import paged
        if c["kind"] == "append":
            paged.append(st["pool"], st["batch"], st["k"], st["v"], q=st["q"], q_out=st["out"],
                         positions=st["positions"], sections=st["sections"], rope_base=BASE)
            return st["out"], st["k_pool"], st["v_pool"]
        if c["kind"] == "attention":
            return paged.attention(st["pool"], st["batch"], st["q"], out=st["out"], cap=c["cap"], causal=c["causal"],
                                   window=c["window"], prefix=st.get("prefix"))
        return paged.shared_attention(st["pool"], st["batch"], st["q"], c["shared"], out=st["out"], cap=c["cap"])
    if c["kind"] == "append":
        return _plain_append(st)
    return _plain_attention(st)


def _plain_append(st):
    c = st["case"]
    n, half = st["starts"][-1], c["rot"] // 2
    axis = torch.repeat_interleave(torch.arange(c["axes"], device="cuda"),
                                   torch.tensor(st["sections"], device="cuda"))
    freq = BASE ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    angle = st["positions"][:n].long()[:, axis].double() * freq
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

    def rotate(x):
        x = x[:n].float()
        a, b = x[..., :half], x[..., half:2 * half]
        return torch.cat([a * cos - b * sin, b * cos + a * sin, x[..., 2 * half:]], -1).to(DTYPES[c["dtype"]])

    new = torch.tensor(st["new"], device="cuda")
    req = torch.repeat_interleave(torch.arange(c["req"], device="cuda"), new)
    place = torch.arange(n, device="cuda") - st["start"].long()[req + 1] + st["kv_len"].long()[req]
    ids = st["pages"].long()[req, place // c["page"]]
    st["out"][:n] = rotate(st["q"])
    st["k_pool"][ids, :, place % c["page"]] = rotate(st["k"])
    st["v_pool"][ids, :, place % c["page"]] = st["v"][:n]
    return st["out"], st["k_pool"], st["v_pool"]


def _plain_attention(st):
    c = st["case"]
    hd, n_kv = c["hd"], c["n_kv"]
    group = c["n_q"] // n_kv
    for r in range(c["req"]):
        a, n, length = st["starts"][r], st["new"][r], st["length"][r]
        ids = st["pages"][r, :-(-length // c["page"])].long()
        k = st["k_pool"][ids].transpose(0, 1).reshape(n_kv, -1, hd)[:, :length].float()
        v = st["v_pool"][ids].transpose(0, 1).reshape(n_kv, -1, hd)[:, :length].float()
        kt = k.transpose(1, 2).contiguous()
        key = torch.arange(length, device="cuda")
        step = max(1, (1 << 27) // (length * c["n_q"]))
        for i in range(0, n, step):
            m = min(step, n - i)
            q = st["q"][a + i:a + i + m].float().reshape(m, n_kv, group, hd).permute(1, 2, 0, 3).reshape(n_kv, -1, hd)
            s = torch.matmul(q, kt).view(n_kv, group, m, length) / math.sqrt(hd)
            if c["cap"]:
                s = c["cap"] * torch.tanh(s / c["cap"])
            if c.get("causal", True):
                p = torch.arange(length - n + i, length - n + i + m, device="cuda")[:, None]
                seen = key <= p
                if c.get("window"):
                    seen &= p - key < c["window"]
                if c.get("prefix"):
                    seen |= key < c["prefix"]
                s.masked_fill_(~seen, -math.inf)
            w = torch.exp(s - s.amax(-1, keepdim=True))
            o = torch.matmul(w.view(n_kv, -1, length), v).view(n_kv, group, m, hd) / w.sum(-1, keepdim=True)
            st["out"][a + i:a + i + m] = o.permute(2, 0, 1, 3).reshape(m, c["n_q"], hd).to(st["out"].dtype)
    return st["out"]


# ------------------------------------------------------------------ the definition in 64 bits


def exact(case, seed):
    st = prepare(case, seed)
    q = st["q"].double()
    out = torch.zeros_like(q)
    if case["kind"] == "append":
        return _exact_append(st, q, out)
    group = case["n_q"] // case["n_kv"]
    for r, (n, length) in enumerate(zip(st["new"], st["length"])):
        j = torch.arange(length, device="cuda")
        page_of, slot = st["pages"][r].long()[j // case["page"]], j % case["page"]
        first = st["starts"][r]
        for h in range(case["n_q"]):
            keys = st["k_pool"][page_of, h // group, slot].double()
            values = st["v_pool"][page_of, h // group, slot].double()
            for lo in range(0, n, 2048):
                hi = min(n, lo + 2048)
                score = q[first + lo:first + hi, h] @ keys.T * case["hd"] ** -0.5
                if case["cap"] > 0:
                    score = torch.tanh(score / case["cap"]) * case["cap"]
                at = torch.arange(lo, hi, device="cuda")[:, None] + (length - n)
                hidden = torch.zeros_like(score, dtype=torch.bool)
                if case.get("causal", True):
                    hidden = j[None, :] > at
                    if case.get("window", 0) > 0:
                        hidden = hidden | (j[None, :] <= at - case["window"])
                    hidden = hidden & (j[None, :] >= case.get("prefix", 0))
                weight = torch.softmax(score.masked_fill(hidden, float("-inf")), dim=1)
                out[first + lo:first + hi, h] = weight @ values
    return out


def _exact_append(st, q, out):
    c = st["case"]
    half = c["rot"] // 2
    k_pool, v_pool = st["k_pool"].double(), st["v_pool"].double()
    pos = st["positions"].cpu().tolist()
    theta = torch.zeros(len(pos), half, dtype=torch.float64)
    inv = [math.exp(-math.log(BASE) * i / half) for i in range(half)]
    i0 = 0
    for a, m in enumerate(st["sections"]):
        theta[:, i0:i0 + m] = torch.tensor([p[a] for p in pos], dtype=torch.float64)[:, None] * torch.tensor(
            inv[i0:i0 + m], dtype=torch.float64)
        i0 += m
    turn = torch.polar(torch.ones_like(theta), theta).cuda()[:, None, :]

    def rotated(x):
        z = torch.complex(x[..., :half], x[..., half:2 * half]) * turn
        return torch.cat([z.real, z.imag, x[..., 2 * half:]], dim=-1)

    rq, rk, v = rotated(q), rotated(st["k"].double()), st["v"].double()
    table = st["pages"].cpu().tolist()
    dst = [(table[r][p // c["page"]], p % c["page"])
           for r, (n, end) in enumerate(zip(st["new"], st["length"])) for p in range(end - n, end)]
    page = torch.tensor([d[0] for d in dst], device="cuda")
    slot = torch.tensor([d[1] for d in dst], device="cuda")
    out[:len(dst)] = rq[:len(dst)]
    k_pool[page, :, slot] = rk[:len(dst)]
    v_pool[page, :, slot] = v[:len(dst)]
    return out, k_pool, v_pool
