"""Plain 64-bit definitions of the paged-cache operators (CPU), the bounds that
their rounding gives, and builders of ragged batches for the tests."""
import math
import random

import numpy as np
import torch

DT = {"bf16": torch.bfloat16, "f32": torch.float32}
HALF = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}     # half a step, relative to the value


class Case:
    """A pool and a ragged batch in host memory. new, length: tokens that each
    request brings and then has. Pages are spread at random over the pool."""

    def __init__(self, new, length, n_q, n_kv, hd, dtype="bf16", page=16, seed=0, shared=0, extra_rows=0, q_scale=2.0,
                 spare=2):
        g = torch.Generator().manual_seed(seed)
        rng = random.Random(seed)
        self.new, self.length, self.n_q, self.n_kv, self.hd, self.dtype = list(new), list(length), n_q, n_kv, hd, dtype
        self.page, self.shared = page, shared
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(int).tolist()
        self.rows = self.starts[-1] + extra_rows
        need = [-(-n // page) for n in length]
        common = shared // page
        total = common + sum(max(0, n - common) for n in need) + spare
        ids = list(range(total))
        rng.shuffle(ids)
        head, rest = ids[:common], ids[common:]
        stride = max(need + [1, common]) + 1
        self.table = []
        for n in need:
            row = head + rest[:max(0, n - common)]
            rest = rest[max(0, n - common):]
            self.table.append(row + [-1] * (stride - len(row)))
        dt = DT[dtype]
        shape = (total, n_kv, page, hd)
        self.k = torch.randn(shape, generator=g).to(dt)
        self.v = torch.randn(shape, generator=g).to(dt)
        self.q = (q_scale * torch.randn(self.rows, n_q, hd, generator=g)).to(dt)

    def gathered(self, r, pool):
        """Request r's keys or values [n_kv][length][hd] in 64 bits, and which of them have a page."""
        n = self.length[r]
        j = torch.arange(n)
        ids = torch.tensor(self.table[r], dtype=torch.long)[j // self.page] if n else torch.zeros(0, dtype=torch.long)
        there = (ids >= 0) & (ids < pool.shape[0])
        x = pool[ids.clamp(0, pool.shape[0] - 1), :, j % self.page].double()     # [n][n_kv][hd]
        return x.transpose(0, 1), there

    def device(self, dev="cuda"):
        """The tensors of this case on the GPU: (KVPool, Batch, q)."""
        from paper_2609_12075_amd import paged
        pool = paged.KVPool(self.k.to(dev), self.v.to(dev))
        return pool, self.batch(dev), self.q.to(dev)

    def batch(self, dev="cuda", max_new=None, max_len=None):
        from paper_2609_12075_amd import paged
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device=dev)   # noqa: E731
        return paged.Batch(i32(self.starts), i32(self.length), i32(self.table), n_tok=self.rows,
                           max_new=max(self.new) if max_new is None else max_new,
                           max_len=max(self.length) if max_len is None else max_len)


def attention_ref(c, cap=0.0, causal=True, window=0, prefix=None, scale=None):
    """The definition in 64 bits. Returns (o, lse, bound): bound is what the
    operator's rounding may move an output by, derived per output below."""
    o = torch.zeros(c.rows, c.n_q, c.hd, dtype=torch.float64)
    lse = torch.full((c.rows, c.n_q), -math.inf, dtype=torch.float64)
    bound = torch.zeros_like(o)
    lbound = torch.zeros_like(lse)
    scale = c.hd ** -0.5 if scale is None else scale
    grp = c.n_q // c.n_kv
    for r, (n, length) in enumerate(zip(c.new, c.length)):
        if n == 0:
            continue
        k, there = c.gathered(r, c.k)
        v, _ = c.gathered(r, c.v)
        rows = slice(c.starts[r], c.starts[r] + n)
        p = torch.arange(n)[:, None] + length - n
        j = torch.arange(length)[None, :]
        see = torch.ones(n, length, dtype=torch.bool)
        if causal:
            see = j <= p
            if window:
                see &= p - j < window
            if prefix is not None:
                see |= j < prefix[r]
        see = see & there[None, :]
        for h in range(c.n_q):
            q = c.q[rows, h].double()
            kk, vv = k[h // grp], v[h // grp]
            # what is not seen takes no part, whatever its bits
            kk = torch.where(see.any(0)[:, None], kk, torch.zeros_like(kk))
            s = torch.where(see, (q @ kk.T) * scale, torch.full((), -math.inf, dtype=torch.float64))
            mag = torch.where(see, (q.abs() @ kk.abs().T) * scale, torch.zeros(())).amax(1, keepdim=True) if length else \
                torch.zeros(n, 1, dtype=torch.float64)
            if cap:
                s = torch.where(see, cap * torch.tanh(s / cap), s)
            m = s.amax(1, keepdim=True) if length else torch.full((n, 1), -math.inf, dtype=torch.float64)
            m0 = torch.where(m == -math.inf, torch.zeros_like(m), m)
            w = torch.where(see, torch.exp(s - m0), torch.zeros((), dtype=torch.float64))
            l = w.sum(1, keepdim=True)
            inv = torch.where(l > 0, 1 / l, torch.zeros_like(l))
            if torch.isfinite(vv).all():
                num, mass = w @ vv, (w @ vv.abs()) * inv
            else:                                      # 0 times an unseen infinity is nothing
                num = torch.stack([(w[i][see[i]][:, None] * vv[see[i]]).sum(0) for i in range(n)])
                mass = torch.stack([(w[i][see[i]][:, None] * vv[see[i]].abs()).sum(0) for i in range(n)]) * inv
            o[rows, h] = num * inv
            lse[rows, h] = (m0 + torch.log(l))[:, 0]
            # A score sums hd products in fp32 (hd 2^-24 of the sum of magnitudes), is scaled, capped (a few 2^-24
            # of the cap) and taken relative to the maximum (a few 2^-24 of its size); that error is the relative
            # error of its weight, in the numerator and in the sum. Sums over the keys: 2^-24 each.
            top = torch.where(see, s.abs(), torch.zeros((), dtype=torch.float64)).amax(1, keepdim=True) if length else mag
            es = c.hd * 2.0 ** -24 * mag + 8 * 2.0 ** -24 * (top + (cap if cap else 0.0)) + 2.0 ** -21
            rel = 2 * es + 2 * (length + 64) * 2.0 ** -24
            weights = 2.0 ** -8 if c.dtype == "bf16" else 0.0       # weights rounded to bf16 in the numerator
            bound[rows, h] = (rel + weights) * mass + HALF[c.dtype] * (o[rows, h].abs() + (rel + weights) * mass) + 1e-30
            lbound[rows, h] = (rel + 2.0 ** -22 * (lse[rows, h].abs()[:, None].nan_to_num(0, 0, 0) + 1))[:, 0]
    return o, lse, bound, lbound


def check_attention(c, got, ref, lse=None, rows=None):
    o, rl, bound, lbound = ref
    n = c.starts[-1]
    got = got.detach().cpu().double()[:n]
    o, bound = o[:n], bound[:n]
    nan = torch.isnan(o)
    assert torch.equal(torch.isnan(got), nan), "NaN in other places"
    inf = torch.isinf(o)
    assert torch.equal(torch.where(inf, got, torch.zeros(())), torch.where(inf, o, torch.zeros(()))), "infinities differ"
    ok = ~(nan | inf)
    err = torch.where(ok, (got - o).abs(), torch.zeros(()))
    lim = torch.where(ok, bound, torch.ones(()))
    worst = float((err / lim).max()) if err.numel() else 0.0
    assert worst <= 1.0, f"off by {worst:.3f} of the bound"
    if lse is not None:
        g, w = lse.detach().cpu().double()[:n], rl[:n]
        assert torch.equal(torch.isinf(g), torch.isinf(w))
        fin = torch.isfinite(w)
        assert ((g - w).abs()[fin] <= lbound[:n][fin]).all(), float(((g - w).abs()[fin] / lbound[:n][fin]).max())
    return worst


def append_ref(c, k, v, q, positions, sections, base):
    """The definition in 64 bits. Returns (q_out, k pool, v pool) and the bound on q_out and the k pool's new rows."""
    half = sum(sections)
    kp, vp, qo = c.k.double().clone(), c.v.double().clone(), q.double().clone()
    touched = torch.zeros(kp.shape[:3], dtype=torch.bool)

    def turn(x, pos):
        y = x.double().clone()
        f = 0
        for a, m in enumerate(sections):
            for i in range(f, f + m):
                t = pos[a] * base ** (-i / half)
                cs, sn = math.cos(t), math.sin(t)
                xa, xb = x[..., i].double(), x[..., i + half].double()
                y[..., i], y[..., i + half] = xa * cs - xb * sn, xb * cs + xa * sn
            f += m
        return y

    for r, (n, length) in enumerate(zip(c.new, c.length)):
        for i in range(n):
            t, p = c.starts[r] + i, length - n + i
            pos = positions[t] if positions is not None else [p]
            qo[t] = turn(q[t], pos)
            pg = c.table[r][p // c.page] if p >= 0 else -1
            if 0 <= pg < kp.shape[0]:
                kp[pg, :, p % c.page] = turn(k[t], pos)
                vp[pg, :, p % c.page] = v[t].double()
                touched[pg, :, p % c.page] = True
    return qo, kp, vp, touched


def rotation_bound(x, dtype):
    """sine and cosine off by a few 2^-24 (angle reduced in fp64, rounded to fp32, function within 2 ulp), two
    products and a sum in fp32: 8 * 2^-24 of |x_a| + |x_b|, at most 8 * 2^-24 * 2 max|row|, then half a step."""
    top = x.abs().amax(-1, keepdim=True)
    return 16 * 2.0 ** -24 * top + HALF[dtype] * (x.abs() + 16 * 2.0 ** -24 * top)
