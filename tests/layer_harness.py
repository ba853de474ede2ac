"""Plumbing of the mc_layer_* tests: a seeded paged cache whose unused rows hold NaN and infinities, and the operators'
definitions in 64 bits on the host, with error bounds derived from the arithmetic the kernels are allowed."""
from __future__ import annotations

import math

import torch

U32 = 2.0 ** -24  # half a step of binary32, relative


def eps_half(dtype):
    return torch.finfo(dtype).eps / 2


class Cache:
    """lens: cached tokens per sequence; marks: positions pool with gaps, in another order per head."""

    def __init__(self, lens, H, Hq, ps, dtype, seed=0, marks=False, weights=False, poison=True, room=1, device="cuda", max_len=None):
        import paper_2405_14366_b200 as mc
        self.mc, self.lens, self.H, self.Hq, self.ps, self.B = mc, list(lens), H, Hq, ps, len(lens)
        self.nq = Hq // H
        self.dt = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
        g = self.g = torch.Generator().manual_seed(seed + 1)
        pages = [-(-(n + room) // ps) if n + room else 0 for n in lens]
        self.mp = max(max(pages), 1, -(-(max_len or 0) // ps))  # (the block table has to reach the declared bound)
        spare = 2  # pages of nobody
        self.n_pages = sum(pages) + spare
        ids = torch.randperm(self.n_pages, generator=g)
        self.table = torch.full((self.B, self.mp), -7, dtype=torch.int32)  # slots past a sequence's pages: not an id
        at = 0
        for b, n in enumerate(pages):
            self.table[b, :n] = ids[at:at + n]
            at += n
        shape = (self.n_pages, H, ps)
        bad = torch.tensor([float("nan"), float("inf"), -float("inf"), 60000.0])[torch.randint(0, 4, shape + (128,), generator=g)]
        fill = (lambda: bad.clone()) if poison else (lambda: torch.zeros(shape + (128,)))
        self.k, self.v = fill().to(self.dt), fill().to(self.dt)
        self.pos = torch.full(shape, -12345, dtype=torch.int32) if marks else None
        self.w = torch.rand(shape, generator=g) if weights else None
        self.dense_k, self.dense_v, self.dense_pos = [], [], []
        self.q_next = []  # position of the next token
        for b, n in enumerate(lens):
            k, v = self.rows(n, H), self.rows(n, H)
            self.dense_k.append(k)
            self.dense_v.append(v)
            pos = torch.arange(n)[:, None].expand(n, H)
            if marks:
                pos = torch.stack([torch.randperm(n, generator=g) for _ in range(H)], 1) if n else pos
                pos = pos + pos // 2
            self.dense_pos.append(pos)
            self.q_next.append(n + n // 2 + 1 if marks else n)
            for x, pool in ((k, self.k), (v, self.v), (pos.int(), self.pos)):
                if pool is not None and n:
                    t = torch.arange(n)
                    pool[self.table[b, t // ps].long(), :, t % ps] = x.to(pool.dtype)
        dev = lambda t: None if t is None else t.to(device)  # noqa: E731
        self.d = {k: dev(getattr(self, k)) for k in ("k", "v", "pos", "w", "table")}
        self.d_lens = torch.tensor(self.lens, dtype=torch.int32, device=device)
        self.cfg = mc.McConfig(H, Hq, ps, dtype)
        self.max_len = max(self.lens) if max_len is None else max_len
        self.batch = mc.Batch(self.d["table"], self.d_lens, self.max_len, self.n_pages)
        self.layer = mc.LayerCache(self.cfg, self.d["k"], self.d["v"], self.d["pos"], self.d["w"])
        self.device = device

    def rows(self, *s):
        x = torch.randn(*s, 128, generator=self.g) / math.sqrt(128.0) * torch.exp(0.5 * torch.randn(*s, 1, generator=self.g))
        return x.to(self.dt)

    def queries(self, *s, scale=2.5):
        return (torch.randn(*s, 128, generator=self.g) * scale * math.sqrt(128.0)).to(self.dt)

    def gathered(self, name, b, n=None):
        """[n][H]... of a device pool, through the block table."""
        n = self.lens[b] if n is None else n
        t = torch.arange(n)
        return self.d[name].cpu()[self.table[b, t // self.ps].long(), :, t % self.ps]

    def workspace(self, op, arg=0, fill=0xFF):
        """Scratch full of NaN patterns: nothing in it may matter."""
        n = self.mc.lib().mc_layer_workspace_bytes(self.cfg, self.batch, op, arg)
        return torch.full((n,), fill, dtype=torch.uint8, device=self.device)


def seen(pos, q_pos, window=0, doc=0, prefix=0):
    ok = pos >= doc
    if window:
        ok &= q_pos - pos < window
    return (ok | (pos < prefix)) & (pos <= q_pos)


def scores64(q, k, pos, q_pos, sm, cap=0.0, slope=0.0):
    """Scores [rows][n] of queries [rows][128] (slope: a number or [rows]) and a bound of their error in binary32."""
    q, k = q.double(), k.double()
    s = q @ k.T * sm
    mag = q.abs() @ k.abs().T * abs(sm)  # what the fp32 sum of 128 exact products can be off by: 128 roundings of it
    err = 130 * U32 * mag
    if cap:
        s = cap * torch.tanh(s / cap)
        err = err + 8 * U32 * cap  # tanh to a few ulp; its slope is at most 1
    dist = (q_pos - pos).double()
    slope = torch.as_tensor(slope, dtype=torch.float64).reshape(-1, 1)
    s = s - slope * dist
    err = err + 4 * U32 * (s.abs() + (slope * dist).abs())  # the scale, log2(e), the bias and their sums
    return s, err


def softmax64(s, err, ok):
    """Probabilities (0 where nothing is seen), log-sum-exp, and a bound of a probability's relative error."""
    s = s.masked_fill(~ok, -math.inf)
    lse = torch.logsumexp(s, 1)
    p = torch.exp(s - lse[:, None])
    p[~ok] = 0.0
    worst = err.masked_fill(~ok, 0.0).amax(1) if s.shape[1] else torch.zeros(s.shape[0], dtype=torch.float64)
    # numerator and sum are off by `worst` each; exp2 of a difference adds a few units of its argument's last place
    rel = 2 * worst + 16 * U32 + 4 * U32 * (s.amax(1) if s.shape[1] else lse).abs().nan_to_num(0.0, 0.0, 0.0) + s.shape[1] ** 0.5 * U32
    return p, lse, rel


def attn64(c, b, h, q, sm, *, k_new=None, v_new=None, cap=0.0, slopes=None, window=0, doc=0, prefix=0, q_pos=None):
    """One (sequence, kv head): out [nq][128], lse [nq], p summed over the group [n_tot], and the three bounds."""
    n = c.lens[b]
    k, v, pos = c.dense_k[b][:, h], c.dense_v[b][:, h], c.dense_pos[b][:, h] if n else torch.zeros(0, dtype=torch.long)
    if q_pos is None:
        q_pos = n if k_new is not None else n - 1
    if k_new is not None:
        k, v = torch.cat([k, k_new[None]]), torch.cat([v, v_new[None]])
        pos = torch.cat([pos, torch.tensor([q_pos if c.pos is not None else n])])  # (no positions pool: its index)
    slope = slopes[h * c.nq:(h + 1) * c.nq] if slopes is not None else 0.0
    s, err = scores64(q, k, pos, q_pos, sm, cap, slope)
    ok = seen(pos, q_pos, window, doc, prefix)[None].expand_as(s)
    p, lse, rel = softmax64(s, err, ok)
    vz = torch.where(ok[0][:, None], v.double(), torch.zeros((), dtype=torch.float64))
    out = p @ vz
    a = p @ vz.abs()
    half = eps_half(c.dt)
    # P rounded to the storage type, the result rounded once, the probabilities' own error, 16-bit underflow of P
    tol = half * a * (1 + half) + half * (out.abs() + a * rel[:, None]) + a * rel[:, None]
    if c.dt == torch.float16:
        tol = tol + 2.0 ** -25 * vz.abs().sum(0)[None] + 2.0 ** -25
    tol = tol + 1e-30
    fin = torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)
    lse_tol = rel + 4 * U32 * (1 + fin.abs())
    return out, lse, p.sum(0), tol, lse_tol, (p * rel[:, None]).sum(0)
