"""Plumbing of the mc_layer_q4_* tests: a seeded 4-bit paged cache whose unused pages and rows hold NaN and infinities, and the
operators' definitions in 64 bits on the host, with error bounds derived from the arithmetic the kernels are allowed."""
from __future__ import annotations

import math

import numpy as np
import torch

import layer_harness as LH
from oracle import minicache_oracle as orc

PAGE = 32
H11 = 2.0 ** -11  # half a step of binary16, relative


def quantise(rows, kind):
    """rows [pages][32][128] float64 -> codes uint8 [pages][32][128], scale, zero (K: [pages][128], V: [pages][32][4])."""
    x = np.asarray(rows, np.float64)
    if kind == "k":
        codes, s, z = orc.q4_quantise(x, 1)
        return codes, s[:, 0], z[:, 0]
    codes, s, z = orc.q4_quantise(x, 2)
    return codes, s, z


def tame(x, dtype):
    most = 65504.0 if dtype == torch.float16 else 65280.0
    return torch.where(torch.isnan(x), torch.zeros_like(x), x.double().clamp(-most, most).to(x.dtype))


def pack(codes):
    c = torch.as_tensor(codes)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def unpack(b):
    return torch.stack([b & 15, b >> 4], -1).flatten(-2)


class Cache:
    """lens: cached tokens per sequence; room: tokens the block table reaches beyond them."""

    def __init__(self, lens, H, Hq, dtype, seed=0, room=1, max_len=None, scale=1.0, empty=False, device="cuda"):
        import paper_2405_14366_b200 as mc
        self.mc, self.lens, self.H, self.Hq, self.B, self.nq = mc, list(lens), H, Hq, len(lens), Hq // H
        self.dt = {"f16": torch.float16, "bf16": torch.bfloat16}[dtype]
        self.device, self.scale = device, scale
        g = self.g = torch.Generator().manual_seed(seed + 1)
        pages = [(n + room) // PAGE for n in lens]  # (a page is needed once it is complete)
        self.max_len = max(self.lens) if max_len is None else max_len
        self.mp = max(max(pages), -(-self.max_len // PAGE), 1)
        self.n_pages = sum(pages) + 2
        ids = torch.randperm(self.n_pages, generator=g)
        self.table = torch.full((self.B, self.mp), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(pages):
            self.table[b, :n] = ids[at:at + n]
            at += n
        bad = torch.tensor([float("nan"), float("inf"), -float("inf"), 60000.0])
        junk = lambda *s: bad[torch.randint(0, 4, s, generator=g)]  # noqa: E731
        P = self.n_pages
        self.kc, self.vc = (torch.randint(0, 256, (P, H, PAGE, 64), generator=g, dtype=torch.uint8) for _ in range(2))
        self.km, self.vm = junk(P, H, 128, 2).half(), junk(P, H, PAGE, 4, 2).half()
        self.rk, self.rv = junk(self.B, H, PAGE, 128).to(self.dt), junk(self.B, H, PAGE, 128).to(self.dt)
        self.raw = []  # per sequence the 16-bit rows (k, v) [n][H][128] that went in
        for b, n in enumerate(lens):
            k, v = self.rows(n, H), self.rows(n, H)
            self.raw.append([k, v])
            if empty:
                continue
            self.put(b, k, v)
        dev = lambda t: t.to(device)  # noqa: E731
        self.d = {x: dev(getattr(self, x)) for x in ("kc", "km", "vc", "vm", "rk", "rv", "table")}
        self.d_lens = torch.tensor([0] * self.B if empty else self.lens, dtype=torch.int32, device=device)
        self.cfg = mc.McConfig(H, Hq, PAGE, dtype)
        self.batch = mc.Batch(self.d["table"], self.d_lens, self.max_len, self.n_pages)
        self.layer = mc.LayerQ4Cache(self.cfg, *(self.d[x] for x in ("kc", "km", "vc", "vm", "rk", "rv")),
                                     status=torch.zeros(4, dtype=torch.int32, device=device))

    def rows(self, *s):
        x = torch.randn(*s, 128, generator=self.g) / math.sqrt(128.0) * torch.exp(0.5 * torch.randn(*s, 1, generator=self.g))
        return (x * self.scale).to(self.dt)

    def queries(self, *s, scale=2.5):
        return (torch.randn(*s, 128, generator=self.g) * min(scale * math.sqrt(128.0) / self.scale, 5000.0)).to(self.dt)

    def put(self, b, k, v):
        """Rows [n][H][128] as sequence b's whole cache, on the host."""
        n, full = len(k), len(k) // PAGE
        for x, codes, meta, res, kind in ((k, self.kc, self.km, self.rk, "k"), (v, self.vc, self.vm, self.rv, "v")):
            if full:
                p = self.table[b, :full].long()
                r = tame(x[:full * PAGE], self.dt).double().view(full, PAGE, self.H, 128).transpose(1, 2).reshape(-1, PAGE, 128)
                c, s, z = quantise(r.numpy(), kind)
                codes[p] = pack(c).view(full, self.H, PAGE, 64)
                sz = torch.from_numpy(np.stack([s, z], -1).astype(np.float16)) + 0.0  # (-0 as +0)
                meta[p] = sz.view(full, self.H, 128, 2) if kind == "k" else sz.view(full, self.H, PAGE, 4, 2)
            if n % PAGE:
                res[b, :, :n % PAGE] = x[full * PAGE:].transpose(0, 1)

    def values(self, b, h, n=None):
        """What the cache holds of (sequence, kv head): parts [tokens][128] code * scale, zero (K), the same of V, in 64 bits;
        rows of the begun page have no code part."""
        n = self.lens[b] if n is None else n
        full = n // PAGE
        p = self.table[b, :full].long()
        out = []
        for codes, meta, res, kind in ((self.kc, self.km, self.rk, "k"), (self.vc, self.vm, self.rv, "v")):
            c, m = unpack(codes[p, h]).double(), meta[p, h].double()
            if kind == "k":
                cs, z = c * m[:, None, :, 0], m[:, None, :, 1].expand_as(c)
            else:
                cs = (c.view(full, PAGE, 4, 32) * m[..., 0, None]).flatten(-2)
                z = m[..., 1, None].expand(full, PAGE, 4, 32).flatten(-2)
            r = res[b, h, :n % PAGE].double()
            out += [torch.cat([cs.reshape(-1, 128), torch.zeros_like(r)]), torch.cat([z.reshape(-1, 128), r])]
        return out

    def workspace(self, op, arg=0):
        """Scratch full of NaN patterns: nothing in it may matter."""
        return torch.full((self.mc.lib().mc_layer_workspace_bytes(self.cfg, self.batch, op, arg),), 0xFF, dtype=torch.uint8, device=self.device)

    def status(self):
        return self.mc.lib().mc_layer_q4_read_status(self.layer, check=False)

    def same_as_host(self):
        """The device's cache is the host's, bit for bit (NaN patterns included)."""
        for x in ("kc", "km", "vc", "vm", "rk", "rv"):
            a, b = self.d[x].cpu(), getattr(self, x)
            a, b = (t.view(torch.int16) if t.element_size() == 2 else t for t in (a, b))
            if not torch.equal(a, b):
                i = (a != b).nonzero()
                return x, len(i), [(j.tolist(), a[tuple(j)].item(), b[tuple(j)].item()) for j in i[:5]]
        return None


def page_bounds(c, q, b, h):
    """Score of every complete page of (sequence, kv head) for queries q [nq][128], numpy float64."""
    full = c.lens[b] // PAGE
    m = c.km[c.table[b, :full].long(), h].double().numpy()
    q = q.double().numpy()
    lo, hi = m[..., 1], m[..., 1] + 15.0 * m[..., 0]
    return sum(np.maximum(x * lo, x * hi).sum(1) for x in q) if full else np.zeros(0)


def select64(c, q, b, h, budget, sink, recent, q_pos, window=0, doc=0, prefix=0):
    full = c.lens[b] // PAGE
    t = torch.arange(full * PAGE)
    ok = LH.seen(t, q_pos, window, doc, prefix).view(full, PAGE).any(1).tolist() if full else []
    cand = [p for p in range(full) if ok[p]]
    s = page_bounds(c, q, b, h)
    key = lambda p: (not (p < sink or p >= full - recent), -s[p] if s[p] == s[p] else math.inf, p)  # noqa: E731
    safe = lambda p: p < sink or p >= full - recent  # noqa: E731
    rank = sorted(cand, key=lambda p: (0, 0.0, p) if safe(p) else (1,) + key(p)[1:])
    return sorted(rank[:budget])


def attn64(c, b, h, q, sm, *, k_new=None, v_new=None, cap=0.0, slopes=None, window=0, doc=0, prefix=0, q_pos=None, pages=None):
    """One (sequence, kv head): out [nq][128], lse [nq], and their bounds."""
    n = c.lens[b]
    kc, kz, vc, vz = c.values(b, h)
    q_pos = (n if k_new is not None else n - 1) if q_pos is None else q_pos
    if k_new is not None:
        zero = torch.zeros(1, 128, dtype=torch.float64)
        kc, kz, vc, vz = torch.cat([kc, zero]), torch.cat([kz, k_new[None].double()]), torch.cat([vc, zero]), torch.cat([vz, v_new[None].double()])
    pos = torch.arange(len(kc))
    ok = LH.seen(pos, q_pos, window, doc, prefix)
    full = n // PAGE * PAGE
    if pages is not None:
        pick = torch.zeros(n // PAGE, dtype=torch.bool)
        pick[torch.as_tensor(pages, dtype=torch.long)] = True
        ok = ok & torch.cat([pick.repeat_interleave(PAGE), torch.ones(len(kc) - full, dtype=torch.bool)])
    for x in (kc, kz, vc, vz):  # what is not seen may hold anything
        x[~ok] = 0.0
    q = q.double()
    s = q @ (kc + kz).T * sm
    # fp32 sums of 256 exact products in two chains and their join (a tensor core's sum may cut instead of rounding: one unit of
    # the last place each); what the query's binary16 form loses below 2^-25 of the unit in which its largest number is 2 to 4
    err = 520 * LH.U32 * (q.abs() @ (kc.abs() + kz.abs()).T) * abs(sm)
    unit = torch.exp2(torch.floor(torch.log2(q.abs().amax(1).clamp(min=2.0 ** -120))) - 1)
    err = err + 2.0 ** -25 * unit[:, None] * (128 * 15 + (kc.abs() + kz.abs()).sum(1)[None]) * abs(sm)
    if cap:
        s = cap * torch.tanh(s / cap)
        err = err + 8 * LH.U32 * cap
    slope = torch.as_tensor(slopes[h * c.nq:(h + 1) * c.nq] if slopes is not None else 0.0, dtype=torch.float64).reshape(-1, 1)
    dist = (q_pos - pos).double()
    s = s - slope * dist
    err = err + 4 * LH.U32 * (s.abs() + (slope * dist).abs())
    p, lse, rel = LH.softmax64(s, err, ok[None].expand_as(s))
    out = p @ (vc + vz)
    a, az = p @ vc.abs(), p @ vz.abs()
    half = LH.eps_half(c.dt)
    begun = torch.arange(len(kc)) >= full
    # p rounded to 11 bits, p scale once more; the begun page's p to the storage type; the result once; the probabilities' own error
    tol = 2 * H11 * (1 + H11) * a + H11 * az + max(half, H11) * (p[:, begun] @ vz[begun].abs()) + half * out.abs() + (1 + half) * (a + az) * rel[:, None]
    # what is below 2^-25 of 2^e: e at least 8 less the exponent of the largest scale, at most 15
    top = float(c.vm[c.table[b, :n // PAGE].long(), h].double()[..., 0].max()) if n >= PAGE else 0.0
    low = max(2.0 ** (math.floor(math.log2(top)) + 1 - 8) if top > 0 else 0.0, 2.0 ** -15)
    tol = tol + 2.0 ** -25 * low * (15.0 * full + vc.abs().sum(0) + vz.abs().sum(0))[None]
    if c.dt == torch.float16:
        tol = tol + 2.0 ** -25 * vz[begun].abs().sum(0)[None] + 2.0 ** -25
    fin = torch.where(torch.isinf(lse), torch.zeros_like(lse), lse)
    return out, lse, tol + 1e-30, rel + 4 * LH.U32 * (1 + fin.abs())
