"""The operators of a layer whose cache is held in 4 bits: writing rows into it and reading them back, single-token
attention over it, and attention over the pages that a cheap score selects.  Cases, inputs, plain forms (32 bits,
elementary torch operations; 64 bits where a value next to a border decides a whole number) and the definitions in 64
bits.

MiniCache merges the layers S .. L-1 of a model; with 4-bit layers (keys per channel over a page of 32 tokens, values per
token over 32 channels) the layers below S stay 4-bit caches, which these operators write, read and attend.  Shapes are
those of the benchmark's workloads (32 heads x 128 in binary16, 8 kv heads under 32 query heads in bfloat16, ragged
serving batches, long sequences)."""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}
PAGE = 32


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def _append(name, **kw):
    c = dict(name=name, op="append", dtype="f16", hq=32, hkv=32, batch=1, n=0, new=512, ragged=False, packed=False)
    c.update(kw)
    return c


def _attn(name, **kw):
    c = dict(name=name, op="attn", dtype="f16", hq=32, hkv=32, batch=1, n=512, ragged=False, append=True, cap=0.0, alibi=False,
             window=0, prefix=0, docs=False)
    c.update(kw)
    return c


def _sparse(name, **kw):
    c = dict(name=name, op="sparse", dtype="f16", hq=32, hkv=32, batch=1, n=8192, ragged=False, append=True, cap=0.0, window=0,
             prefix=0, docs=False, budget=64, sink=1, recent=2)
    c.update(kw)
    return c


def listed():
    return [
        # one user's prompt goes into the cache and is read back for the prompt's own attention: nothing but latency
        _append("append_prompt", batch=1, new=500),
        # the next chunk of a batch of prompts, out of a packed projection, behind odd lengths: pages begun are completed
        _append("append_chunks", dtype="bf16", hkv=8, batch=16, n=3000, new=2048, ragged=True, packed=True),
        # the benchmark's batch of prompts
        _append("append_7b_batch", batch=8, new=4096),
        # one user's first generated tokens: a page and a begun one
        _attn("attn_first_tokens", batch=1, n=45),
        # the benchmark's batch, a layer below the merged half: plain causal attention, the step's rows appended
        _attn("attn_7b_batch", batch=8, n=4109),
        # grouped heads, scores capped by a tanh, a long batch
        _attn("attn_gqa_capped", dtype="bf16", hkv=8, batch=16, n=8192, cap=50.0),
        # a serving batch of all lengths, packed documents, a sliding window behind four sink tokens
        _attn("attn_ragged_window", batch=64, n=2048, ragged=True, window=512, prefix=4, docs=True),
        # a long context with a distance bias, nothing appended
        _attn("attn_alibi_long", dtype="bf16", hkv=8, batch=4, n=32749, alibi=True, append=False),
        # one user's decode step over the best 32 of 256 pages
        _sparse("sparse_one_user", batch=1, n=8200, budget=32),
        # a batch with grouped heads, a quarter of the pages
        _sparse("sparse_gqa", dtype="bf16", hkv=8, batch=16, n=8192, budget=64),
        # very long contexts: 64 of 4096 pages
        _sparse("sparse_long", dtype="bf16", hkv=8, batch=4, n=131060, budget=64, sink=2, recent=8),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["append", "attn", "attn", "sparse"])
    dtype = rng.choice(["f16", "bf16"])
    hkv, hq = rng.choice([(32, 32), (8, 32), (4, 32), (8, 16), (1, 8), (5, 10), (2, 2)])
    batch = _log_int(rng, 1, 64)
    # no more (token, kv head) rows than the largest listed case of the operator has
    most = min(131072 if op == "sparse" else 32768, max(64, (1 << (22 if op == "sparse" else 20)) // (batch * hkv)))
    base = dict(dtype=dtype, hq=hq, hkv=hkv, batch=batch, ragged=rng.random() < 0.5)
    if op == "append":
        c = _append("", **base, n=rng.choice([0, _log_int(rng, 1, 4096)]), new=_log_int(rng, 1, most), packed=rng.random() < 0.5)
    else:
        score = dict(n=_log_int(rng, 1, most), append=rng.random() < 0.7, cap=rng.choice([0.0, 0.0, 30.0, 50.0]),
                     window=rng.choice([0, 0, 1, _log_int(rng, 2, 4096)]), prefix=rng.choice([0, 0, 4, 17]), docs=rng.random() < 0.25)
        if op == "attn":
            c = _attn("", **base, **score, alibi=rng.random() < 0.3)
        else:
            c = _sparse("", **base, **score, budget=_log_int(rng, 1, 256))
            c["sink"] = min(rng.choice([0, 1, 2]), c["budget"])
            c["recent"] = rng.randint(0, min(16, c["budget"] - c["sink"]))
    del c["name"]
    return c


def _spread(c, most, least, at):
    """A length per sequence: a property of the case (its work follows from it), not of the seed."""
    if not c["ragged"]:
        return [most] * c["batch"]
    lo, out = max(1, most // 16), []
    for i in range(c["batch"]):
        f = (at + 0.618034 * i) % 1.0
        out.append(max(least, min(most, int(round(lo * (most / lo) ** f)))))
    out[0] = most
    return out


def _lens(c):
    """Cached tokens per sequence when the call is made."""
    out = _spread(c, c["n"], 1, 0.381) if c["n"] else [0] * c["batch"]
    if c["ragged"] and c["batch"] > 3 and c["op"] != "append":
        out[2] = 0  # a slot without a sequence
    if c["op"] != "append":
        out = [n - 1 if n % PAGE == PAGE - 1 else n for n in out]  # (a page that fills is the append cases' business)
    return out


def _news(c):
    out = _spread(c, c["new"], 1, 0.77)
    if c["ragged"] and c["batch"] > 3:
        out[2] = 0  # a sequence that gets nothing
    return out


def _doc_starts(c, lens):
    return [n // 3 if c["docs"] and i % 2 else 0 for i, n in enumerate(lens)]


def _ranges(c, n, doc):
    """The cached tokens [0, a) and [lo, hi) that the query behind (or at the end of) n of them sees."""
    q_pos = n if c["append"] else n - 1
    a = min(n, c["prefix"], q_pos + 1)
    lo = max(doc, q_pos - c["window"] + 1 if c["window"] else 0, a)
    return a, lo, max(lo, min(n, q_pos + 1))


def _candidates(c, n, doc):
    """Complete pages with a token that the query sees."""
    a, lo, hi = _ranges(c, n, doc)
    full = n // PAGE
    return sum(1 for p in range(full) if p * PAGE < a or (p * PAGE < hi and (p + 1) * PAGE > lo and hi > lo))


def work(c):
    H, nq = c["hkv"], c["hq"] // c["hkv"]
    row = 160  # codes and group parameters of a token's key and value
    if c["op"] == "append":
        rows = 0
        b = 0
        for n, m in zip(_lens(c), _news(c)):
            done = (n + m) // PAGE * PAGE - n // PAGE * PAGE  # tokens of pages that are completed
            left = (n + m) % PAGE if done else m  # rows that stay in 16 bits
            rows += m
            b += (n % PAGE if done else 0) * 512 + done * row + left * 512  # written (and the begun page read)
            b += max(0, (n + m) // PAGE * PAGE - n) * row + min(m, (n + m) % PAGE) * 512  # read back
        return {"bytes": H * (b + rows * 2 * 512), "flops": 0}
    tokens = b = 0
    for n, d in zip(_lens(c), _doc_starts(c, _lens(c))):
        a, lo, hi = _ranges(c, n, d)
        full = n // PAGE * PAGE
        tail = max(0, a - full) + max(0, hi - max(lo, full))  # visible rows of the begun page
        if c["op"] == "sparse":
            cand = _candidates(c, n, d)
            inside = min(c["budget"], cand) * PAGE
            b += H * cand * 512
        else:
            inside = a + hi - lo - tail
        tokens += inside + tail
        b += H * (inside * row + tail * 512)
    new = c["batch"] * H
    b += c["batch"] * c["hq"] * (512 + 4) + (new * 1024 if c["append"] else 0)
    return {"bytes": b, "flops": 4 * 128 * nq * (H * tokens + (new if c["append"] else 0))}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _pack(codes):
    """Codes [...][128] to bytes [...][64]: channel 2i in the low half of byte i, channel 2i + 1 in the high one."""
    c = codes.to(torch.uint8)
    return c[..., 0::2] | (c[..., 1::2] << 4)


def _fill(s, g, n_pages, H, dt):
    """Pools full of quantised rows (unit directions of log-normal length), a few pages at a time."""
    s["k_codes"] = torch.empty(n_pages, H, PAGE, 64, dtype=torch.uint8, device="cuda")
    s["v_codes"] = torch.empty_like(s["k_codes"])
    s["k_meta"] = torch.empty(n_pages, H, 128, 2, dtype=torch.float16, device="cuda")
    s["v_meta"] = torch.empty(n_pages, H, PAGE, 4, 2, dtype=torch.float16, device="cuda")
    step = max(1, (1 << 25) // (H * PAGE * 128))
    for i in range(0, n_pages, step):
        p = min(step, n_pages - i)
        for name in ("k", "v"):
            x = _rows(g, p, H, PAGE, dtype=dt).float()
            x = x if name == "k" else x.view(p, H, PAGE, 4, 32)
            axis = 2 if name == "k" else 4
            lo, hi = x.amin(axis, keepdim=True), x.amax(axis, keepdim=True)
            zero, scale = lo.half(), ((hi - lo) / 15.0).half()
            scale = torch.where(scale == 0, torch.ones_like(scale), scale)
            code = torch.round((x - zero.float()) / scale.float()).clamp(0, 15).view(p, H, PAGE, 128)
            s[name + "_codes"][i:i + p] = _pack(code)
            s[name + "_meta"][i:i + p] = torch.stack([scale, zero], -1).squeeze(axis)


def _rows(g, *shape, dtype):
    x = torch.randn(*shape, 128, generator=g, device="cuda") * (1 / math.sqrt(128.0))
    return (x * torch.exp(0.5 * torch.randn(*shape, 1, generator=g, device="cuda"))).to(dtype)


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * seed + 29)
    dt, H, B = DTYPES[c["dtype"]], c["hkv"], c["batch"]
    lens = _lens(c)
    news = _news(c) if c["op"] == "append" else [1 if c["append"] else 0] * B
    pages = [max(1, -(-(n + m) // PAGE)) for n, m in zip(lens, news)]
    n_pages, mp = sum(pages), max(pages)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(B, mp, dtype=torch.int32, device="cuda")
    table[torch.arange(mp, device="cuda")[None, :] < torch.tensor(pages, device="cuda")[:, None]] = order
    s = dict(c=dict(c), lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), table=table, n_pages=n_pages,
             max_len=max(lens) + (max(news) if c["op"] == "append" else 0), status=torch.zeros(4, dtype=torch.int32, device="cuda"))
    _fill(s, g, n_pages, H, dt)
    # the begun pages; slots behind a sequence's rows hold what an earlier page left there
    s["res_k"], s["res_v"] = _rows(g, B, H, PAGE, dtype=dt), _rows(g, B, H, PAGE, dtype=dt)
    if c["op"] == "append":
        rows = sum(news)
        s["total"] = s["lens"] + torch.tensor(news, dtype=torch.int32, device="cuda")
        s["offsets"] = torch.tensor([0] + torch.tensor(news).cumsum(0).tolist(), dtype=torch.int32, device="cuda")
        if c["packed"]:
            qkv = torch.empty(rows, c["hq"] + 2 * H, 128, dtype=dt, device="cuda")
            s["k"], s["v"] = qkv[:, c["hq"]:c["hq"] + H], qkv[:, c["hq"] + H:]
        else:
            s["k"], s["v"] = (torch.empty(rows, H, 128, dtype=dt, device="cuda") for _ in range(2))
        for i in range(0, rows, 1 << 15):
            for x in (s["k"], s["v"]):
                x[i:i + (1 << 15)] = _rows(g, min(1 << 15, rows - i), H, dtype=dt)
        s["res0"] = (s["res_k"].clone(), s["res_v"].clone())  # put back ahead of every pass, which meets the same cache
        s["back_k"], s["back_v"] = (torch.zeros(rows, H, 128, dtype=dt, device="cuda") for _ in range(2))
        return s
    s["q"] = (torch.randn(B, c["hq"], 128, generator=g, device="cuda") * (2.5 * math.sqrt(128.0))).to(dt)
    s["k_new"], s["v_new"] = (_rows(g, B, H, dtype=dt), _rows(g, B, H, dtype=dt)) if c["append"] else (None, None)
    s["out"] = torch.zeros_like(s["q"])
    s["lse"] = torch.zeros(B, c["hq"], device="cuda")
    s["prefix"] = torch.full((B,), c["prefix"], dtype=torch.int32, device="cuda") if c["prefix"] else None
    s["docs"] = torch.tensor(_doc_starts(c, lens), dtype=torch.int32, device="cuda") if c["docs"] else None
    s["slopes"] = torch.exp2(-8.0 * torch.arange(1, c["hq"] + 1, device="cuda") / c["hq"]).float() if c.get("alibi") else None
    # (the selection takes the step's position, which without a new row is the last cached token's)
    s["q_pos"] = s["lens"] - (0 if c["append"] else 1)
    if c["op"] == "sparse":
        s["pages"] = torch.full((B, H, c["budget"]), -1, dtype=torch.int32, device="cuda")
        s["counts"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------
def _half(x):
    """float64 rounded once to binary16 (a conversion by way of binary32 rounds twice), as float64."""
    ulp = torch.exp2((torch.frexp(x)[1] - 11).clamp(min=-24).double())
    return torch.round(x / ulp) * ulp


def _quantise(x, axis):
    """float64 codes, scale and zero of groups along axis: what decides a code is formed in 64 bits."""
    lo, hi = x.amin(axis, keepdim=True), x.amax(axis, keepdim=True)
    scale, zero = _half((hi - lo) / 15.0), _half(lo)
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    return torch.round((x - zero) / scale).clamp(0, 15), scale, zero


def _values(s, pages):
    """Keys and values [pages][H][32][128] in binary32 that the codes of these pages stand for."""
    out = []
    for name in ("k", "v"):
        b = s[name + "_codes"][pages]
        code = torch.stack([b & 15, b >> 4], -1).flatten(-2).float()
        m = s[name + "_meta"][pages].float()
        if name == "k":
            out.append(code * m[:, :, None, :, 0] + m[:, :, None, :, 1])
        else:
            out.append((code.view(*code.shape[:3], 4, 32) * m[..., 0, None] + m[..., 1, None]).flatten(-2))
    return out


def _plain_append(s):
    c = s["c"]
    H = c["hkv"]
    s["res_k"].copy_(s["res0"][0])
    s["res_v"].copy_(s["res0"][1])
    at = 0
    for b, (n, m) in enumerate(zip(_lens(c), _news(c))):
        k, v = s["k"][at:at + m], s["v"][at:at + m]
        begun, first = n % PAGE, n // PAGE
        k, v = torch.cat([s["res_k"][b, :, :begun].transpose(0, 1), k]), torch.cat([s["res_v"][b, :, :begun].transpose(0, 1), v])
        full = len(k) // PAGE
        pages = s["table"][b, first:first + full].long()
        step = max(1, (1 << 24) // (H * PAGE * 128))
        for i in range(0, full, step):
            p = pages[i:i + step]
            xk, xv = (x[i * PAGE:(i + len(p)) * PAGE].reshape(len(p), PAGE, H, 128).transpose(1, 2).double() for x in (k, v))
            code, scale, zero = _quantise(xk, 2)
            s["k_codes"][p], s["k_meta"][p] = _pack(code), torch.stack([scale, zero], -1)[:, :, 0].half()
            code, scale, zero = _quantise(xv.reshape(len(p), H, PAGE, 4, 32), 4)
            s["v_codes"][p], s["v_meta"][p] = _pack(code.flatten(-2)), torch.stack([scale, zero], -1)[..., 0, :].half()
        lo = begun if full == 0 else 0  # (rows of the begun page stay where they are)
        tail = len(k) - full * PAGE
        s["res_k"][b, :, lo:tail] = k[full * PAGE + lo:].transpose(0, 1)
        s["res_v"][b, :, lo:tail] = v[full * PAGE + lo:].transpose(0, 1)
        # and read back: the rows as the cache holds them
        for i in range(0, full, step):
            xk, xv = (x.transpose(1, 2).reshape(-1, H, 128) for x in _values(s, pages[i:i + step]))
            cut = max(0, begun - i * PAGE)
            to = at + max(0, i * PAGE - begun)
            s["back_k"][to:to + len(xk) - cut], s["back_v"][to:to + len(xk) - cut] = xk[cut:].to(k.dtype), xv[cut:].to(k.dtype)
        s["back_k"][at + m - (tail - lo):at + m] = s["res_k"][b, :, lo:tail].transpose(0, 1)
        s["back_v"][at + m - (tail - lo):at + m] = s["res_v"][b, :, lo:tail].transpose(0, 1)
        at += m


def _seen(c, s, pos, q_pos):
    """Which positions [B][...] the queries see."""
    shape = (-1,) + (1,) * (pos.dim() - 1)
    near = pos >= (s["docs"].view(shape) if s["docs"] is not None else 0)
    if c["window"]:
        near = near & (q_pos.view(shape) - pos < c["window"])
    if s["prefix"] is not None:
        near = near | (pos < s["prefix"].view(shape))
    return near & (pos <= q_pos.view(shape))


def _plain_select(s):
    c = s["c"]
    B, H, nq, budget = c["batch"], c["hkv"], c["hq"] // c["hkv"], c["budget"]
    q = s["q"].double().view(B, H, nq, 128)
    total, above = q.sum(2), q.clamp(min=0).sum(2)
    P = s["table"].shape[1]
    score = torch.empty(B, H, P, dtype=torch.float64, device="cuda")
    for b in range(B):  # (64 bits: which page is the last one in must not hang on the order of a sum)
        m = s["k_meta"][s["table"][b].long()].double()  # [P][H][128][2]
        score[b] = torch.einsum("phc,hc->hp", m[..., 1], total[b]) + 15.0 * torch.einsum("phc,hc->hp", m[..., 0], above[b])
    n, q_pos = s["lens"].long(), s["q_pos"].long()
    tok = torch.arange(P * PAGE, device="cuda")[None].expand(B, -1)
    page = torch.arange(P, device="cuda")[None]
    full = (n // PAGE)[:, None]
    cand = (_seen(c, s, tok, q_pos) & (tok < n[:, None])).view(B, P, PAGE).any(2) & (page < full)
    guarded = (page < c["sink"]) | (page >= full - c["recent"])
    key = torch.where(guarded[:, None], torch.full_like(score, math.inf), score).masked_fill(~cand[:, None], -math.inf)
    order = torch.sort(key, dim=2, descending=True, stable=True)[1][:, :, :budget]
    kept = torch.zeros_like(key, dtype=torch.bool).scatter_(2, order, True) & cand[:, None]
    s["counts"].copy_(cand.sum(1).clamp(max=budget))
    b, h, p = kept.nonzero(as_tuple=True)  # (in ascending order of the page)
    s["pages"][b, h, (kept.cumsum(2) - 1)[b, h, p]] = p.to(torch.int32)
    return kept


def _plain_attn(s, kept=None):
    c = s["c"]
    B, H, nq = c["batch"], c["hkv"], c["hq"] // c["hkv"]
    n = s["lens"].long()
    q_pos = s["q_pos"].long()
    P = s["table"].shape[1]
    at = torch.arange(P * PAGE + PAGE, device="cuda")[None].expand(B, -1)  # every page's slots, then the begun page's
    full = (n // PAGE * PAGE)[:, None]
    pos = torch.where(at < P * PAGE, at, full + at - P * PAGE)
    if c["append"]:
        s["res_k"][torch.arange(B, device="cuda"), :, n % PAGE] = s["k_new"]
        s["res_v"][torch.arange(B, device="cuda"), :, n % PAGE] = s["v_new"]
    total = (n + 1 if c["append"] else n)[:, None]
    held = torch.where(at < P * PAGE, at < full, pos < total)
    ok = (_seen(c, s, pos, q_pos) & held)[:, None]
    if kept is not None:
        pick = torch.ones(B, H, P * PAGE + PAGE, dtype=torch.bool, device="cuda")
        pick[:, :, :P * PAGE] = kept.repeat_interleave(PAGE, 2)
        ok = ok & pick
    for b in range(B):
        k, v = (x.transpose(0, 1).reshape(H, P * PAGE, 128) for x in _values(s, s["table"][b].long()))
        k, v = torch.cat([k, s["res_k"][b].float()], 1), torch.cat([v, s["res_v"][b].float()], 1)
        x = (s["q"][b].float().view(H, nq, 128) @ k.transpose(1, 2)) * (1.0 / math.sqrt(128.0))
        if c["cap"]:
            x = c["cap"] * torch.tanh(x / c["cap"])
        if s["slopes"] is not None:
            x = x - s["slopes"].view(H, nq, 1) * (q_pos[b] - pos[b]).float()
        mask = ok[b][:, None]
        x = x.masked_fill(~mask, -math.inf)
        m = x.amax(2, keepdim=True)
        e = torch.exp(x - torch.where(m == -math.inf, torch.zeros_like(m), m))
        l = e.sum(2, keepdim=True)
        v = torch.where(ok[b][..., None].expand(H, -1, 1), v, torch.zeros_like(v))
        s["out"][b] = ((e / torch.where(l > 0, l, torch.ones_like(l))) @ v).reshape(c["hq"], 128).to(s["out"].dtype)
        s["lse"][b] = (m + torch.log(l)).reshape(c["hq"])


# ---------------------------------------------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------------------------------------------
def _handle(s):
    """What a user's program sets up once per cache: the configuration, the batch and cache descriptions, scratch memory."""
    import paper_2405_14366_b200 as mc
    c = s["c"]
    lib = mc.lib()
    cfg = mc.McConfig(c["hkv"], c["hq"], PAGE, c["dtype"])
    batch = mc.Batch(s["table"], s["lens"], s["max_len"], s["n_pages"])
    layer = mc.LayerQ4Cache(cfg, s["k_codes"], s["k_meta"], s["v_codes"], s["v_meta"], s["res_k"], s["res_v"], s["status"])
    if c["op"] == "append":
        return lib, cfg, batch, mc.Batch(s["table"], s["total"], s["max_len"], s["n_pages"]), layer
    opts = mc.ScoreOpts(1.0 / math.sqrt(128.0), softcap=c["cap"], alibi_slopes=s["slopes"], window=c["window"], doc_start=s["docs"],
                        prefix_len=s["prefix"], q_pos=s["q_pos"])
    flags = mc.MC_LAYER_APPEND if c["append"] else 0
    need = lib.mc_layer_workspace_bytes(cfg, batch, mc.MC_OP_LAYER_Q4_ATTN, flags)
    keep = None
    if c["op"] == "sparse":
        keep = mc.PageSelection(c["budget"], n_sink=c["sink"], n_recent=c["recent"])
        need = max(need, lib.mc_layer_workspace_bytes(cfg, batch, mc.MC_OP_LAYER_Q4_SELECT, 0))
    return lib, cfg, batch, layer, opts, flags, keep, torch.empty(need, dtype=torch.uint8, device="cuda")


def _call(s):
    if "handle" not in s:
        s["handle"] = _handle(s)
    c = s["c"]
    if c["op"] == "append":
        lib, cfg, batch, after, layer = s["handle"]
        s["res_k"].copy_(s["res0"][0])
        s["res_v"].copy_(s["res0"][1])
        lib.mc_layer_q4_append(cfg, batch, layer, s["k"], s["v"], s["offsets"])
        lib.mc_layer_q4_read(cfg, after, layer, s["lens"], s["back_k"], s["back_v"], s["offsets"])
        return
    lib, cfg, batch, layer, opts, flags, keep, ws = s["handle"]
    pages = counts = None
    if keep is not None:
        pages, counts = s["pages"], s["counts"]
        lib.mc_layer_q4_select(cfg, batch, layer, opts, keep, s["q"], pages, counts, ws)
    lib.mc_layer_q4_attn(cfg, batch, layer, opts, pages, counts, s["q"], s["k_new"], s["v_new"], flags, s["out"], s["lse"], ws)


def run(state):
    s = state
    if own:
        _call(s)
    elif s["c"]["op"] == "append":
        _plain_append(s)
    else:
        _plain_attn(s, _plain_select(s) if s["c"]["op"] == "sparse" else None)
    if s["c"]["op"] == "append":
        return {"k": s["back_k"], "v": s["back_v"], "res_k": s["res_k"], "res_v": s["res_v"]}
    r = {"out": s["out"], "lse": s["lse"]}
    if s["c"]["append"]:
        r.update(res_k=s["res_k"], res_v=s["res_v"])
    if s["c"]["op"] == "sparse":
        r.update(pages=s["pages"], counts=s["counts"])
    return r


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits, one sequence and one head after the other
# ---------------------------------------------------------------------------------------------------------------
def _group64(x):
    """Values [...][32] of one group each -> the values that their codes stand for."""
    import numpy as np
    least, most = x.min(-1)[0], x.max(-1)[0]
    to16 = lambda t: torch.from_numpy(t.cpu().numpy().astype(np.float16).astype(np.float64)).to(t.device)  # noqa: E731 (one rounding)
    step, base = to16((most - least) / 15), to16(least)
    step[step == 0] = 1.0
    code = torch.clip(((x - base[..., None]) / step[..., None]).round(), 0.0, 15.0)
    return base[..., None] + step[..., None] * code


def _unpacked64(codes):
    c = codes.long()
    out = torch.empty(*c.shape[:-1], 128, dtype=torch.float64, device=c.device)
    out[..., 0::2], out[..., 1::2] = (c % 16).double(), (c // 16).double()
    return out


def exact(c, seed):
    c = dict(c)
    lens, H, nq = _lens(c), c["hkv"], c["hq"] // c["hkv"]
    if sum(1 for n in lens if n) * H > 20_000:
        return None
    s = prepare(c, seed)
    if c["op"] == "append":
        off = s["offsets"].tolist()
        back = {x: torch.zeros(s["k"].shape, dtype=torch.float64, device="cuda") for x in "kv"}
        for b, n in enumerate(lens):
            old, m = n % PAGE, off[b + 1] - off[b]
            done = (old + m) // PAGE * PAGE
            for x in "kv":
                for h in range(H):
                    r = torch.cat([s["res_" + x][b, h, :old], s[x][off[b]:off[b + 1], h]])
                    d = r.double()
                    if done:
                        pages = d[:done].view(-1, PAGE, 128)
                        d[:done] = (_group64(pages.transpose(1, 2)).transpose(1, 2) if x == "k" else
                                    _group64(pages.reshape(-1, PAGE, 4, 32))).reshape(done, 128)
                    back[x][off[b]:off[b + 1], h] = d[old:]
                    s["res_" + x][b, h, :len(r) - done] = r[done:]
        return {"k": back["k"], "v": back["v"], "res_k": s["res_k"], "res_v": s["res_v"]}
    out = torch.zeros(c["batch"], c["hq"], 128, dtype=torch.float64, device="cuda")
    lse = torch.full((c["batch"], c["hq"]), -math.inf, dtype=torch.float64, device="cuda")
    docs = _doc_starts(c, lens)
    for b, n in enumerate(lens):
        a, lo, hi = _ranges(c, n, docs[b])
        full = n // PAGE
        q_pos = n if c["append"] else n - 1
        if c["append"]:
            s["res_k"][b, :, n % PAGE], s["res_v"][b, :, n % PAGE] = s["k_new"][b], s["v_new"][b]
        see = [t < a or lo <= t < hi for t in range(n)] + ([True] if c["append"] else [])
        seen = torch.tensor(see, dtype=torch.bool, device="cuda")
        cands = [p for p in range(full) if any(see[p * PAGE:(p + 1) * PAGE])]
        ids = s["table"][b, :full].long()
        for h in range(H):
            km, vm = s["k_meta"][ids, h].double(), s["v_meta"][ids, h].double()
            q = s["q"][b, h * nq:(h + 1) * nq].double()
            use = list(range(full))
            if c["op"] == "sparse":
                low, high = km[..., 1], km[..., 1] + 15.0 * km[..., 0]
                reach = sum(torch.maximum(q[j] * low, q[j] * high).sum(1) for j in range(nq)).tolist()
                safe = lambda p: p < c["sink"] or p >= full - c["recent"]  # noqa: E731
                use = sorted(sorted(cands, key=lambda p: (not safe(p), 0.0 if safe(p) else -reach[p], p))[:c["budget"]])
                s["pages"][b, h, :len(use)] = torch.tensor(use, dtype=torch.int32, device="cuda")
                s["counts"][b] = len(use)
            u = torch.tensor(use, dtype=torch.long, device="cuda")
            k = _unpacked64(s["k_codes"][ids[u], h]) * km[u][:, None, :, 0] + km[u][:, None, :, 1]
            v = _unpacked64(s["v_codes"][ids[u], h]).view(-1, PAGE, 4, 32) * vm[u][..., :1] + vm[u][..., 1:]
            t = (u[:, None] * PAGE + torch.arange(PAGE, device="cuda")).flatten()
            rest = torch.arange(full * PAGE, len(see), device="cuda")
            k = torch.cat([k.reshape(-1, 128), s["res_k"][b, h, rest % PAGE].double()])
            v = torch.cat([v.reshape(-1, 128), s["res_v"][b, h, rest % PAGE].double()])
            t = torch.cat([t, rest])
            k, v, t = k[seen[t]], v[seen[t]], t[seen[t]]
            if not len(t):
                continue
            x = q @ k.T / math.sqrt(128.0)
            if c["cap"]:
                x = torch.tanh(x / c["cap"]) * c["cap"]
            if c.get("alibi"):
                x = x + s["slopes"][h * nq:(h + 1) * nq].double()[:, None] * (t - q_pos).double()
            z = torch.logsumexp(x, 1)
            out[b, h * nq:(h + 1) * nq], lse[b, h * nq:(h + 1) * nq] = torch.exp(x - z[:, None]) @ v, z
    r = {"out": out, "lse": lse}
    if c["append"]:
        r.update(res_k=s["res_k"], res_v=s["res_v"])
    if c["op"] == "sparse":
        r.update(pages=s["pages"], counts=s["counts"])
    return r
