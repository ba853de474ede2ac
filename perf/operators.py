"""The operators of an uncompressed layer's paged cache: single-token attention with capped, distance-biased and
masked scores, the attention weight that a prompt's last queries give to every cached token, and eviction of the
tokens that got the least.  Cases, inputs, plain forms (32 bits, elementary torch operations) and the definitions
in 64 bits.

MiniCache merges the layers S .. L-1 of a model; the layers below S keep ordinary caches, which these operators
attend and bound.  Shapes are those of the benchmark's workloads (32 heads x 128 in binary16, 8 kv heads under 32
query heads in bfloat16, pages of 16, 32 and 64 tokens, ragged serving batches, 32768-token sequences)."""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


# ---------------------------------------------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------------------------------------------
def _attn(name, **kw):
    c = dict(name=name, op="attn", dtype="f16", hq=32, hkv=32, ps=16, batch=1, n=512, ragged=False, append=True, cap=0.0,
             alibi=False, window=0, prefix=0, docs=False, marked=False, gather=False)
    c.update(kw)
    return c


def _observe(name, **kw):
    c = dict(name=name, op="observe", dtype="f16", hq=32, hkv=32, ps=16, batch=1, n=512, ragged=False, n_obs=32, cap=0.0,
             alibi=False, window=0, prefix=0, docs=False)
    c.update(kw)
    return c


def _evict(name, **kw):
    c = dict(name=name, op="evict", dtype="f16", hq=32, hkv=32, ps=16, batch=1, n=1025, ragged=False, budget=1024, sink=4,
             recent=64)
    c.update(kw)
    return c


def listed():
    return [
        # one user's first generated tokens: nothing but latency
        _attn("attn_first_tokens", batch=1, n=33),
        # the benchmark's batch, a layer below the merged half: plain causal attention, the step's rows appended
        _attn("attn_7b_batch", batch=8, n=4096),
        # grouped heads, scores capped by a tanh (models that cap their logits), a long batch
        _attn("attn_gqa_capped", dtype="bf16", hkv=8, batch=16, n=8192, cap=50.0),
        # a serving batch of all lengths, packed documents, a sliding window behind four sink tokens
        _attn("attn_ragged_window", ps=32, batch=64, n=2048, ragged=True, window=512, prefix=4, docs=True),
        # a long context whose cache has been evicted from: rows carry their positions, distance bias, weights gathered
        _attn("attn_alibi_long", dtype="bf16", hkv=8, ps=64, batch=4, n=32768, alibi=True, marked=True, gather=True),
        # the steady state of a bounded cache: one token more than the budget, weights gathered
        _attn("attn_bounded_step", dtype="bf16", hkv=8, batch=16, n=1024, marked=True, gather=True),
        # the weights of one short prompt
        _observe("observe_prompt", batch=1, n=512, n_obs=32),
        # the weights of a batch of prompts, grouped heads, capped scores
        _observe("observe_gqa_capped", dtype="bf16", hkv=8, batch=16, n=8192, n_obs=32, cap=50.0),
        # long prompts of odd lengths, a wide window of queries
        _observe("observe_long", dtype="bf16", hkv=8, ps=64, batch=4, n=32749, n_obs=64),
        # every decode step of a bounded cache: one token goes
        _evict("evict_step", batch=8, n=1025, budget=1024),
        # after the prompt: 4096 tokens down to an odd budget
        _evict("evict_prompt", batch=8, n=4096, budget=1000),
        # after a long prompt
        _evict("evict_long", dtype="bf16", hkv=8, ps=64, batch=4, n=32768, budget=4096),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["attn", "attn", "observe", "evict"])
    dtype = rng.choice(["f16", "bf16"])
    hkv, hq = rng.choice([(32, 32), (8, 32), (4, 32), (8, 16), (1, 8), (5, 10), (2, 2)])
    ps = rng.choice([16, 32, 64])
    batch = _log_int(rng, 1, 64)
    # no more cached rows than the largest listed case of the operator has (batch x tokens x kv heads)
    most = min(32768, max(32, (1 << 20) // (batch * hkv)))
    n = _log_int(rng, 1, most)
    ragged = rng.random() < 0.5
    base = dict(dtype=dtype, hq=hq, hkv=hkv, ps=ps, batch=batch, n=n, ragged=ragged)
    score = dict(cap=rng.choice([0.0, 0.0, 30.0, 50.0]), alibi=rng.random() < 0.3,
                 window=rng.choice([0, 0, 1, _log_int(rng, 2, 4096)]), prefix=rng.choice([0, 0, 4, 17]),
                 docs=rng.random() < 0.25)
    if op == "attn":
        c = _attn("", **base, **score, append=rng.random() < 0.7, marked=rng.random() < 0.4, gather=rng.random() < 0.4)
    elif op == "observe":
        c = _observe("", **base, **score, n_obs=_log_int(rng, 1, 256 // (hq // hkv) if hq // hkv > 3 else 64))
    else:
        c = _evict("", **base, budget=_log_int(rng, 1, n), sink=rng.choice([0, 1, 4]), recent=0)
        c["sink"] = min(c["sink"], c["budget"])
        c["recent"] = rng.randint(0, c["budget"] - c["sink"])
    del c["name"]
    return c


def _lens(c):
    """Cached tokens per sequence: a property of the case (its work follows from it), not of the seed."""
    if not c["ragged"]:
        return [c["n"]] * c["batch"]
    lo, out = max(1, c["n"] // 16), []
    for i in range(c["batch"]):
        f = (0.381 + 0.618034 * i) % 1.0
        out.append(max(1, min(c["n"], int(round(lo * (c["n"] / lo) ** f)))))
    out[0] = c["n"]
    if c["batch"] > 3:
        out[2] = 0  # a slot without a sequence
    return out


def _doc_starts(c, lens):
    return [n // 3 if c["docs"] and i % 2 else 0 for i, n in enumerate(lens)]


def _visible(c, n_cached, q_pos, doc):
    """Cached tokens (indices = positions) that a query at q_pos sees."""
    a = min(n_cached, c["prefix"], q_pos + 1)
    lo = max(doc, q_pos - c["window"] + 1 if c["window"] else 0)
    lo, hi = max(lo, a), min(n_cached, q_pos + 1)
    return a + max(0, hi - lo)


def work(c):
    lens, nq = _lens(c), c["hq"] // c["hkv"]
    if c["op"] == "attn":
        rows = 0  # cached token rows per kv head that some query needs
        for n, d in zip(lens, _doc_starts(c, lens)):
            # (positions of an evicted cache: every third one is missing, so a window sees about two thirds of its width)
            q_pos = _span(c, n) if c["append"] else _span(c, n) - 1
            rows += n if c["marked"] and not c["window"] and not c["docs"] else _visible(c, n, q_pos, d)
        th = rows * c["hkv"]
        new = c["batch"] * c["hkv"]
        b = th * 512 + new * (512 + 512 if c["append"] else 0) + c["batch"] * c["hq"] * (512 + 4)
        b += sum(lens) * c["hkv"] * 4 if c["marked"] else 0
        b += th * 8 if c["gather"] else 0
        return {"bytes": b, "flops": 4 * 128 * nq * (th + (new if c["append"] else 0))}
    if c["op"] == "observe":
        th = sum(lens) * c["hkv"]
        return {"bytes": th * (256 + 4) + c["batch"] * c["n_obs"] * c["hq"] * 256, "flops": 2 * 128 * nq * c["n_obs"] * th}
    b, k = 0, c["budget"]
    for n in lens:
        if n <= k:
            continue
        fixed = c["sink"] + c["recent"]
        free = k - fixed  # kept by weight: spread evenly over what is not protected
        behind = max(0, n - k - c["recent"]) / max(1, n - fixed)
        moved = min(c["recent"], n - k) + free * behind
        b += c["hkv"] * (n * 8 + moved * (2 * 512 + 8))
    return {"bytes": max(b, 8 * c["batch"]), "flops": 0}


# ---------------------------------------------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------------------------------------------
def _span(c, n):
    """Position behind a sequence of n cached tokens: with marks every third position has been evicted."""
    return n + n // 2 if c.get("marked") else n


def prepare(c, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(1_000_003 * seed + 17)
    dt, ps, H, B = DTYPES[c["dtype"]], c["ps"], c["hkv"], c["batch"]
    lens = _lens(c)
    pages = [max(1, -(-(n + 1) // ps)) for n in lens]
    n_pages, mp = sum(pages), max(pages)
    order = torch.randperm(n_pages, generator=g, device="cuda").to(torch.int32)
    table = torch.zeros(B, mp, dtype=torch.int32, device="cuda")
    held = torch.arange(mp, device="cuda")[None, :] < torch.tensor(pages, device="cuda")[:, None]
    table[held] = order
    randn = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731

    def rows(*s):  # unit directions of log-normal length
        x = torch.empty(*s, 128, dtype=dt, device="cuda")
        for i in range(0, s[0], 4096):  # (a large pool in parts: the 32-bit intermediate stays small)
            p = (min(4096, s[0] - i),) + s[1:]
            x[i:i + p[0]] = (randn(*p, 128) * (1 / math.sqrt(128.0)) * torch.exp(0.5 * randn(*p, 1))).to(dt)
        return x

    s = dict(c=dict(c), lens=torch.tensor(lens, dtype=torch.int32, device="cuda"), max_len=max(lens), table=table, n_pages=n_pages,
             k=rows(n_pages, H, ps), v=rows(n_pages, H, ps), status=torch.zeros(4, dtype=torch.int32, device="cuda"))
    tok = (torch.arange(mp * ps, device="cuda").view(1, mp, 1, ps)).expand(B, mp, H, ps)  # token index of every slot
    if c["op"] == "attn":
        s["q"] = (randn(B, c["hq"], 128) * (2.5 * math.sqrt(128.0))).to(dt)
        s["k_new"], s["v_new"] = (rows(B, H), rows(B, H)) if c["append"] else (None, None)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros(B, c["hq"], device="cuda")
        if c["marked"]:  # positions 0, 1, 3, 4, 6, 7, ... in an order that eviction has stirred, alike in no two heads
            s["pos"] = torch.zeros(n_pages, H, ps, dtype=torch.int32, device="cuda")
            nn = s["lens"].long().view(B, 1, 1, 1)
            head = torch.arange(H, device="cuda").view(1, 1, H, 1)
            i = torch.where(tok < nn, (tok + 7 * head) % nn.clamp(min=1), tok)
            s["pos"][table[held].long()] = (i + i // 2).to(torch.int32)[held]
            s["q_pos"] = torch.tensor([_span(c, n) - (0 if c["append"] else 1) for n in lens], dtype=torch.int32, device="cuda")
        if c["gather"]:
            s["weights0"] = torch.rand(n_pages, H, ps, generator=g, device="cuda")
            s["weights"] = s["weights0"].clone()
    elif c["op"] == "observe":
        s["q"] = (randn(B, c["n_obs"], c["hq"], 128) * (2.5 * math.sqrt(128.0))).to(dt)
        s["weights"] = torch.zeros(n_pages, H, ps, device="cuda")
    else:
        # weights of a long tail, on a grid so that ties happen; positions and weights side by side: the pass puts
        # both back first, so that every pass meets the same cache (the rows behind the budget are never written)
        s["marks0"] = torch.empty(2, n_pages, H, ps, device="cuda")
        s["marks0"][0] = torch.round(torch.exp(2.0 * randn(n_pages, H, ps)) * 64.0) / 64.0
        pos = torch.zeros(n_pages, H, ps, dtype=torch.int32, device="cuda")
        pos[table[held].long()] = tok.to(torch.int32)[held]
        s["marks0"][1] = pos.view(torch.float32)
        s["marks"] = s["marks0"].clone()
        s["new_lens"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    if c["op"] != "evict":
        s["prefix"] = torch.full((B,), c["prefix"], dtype=torch.int32, device="cuda") if c["prefix"] else None
        s["docs"] = torch.tensor(_doc_starts(c, lens), dtype=torch.int32, device="cuda") if c["docs"] else None
        s["slopes"] = torch.exp2(-8.0 * torch.arange(1, c["hq"] + 1, device="cuda") / c["hq"]).float() if c["alibi"] else None
    return s


# ---------------------------------------------------------------------------------------------------------------
# plain forms
# ---------------------------------------------------------------------------------------------------------------
def _dense(pool, table):
    """[pages][H][ps][...] -> [B][H][tokens][...] through the block table."""
    x = pool[table.long()]  # [B][mp][H][ps]...
    x = x.transpose(1, 2)
    return x.reshape(x.shape[0], x.shape[1], x.shape[2] * x.shape[3], *x.shape[4:])


def _seen(c, s, pos, q_pos):
    """Which positions a query at q_pos sees; both broadcast, the sequence is the first axis."""
    shape = (-1,) + (1,) * (pos.dim() - 1)
    lo = s["docs"].view(shape) if s["docs"] is not None else 0
    near = pos >= lo
    if c["window"]:
        near = near & (q_pos - pos < c["window"])
    if s["prefix"] is not None:
        near = near | (pos < s["prefix"].view(shape))
    return near & (pos <= q_pos)


def _scores(c, s, dots, pos, q_pos, head_axis):
    x = dots * (1.0 / math.sqrt(128.0))
    if c["cap"]:
        x = c["cap"] * torch.tanh(x / c["cap"])
    if s["slopes"] is not None:
        shape = [1] * x.dim()
        shape[head_axis], shape[head_axis + 1] = c["hkv"], c["hq"] // c["hkv"]
        x = x - s["slopes"].view(shape) * (q_pos - pos).float()
    return x


def _plain_attn(s):
    c = s["c"]
    B, H, ps, nq = c["batch"], c["hkv"], c["ps"], c["hq"] // c["hkv"]
    n = s["lens"].long()
    if c["append"]:
        page = s["table"].long()[torch.arange(B, device="cuda"), n // ps]
        s["k"][page, :, n % ps], s["v"][page, :, n % ps] = s["k_new"], s["v_new"]
        if c["marked"]:
            s["pos"][page, :, n % ps] = s["q_pos"][:, None]
        total = n + 1
    else:
        total = n
    k, v = _dense(s["k"], s["table"]).float(), _dense(s["v"], s["table"]).float()
    at = torch.arange(k.shape[2], device="cuda").view(1, 1, 1, -1)
    pos = _dense(s["pos"], s["table"])[:, :, None].long() if c["marked"] else at
    q_pos = (s["q_pos"].long() if c["marked"] else total - 1).view(B, 1, 1, 1)
    dots = s["q"].float().view(B, H, nq, 128) @ k.transpose(2, 3)
    x = _scores(c, s, dots, pos, q_pos, 1)
    x = x.masked_fill(~(_seen(c, s, pos, q_pos) & (at < total.view(B, 1, 1, 1))), -math.inf)
    m = x.amax(3, keepdim=True)
    e = torch.exp(x - torch.where(m == -math.inf, torch.zeros_like(m), m))
    l = e.sum(3, keepdim=True)
    p = e / torch.where(l > 0, l, torch.ones_like(l))
    s["out"].copy_((p @ v).reshape(B, c["hq"], 128).to(s["out"].dtype))
    s["lse"].copy_((m + torch.log(l)).reshape(B, c["hq"]))
    if c["gather"]:
        s["weights"].copy_(s["weights0"])
        held = at[:, :, 0] < total.view(B, 1, 1)
        w = _dense(s["weights"], s["table"]).clone()
        if c["append"]:
            w = torch.where(at[:, :, 0] == n.view(B, 1, 1), torch.zeros_like(w), w)  # the new row begins at nothing
        _put(s["weights"], s["table"], w + p.sum(2), held)


def _put(pool, table, dense, held):
    """The held tokens of [B][H][tokens] back into [pages][H][ps]."""
    b, h, t = held.expand_as(dense).nonzero(as_tuple=True)
    ps = pool.shape[2]
    pool[table.long()[b, t // ps], h, t % ps] = dense[b, h, t]


def _plain_observe(s):
    c = s["c"]
    B, H, nq, J = c["batch"], c["hkv"], c["hq"] // c["hkv"], c["n_obs"]
    n = s["lens"].long()
    k = _dense(s["k"], s["table"]).float()
    at = torch.arange(k.shape[2], device="cuda").view(1, 1, 1, 1, -1)
    q = s["q"].float().view(B, J, H, nq, 128).permute(0, 2, 3, 1, 4)  # [B][H][nq][J][128]
    q_pos = n.view(B, 1, 1, 1, 1) - J + torch.arange(J, device="cuda").view(1, 1, 1, -1, 1)
    x = _scores(c, s, (q.reshape(B, H, -1, 128) @ k.transpose(2, 3)).view(B, H, nq, J, -1), at, q_pos, 1)
    x = x.masked_fill(~(_seen(c, s, at, q_pos) & (q_pos >= 0)), -math.inf)
    m = x.amax(4, keepdim=True)
    e = torch.exp(x - torch.where(m == -math.inf, torch.zeros_like(m), m))
    l = e.sum(4, keepdim=True)
    w = (e / torch.where(l > 0, l, torch.ones_like(l))).sum((2, 3))
    _put(s["weights"], s["table"], w, at[:, :, 0, 0] < n.view(B, 1, 1))


def _plain_evict(s):
    c = s["c"]
    B, H, ps, budget = c["batch"], c["hkv"], c["ps"], c["budget"]
    s["marks"].copy_(s["marks0"])
    weights, pos = s["marks"][0], s["marks"][1].view(torch.int32)
    n = s["lens"].long()
    w, p = _dense(weights, s["table"]), _dense(pos, s["table"]).long()
    at = torch.arange(w.shape[2], device="cuda").view(1, 1, -1)
    nn = n.view(B, 1, 1)
    guarded = (p < c["sink"]) | (p > nn - 1 - c["recent"])
    key = torch.where(guarded, torch.full_like(w, math.inf), w).masked_fill(at >= nn, -math.inf)
    order = torch.sort(key, dim=2, descending=True, stable=True)[1]
    kept = torch.zeros_like(key, dtype=torch.bool).scatter_(2, order[:, :, :budget], True) & (at < nn)
    over = nn > budget
    src = (kept & (at >= budget) & over).nonzero(as_tuple=True)
    dst = (~kept & (at < budget) & over).nonzero(as_tuple=True)  # as many per (sequence, head), in the same order
    slot = lambda x: (s["table"].long()[x[0], x[2] // ps], x[1], x[2] % ps)  # noqa: E731
    for pool in (s["k"], s["v"], weights, pos):
        pool[slot(dst)] = pool[slot(src)]
    s["new_lens"].copy_(n.clamp(max=budget).to(torch.int32))


# ---------------------------------------------------------------------------------------------------------------
# the framework's calls
# ---------------------------------------------------------------------------------------------------------------
def _handle(s):
    """What a user's program sets up once per cache: the configuration, the batch and cache descriptions, scratch memory."""
    import paper_2405_14366_b200 as mc
    c = s["c"]
    lib = mc.lib()
    cfg = mc.McConfig(c["hkv"], c["hq"], c["ps"], c["dtype"])
    batch = mc.Batch(s["table"], s["lens"], s["max_len"], s["n_pages"])
    flags = (mc.MC_LAYER_APPEND if c.get("append") else 0) | (mc.MC_LAYER_ACCUMULATE if c.get("gather") else 0)
    if c["op"] == "evict":
        layer = mc.LayerCache(cfg, s["k"], s["v"], positions=s["marks"][1].view(torch.int32), weights=s["marks"][0], status=s["status"])
        opts, op = mc.EvictOpts(c["budget"], c["sink"], c["recent"]), mc.MC_OP_LAYER_EVICT
    else:
        layer = mc.LayerCache(cfg, s["k"], s["v"], positions=s.get("pos"), weights=s.get("weights"), status=s["status"])
        opts = mc.ScoreOpts(1.0 / math.sqrt(128.0), softcap=c["cap"], alibi_slopes=s["slopes"], window=c["window"],
                            doc_start=s["docs"], prefix_len=s["prefix"], q_pos=s.get("q_pos"))
        op = mc.MC_OP_LAYER_ATTN if c["op"] == "attn" else mc.MC_OP_LAYER_OBSERVE
    ws = torch.empty(lib.mc_layer_workspace_bytes(cfg, batch, op, c.get("n_obs", flags)), dtype=torch.uint8, device="cuda")
    return lib, cfg, batch, layer, opts, flags, ws


def _call(s):
    if "handle" not in s:
        s["handle"] = _handle(s)
    lib, cfg, batch, layer, opts, flags, ws = s["handle"]
    c = s["c"]
    if c["op"] == "attn":
        if c["gather"]:
            s["weights"].copy_(s["weights0"])  # every pass adds to the same weights
        lib.mc_layer_attn(cfg, batch, layer, opts, s["q"], s["k_new"], s["v_new"], flags, s["out"], s["lse"], ws)
    elif c["op"] == "observe":
        lib.mc_layer_observe(cfg, batch, layer, opts, s["q"], 0, ws)
    else:
        s["marks"].copy_(s["marks0"])
        lib.mc_layer_evict(cfg, batch, layer, opts, s["new_lens"], ws)


def _outputs(s):
    c = s["c"]
    if c["op"] == "observe":
        return {"weights": s["weights"]}
    if c["op"] == "evict":
        return {"k": s["k"], "v": s["v"], "weights": s["marks"][0], "pos": s["marks"][1].view(torch.int32), "lens": s["new_lens"]}
    r = {"out": s["out"], "lse": s["lse"]}
    if c["append"]:
        r.update(k=s["k"], v=s["v"])
        if c["marked"]:
            r["pos"] = s["pos"]
    if c["gather"]:
        r["weights"] = s["weights"]
    return r


def run(state):
    if own:
        _call(state)
    else:
        {"attn": _plain_attn, "observe": _plain_observe, "evict": _plain_evict}[state["c"]["op"]](state)
    return _outputs(state)


# ---------------------------------------------------------------------------------------------------------------
# the definitions in 64 bits, one sequence and one query after the other
# ---------------------------------------------------------------------------------------------------------------
def _rows64(pool, table_row, h, n, ps):
    """Rows (or marks) of the first n tokens of a sequence, kv head h (or all heads: a slice)."""
    t = torch.arange(n, device="cuda")
    return pool[table_row[t // ps].long(), h, t % ps]


def _softmax64(c, s, b, h, keys, pos, q, q_pos):
    """Probabilities of kv head h's queries [nq][128] at q_pos over n keys, and their log-sum-exps."""
    nq = c["hq"] // c["hkv"]
    x = q.double() @ keys.double().T / math.sqrt(128.0)
    if c["cap"]:
        x = torch.tanh(x / c["cap"]) * c["cap"]
    if c["alibi"]:
        slope = s["slopes"][h * nq:(h + 1) * nq].double()
        x = x + slope[:, None] * (pos.double() - float(q_pos))[None, :]
    ok = pos <= q_pos
    near = torch.ones_like(ok)
    if c["docs"]:
        near &= pos >= int(s["docs"][b])
    if c["window"]:
        near &= pos > q_pos - c["window"]
    if c["prefix"]:
        near |= pos < c["prefix"]
    x[:, ~(ok & near)] = -math.inf
    lse = torch.logsumexp(x, 1)
    p = torch.exp(x - lse[:, None])
    p[:, ~(ok & near)] = 0.0  # (a query that sees nothing has no probabilities)
    return p, lse


def exact(c, seed):
    c = dict(c)
    lens, ps, H, nq = _lens(c), c["ps"], c["hkv"], c["hq"] // c["hkv"]
    steps = sum(1 for n in lens if n) * H * (c["n_obs"] if c["op"] == "observe" else 1)
    if steps > 40_000:
        return None
    s = prepare(c, seed)
    if c["op"] == "evict":
        k, v, w, pos = s["k"], s["v"], s["marks0"][0], s["marks0"][1].view(torch.int32)
        for b, n in enumerate(lens):
            if n <= c["budget"]:
                continue
            where = [(s["table"][b, t // ps].item(), t % ps) for t in range(0, n, ps)]
            page = torch.tensor([x for x, _ in where], device="cuda").repeat_interleave(ps)[:n]
            slot = torch.arange(n, device="cuda") % ps
            for h in range(H):
                ww, pp = w[page, h, slot].double().cpu(), pos[page, h, slot].cpu()
                safe = (pp < c["sink"]) | (pp >= n - c["recent"])
                rank = sorted(range(n), key=lambda i, a=safe.tolist(), x=ww.tolist(): (not a[i], -x[i], i)) if n <= 4096 else \
                    torch.sort(torch.where(safe, torch.full_like(ww, math.inf), ww), descending=True, stable=True)[1].tolist()
                keep = set(rank[:c["budget"]])
                holes = [i for i in range(c["budget"]) if i not in keep]
                movers = sorted(i for i in keep if i >= c["budget"])
                a, z = torch.tensor(movers, device="cuda", dtype=torch.long), torch.tensor(holes, device="cuda", dtype=torch.long)
                for x in (k, v, w, pos):
                    x[page[z], h, slot[z]] = x[page[a], h, slot[a]]
        return {"k": k, "v": v, "weights": w, "pos": pos, "lens": torch.tensor([min(n, c["budget"]) for n in lens], dtype=torch.int32)}
    if c["op"] == "observe":
        w = torch.zeros(s["weights"].shape, dtype=torch.float64, device="cuda")
        for b, n in enumerate(lens):
            if not n:
                continue
            t = torch.arange(n, device="cuda")
            page = s["table"][b, t // ps].long()
            for h in range(H):
                keys = _rows64(s["k"], s["table"][b], h, n, ps)
                for j in range(c["n_obs"]):
                    if (q_pos := n - c["n_obs"] + j) >= 0:
                        w[page, h, t % ps] += _softmax64(c, s, b, h, keys, t, s["q"][b, j, h * nq:(h + 1) * nq], q_pos)[0].sum(0)
        return {"weights": w}
    out = torch.zeros(c["batch"], c["hq"], 128, dtype=torch.float64, device="cuda")
    lse = torch.full((c["batch"], c["hq"]), -math.inf, dtype=torch.float64, device="cuda")
    w = s["weights0"].double() if c["gather"] else None
    for b, n in enumerate(lens):
        if c["append"]:
            page = s["table"][b, n // ps].item()
            s["k"][page, :, n % ps], s["v"][page, :, n % ps] = s["k_new"][b], s["v_new"][b]
            if c["marked"]:
                s["pos"][page, :, n % ps] = s["q_pos"][b]
            if c["gather"]:
                w[page, :, n % ps] = 0.0
            n += 1
        if not n:
            continue
        q_pos = int(s["q_pos"][b]) if c["marked"] else n - 1
        t = torch.arange(n, device="cuda")
        for h in range(H):
            keys, vals = _rows64(s["k"], s["table"][b], h, n, ps), _rows64(s["v"], s["table"][b], h, n, ps)
            pos = _rows64(s["pos"], s["table"][b], h, n, ps) if c["marked"] else t
            p, z = _softmax64(c, s, b, h, keys, pos, s["q"][b, h * nq:(h + 1) * nq], q_pos)
            out[b, h * nq:(h + 1) * nq], lse[b, h * nq:(h + 1) * nq] = p @ vals.double(), z
            if c["gather"]:
                w[s["table"][b, t // ps].long(), h, t % ps] += p.sum(0)
    r = {"out": out, "lse": lse}
    if c["append"]:
        r.update(k=s["k"], v=s["v"])
        if c["marked"]:
            r["pos"] = s["pos"]
    if c["gather"]:
        r["weights"] = w
    return r
