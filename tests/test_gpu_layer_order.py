"""The mc_layer_* calls next to other work: behind a kernel that uses tensor memory, from several host threads, and with
other contents in the rows that do not count."""
import math

import numpy as np
import pytest
import torch

import gen
from gen import CONFIGS

pytestmark = pytest.mark.gpu

SM = 1.0 / math.sqrt(128.0)


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2405_14366_b200.build import build_library
    build_library()
    import layer_harness
    return layer_harness


@pytest.mark.parametrize("lens,Hq,J", [([512, 300], 8, 40), ([700, 1], 2, 128), ([4200, 77], 8, 20)])
@pytest.mark.parametrize("graph", [False, True])
def test_observe_behind_a_prefill_merge(L, lens, Hq, J, graph):
    """Both take tensor memory: the merge in a layer's projection, then the weights of a prompt, without a pause, in turn: the
    bits of calls that find the device idle.  (Short prompts of more than 128 rows, of one and of two tiles per CTA; a long one.)"""
    import mc_harness
    wl = CONFIGS["c1"].scaled("pf", n_kv_heads=8, n_q_heads=8, dtype="bf16", batch=4, seq_len=512, index=68)
    case = {k: v.cuda() for k, v in gen.make_projection_case(wl, 0, 1024, 512).items()}
    zeros = torch.zeros_like(case["k_lm1"]).cpu()
    p = mc_harness.Problem(wl, seq_lens=np.asarray([512, 512, 400, 512], np.int32),
                           tensors={"k_lm1": case["k_lm1"].cpu(), "v_lm1": case["v_lm1"].cpu(), "k_l": zeros, "v_l": zeros.clone()})
    ws_p, pools = p.workspace(0), [p.pools[k] for k in ("k_lm1", "v_lm1", "k_l", "v_l")]
    c = L.Cache(lens, 2, Hq, 16, "bf16", seed=3, weights=True)
    mc, lib = c.mc, c.mc.lib()
    q, ws = c.queries(len(lens), J, Hq).cuda(), c.workspace(mc.MC_OP_LAYER_OBSERVE, J)

    def run(pause, times):
        for i in range(times):
            lib.mc_prefill_merge_pair(p.cfg, p.batch(), case["x"], case["w_k"], case["w_v"], *pools, p.pair, 0.9, i % 2 == 0, ws_p)
            pause()
            lib.mc_layer_observe(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), q, mc.MC_LAYER_ACCUMULATE if i else 0, ws)
            pause()
    got = []
    for idle in (True, False):
        c.d["w"].zero_()
        p.pair.e_k.zero_()
        torch.cuda.synchronize()
        if idle or not graph:
            run(torch.cuda.synchronize if idle else lambda: None, 20)
        else:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                run(lambda: None, 20)
            g.replay()
        torch.cuda.synchronize()
        assert lib.mc_layer_read_status(c.layer, check=False)[1] == 0
        got.append([c.d["w"].clone(), p.pair.e_k.clone().view(torch.int16)])
    assert all(torch.equal(a, b) for a, b in zip(*got)) and float(got[0][0].sum()) > 0


@pytest.mark.parametrize("lens,Hq,J", [([512, 300], 8, 40), ([700, 1], 2, 128), ([4200, 77], 8, 20)])
def test_observe_next_to_a_prefill_merge(L, lens, Hq, J):
    """The same two operators at the same time, on streams of their own: each gets what it gets alone.  (A CTA that holds tensor
    memory never waits for one that may not have it: the merge's wait for nobody, a cluster's wait for CTAs that wait for those.)"""
    import mc_harness
    wl = CONFIGS["c1"].scaled("pf", n_kv_heads=8, n_q_heads=8, dtype="bf16", batch=4, seq_len=512, index=68)
    case = {k: v.cuda() for k, v in gen.make_projection_case(wl, 0, 1024, 512).items()}
    zeros = torch.zeros_like(case["k_lm1"]).cpu()
    p = mc_harness.Problem(wl, seq_lens=np.asarray([512, 512, 400, 512], np.int32),
                           tensors={"k_lm1": case["k_lm1"].cpu(), "v_lm1": case["v_lm1"].cpu(), "k_l": zeros, "v_l": zeros.clone()})
    ws_p, pools = p.workspace(0), [p.pools[k] for k in ("k_lm1", "v_lm1", "k_l", "v_l")]
    c = L.Cache(lens, 2, Hq, 16, "bf16", seed=3, weights=True)
    mc, lib = c.mc, c.mc.lib()
    q, ws = c.queries(len(lens), J, Hq).cuda(), c.workspace(mc.MC_OP_LAYER_OBSERVE, J)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    for times in (1, 100):
        torch.cuda.synchronize()
        for _ in range(times):
            lib.mc_prefill_merge_pair(p.cfg, p.batch(), case["x"], case["w_k"], case["w_v"], *pools, p.pair, 0.9, False, ws_p, stream=streams[0])
            if times == 1:
                torch.cuda.synchronize()
            lib.mc_layer_observe(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), q, 0, ws, stream=streams[1])
        torch.cuda.synchronize()
        assert lib.mc_layer_read_status(c.layer, check=False)[1] == 0
        got.append([c.d["w"].clone(), p.pair.e_k.clone().view(torch.int16)])
    assert all(torch.equal(a, b) for a, b in zip(*got)) and float(got[0][0].sum()) > 0


def unseen_filled(L, lens, H, Hq, ps, dtype, fill, visible, seed=11, max_len=None):
    """A cache whose rows outside visible(b) (a truth value per token) all hold `fill`: hidden, behind the sequence, of nobody."""
    c = L.Cache(lens, H, Hq, ps, dtype, seed=seed, weights=True, poison=False, max_len=max_len)
    keep = torch.zeros(c.n_pages, ps, dtype=torch.bool)
    for b, n in enumerate(lens):
        t = torch.arange(n)
        keep[c.table[b, t // ps].long(), t % ps] = visible(b)
    for k in ("k", "v"):
        c.d[k].copy_(torch.where(keep[:, None, :, None], getattr(c, k), torch.full((), fill).to(c.dt)))
    return c


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("window,prefix,doc", [(0, 0, 0), (20, 3, 0), (0, 0, 9)])
@pytest.mark.parametrize("lens,ps", [([32, 48, 7, 160], 16), ([64, 128, 33, 1], 64), ([500, 2000, 176], 32)])
def test_attention_under_a_cap_does_not_see_what_it_must_not(L, lens, ps, window, prefix, doc, dtype):
    """Which form of the cap a visible score takes may not follow from rows that do not count, nor from what another call left
    in shared memory: the same bits whatever they are.  (A new row that opens a slice of 16 tokens stands among stale rows.)"""
    H, Hq, B = 2, 8, len(lens)
    got = []
    for fill in (0.0, 6.0e4, float("nan"), float("inf"), -6.0e4):
        c = unseen_filled(L, lens, H, Hq, ps, dtype, fill, lambda b: L.seen(torch.arange(lens[b]), lens[b], window, doc, prefix))
        mc, lib = c.mc, c.mc.lib()
        flags = mc.MC_LAYER_APPEND | mc.MC_LAYER_ACCUMULATE
        ten = lambda x: torch.full((B,), x, dtype=torch.int32, device="cuda") if x else None  # noqa: E731
        ws = c.workspace(mc.MC_OP_LAYER_ATTN, flags)
        q, kn, vn = c.queries(B, Hq).cuda(), c.rows(B, H).cuda(), c.rows(B, H).cuda()
        out, lse = torch.zeros_like(q), torch.zeros(B, Hq, device="cuda")

        def before(value):  # every SM's stages full of `value`
            d = L.Cache([300] * 64, H, Hq, 16, dtype, poison=False)
            for k in ("k", "v"):
                d.d[k].fill_(value)
            x = torch.full((64, Hq, 128), 1.0, dtype=d.dt, device="cuda")
            lib.mc_layer_attn(d.cfg, d.batch, d.layer, mc.ScoreOpts(SM, softcap=50.0), x, None, None, 0, torch.zeros_like(x), None,
                              d.workspace(mc.MC_OP_LAYER_ATTN))
        before(0.0 if fill != fill else fill)
        torch.cuda.synchronize()
        lib.mc_layer_attn(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM, softcap=50.0, window=window, prefix_len=ten(prefix), doc_start=ten(doc)),
                          q, kn, vn, flags, out, lse, ws)
        torch.cuda.synchronize()
        assert lib.mc_layer_read_status(c.layer, check=False)[1] == 0
        w = [c.gathered("w", b, n + 1) for b, n in enumerate(lens)]
        got.append([out.view(torch.int16).cpu(), lse.cpu()] + w)
    assert not torch.isnan(got[0][1]).any()  # (-inf: a document that begins behind a short sequence's query)
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))


@pytest.mark.parametrize("dtype,marks", [("f16", False), ("bf16", False), ("bf16", True)])
@pytest.mark.parametrize("window,prefix,doc", [(0, 0, 0), (60, 3, 0), (0, 0, 90)])
@pytest.mark.parametrize("lens,J", [([77, 512, 300], 5), ([1000, 130, 17], 17), ([1, 700, 257], 40), ([4200, 77, 200], 5), ([2300, 300, 129], 40),
                                    ([4301, 1, 255], 13)])
def test_weights_under_a_cap_do_not_see_what_they_must_not(L, lens, J, window, prefix, doc, marks, dtype):
    """The same for a prompt's weights: tokens behind a sequence (their pages are copied or not), hidden ones, and the rows between
    a group's queries and the tile's 32, 64 or 128 (nothing fills them).  Prompts in one launch and in two, one and two row tiles."""
    H, Hq, B, ps = 2, 8, len(lens), 16
    got = []
    for fill in (0.0, 6.0e4, float("nan"), float("inf"), -6.0e4):
        spots = (lambda b: torch.ones(lens[b], dtype=torch.bool)) if marks else \
            (lambda b: torch.stack([L.seen(torch.arange(lens[b]), lens[b] - J + j, window, doc, prefix) for j in range(J)]).any(0))
        c = unseen_filled(L, lens, H, Hq, ps, dtype, fill, spots)
        mc, lib = c.mc, c.mc.lib()
        layer = c.layer
        if marks:  # positions as the tokens' own: nothing is left out, every tile is looked at token by token
            pos = torch.full((c.n_pages, H, ps), -5, dtype=torch.int32)
            for b, n in enumerate(lens):
                t = torch.arange(n)
                pos[c.table[b, t // ps].long(), :, t % ps] = t.int()[:, None].expand(n, H)
            layer = mc.LayerCache(c.cfg, c.d["k"], c.d["v"], pos.cuda(), c.d["w"], status=c.layer.status)
        ten = lambda x: torch.full((B,), x, dtype=torch.int32, device="cuda") if x else None  # noqa: E731
        ws = c.workspace(mc.MC_OP_LAYER_OBSERVE, J)
        q = c.queries(B, J, Hq).cuda()
        for n, m in ((c.max_len, 64), (600, 32)):  # tiles, queries and tensor memory full of `fill`
            d = L.Cache([n] * 8, H, Hq, ps, dtype, poison=False, weights=True)
            x = 0.0 if fill != fill else fill
            d.d["k"].fill_(x)
            lib.mc_layer_observe(d.cfg, d.batch, d.layer, mc.ScoreOpts(SM, softcap=50.0), torch.full((8, m, Hq, 128), x, dtype=d.dt, device="cuda"),
                                 0, d.workspace(mc.MC_OP_LAYER_OBSERVE, m))
        torch.cuda.synchronize()
        lib.mc_layer_observe(c.cfg, c.batch, layer, mc.ScoreOpts(SM, softcap=50.0, window=window, prefix_len=ten(prefix), doc_start=ten(doc)), q, 0, ws)
        torch.cuda.synchronize()
        assert lib.mc_layer_read_status(layer, check=False)[1] == 0
        got.append([c.gathered("w", b, n) for b, n in enumerate(lens)])
    assert all(torch.isfinite(w).all() for w in got[0]) and float(sum(w.sum() for w in got[0])) > 0
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))



@pytest.mark.parametrize("op", ["attn", "observe", "observe long", "evict", "prefill"])
def test_the_first_call_of_a_host_thread(L, op):
    """A thread that has made no CUDA call of its own yet: the same results as from the thread that made the tensors."""
    import threading
    c = L.Cache([4200 if op == "observe long" else 100, 30], 2, 8, 16, "bf16", marks=op == "evict", weights=True)
    mc, lib = c.mc, c.mc.lib()
    if op == "attn":
        q = c.queries(2, 8).cuda()
        got, ws = torch.zeros_like(q), c.workspace(mc.MC_OP_LAYER_ATTN)
        call = lambda s: lib.mc_layer_attn(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), q, None, None, 0, got, None, ws, stream=s)  # noqa: E731
    elif op == "evict":
        got, ws = torch.zeros_like(c.d_lens), c.workspace(mc.MC_OP_LAYER_EVICT)
        call = lambda s: lib.mc_layer_evict(c.cfg, c.batch, c.layer, mc.EvictOpts(50), got, ws, stream=s)  # noqa: E731
    elif op == "prefill":
        import mc_harness
        wl = CONFIGS["c1"].scaled("pf", n_kv_heads=2, n_q_heads=2, dtype="bf16", batch=1, seq_len=128, index=68)
        case = {k: v.cuda() for k, v in gen.make_projection_case(wl, 0, 128, 128).items()}
        zeros = torch.zeros_like(case["k_lm1"]).cpu()
        p = mc_harness.Problem(wl, seq_lens=np.asarray([128], np.int32),
                               tensors={"k_lm1": case["k_lm1"].cpu(), "v_lm1": case["v_lm1"].cpu(), "k_l": zeros, "v_l": zeros.clone()})
        got, ws = p.pair.e_k.view(torch.int16), p.workspace(0)
        call = lambda s: lib.mc_prefill_merge_pair(p.cfg, p.batch(), case["x"], case["w_k"], case["w_v"],  # noqa: E731
                                                   *[p.pools[k] for k in ("k_lm1", "v_lm1", "k_l", "v_l")], p.pair, 0.9, True, ws, stream=s)
    else:
        q, ws, got = c.queries(2, 8, 8).cuda(), c.workspace(mc.MC_OP_LAYER_OBSERVE, 8), c.d["w"]
        call = lambda s: lib.mc_layer_observe(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), q, 0, ws, stream=s)  # noqa: E731
    stream, start, failed = torch.cuda.Stream(), got.clone(), []

    def work():
        try:
            call(stream)
        except Exception as e:  # noqa: BLE001
            failed.append(e)
    torch.cuda.synchronize()
    t = threading.Thread(target=work)
    t.start()
    t.join()
    assert not failed, failed
    torch.cuda.synchronize()
    there = got.clone()
    got.copy_(start)
    if op == "evict":  # (both find all rows in place)
        assert there.tolist() == [50, 30]
        return
    torch.cuda.synchronize()
    call(stream)
    torch.cuda.synchronize()
    assert torch.equal(there, got) and not torch.equal(there, start)


@pytest.mark.parametrize("op", ["attn", "observe", "observe long", "evict"])
def test_threads_with_calls_of_different_sizes(L, op):
    """Host threads, a stream and a workspace each, whose calls need different amounts of shared memory: none is refused, and
    each gets what it gets alone.  (The library's own entry points, so that the threads meet inside them.)"""
    import sys
    import threading
    small, large = {"attn": ([40] * 2, [40] * 512), "observe": ([500], [500]), "observe long": ([4200], [9] * 511 + [4200]),
                    "evict": ([60] * 8, [60] * 8)}[op]
    sides = []
    for i, lens in enumerate((small, large, small, large)):
        c = L.Cache(lens, 1, 8, 16, "bf16", seed=i, marks=op == "evict", weights=True, max_len=30000 if op == "evict" and i % 2 else None)
        mc, lib, s = c.mc, c.mc.lib(), torch.cuda.Stream()
        raw, made = lib._lib, []

        class Spy:  # the entry point and the arguments that the binding gives it
            def __getattr__(self, name):
                def call(*a):
                    made.append((getattr(raw, name), a))
                    return getattr(raw, name)(*a)
                return call
        if op == "attn":
            q = c.queries(c.B, 8).cuda()
            keep = [q, torch.zeros_like(q), c.workspace(mc.MC_OP_LAYER_ATTN)]
            args = ("mc_layer_attn", c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), q, None, None, 0, keep[1], None, keep[2])
        elif op == "evict":
            keep = [None, torch.zeros_like(c.d_lens), c.workspace(mc.MC_OP_LAYER_EVICT)]
            args = ("mc_layer_evict", c.cfg, c.batch, c.layer, mc.EvictOpts(60), keep[1], keep[2])
        else:
            J = 20 if i % 2 else 4
            keep = [c.queries(c.B, J, 8).cuda(), c.d["w"], c.workspace(mc.MC_OP_LAYER_OBSERVE, J)]
            args = ("mc_layer_observe", c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), keep[0], 0, keep[2])
        torch.cuda.synchronize()
        lib._lib = Spy()
        try:
            getattr(lib, args[0])(*args[1:], stream=s)
        finally:
            lib._lib = raw
        torch.cuda.synchronize()
        sides.append((made[-1], keep[1], keep[1].clone(), c, keep, args, s))
    refused, start = [0] * len(sides), threading.Barrier(len(sides))
    times = 20000 if op == "evict" else 2000

    def work(k):
        call, a = sides[k][0]
        start.wait()
        for _ in range(times):
            refused[k] += 1 if call(*a) else 0
    threads = [threading.Thread(target=work, args=(k,)) for k in range(len(sides))]
    was = sys.getswitchinterval()
    sys.setswitchinterval(1e-6)
    try:
        for t in threads:
            t.start()
        for t in threads:
            t.join()
    finally:
        sys.setswitchinterval(was)
    torch.cuda.synchronize()
    assert refused == [0] * len(sides)
    for _, got, alone, c, *_ in sides:
        assert torch.equal(got, alone) and c.mc.lib().mc_layer_read_status(c.layer, check=False)[1] == 0


def drawn(seed):
    import random
    r = random.Random(seed)
    nq, H = r.choice([1, 2, 4, 8]), r.choice([1, 2, 3])
    return dict(H=H, Hq=H * nq, nq=nq, ps=r.choice([16, 32, 64]), dtype=r.choice(["f16", "bf16"]), marks=r.random() < 0.5,
                lens=[r.choice([0, 1, 15, 16, 17, 63, 64, 130, 700, 1500]) for _ in range(r.randint(1, 5))] + [r.choice([33, 600, 4500])],
                cap=r.choice([0.0, 0.5, 5.0, 50.0]), alibi=r.random() < 0.4, window=r.choice([0, 0, 1, 40, 900]), prefix=r.choice([0, 0, 5]),
                doc=r.choice([0, 0, 30]), J=r.randint(1, 200 // nq if nq > 1 else 64), append=r.random() < 0.5, sm=r.choice([SM, -SM, 0.5]))


@pytest.mark.parametrize("seed", range(40))
def test_no_bit_follows_from_what_is_not_seen(L, seed):
    """Drawn shapes and options: the rows that no query of a head sees, those behind the sequences and nobody's pages change, and
    so does what the call before left behind; out, lse and weights do not."""
    o = drawn(seed)
    lens, H, Hq, ps, B, J = o["lens"], o["H"], o["Hq"], o["ps"], len(o["lens"]), o["J"]
    got = []
    for fill in (0.0, 6.0e4, float("nan"), -float("inf")):
        c = L.Cache(lens, H, Hq, ps, o["dtype"], seed=seed, marks=o["marks"], weights=True, poison=False)
        mc, lib = c.mc, c.mc.lib()
        last = [x - 1 for x in c.q_next] if o["marks"] else [n - 1 for n in lens]
        keeps = []
        for queries in (1, J):  # the step's query stands at last + 1 if its row is new; the observed ones end at last
            keep = torch.zeros(c.n_pages, H, ps, dtype=torch.bool)
            for b, n in enumerate(lens):
                t, p = torch.arange(n), c.dense_pos[b]
                at = [last[b] + (1 if o["append"] else 0)] if queries == 1 else [last[b] - j for j in range(J) if last[b] - j >= 0]
                ok = torch.zeros(n, H, dtype=torch.bool)
                for x in at:
                    ok |= L.seen(p, x, o["window"], o["doc"], o["prefix"])
                keep[c.table[b, t // ps].long(), :, t % ps] = ok
            keeps.append(keep)
        ten = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        some = lambda x: ten([x] * B) if x else None  # noqa: E731
        slopes = torch.exp2(-8.0 * torch.arange(1, Hq + 1) / Hq).cuda() if o["alibi"] else None
        opts = lambda q_pos: mc.ScoreOpts(o["sm"], softcap=o["cap"], alibi_slopes=slopes, window=o["window"], prefix_len=some(o["prefix"]),  # noqa: E731
                                          doc_start=some(o["doc"]), q_pos=ten(q_pos) if o["marks"] else None)
        q, qo, kn, vn = c.queries(B, Hq).cuda(), c.queries(B, J, Hq).cuda(), c.rows(B, H).cuda(), c.rows(B, H).cuda()
        flags = mc.MC_LAYER_ACCUMULATE | (mc.MC_LAYER_APPEND if o["append"] else 0)
        out, lse = torch.zeros_like(q), torch.zeros(B, Hq, device="cuda")
        stale = L.Cache([max(lens)] * 4, H, Hq, ps, o["dtype"], poison=False, weights=True)
        stale.d["k"].fill_(0.0 if fill != fill else fill)
        results = []
        for i in (1, 0):
            for k in ("k", "v"):
                c.d[k].copy_(torch.where(keeps[i][..., None], getattr(c, k), torch.full((), fill).to(c.dt)))
            lib.mc_layer_observe(stale.cfg, stale.batch, stale.layer, mc.ScoreOpts(o["sm"], softcap=o["cap"]), c.queries(4, J, Hq).cuda() * 30, 0,
                                 stale.workspace(mc.MC_OP_LAYER_OBSERVE, J))
            if i:
                lib.mc_layer_observe(c.cfg, c.batch, c.layer, opts(last), qo, 0, c.workspace(mc.MC_OP_LAYER_OBSERVE, J))
            else:
                lib.mc_layer_attn(c.cfg, c.batch, c.layer, opts([x + (1 if o["append"] else 0) for x in last]), q, kn if o["append"] else None,
                                  vn if o["append"] else None, flags, out, lse, c.workspace(mc.MC_OP_LAYER_ATTN, flags))
            torch.cuda.synchronize()
            results += [c.gathered("w", b, n) for b, n in enumerate(lens)]
        assert lib.mc_layer_read_status(c.layer, check=False)[1] == 0
        got.append(results + [out.cpu().view(torch.int16), lse.cpu()])
    assert not any(torch.isnan(x.float()).any() for x in got[0])
    for other in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(got[0], other))
