"""The three operators of an uncompressed layer together, as a serving loop uses them: the prompt's weights, the first
eviction, then decode steps that attend, append, gather weights and evict -- every step against the definitions in 64
bits over the rows that the cache is supposed to hold; and the same loop replayed from a CUDA graph."""
import math

import pytest
import torch

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


class Loop:
    def __init__(self, L, lens, H, Hq, ps, dtype, budget, sink, recent, n_obs, opts_kw, steps, seed=0):
        self.c = c = L.Cache(lens, H, Hq, ps, dtype, seed=seed, marks=False, weights=True, room=max(steps, budget + 1))
        mc = c.mc
        c.d["pos"] = torch.full((c.n_pages, H, ps), -1, dtype=torch.int32, device="cuda")
        for b, n in enumerate(lens):
            t = torch.arange(n)
            c.d["pos"][c.table[b, t // ps].long().cuda(), :, (t % ps).cuda()] = t.int().cuda()[:, None].expand(n, H)
        c.layer = mc.LayerCache(c.cfg, c.d["k"], c.d["v"], c.d["pos"], c.d["w"])
        self.lens = c.d_lens.clone()
        self.new_lens = torch.zeros_like(self.lens)
        self.pos = self.lens.clone()  # the next token's position
        self.last = self.lens - 1     # the newest token's position
        self.max_len = max(max(lens), budget) + 1
        self.batch = mc.Batch(c.d["table"], self.lens, min(self.max_len, c.mp * ps), c.n_pages)
        self.score = mc.ScoreOpts(SM, q_pos=self.pos, **opts_kw)
        self.score_obs = mc.ScoreOpts(SM, q_pos=self.last, **opts_kw)
        self.evict_opts = mc.EvictOpts(budget, sink, recent, self.last)
        self.budget, self.sink, self.recent, self.n_obs = budget, sink, recent, n_obs
        need = [c.mc.lib().mc_layer_workspace_bytes(c.cfg, self.batch, op, arg)
                for op, arg in ((mc.MC_OP_LAYER_ATTN, 3), (mc.MC_OP_LAYER_OBSERVE, n_obs), (mc.MC_OP_LAYER_EVICT, 0))]
        self.ws = torch.full((max(need),), 0xFF, dtype=torch.uint8, device="cuda")  # one workspace for all: the calls follow each other
        self.q = torch.zeros(c.B, Hq, 128, dtype=c.dt, device="cuda")
        self.kn, self.vn = (torch.zeros(c.B, H, 128, dtype=c.dt, device="cuda") for _ in range(2))
        self.out, self.lse = torch.zeros_like(self.q), torch.zeros(c.B, Hq, device="cuda")

    def observe(self, q):
        self.c.mc.lib().mc_layer_observe(self.c.cfg, self.batch, self.c.layer, self.score_obs, q, 0, self.ws)

    def evict(self):
        self.c.mc.lib().mc_layer_evict(self.c.cfg, self.batch, self.c.layer, self.evict_opts, self.new_lens, self.ws)
        self.lens.copy_(self.new_lens)

    def attend(self):
        mc = self.c.mc
        mc.lib().mc_layer_attn(self.c.cfg, self.batch, self.c.layer, self.score, self.q, self.kn, self.vn,
                               mc.MC_LAYER_APPEND | mc.MC_LAYER_ACCUMULATE, self.out, self.lse, self.ws)
        self.lens.add_(1)

    def step(self):
        self.attend()
        self.last.copy_(self.pos)
        self.pos.add_(1)
        self.evict()

    def state(self):
        """Per sequence: rows, positions and weights of the tokens the cache holds, [n][H]..."""
        c, got = self.c, []
        host = {k: c.d[k].cpu() for k in ("k", "v", "pos", "w")}
        for b, n in enumerate(self.lens.tolist()):
            t = torch.arange(n)
            pg = c.table[b, t // c.ps].long()
            got.append({k: host[k][pg, :, t % c.ps] for k in host})
        return got


def check_evicted(loop, before, after, last):
    """`after` is what the rule makes of `before`, slot by slot."""
    for b, (x, y) in enumerate(zip(before, after)):
        n = x["w"].shape[0]
        keep_n = min(n, loop.budget)
        assert y["w"].shape[0] == keep_n
        for h in range(loop.c.H):
            w, p = x["w"][:, h].tolist(), x["pos"][:, h].tolist()
            rank = sorted(range(n), key=lambda i: (not (p[i] < loop.sink or p[i] > last[b] - loop.recent), -w[i], i))
            keep = sorted(rank[:keep_n])
            slots = [i if i in set(keep) else -1 for i in range(keep_n)]
            movers = iter(i for i in keep if i >= keep_n)
            src = torch.tensor([i if i >= 0 else next(movers) for i in slots], dtype=torch.long)
            for k in ("k", "v", "pos", "w"):
                assert torch.equal(y[k][:, h], x[k][src, h]), (b, h, k)


@pytest.mark.parametrize("dtype,ps,opts", [("f16", 16, {}), ("bf16", 32, dict(softcap=20.0)), ("bf16", 16, dict(alibi=True)), ("f16", 64, dict(window=48))])
def test_prompt_eviction_and_decode(L, dtype, ps, opts):
    lens, H, Hq, budget, sink, recent, J, steps = [300, 41, 1, 129], 2, 8, 64, 4, 16, 16, 30
    nq = Hq // H
    slopes = torch.exp2(-8.0 * torch.arange(1, Hq + 1).double() / Hq).float() if opts.pop("alibi", False) else None
    kw = dict(opts, alibi_slopes=None if slopes is None else slopes.cuda())
    loop = Loop(L, lens, H, Hq, ps, dtype, budget, sink, recent, J, kw, steps)
    c = loop.c
    cap, window = opts.get("softcap", 0.0), opts.get("window", 0)
    qo = c.queries(c.B, J, Hq)
    loop.observe(qo.cuda())
    st = loop.state()
    for b, n in enumerate(lens):
        for h in range(H):
            at = (n - J + torch.arange(J)).repeat_interleave(nq)[:, None]
            pos = torch.arange(n)[None]
            s, err = L.scores64(qo[b, :, h * nq:(h + 1) * nq].reshape(-1, 128), c.dense_k[b][:, h], pos, at, SM, cap,
                                slopes[h * nq:(h + 1) * nq].repeat(J) if slopes is not None else 0.0)
            p, _, rel = L.softmax64(s, err, L.seen(pos.expand_as(s), at, window) & (at >= 0))
            tol = (p * (rel[:, None] + 64 * L.U32)).sum(0) + 1e-30
            assert ((st[b]["w"][:, h].double() - p.sum(0)).abs() <= tol).all()
    loop.evict()
    after = loop.state()
    check_evicted(loop, st, after, [n - 1 for n in lens])
    rows_k = [dict(enumerate(c.dense_k[b])) for b in range(c.B)]  # position -> [H][128]
    rows_v = [dict(enumerate(c.dense_v[b])) for b in range(c.B)]
    for step in range(steps):
        q, kn, vn = c.queries(c.B, Hq), c.rows(c.B, H), c.rows(c.B, H)
        loop.q.copy_(q)
        loop.kn.copy_(kn)
        loop.vn.copy_(vn)
        held, pos0 = loop.state(), loop.pos.tolist()
        loop.attend()
        mid = loop.state()
        for b in range(c.B):
            rows_k[b][pos0[b]], rows_v[b][pos0[b]] = kn[b], vn[b]
            x = mid[b]
            for h in range(H):
                ps_ = x["pos"][:, h].tolist()
                assert len(set(ps_)) == len(ps_) and ps_[-1] == pos0[b]
                k = torch.stack([rows_k[b][i][h] for i in ps_])
                v = torch.stack([rows_v[b][i][h] for i in ps_])
                assert torch.equal(k, x["k"][:, h]) and torch.equal(v, x["v"][:, h])  # the rows are the ones of their positions
                rows = slice(h * nq, (h + 1) * nq)
                pt = torch.tensor(ps_)
                s, err = L.scores64(q[b, rows], k, pt, pos0[b], SM, cap, slopes[rows] if slopes is not None else 0.0)
                p, lse, rel = L.softmax64(s, err, L.seen(pt, pos0[b], window)[None].expand_as(s))
                a, half = p @ v.double().abs(), L.eps_half(c.dt)
                o = p @ v.double()
                tol = half * a * (1 + half) + half * (o.abs() + a * rel[:, None]) + a * rel[:, None] + \
                    (2.0 ** -25 * (v.double().abs().sum(0)[None] + 1) if c.dt == torch.float16 else 0.0) + 1e-30
                assert ((loop.out[b, rows].cpu().double() - o).abs() <= tol).all(), (step, b, h)
                assert ((loop.lse[b, rows].cpu().double() - lse).abs() <= rel + 4 * L.U32 * (1 + lse.abs())).all()
                w0 = torch.cat([held[b]["w"][:, h].double(), torch.zeros(1, dtype=torch.float64)])
                want = w0 + p.sum(0)
                assert ((x["w"][:, h].double() - want).abs() <= (p * rel[:, None]).sum(0) + 4 * L.U32 * want + 1e-30).all()
        loop.last.copy_(loop.pos)
        loop.pos.add_(1)
        loop.evict()
        check_evicted(loop, mid, loop.state(), pos0)
    words, code = c.mc.lib().mc_layer_read_status(c.layer, check=False)
    assert code == 0, words


def test_the_loop_from_a_graph_equals_the_eager_one(L):
    args = ([200, 64, 7], 2, 8, 16, "bf16", 64, 4, 16, 8, {}, 24)
    g = torch.Generator().manual_seed(9)
    tok = [[(torch.randn(3, n, 128, generator=g) * s).to(torch.bfloat16).cuda() for n, s in ((8, 28.0), (2, 0.1), (2, 0.1))] for _ in range(20)]
    qo = (torch.randn(3, 8, 8, 128, generator=g) * 28).to(torch.bfloat16).cuda()
    ends = []
    for graphed in (False, True):
        loop = Loop(L, *args)
        loop.observe(qo)
        loop.evict()
        feed = [torch.zeros_like(x) for x in tok[0]]
        outs = []

        def one():
            loop.q.copy_(feed[0])
            loop.kn.copy_(feed[1])
            loop.vn.copy_(feed[2])
            loop.step()
        if graphed:
            keep = {k: v.clone() for k, v in dict(loop.c.d, lens=loop.lens, pos_=loop.pos, last=loop.last).items()}
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                one()  # warm-up; undone below
            torch.cuda.current_stream().wait_stream(s)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                one()
            for k, v in keep.items():
                {"lens": loop.lens, "pos_": loop.pos, "last": loop.last}.get(k, loop.c.d.get(k)).copy_(v)
        for t in tok:
            for f, x in zip(feed, t):
                f.copy_(x)
            graph.replay() if graphed else one()
            outs.append(loop.out.clone())
        torch.cuda.synchronize()
        bits = {k: v.clone().view({2: torch.int16, 4: torch.int32}[v.element_size()]) for k, v in loop.c.d.items() if k != "table"}
        ends.append((outs, bits, loop.lens.tolist()))
        words, code = loop.c.mc.lib().mc_layer_read_status(loop.c.layer, check=False)
        assert code == 0, words
    assert ends[0][2] == ends[1][2]
    assert all(torch.equal(a, b) for a, b in zip(ends[0][0], ends[1][0]))
    for k in ends[0][1]:
        assert torch.equal(ends[0][1][k], ends[1][1][k]), k


def test_rows_past_four_gigabytes(L):
    """Pools of more than 2^32 bytes: the pages in use are the last ones."""
    import paper_2405_14366_b200 as mc
    H, ps, n_pages, n = 8, 64, 34000, 150  # 8 * 64 * 256 bytes per page: 4.46 GB
    k, v = (torch.zeros(n_pages, H, ps, 128, dtype=torch.float16, device="cuda") for _ in range(2))
    pos, w = torch.zeros(n_pages, H, ps, dtype=torch.int32, device="cuda"), torch.zeros(n_pages, H, ps, device="cuda")
    g = torch.Generator().manual_seed(3)
    kd, vd = (torch.randn(n, H, 128, generator=g).half() * 0.1 for _ in range(2))
    table = torch.tensor([[n_pages - 1, n_pages - 3, n_pages - 2]], dtype=torch.int32)
    t = torch.arange(n)
    for x, pool in ((kd, k), (vd, v), (t.int()[:, None].expand(n, H), pos)):
        pool[table[0, t // ps].long().cuda(), :, (t % ps).cuda()] = x.cuda().to(pool.dtype)
    cfg, lens = mc.McConfig(H, H, ps, "f16"), torch.tensor([n], dtype=torch.int32, device="cuda")
    batch, layer, lib = mc.Batch(table.cuda(), lens, n, n_pages), mc.LayerCache(cfg, k, v, pos, w), mc.lib()
    q, kn, vn = ((torch.randn(1, H, 128, generator=g) * s).half() for s in (28.0, 0.1, 0.1))
    qo = (torch.randn(1, 4, H, 128, generator=g) * 28).half()
    out, new = torch.zeros(1, H, 128, dtype=torch.float16, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = [torch.empty(lib.mc_layer_workspace_bytes(cfg, batch, op, a), dtype=torch.uint8, device="cuda") for op, a in ((2, 3), (3, 4), (4, 0))]
    lib.mc_layer_observe(cfg, batch, layer, mc.ScoreOpts(SM), qo.cuda(), 0, ws[1])
    lib.mc_layer_attn(cfg, batch, layer, mc.ScoreOpts(SM), q.cuda(), kn.cuda(), vn.cuda(), 3, out, None, ws[0])
    got = w[table[0, t // ps].long().cuda(), :, (t % ps).cuda()].cpu().double()
    for h in range(H):
        kk, vv = torch.cat([kd[:, h], kn[0, h][None]]).double(), torch.cat([vd[:, h], vn[0, h][None]]).double()
        p = torch.softmax(q[0, h].double() @ kk.T * SM, 0)
        assert ((out[0, h].cpu().double() - p @ vv).abs() <= 3 * 2.0 ** -11 * (p @ vv.abs()) + 1e-5).all()
        s = qo[0, :, h].double() @ kd[:, h].double().T * SM
        s = s.masked_fill(t[None] > n - 4 + torch.arange(4)[:, None], -math.inf)
        want = torch.softmax(s, 1).sum(0) + p[:n]
        assert ((got[:, h] - want).abs() <= 1e-5 * want + 1e-12).all()
    lib.mc_layer_evict(cfg, batch, layer, mc.EvictOpts(100, 0, 8), new, ws[2])
    words, code = lib.mc_layer_read_status(layer, check=False)
    assert code == 0 and new.item() == 100, words
    u = torch.arange(100)
    kept_pos = pos[table[0, u // ps].long().cuda(), :, (u % ps).cuda()].cpu().long()
    kept_k = k[table[0, u // ps].long().cuda(), :, (u % ps).cuda()].cpu()
    for h in range(H):
        assert torch.equal(kept_k[:, h], kd[kept_pos[:, h], h])
        order = sorted(range(n), key=lambda i: (i <= n - 1 - 8, -got[i, h].item(), i))[:100]
        assert set(kept_pos[:, h].tolist()) == set(order)


@pytest.mark.parametrize("graph", [False, True])
def test_new_lengths_passed_straight_on(L, graph):
    """The eviction's new lengths as the lengths of the next calls, two buffers in turn, without a kernel between: the same
    bits as with the device idle after every call."""
    lens, budget, steps = [700, 90, 1300], 64, 6
    got = []
    for wait in (True, False):
        c = L.Cache(lens, 4, 16, 16, "bf16", seed=21, marks=True, weights=True, poison=False)
        mc, lib = c.mc, c.mc.lib()
        pos = torch.tensor(c.q_next, dtype=torch.int32, device="cuda")
        bufs = [c.d_lens.clone(), torch.zeros_like(c.d_lens)]
        batches = [mc.Batch(c.d["table"], x, c.max_len, c.n_pages) for x in bufs]
        ws = torch.zeros(max(lib.mc_layer_workspace_bytes(c.cfg, c.batch, op, arg)
                             for op, arg in ((mc.MC_OP_LAYER_ATTN, 2), (mc.MC_OP_LAYER_OBSERVE, 8), (mc.MC_OP_LAYER_EVICT, 0))),
                         dtype=torch.uint8, device="cuda")
        q, q_obs = c.queries(3, 16).cuda(), c.queries(3, 8, 16).cuda()
        outs = [torch.zeros_like(q) for _ in range(steps)]
        score, less = mc.ScoreOpts(SM, q_pos=pos), [mc.EvictOpts(budget * (steps - i), 2, 8, pos) for i in range(steps)]

        def run(pause):
            for i in range(steps):
                now, then = batches[i % 2], batches[1 - i % 2]
                lib.mc_layer_evict(c.cfg, now, c.layer, less[i], bufs[1 - i % 2], ws)
                pause()
                lib.mc_layer_attn(c.cfg, then, c.layer, score, q, None, None, mc.MC_LAYER_ACCUMULATE, outs[i], None, ws)
                pause()
                lib.mc_layer_observe(c.cfg, then, c.layer, score, q_obs, mc.MC_LAYER_ACCUMULATE, ws)
                pause()
        torch.cuda.synchronize()
        if wait or not graph:
            run(torch.cuda.synchronize if wait else lambda: None)
        else:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                run(lambda: None)
            g.replay()
        torch.cuda.synchronize()
        assert bufs[0].tolist() == [budget] * 3
        got.append((torch.stack(outs), c.gathered("w", 0, budget), c.gathered("pos", 2, budget)))
        assert lib.mc_layer_read_status(c.layer, check=False)[1] == 0
    assert all(torch.equal(a, b) for a, b in zip(*got)) and torch.isfinite(got[0][0].float()).all()


@pytest.mark.parametrize("shift", [4, 12, 16])
def test_positions_and_weights_inside_one_allocation(L, shift):
    """Positions and weights that begin 16, 48 and 64 bytes into their storage: the bits of those that begin at a pool's own."""
    got = []
    for off in (0, shift):
        c = L.Cache([300, 77, 130], 1, 4, 16, "bf16", seed=31, marks=True, weights=True)
        mc, lib = c.mc, c.mc.lib()
        pos, w = (torch.zeros(c.d[k].numel() + off, dtype=c.d[k].dtype, device="cuda")[off:].view(c.d[k].shape) for k in ("pos", "w"))
        pos.copy_(c.d["pos"])
        w.copy_(c.d["w"])
        layer = mc.LayerCache(c.cfg, c.d["k"], c.d["v"], pos, w)
        q_pos = torch.tensor(c.q_next, dtype=torch.int32, device="cuda")
        q, q_obs, kn, vn = c.queries(3, 4).cuda(), c.queries(3, 8, 4).cuda(), c.rows(3, 1).cuda(), c.rows(3, 1).cuda()
        flags = mc.MC_LAYER_APPEND | mc.MC_LAYER_ACCUMULATE
        ws = torch.zeros(max(lib.mc_layer_workspace_bytes(c.cfg, c.batch, op, arg)
                             for op, arg in ((mc.MC_OP_LAYER_ATTN, flags), (mc.MC_OP_LAYER_OBSERVE, 8), (mc.MC_OP_LAYER_EVICT, 0))),
                         dtype=torch.uint8, device="cuda")
        out, new = torch.empty_like(q), torch.zeros_like(c.d_lens)
        lib.mc_layer_observe(c.cfg, c.batch, layer, mc.ScoreOpts(SM, q_pos=q_pos - 1), q_obs, 0, ws)
        lib.mc_layer_attn(c.cfg, c.batch, layer, mc.ScoreOpts(SM, q_pos=q_pos, window=90), q, kn, vn, flags, out, None, ws)
        lib.mc_layer_evict(c.cfg, c.batch, layer, mc.EvictOpts(64, 2, 8, q_pos), new, ws)
        torch.cuda.synchronize()
        assert lib.mc_layer_read_status(layer, check=False)[1] == 0
        held = [x.cpu()[c.table[b, :4].long()] for b in range(3) for x in (pos, w)]
        got.append([out.cpu(), new.cpu()] + held + [c.gathered("k", b, 64) for b in range(3)])
    for a, b in zip(*got):
        assert torch.equal(a.float().nan_to_num(7.0), b.float().nan_to_num(7.0))
    assert torch.isfinite(got[0][0].float()).all()
