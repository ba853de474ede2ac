"""The operators of a 4-bit layer together, as a serving loop uses them -- prompts appended in chunks, decode steps that select
pages, attend and append --, eager and from a graph; on streams of their own; over pools past 4 GB; and what must not matter."""
import math

import numpy as np
import pytest
import torch

import test_gpu_layer_q4_attn as A
import test_gpu_layer_q4_rows as R

pytestmark = pytest.mark.gpu
SM = A.SM


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2405_14366_b200.build import build_library
    build_library()
    import q4_layer_harness
    return q4_layer_harness


@pytest.mark.parametrize("dtype,H,Hq,kw", [("f16", 2, 2, {}), ("bf16", 2, 8, dict(window=90, prefix=[33, 4, 0, 0])), ("bf16", 1, 8, dict(cap=20.0))])
def test_prompts_in_chunks_then_decode_steps(Q, dtype, H, Hq, kw):
    c = Q.Cache([0] * 4, H, Hq, dtype, seed=31, room=420, max_len=448, empty=True)
    for news in ([200, 31, 1, 0], [150, 1, 33, 64], [13, 40, 29, 1]):
        R.grow(Q, c, news, packed=True)
    masks = {k: v for k, v in kw.items() if k != "cap"}
    for step in range(34):
        q = c.queries(4, Hq)
        pages, counts = A.select(Q, c, q, 4, 1, 1, **masks)
        if step % 3 == 0:  # every page
            A.run(Q, c, q=q, append=True, check=step % 4 == 0, **kw)
        else:
            A.run(Q, c, q=q, append=True, pages=pages, counts=counts.tolist(), check=step % 4 == 0, **kw)
    assert c.same_as_host() is None and c.status()[1] == 0
    # the whole of every sequence, read back
    total = sum(c.lens)
    k, v = (torch.zeros(total, H, 128, dtype=c.dt, device="cuda") for _ in range(2))
    off = torch.tensor([0] + np.cumsum(c.lens).tolist(), dtype=torch.int32, device="cuda")
    c.mc.lib().mc_layer_q4_read(c.cfg, c.batch, c.layer, None, k, v, off)
    at = 0
    for b, n in enumerate(c.lens):
        for h in range(H):
            kc, kz, vc, vz = c.values(b, h)
            for got, want in ((k, kc + kz), (v, vc + vz)):
                d = (got[at:at + n, h].cpu().double() - want).abs()
                assert (d <= want.abs() * torch.finfo(c.dt).eps / 2 * (1 + 2.0 ** -15) + 2.0 ** -25).all()
        at += n


class Loop:
    """Decode steps over a prompt, every buffer fixed, so that a graph can hold a step."""

    def __init__(self, Q, seed=5, lens=(70, 31, 0, 250), H=2, Hq=8, dtype="bf16", steps=40):
        self.c = c = Q.Cache(list(lens), H, Hq, dtype, seed=seed, room=steps, max_len=max(lens) + steps)
        mc = self.mc = c.mc
        B = c.B
        self.q = torch.zeros(B, Hq, 128, dtype=c.dt, device="cuda")
        self.kn, self.vn = (torch.zeros(B, H, 128, dtype=c.dt, device="cuda") for _ in range(2))
        self.out, self.lse = torch.zeros_like(self.q), torch.zeros(B, Hq, device="cuda")
        self.pages, self.counts = torch.full((B, H, 5), -1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
        self.ws = torch.cat([c.workspace(mc.MC_OP_LAYER_Q4_ATTN, 1), c.workspace(mc.MC_OP_LAYER_Q4_SELECT)])
        self.opts = mc.ScoreOpts(SM, softcap=30.0, window=200)

    def step(self):
        mc, c = self.mc, self.c
        mc.lib().mc_layer_q4_select(c.cfg, c.batch, c.layer, self.opts, mc.PageSelection(5, 1, 1), self.q, self.pages, self.counts, self.ws)
        mc.lib().mc_layer_q4_attn(c.cfg, c.batch, c.layer, self.opts, self.pages, self.counts, self.q, self.kn, self.vn, mc.MC_LAYER_APPEND,
                                  self.out, self.lse, self.ws)
        c.d_lens.add_(1)

    def state(self):
        bits = lambda t: t.view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()]).clone()  # noqa: E731
        return {k: bits(v) for k, v in dict(self.c.d, lens=self.c.d_lens, out=self.out, lse=self.lse, pages=self.pages, counts=self.counts).items()}


def feed(steps, B=4, Hq=8, H=2, dt=torch.bfloat16):
    g = torch.Generator().manual_seed(77)
    return [[(torch.randn(B, n, 128, generator=g) * s).to(dt).cuda() for n, s in ((Hq, 28.0), (H, 0.1), (H, 0.1))] for _ in range(steps)]


def test_the_loop_from_a_graph_equals_the_eager_one(Q):
    tokens, ends = feed(40), []
    for graphed in (False, True):
        loop = Loop(Q)
        if graphed:
            keep = {k: v.clone() for k, v in dict(loop.c.d, lens=loop.c.d_lens).items()}
            s = torch.cuda.Stream()
            s.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(s):
                loop.step()  # warm-up; undone below
            torch.cuda.current_stream().wait_stream(s)
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph):
                loop.step()
            for k, v in keep.items():
                (loop.c.d_lens if k == "lens" else loop.c.d[k]).copy_(v)
            loop.pages.fill_(-1)
        states = []
        for t in tokens:
            for f, x in zip((loop.q, loop.kn, loop.vn), t):
                f.copy_(x)
            graph.replay() if graphed else loop.step()
            states.append(loop.state())
        torch.cuda.synchronize()
        assert loop.c.status()[1] == 0
        ends.append(states)
    for i, (x, y) in enumerate(zip(*ends)):
        for k in x:
            assert torch.equal(x[k], y[k]), (i, k)


def test_loops_on_two_streams_at_once(Q):
    """Two caches, two workspaces, two streams, nothing that orders them: each ends as it does alone."""
    tokens = feed(30)
    alone = []
    for seed in (5, 6):
        loop = Loop(Q, seed=seed)
        for t in tokens:
            for f, x in zip((loop.q, loop.kn, loop.vn), t):
                f.copy_(x)
            loop.step()
        torch.cuda.synchronize()
        alone.append(loop.state())
    loops, streams = [Loop(Q, seed=s) for s in (5, 6)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for t in tokens:
        for loop, s in zip(loops, streams):
            with torch.cuda.stream(s):
                for f, x in zip((loop.q, loop.kn, loop.vn), t):
                    f.copy_(x)
                loop.step()
    torch.cuda.synchronize()
    for loop, want in zip(loops, alone):
        got = loop.state()
        for k in want:
            assert torch.equal(got[k], want[k]), k


def test_calls_right_behind_each_other(Q):
    """Append, attend, append, read with nothing in between (each may start while the one before it drains): as with waits."""
    def go(wait):
        c = Q.Cache([40, 0, 95], 2, 4, "f16", seed=8, room=300, max_len=400)
        mc, lib = c.mc, c.mc.lib()
        g = torch.Generator().manual_seed(4)
        ws, outs = c.workspace(mc.MC_OP_LAYER_Q4_ATTN, 1), []
        for i in range(12):
            news = [(7 * i + 5 * b) % 24 for b in range(3)]
            rows = sum(news)
            k, v = ((torch.randn(max(rows, 1), 2, 128, generator=g) * 0.1).half().cuda()[:rows] for _ in range(2))
            off = torch.tensor([0] + np.cumsum(news).tolist(), dtype=torch.int32).cuda()
            add = torch.tensor(news, dtype=torch.int32).cuda()
            q = (torch.randn(3, 4, 128, generator=g) * 28).half().cuda()
            out, lse = torch.zeros_like(q), torch.zeros(3, 4, device="cuda")
            back = [torch.zeros(rows, 2, 128, dtype=torch.float16, device="cuda") for _ in range(2)]
            before = c.d_lens.clone()
            torch.cuda.synchronize()
            lib.mc_layer_q4_append(c.cfg, c.batch, c.layer, k, v, off)
            c.d_lens.add_(add)
            if wait:
                torch.cuda.synchronize()
            lib.mc_layer_q4_attn(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), None, None, q, k.new_zeros(3, 2, 128) + 0.1, k.new_zeros(3, 2, 128) + 0.2,
                                 mc.MC_LAYER_APPEND, out, lse, ws)
            c.d_lens.add_(1)
            if wait:
                torch.cuda.synchronize()
            lib.mc_layer_q4_read(c.cfg, c.batch, c.layer, before, *back, off)
            outs += [out, lse] + back
        torch.cuda.synchronize()
        assert c.status()[1] == 0
        return outs, {k: v.clone().view(torch.uint8) for k, v in c.d.items()}
    (a, x), (b, y) = go(True), go(False)
    assert all(torch.equal(p, q) for p, q in zip(a, b)) and all(torch.equal(x[k], y[k]) for k in x)


@pytest.mark.parametrize("Hq", [2, 8, 16])
def test_what_is_not_seen_has_no_say(Q, Hq):
    """Hidden pages, hidden rows of a page's values, slots behind the last row, pages of nobody, scratch: no bit of the output."""
    kw = dict(softcap=25.0, window=150, prefix_len=A.dev([20, 0, 40]), doc_start=A.dev([0, 100, 0]))
    outs = []
    for fill in range(3):
        c = Q.Cache([300, 131, 97], 2, Hq, "bf16", seed=14)
        mc = c.mc
        g = torch.Generator().manual_seed(fill)
        q, kn, vn = ((torch.randn(3, n, 128, generator=torch.Generator().manual_seed(9)) * s).bfloat16().cuda() for n, s in ((Hq, 28.0), (2, 0.1), (2, 0.1)))
        if fill:
            used = torch.zeros(c.n_pages, dtype=torch.bool)
            for b, n in enumerate(c.lens):
                lo = max(n - 149, [0, 100, 0][b])
                for s in range(n // 32):
                    t = torch.arange(32 * s, 32 * s + 32)
                    see = (t >= lo) | (t < [20, 0, 40][b])
                    page = int(c.table[b, s])
                    used[page] = see.any()
                    hide = (~see).nonzero().flatten().cuda()
                    c.d["vm"][page, :, hide] = torch.randn(2, len(hide), 4, 2, generator=g).half().cuda() * 1e4
                    c.d["vc"][page, :, hide] = torch.randint(0, 256, (2, len(hide), 64), generator=g, dtype=torch.uint8).cuda()
                    c.d["kc"][page, :, hide] = torch.randint(0, 256, (2, len(hide), 64), generator=g, dtype=torch.uint8).cuda()
                c.d["rk"][b, :, n % 32:] = float("nan") if fill == 1 else 1e4
                c.d["rv"][b, :, n % 32:] = float("nan") if fill == 1 else -1e4
            free = (~used).nonzero().flatten().cuda()
            for x in ("km", "vm"):
                c.d[x][free] = float("nan") if fill == 1 else 3.0
        ws = c.workspace(mc.MC_OP_LAYER_Q4_ATTN, 0)
        ws.fill_(0xFF if fill == 1 else 0x3C)
        out, lse = torch.zeros(3, Hq, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(3, Hq, device="cuda")
        mc.lib().mc_layer_q4_attn(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM, **kw), None, None, q, kn, vn, 0, out, lse, ws)
        torch.cuda.synchronize()
        assert c.status()[1] == 0
        outs.append((out.view(torch.int16), lse.view(torch.int32)))
    for o in outs[1:]:
        assert torch.equal(o[0], outs[0][0]) and torch.equal(o[1], outs[0][1])


def test_no_output_beyond_what_is_asked_for(Q):
    """lse is optional; out and lse are written for every sequence, an empty one's too, and nothing of the cache without a flag."""
    c = Q.Cache([0, 64, 33], 2, 4, "f16", seed=3)
    mc = c.mc
    out = torch.full((3, 4, 128), 5.0, dtype=c.dt, device="cuda")
    mc.lib().mc_layer_q4_attn(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), None, None, c.queries(3, 4).cuda(), None, None, 0, out, None,
                              c.workspace(mc.MC_OP_LAYER_Q4_ATTN, 0))
    torch.cuda.synchronize()
    assert (out[0] == 0).all() and not (out[1:] == 5).any() and c.same_as_host() is None


def test_the_readme_snippet(Q, repo_root):
    """README's loop over a 4-bit layer, as it stands there: every step against the definition over what the cache should hold."""
    import os
    import re
    with open(os.path.join(repo_root, "README.md")) as f:
        (code,) = [b for b in re.findall(r"```python\n(.*?)```", f.read(), re.S) if "LayerQ4Cache.empty(" in b]
    lens, H, Hq, n_steps = [2500, 70, 1], 2, 8, 40
    c = Q.Cache([0] * 3, H, Hq, "f16", seed=3, room=max(lens) + n_steps, max_len=2560, empty=True)
    mc, g = c.mc, c.g
    rows = [[c.rows(n + n_steps, H) for n in lens] for _ in range(2)]
    k, v = (torch.cat([x[:n] for x, n in zip(r, lens)]).cuda() for r in rows)
    off = torch.tensor([0] + np.cumsum(lens).tolist(), dtype=torch.int32, device="cuda")
    ends = [n + n_steps for n in lens]
    steps = [(c.queries(3, Hq).cuda(), *(torch.stack([x[n + i] for x, n in zip(r, lens)]).cuda() for r in rows)) for i in range(n_steps)]
    back = [torch.zeros(sum(ends), H, 128, dtype=c.dt, device="cuda") for _ in range(2)]
    space = dict(mc=mc, torch=torch, lib=mc.lib(), cfg=c.cfg, batch_size=3, n_pages=c.n_pages, block_table=c.d["table"], max_seq_len=2560, k=k, v=v,
                 offsets=off, sm_scale=SM, steps=steps, out=torch.zeros(3, Hq, 128, dtype=c.dt, device="cuda"), lse=torch.zeros(3, Hq, device="cuda"),
                 k_back=back[0], v_back=back[1], row_offsets=torch.tensor([0] + np.cumsum(ends).tolist(), dtype=torch.int32, device="cuda"))
    exec(compile(code, "README.md", "exec"), space)
    torch.cuda.synchronize()
    assert mc.lib().mc_layer_q4_read_status(space["layer"], check=False)[1] == 0 and space["seq_lens"].tolist() == ends
    at = 0
    for b, n in enumerate(lens):  # the host's cache one step before the end
        c.put(b, *(r[b][:n + n_steps - 1] for r in rows))
        c.lens[b] = n + n_steps - 1
    q, kn, vn = (x.cpu() for x in steps[-1])
    for b, n in enumerate(c.lens):
        for h in range(H):
            r = slice(4 * h, 4 * h + 4)
            want = Q.select64(c, q[b, r], b, h, 64, 1, 2, n)
            assert space["pages"][b, h, :len(want)].tolist() == want and int(space["counts"][b]) == len(want)
            o, z, tol, ztol = Q.attn64(c, b, h, q[b, r], SM, k_new=kn[b, h], v_new=vn[b, h], pages=want)
            assert ((space["out"][b, r].cpu().double() - o).abs() <= tol).all() and ((space["lse"][b, r].cpu().double() - z).abs() <= ztol).all()
            kc, kz, vc, vz = c.values(b, h)
            full = (n + 1) // 32 * 32 if (n + 1) % 32 == 0 else n // 32 * 32
            keep = min(full, n // 32 * 32)
            for got, want64 in ((back[0], kc + kz), (back[1], vc + vz)):
                d = (got[at:at + keep, h].cpu().double() - want64[:keep]).abs()
                assert (d <= want64[:keep].abs() * Q.H11 + 2.0 ** -25).all()
        at += n + 1


def test_pools_past_four_gigabytes(Q):
    """Pools of more than 2^32 bytes: the pages in use are the last ones."""
    import paper_2405_14366_b200 as mc
    H, Hq, n_pages, n = 8, 32, 270000, 150
    cfg = mc.McConfig(H, Hq, 32, "bf16")
    layer = mc.LayerQ4Cache.empty(cfg, 1, n_pages)
    assert layer.k_codes.numel() > 1 << 32
    table = torch.tensor([[n_pages - 1, n_pages - 5, n_pages - 2, n_pages - 3, n_pages - 4]], dtype=torch.int32, device="cuda")
    lens = torch.zeros(1, dtype=torch.int32, device="cuda")
    batch, lib = mc.Batch(table, lens, 160, n_pages), mc.lib()
    c = Q.Cache([n], H, Hq, "bf16", seed=2)  # the host's copy of the same rows
    k, v = c.raw[0]
    off = torch.tensor([0, n], dtype=torch.int32, device="cuda")
    lib.mc_layer_q4_append(cfg, batch, layer, k.cuda(), v.cuda(), off)
    lens.fill_(n)
    back = [torch.zeros(n, H, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lib.mc_layer_q4_read(cfg, batch, layer, None, *back, off)
    q = c.queries(1, Hq)
    opts = mc.ScoreOpts(SM, q_pos=A.dev([n - 1]))
    ws = torch.empty(max(lib.mc_layer_workspace_bytes(cfg, batch, op, 0) for op in (5, 6)), dtype=torch.uint8, device="cuda")
    pages, counts = torch.zeros(1, H, 2, dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    lib.mc_layer_q4_select(cfg, batch, layer, opts, mc.PageSelection(2), q.cuda(), pages, counts, ws)
    out = torch.zeros(1, Hq, 128, dtype=torch.bfloat16, device="cuda")
    lib.mc_layer_q4_attn(cfg, batch, layer, opts, pages, counts, q.cuda(), None, None, 0, out, None, ws)
    assert lib.mc_layer_q4_read_status(layer, check=False)[1] == 0
    for h in range(H):
        kc, kz, vc, vz = c.values(0, h)
        for got, want in ((back[0], kc + kz), (back[1], vc + vz)):
            assert ((got[:, h].cpu().double() - want).abs() <= want.abs() * 2.0 ** -8 * (1 + 2.0 ** -15)).all()
        rows = slice(4 * h, 4 * h + 4)
        want = Q.select64(c, q[0, rows], 0, h, 2, 0, 0, n - 1)
        assert pages[0, h].tolist() == want
        o, _, tol, _ = Q.attn64(c, 0, h, q[0, rows], SM, pages=want)
        assert ((out[0, rows].cpu().double() - o).abs() <= tol).all()
