"""Calls of a 4-bit layer with nothing at all between them in the stream, so that each starts while the one before it drains: every
length, offset and row is made ahead of the first call, and a wait at the head of the stream lets the host get ahead of the device."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

SM = 1.0 / math.sqrt(128.0)


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2405_14366_b200.build import build_library
    build_library()
    import q4_layer_harness
    return q4_layer_harness


class Steps:
    """Several layers, several steps: append, attend and append, select, attend the selected pages, read back; a layer's output is
    the next layer's query, and all share one workspace."""

    def __init__(self, Q, dtype, H, Hq, lens, layers=3, steps=5, seed=50):
        self.caches = [Q.Cache(lens, H, Hq, dtype, seed=seed + i, room=40 * steps, max_len=max(lens) + 40 * steps) for i in range(layers)]
        c = self.caches[0]
        mc, B, dt = c.mc, c.B, c.dt
        g = torch.Generator().manual_seed(seed)
        i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
        rows = lambda n, s: (torch.randn(n, H, 128, generator=g) * s).to(dt).cuda()  # noqa: E731
        self.opts = [mc.ScoreOpts(SM), mc.ScoreOpts(SM, softcap=30.0, window=150, prefix_len=i32([5] * B))]
        self.ws = torch.full((max(c.workspace(mc.MC_OP_LAYER_Q4_ATTN, 1).numel(), c.workspace(mc.MC_OP_LAYER_Q4_SELECT).numel()),), 0xFF,
                             dtype=torch.uint8, device="cuda")
        self.calls, self.results = [], []
        lib, now = mc.lib(), list(lens)
        q = (torch.randn(B, Hq, 128, generator=g) * 28).to(dt).cuda()
        for step in range(steps):
            news = [(11 * step + 7 * b + 3) % 38 for b in range(B)]
            off, at = i32([0] + np.cumsum(news).tolist()), [i32(now), i32([n + m for n, m in zip(now, news)]), i32([n + m + 1 for n, m in zip(now, news)])]
            back_off = i32([0] + np.cumsum([m + 1 for m in news]).tolist())
            now = [n + m + 1 for n, m in zip(now, news)]
            for c in self.caches:
                before, middle, after = (mc.Batch(c.d["table"], n, c.max_len, c.n_pages) for n in at)
                k, v, kn, vn = rows(sum(news), 0.1), rows(sum(news), 0.1), rows(B, 0.1), rows(B, 0.1)
                out = [torch.full_like(q, 7.0) for _ in range(2)]
                lse = [torch.zeros(B, Hq, device="cuda") for _ in range(2)]
                pages, counts = torch.full((B, H, 4), -1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
                back = [torch.zeros(sum(news) + B, H, 128, dtype=dt, device="cuda") for _ in range(2)]
                # (defaults: what a call takes is fixed here)
                self.calls += [
                    lambda c=c, b=before, k=k, v=v, off=off: lib.mc_layer_q4_append(c.cfg, b, c.layer, k, v, off),
                    lambda c=c, b=middle, q=q, kn=kn, vn=vn, o=out[0], z=lse[0], s=step: lib.mc_layer_q4_attn(
                        c.cfg, b, c.layer, self.opts[s % 2], None, None, q, kn, vn, mc.MC_LAYER_APPEND, o, z, self.ws),
                    lambda c=c, b=after, q=out[0], p=pages, n=counts: lib.mc_layer_q4_select(c.cfg, b, c.layer, self.opts[0], mc.PageSelection(4, 1, 1), q, p, n, self.ws),
                    lambda c=c, b=after, q=out[0], p=pages, n=counts, o=out[1], z=lse[1]: lib.mc_layer_q4_attn(
                        c.cfg, b, c.layer, self.opts[0], p, n, q, None, None, 0, o, z, self.ws),
                    lambda c=c, b=after, f=at[0], back=back, off=back_off: lib.mc_layer_q4_read(c.cfg, b, c.layer, f, *back, off)]
                self.results += out + lse + [pages, counts] + back
                q = out[1]

    def state(self):
        torch.cuda.synchronize()
        assert all(c.status()[1] == 0 for c in self.caches)
        return [t.view(torch.uint8).clone() for t in self.results + [x for c in self.caches for x in c.d.values()]]


def run(Q, how, *args):
    s = Steps(Q, *args)
    torch.cuda.synchronize()
    if how == "graph":
        stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            for call in s.calls:
                call()
        graph.replay()
    else:
        if how == "queued":
            torch.cuda._sleep(40_000_000)  # about 20 ms: the host is through before the first call starts
        for call in s.calls:
            call()
            if how == "waits":
                torch.cuda.synchronize()
    return s.state()


@pytest.mark.parametrize("dtype,H,Hq,lens", [("f16", 2, 4, [40, 0, 95, 300]), ("bf16", 4, 32, [31, 700, 64, 5, 130, 0]), ("f16", 32, 32, [2000, 33])])
def test_nothing_between_the_calls(Q, dtype, H, Hq, lens):
    want = run(Q, "waits", dtype, H, Hq, lens)
    for how in ("queued", "graph", "queued"):
        got = run(Q, how, dtype, H, Hq, lens)
        assert len(got) == len(want)
        for i, (x, y) in enumerate(zip(got, want)):
            assert torch.equal(x, y), (how, i)
