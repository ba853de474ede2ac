"""mc_layer_evict against a sort: which rows stay, where they move, and that nothing else changes."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def L():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2405_14366_b200.build import build_library
    build_library()
    import layer_harness
    return layer_harness


def weights_of(kind, shape, g):
    if kind == "tail":
        return torch.exp(2 * torch.randn(shape, generator=g))
    if kind == "ties":
        return torch.randint(0, 4, shape, generator=g).float() / 4
    if kind == "equal":
        return torch.full(shape, 0.25)
    if kind == "signed zeros":
        return torch.randint(0, 2, shape, generator=g).float() * -0.0 + 0.0 * torch.rand(shape, generator=g)
    special = torch.tensor([float("nan"), float("inf"), -float("inf"), -0.0, 0.0, 1e-45, -1.5, 3.4e38])
    return special[torch.randint(0, 8, shape, generator=g)]


def run(L, lens, budget, sink=0, recent=0, H=2, Hq=2, ps=16, dtype="f16", marks=True, kind="tail", seed=0, q_pos=False, stream=None, max_len=None):
    c = L.Cache(lens, H, Hq, ps, dtype, seed=seed, marks=True, weights=True, max_len=max_len)
    mc, lib, B = c.mc, c.mc.lib(), c.B
    if not marks:  # never evicted from: index order
        for b, n in enumerate(c.lens):
            t = torch.arange(n)
            c.pos[c.table[b, t // ps].long(), :, t % ps] = t[:, None].expand(n, H).int()
        c.d["pos"].copy_(c.pos)
    c.w.copy_(weights_of(kind, c.w.shape, c.g))
    c.d["w"].copy_(c.w)
    last = [x - 1 for x in c.q_next] if marks or q_pos else [n - 1 for n in c.lens]
    qp = torch.tensor(last, dtype=torch.int32, device="cuda") if marks or q_pos else None
    new = torch.full((B,), -9, dtype=torch.int32, device="cuda")
    ws = c.workspace(mc.MC_OP_LAYER_EVICT)
    torch.cuda.synchronize()
    lib.mc_layer_evict(c.cfg, c.batch, c.layer, mc.EvictOpts(budget, sink, recent, qp), new, ws, stream=stream)
    torch.cuda.synchronize()
    words, code = lib.mc_layer_read_status(c.layer, check=False)
    assert code == 0, words
    assert new.tolist() == [min(n, budget) for n in c.lens]
    want = {k: getattr(c, k).clone() for k in ("k", "v", "pos", "w")}
    for b, n in enumerate(c.lens):
        if n <= budget:
            continue
        t = torch.arange(n)
        pg, sl = c.table[b, t // ps].long(), t % ps
        for h in range(H):
            w, p = c.w[pg, h, sl].tolist(), c.pos[pg, h, sl].tolist()

            def rank(i):
                nan = w[i] != w[i]
                return (not (p[i] < sink or p[i] > last[b] - recent), nan, 0.0 if nan else -w[i], i)
            keep = set(sorted(range(n), key=rank)[:budget])
            holes = [i for i in range(budget) if i not in keep]
            movers = [i for i in range(budget, n) if i in keep]
            assert len(holes) == len(movers)
            hi, mi = torch.tensor(holes, dtype=torch.long), torch.tensor(movers, dtype=torch.long)
            for k, pool in want.items():
                pool[pg[hi], h, sl[hi]] = getattr(c, k)[pg[mi], h, sl[mi]]
    for k, pool in want.items():
        as_int = {torch.float16: torch.int16, torch.bfloat16: torch.int16, torch.float32: torch.int32, torch.int32: torch.int32}[pool.dtype]
        assert torch.equal(c.d[k].cpu().view(as_int), pool.view(as_int)), k
    return c


KINDS = ["tail", "ties", "equal", "signed zeros", "special"]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("H,ps,dtype", [(1, 16, "f16"), (3, 32, "bf16"), (40, 64, "f16")])
def test_lengths(L, kind, H, ps, dtype):
    run(L, [1, 0, 2, 33, 100, 129, 257], 32, H=H, Hq=H, ps=ps, dtype=dtype, kind=kind)
    run(L, [100, 129, 257, 256, 7], 100, 4, 20, H=H, Hq=H, ps=ps, dtype=dtype, kind=kind, marks=False)


@pytest.mark.parametrize("budget,sink,recent", [(1, 0, 0), (1, 1, 0), (1, 0, 1), (50, 50, 0), (50, 0, 50), (50, 20, 30), (999, 0, 0), (998, 4, 64),
                                                (2 ** 31 - 1, 0, 0)])
@pytest.mark.parametrize("kind", ["tail", "ties", "special"])
def test_budgets(L, budget, sink, recent, kind):
    run(L, [1000, 999, 64], budget, sink, recent, kind=kind)
    run(L, [1000, 999, 64], budget, sink, recent, kind=kind, marks=False, ps=64)


@pytest.mark.parametrize("n", [2047, 2049, 4097, 8200, 20000])
def test_clusters(L, n):
    run(L, [n, 5, n // 2], n // 3, 4, 100, kind="tail")
    run(L, [n, 5, n // 2], n - 1, 4, 100, kind="ties", ps=32)
    run(L, [n], n // 2, kind="equal")


def test_shares_longer_than_shared_memory(L):
    run(L, [330000], 1000, 4, 64, H=1, Hq=1, ps=64, kind="ties")
    run(L, [100, 3000], 64, H=1, Hq=1, max_len=400000)


def test_other_streams_and_a_second_eviction(L):
    run(L, [700, 300], 128, 4, 16, stream=torch.cuda.Stream())
    c = run(L, [700, 300], 128, 4, 16)
    mc, lib = c.mc, c.mc.lib()
    new, again = torch.tensor([128, 128], dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    before = {k: v.clone() for k, v in c.d.items() if v is not None}
    lib.mc_layer_evict(c.cfg, mc.Batch(c.d["table"], new, 700, c.n_pages), c.layer, mc.EvictOpts(128, 4, 16), again, c.workspace(mc.MC_OP_LAYER_EVICT))
    torch.cuda.synchronize()
    assert again.tolist() == [128, 128]
    for k, v in before.items():
        as_int = {2: torch.int16, 4: torch.int32}[v.element_size()]
        assert torch.equal(v.view(as_int), c.d[k].view(as_int))


def test_bad_pages_and_lengths_are_flagged(L):
    c = L.Cache([300, 200], 2, 2, 16, "f16", marks=True, weights=True)
    mc, lib = c.mc, c.mc.lib()
    new, ws = torch.zeros(2, dtype=torch.int32, device="cuda"), c.workspace(mc.MC_OP_LAYER_EVICT)
    c.d["table"][0, 1], c.d["table"][0, 18] = -1, 10 ** 6
    lib.mc_layer_evict(c.cfg, c.batch, c.layer, mc.EvictOpts(64), new, ws)
    words, code = lib.mc_layer_read_status(c.layer, check=False)
    assert code == 8 and words[0] == 4 and new.tolist() == [64, 64]
    c.layer.status.zero_()
    c.d["table"].copy_(c.table)
    c.d_lens.copy_(torch.tensor([301, -5]))
    lib.mc_layer_evict(c.cfg, c.batch, c.layer, mc.EvictOpts(64), new, ws)
    words, code = lib.mc_layer_read_status(c.layer, check=False)
    assert code == 8 and words[0] == 4 and new.tolist() == [64, 0]
