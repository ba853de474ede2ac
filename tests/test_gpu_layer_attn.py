"""mc_layer_attn against the definition in 64 bits: masks, caps, biases, positions, the appended row, gathered weights."""
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


def run(L, lens, H=2, Hq=4, ps=16, dtype="f16", new=True, append=False, acc=False, marks=False, cap=0.0, alibi=False, window=0,
        docs=None, prefixes=None, q_pos=None, sm=SM, seed=0, lse=True, max_len=None, stream=None):
    c = L.Cache(lens, H, Hq, ps, dtype, seed=seed, marks=marks, weights=acc or append, max_len=max_len)
    mc, lib, B = c.mc, c.mc.lib(), c.B
    q = c.queries(B, Hq)
    kn, vn = (c.rows(B, H), c.rows(B, H)) if new else (None, None)
    if q_pos is None and marks:
        q_pos = [x if new else x - 1 for x in c.q_next]
    slopes = torch.exp2(-8.0 * torch.arange(1, Hq + 1).double() / Hq).float() if alibi else None
    ten = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    opts = mc.ScoreOpts(sm, softcap=cap, alibi_slopes=None if slopes is None else slopes.cuda(), window=window, doc_start=ten(docs),
                        prefix_len=ten(prefixes), q_pos=ten(q_pos))
    flags = (mc.MC_LAYER_APPEND if append else 0) | (mc.MC_LAYER_ACCUMULATE if acc else 0)
    out = torch.full((B, Hq, 128), float("nan"), dtype=c.dt, device="cuda")
    z = torch.full((B, Hq), float("nan"), device="cuda") if lse else None
    before = {k: None if v is None else v.clone() for k, v in c.d.items()}
    ws = c.workspace(mc.MC_OP_LAYER_ATTN, flags)
    dq, dk, dv = q.cuda(), None if kn is None else kn.cuda(), None if vn is None else vn.cuda()
    torch.cuda.synchronize()
    lib.mc_layer_attn(c.cfg, c.batch, c.layer, opts, dq, dk, dv, flags, out, z, ws, stream=stream)
    torch.cuda.synchronize()
    words, code = lib.mc_layer_read_status(c.layer, check=False)
    assert code == 0, words
    worst = 0.0
    expect = {k: None if v is None else v.cpu().clone() for k, v in before.items()}
    w_tol = torch.zeros(c.n_pages, H, ps, dtype=torch.float64)
    w64 = None if expect["w"] is None else expect["w"].double()
    for b, n in enumerate(c.lens):
        if append:
            pg = int(c.table[b, n // ps])
            expect["k"][pg, :, n % ps], expect["v"][pg, :, n % ps] = kn[b], vn[b]
            if marks:
                expect["pos"][pg, :, n % ps] = q_pos[b]
            w64[pg, :, n % ps] = 0.0
        for h in range(H):
            rows = slice(h * c.nq, (h + 1) * c.nq)
            o, l, p, tol, ltol, ptol = L.attn64(c, b, h, q[b, rows], sm, k_new=kn[b, h] if new else None,
                                                v_new=vn[b, h] if new else None, cap=cap, slopes=slopes, window=window,
                                                doc=docs[b] if docs else 0, prefix=prefixes[b] if prefixes else 0,
                                                q_pos=q_pos[b] if q_pos else None)
            got = out[b, rows].double().cpu()
            ratio = ((got - o).abs() / tol).max().item()
            assert ratio <= 1.0, (b, h, n, ratio)
            worst = max(worst, ratio)
            if lse:
                gl = z[b, rows].double().cpu()
                assert torch.equal(torch.isinf(gl), torch.isinf(l)) and (gl[torch.isinf(l)] < 0).all()
                fin = ~torch.isinf(l)
                assert ((gl - l).abs()[fin] <= ltol[fin]).all(), (b, h)
            if acc:
                m = len(p) if append or not new else len(p) - 1
                t = torch.arange(m)
                pg = c.table[b, t // ps].long()
                w64[pg, h, t % ps] += p[:m]
                w_tol[pg, h, t % ps] = ptol[:m] + 2 * L.U32 * w64[pg, h, t % ps] + 1e-30
    for name in ("k", "v", "pos"):
        if expect[name] is not None:  # bit for bit, NaN rows too
            bits = {torch.float16: torch.int16, torch.bfloat16: torch.int16, torch.int32: torch.int32}[expect[name].dtype]
            assert torch.equal(c.d[name].cpu().view(bits), expect[name].view(bits)), name
    if w64 is not None:
        assert ((c.d["w"].double().cpu() - w64).abs() <= w_tol).all()
    return c, out, z


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("H,Hq,ps", [(1, 1, 16), (2, 4, 16), (3, 12, 32), (2, 16, 64), (40, 40, 16)])
def test_plain_lengths(L, H, Hq, ps, dtype):
    run(L, [1, 0, 15, 16, 17, 128, 300], H=H, Hq=Hq, ps=ps, dtype=dtype)
    run(L, [1, 0, 31, 127, 129, 256], H=H, Hq=Hq, ps=ps, dtype=dtype, new=False, seed=3)


@pytest.mark.parametrize("lens", [[0], [1], [127], [128], [5000], [0, 0, 0], [4000, 3, 0, 129, 1]])
@pytest.mark.parametrize("marks", [False, True])
def test_append_and_gather(L, lens, marks):
    run(L, lens, H=2, Hq=8, ps=32, dtype="bf16", append=True, acc=True, marks=marks)
    run(L, lens, H=2, Hq=2, ps=16, dtype="f16", append=True, marks=marks, lse=False)
    run(L, lens, H=2, Hq=4, ps=16, dtype="f16", acc=True, marks=marks, new=False)
    run(L, lens, H=1, Hq=8, ps=64, dtype="f16", acc=True, marks=marks, new=True)


@pytest.mark.parametrize("marks", [False, True])
@pytest.mark.parametrize("window,prefix,doc", [(1, 0, 0), (7, 4, 0), (130, 0, 50), (64, 200, 0), (0, 17, 333), (0, 0, 10 ** 6),
                                               (5, 3, 10 ** 6), (2 ** 31 - 1, 0, 0), (300, 2 ** 31 - 1, 9)])
def test_masks(L, window, prefix, doc, marks):
    lens = [700, 129, 1, 0, 512]
    for append in (False, True):
        run(L, lens, H=2, Hq=8, ps=16, window=window, prefixes=[prefix] * 5, docs=[doc, doc // 2, 0, doc, 5], append=append, acc=append,
            marks=marks, dtype="bf16")
    run(L, lens, H=2, Hq=4, ps=32, window=window, prefixes=[prefix] * 5, docs=[doc, doc // 2, 0, doc, 5], new=False, marks=marks)


@pytest.mark.parametrize("q_pos", [[-1, 0, 5], [300, 10 ** 6, 2 ** 31 - 1], [-(2 ** 31), 100, 255]])
def test_query_positions(L, q_pos):
    """A query before some or all of the cached tokens, or far behind them."""
    for new in (False, True):
        run(L, [300, 200, 129], H=2, Hq=8, ps=16, q_pos=[max(x, -1) for x in q_pos] if not new else [max(x, 0) for x in q_pos], new=new)
        run(L, [300, 200, 129], H=2, Hq=8, ps=16, q_pos=[max(x, 0) for x in q_pos], new=new, window=90, append=new, acc=True)


@pytest.mark.parametrize("cap", [0.5, 5.0, 50.0])
@pytest.mark.parametrize("alibi", [False, True])
def test_cap_and_bias(L, cap, alibi):
    run(L, [900, 65, 2], H=2, Hq=8, ps=32, dtype="f16", cap=cap, alibi=alibi, append=True, acc=True)
    run(L, [900, 65, 2], H=4, Hq=4, ps=16, dtype="bf16", cap=cap, alibi=alibi, marks=True, sm=3.0)
    run(L, [900, 65, 2], H=4, Hq=4, ps=16, dtype="bf16", alibi=alibi, marks=True, sm=-0.2)


@pytest.mark.parametrize("H,Hq,ps", [(1, 1, 16), (32, 32, 16), (40, 80, 32), (64, 64, 16), (8, 64, 64), (3, 12, 16)])
@pytest.mark.parametrize("marks", [False, True])
def test_short_sequences(L, H, Hq, ps, marks):
    """Up to a few hundred tokens: whole sequences per CTA, several kv heads per CTA, nothing to see, each kind of mask."""
    run(L, [33], H=H, Hq=Hq, ps=ps, append=True, acc=True, marks=marks)
    run(L, [0, 1, 62, 0, 63], H=H, Hq=Hq, ps=ps, dtype="bf16", append=True, acc=True, marks=marks, alibi=True)
    run(L, [0, 17, 62, 63, 64], H=H, Hq=Hq, ps=ps, new=False, acc=True, marks=marks, cap=5.0)
    run(L, [64, 127, 5], H=H, Hq=Hq, ps=ps, marks=marks, window=20, prefixes=[3, 0, 9], docs=[0, 10 ** 6, 2], append=True)
    run(L, [130, 191, 0], H=H, Hq=Hq, ps=ps, dtype="bf16", new=False, marks=marks, window=64, prefixes=[70, 0, 0], docs=[100, 10 ** 6, 0])


def test_short_sequences_that_fill_the_gpu(L):
    for n in (60, 120, 180, 255):
        run(L, [max(n - 7 * i, 0) for i in range(9)], H=32, Hq=32, ps=16, append=True, acc=True)
    run(L, [255, 0, 3, 200, 64, 129] * 6, H=8, Hq=32, ps=32, dtype="bf16", marks=True, append=True, acc=True, alibi=True)


def test_long_and_many(L):
    run(L, [20000], H=2, Hq=8, ps=64, dtype="bf16", alibi=True, marks=True, acc=True, append=True)
    run(L, [70 + 13 * i for i in range(64)], H=2, Hq=2, ps=16, append=True)
    run(L, [3] * 512, H=1, Hq=2, ps=16, append=True, acc=True)
    run(L, [10, 40], H=2, Hq=2, ps=16, max_len=100000)  # a bound far above the lengths
    run(L, [10, 40, 3000], H=2, Hq=2, ps=16, max_len=100000, acc=True, append=True)
    run(L, [2600] * 80, H=8, Hq=8, ps=64, dtype="bf16", acc=True, append=True, alibi=True)  # weight blocks with several chunks


def test_results_do_not_depend_on_the_call_before(L):
    c, a, za = run(L, [500, 77, 0, 1300], H=4, Hq=16, ps=16, acc=True, append=True, seed=5)
    run(L, [9, 2000], H=2, Hq=2, ps=32, seed=6)
    c, b, zb = run(L, [500, 77, 0, 1300], H=4, Hq=16, ps=16, acc=True, append=True, seed=5)
    assert torch.equal(a, b) and torch.equal(za, zb)


def test_another_stream_and_a_captured_graph(L):
    s = torch.cuda.Stream()
    run(L, [500, 77], H=2, Hq=8, ps=16, append=True, acc=True, stream=s)
    c = L.Cache([333, 64], 2, 8, 16, "bf16", seed=2, weights=True)
    mc, lib = c.mc, c.mc.lib()
    q, kn, vn = c.queries(2, 8).cuda(), c.rows(2, 2).cuda(), c.rows(2, 2).cuda()
    o1, o2 = torch.zeros(2, 8, 128, dtype=c.dt, device="cuda"), torch.zeros(2, 8, 128, dtype=c.dt, device="cuda")
    opts = mc.ScoreOpts(SM)
    ws = c.workspace(mc.MC_OP_LAYER_ATTN, 3)
    lib.mc_layer_attn(c.cfg, c.batch, c.layer, opts, q, kn, vn, 1, o1, None, ws)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        lib.mc_layer_attn(c.cfg, c.batch, c.layer, opts, q, kn, vn, 1, o2, None, ws)
        c.d_lens.add_(1)
    c.d_lens.copy_(torch.tensor(c.lens))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(o1, o2)
    g.replay()  # one token further: the row appended by the first replay is a cached one now
    torch.cuda.synchronize()
    for b, n in enumerate(c.lens):
        for h in range(2):
            c2_k, c2_v = torch.cat([c.dense_k[b][:, h], kn[b, h].cpu()[None]]), torch.cat([c.dense_v[b][:, h], vn[b, h].cpu()[None]])
            k2, v2 = torch.cat([c2_k, kn[b, h].cpu()[None]]), torch.cat([c2_v, vn[b, h].cpu()[None]])
            s = q[b, 4 * h:4 * h + 4].cpu().double() @ k2.double().T * SM
            p = torch.softmax(s, 1)
            tol = 3 * L.eps_half(c.dt) * (p @ v2.double().abs()) + 1e-6
            assert ((o2[b, 4 * h:4 * h + 4].cpu().double() - p @ v2.double()).abs() <= tol).all()


def test_one_call_s_output_as_the_next_one_s_query(L):
    """Calls chained without a kernel between them give what the same calls give with the device idle between them."""
    c = L.Cache([700, 40, 1500], 4, 16, 16, "bf16", seed=8)
    mc, lib = c.mc, c.mc.lib()
    q = c.queries(3, 16).cuda()
    outs = []
    for wait in (True, False):
        a, b, ws = q.clone(), torch.zeros_like(q), c.workspace(mc.MC_OP_LAYER_ATTN, 0)
        torch.cuda.synchronize()
        for _ in range(12):
            lib.mc_layer_attn(c.cfg, c.batch, c.layer, mc.ScoreOpts(300.0), a, None, None, 0, b, None, ws)
            if wait:
                torch.cuda.synchronize()
            a, b = b, a
        torch.cuda.synchronize()
        outs.append(a.clone())
    assert torch.equal(outs[0], outs[1]) and torch.isfinite(outs[0].float()).all()


def test_a_query_of_nan_leaves_the_weights_of_rows_it_does_not_see(L):
    c = L.Cache([300, 90], 2, 8, 16, "bf16", seed=9, marks=True, weights=True)
    mc, lib = c.mc, c.mc.lib()
    pos = torch.tensor(c.q_next, dtype=torch.int32, device="cuda")
    q = c.queries(2, 8).cuda()
    q[0, 1] = float("nan")  # of kv head 0
    out, before = torch.empty_like(q), c.d["w"].clone()
    window = 100
    lib.mc_layer_attn(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM, window=window, q_pos=pos), q, None, None, mc.MC_LAYER_ACCUMULATE, out, None,
                      c.workspace(mc.MC_OP_LAYER_ATTN, mc.MC_LAYER_ACCUMULATE))
    torch.cuda.synchronize()
    after, other = c.gathered("w", 0), c.gathered("w", 1)
    c.d["w"] = before
    was = c.gathered("w", 0)
    seen = L.seen(c.dense_pos[0], c.q_next[0], window=window)
    assert seen.any() and not seen.all()
    assert torch.equal(after[~seen], was[~seen])
    assert after[:, 0][seen[:, 0]].isnan().all() and torch.isfinite(after[:, 1]).all()
    assert out[0, 1].isnan().all() and torch.isfinite(out[0, 4:].float()).all() and torch.isfinite(out[1].float()).all()
    assert torch.isfinite(other).all()


def test_calls_around_one_whose_sequences_are_all_empty(L):
    """A call with nothing to do between two others, all on one workspace and without a pause: results as with pauses."""
    c = L.Cache([20000, 9000], 4, 16, 64, "bf16", seed=10, weights=True)
    mc, lib = c.mc, c.mc.lib()
    q = c.queries(2, 16).cuda()
    none = mc.Batch(c.d["table"], torch.zeros_like(c.d_lens), c.max_len, c.n_pages)
    start, got = c.d["w"].clone(), []
    for wait in (True, False):
        c.d["w"].copy_(start)
        ws, outs = c.workspace(mc.MC_OP_LAYER_ATTN, mc.MC_LAYER_ACCUMULATE), [torch.full_like(q, 7.0) for _ in range(9)]
        torch.cuda.synchronize()
        for i, o in enumerate(outs):
            lib.mc_layer_attn(c.cfg, none if i % 3 else c.batch, c.layer, mc.ScoreOpts(SM), q, None, None, mc.MC_LAYER_ACCUMULATE, o, None, ws)
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        got.append((torch.stack(outs), c.d["w"].clone()))
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    assert not got[0][0][1].any() and got[0][0][0].any()


def test_bad_pages_and_lengths_are_flagged(L):
    c = L.Cache([100, 50], 2, 4, 16, "f16", poison=False)
    mc, lib = c.mc, c.mc.lib()
    q, kn, vn = c.queries(2, 4).cuda(), c.rows(2, 2).cuda(), c.rows(2, 2).cuda()
    out = torch.zeros(2, 4, 128, dtype=c.dt, device="cuda")
    ws = c.workspace(mc.MC_OP_LAYER_ATTN, 1)
    k0 = c.d["k"].clone()
    c.d["table"][0, 2] = 10 ** 6
    c.d["table"][1, 3] = -1  # the page of the row to append
    lib.mc_layer_attn(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), q, kn, vn, 1, out, None, ws)
    words, code = lib.mc_layer_read_status(c.layer, check=False)
    assert code == 8 and words[0] == 4
    changed = (c.d["k"] != k0).any(3).any(1).nonzero()
    assert changed.tolist() == [[int(c.table[0, 6]), 4]]  # sequence 0's row only
    c.layer.status.zero_()
    c.d["table"].copy_(c.table)
    c.d_lens.copy_(torch.tensor([101, -3]))
    lib.mc_layer_attn(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), q, None, None, 0, out, None, ws)
    words, code = lib.mc_layer_read_status(c.layer, check=False)
    assert code == 8 and words[0] == 4 and (out[1] == 0).all()
