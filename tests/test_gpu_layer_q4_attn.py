"""mc_layer_q4_attn and mc_layer_q4_select against the definitions in 64 bits over the values that the codes stand for."""
import math

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


def dev(x, dt=torch.int32):
    return None if x is None else torch.as_tensor(x, dtype=dt).cuda()


def run(Q, c, *, new=True, append=False, cap=0.0, alibi=False, window=0, docs=None, prefix=None, q_pos=None, pages=None, counts=None, q=None,
        sm=SM, q_scale=2.5, check=True):
    mc = c.mc
    B, H, Hq, nq = c.B, c.H, c.Hq, c.nq
    q = c.queries(B, Hq, scale=q_scale) if q is None else q
    kn, vn = (c.rows(B, H), c.rows(B, H)) if new else (None, None)
    slopes = torch.exp2(-8.0 * torch.arange(1, Hq + 1) / Hq).float() if alibi else None
    opts = mc.ScoreOpts(sm, softcap=cap, alibi_slopes=dev(slopes, torch.float32), window=window, doc_start=dev(docs), prefix_len=dev(prefix),
                        q_pos=dev(q_pos))
    flags = mc.MC_LAYER_APPEND if append else 0
    out = torch.full((B, Hq, 128), 9.0, dtype=c.dt, device="cuda")
    lse = torch.full((B, Hq), 9.0, device="cuda")
    dp = None if pages is None else pages if torch.is_tensor(pages) else dev(pages)
    dc = None if counts is None else dev(counts)
    mc.lib().mc_layer_q4_attn(c.cfg, c.batch, c.layer, opts, dp, dc, q.cuda(), None if kn is None else kn.cuda(), None if vn is None else vn.cuda(),
                              flags, out, lse, c.workspace(mc.MC_OP_LAYER_Q4_ATTN, flags))
    torch.cuda.synchronize()
    if check:
        assert c.status()[1] == 0, c.status()
        worst = 0.0
        for b in range(B):
            for h in range(H):
                kw = dict(k_new=kn[b, h], v_new=vn[b, h]) if new else {}
                sel = None if pages is None else dp[b, h, :int(dc[b])].tolist()
                o, z, tol, ztol = Q.attn64(c, b, h, q[b, h * nq:(h + 1) * nq], sm, cap=cap, slopes=slopes, window=window,
                                           doc=docs[b] if docs else 0, prefix=prefix[b] if prefix else 0,
                                           q_pos=max(q_pos[b], -1) if q_pos else None, pages=sel, **kw)
                go, gz = out[b, h * nq:(h + 1) * nq].cpu().double(), lse[b, h * nq:(h + 1) * nq].cpu().double()
                d = (go - o).abs()
                assert (d <= tol).all(), (b, h, float((d / tol).max()))
                worst = max(worst, float((d / tol).max()))
                inf = torch.isinf(z)
                assert torch.equal(gz[inf], z[inf])
                assert ((gz - z)[~inf].abs() <= ztol[~inf]).all(), (b, h, float(((gz - z)[~inf].abs() / ztol[~inf]).max()))
    if append:
        for b in range(B):  # the host's cache takes the row too
            n = c.lens[b]
            c.raw[b] = [torch.cat([x, r[b][None]]) for x, r in zip(c.raw[b], (kn, vn))]
            if n % 32 == 31:
                at = [int(c.table[b, n // 32])]
                c.rk[b, :, 31], c.rv[b, :, 31] = kn[b], vn[b]
                for x, codes, meta, res, kind in ((c.raw[b][0], c.kc, c.km, c.rk, "k"), (c.raw[b][1], c.vc, c.vm, c.rv, "v")):
                    r = res[b].double()
                    cd, s, z = Q.quantise(r.numpy(), kind)
                    codes[at[0]] = Q.pack(cd)
                    meta[at[0], ..., 0], meta[at[0], ..., 1] = (torch.from_numpy(y).half() for y in (s, z))
            else:
                c.rk[b, :, n % 32], c.rv[b, :, n % 32] = kn[b], vn[b]
        assert c.same_as_host() is None, c.same_as_host()
        c.lens = [n + 1 for n in c.lens]
        c.d_lens.add_(1)
    return out, lse, q, kn, vn


HEADS = [(1, 1), (2, 4), (2, 8), (1, 8), (5, 10), (32, 32), (8, 32), (4, 32)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("H,Hq", HEADS)
def test_lengths(Q, dtype, H, Hq):
    c = Q.Cache([0, 1, 31, 32, 33, 63, 64, 95, 129, 700], H, Hq, dtype, seed=H + Hq)
    run(Q, c, new=True)
    run(Q, c, new=False)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("H,Hq", [(2, 2), (2, 8), (2, 16)])
@pytest.mark.parametrize("kw", [dict(cap=50.0), dict(cap=5.0, q_scale=10.0), dict(alibi=True), dict(window=1), dict(window=40), dict(window=33, prefix=[4] * 7),
                                dict(docs=[0, 5, 32, 40, 64, 100, 333]), dict(docs=[0, 9, 50, 40, 64, 100, 333], prefix=[0, 3, 0, 40, 33, 0, 64], window=100, cap=30.0, alibi=True),
                                dict(q_pos=[0, -1, 10, 40, 20, 500, 300]), dict(q_pos=[-5, 31, 32, 1000, 63, 64, 95], alibi=True)],
                         ids=lambda d: "-".join(d))
def test_masks_caps_and_biases(Q, dtype, H, Hq, kw):
    c = Q.Cache([3, 33, 64, 70, 96, 200, 510], H, Hq, dtype, seed=7)
    run(Q, c, new=True, **kw)
    run(Q, c, new=False, **kw)


@pytest.mark.parametrize("kw", [dict(docs=[500] * 4), dict(q_pos=[-1] * 4), dict(window=3, q_pos=[2000] * 4)], ids=["doc", "before", "window"])
def test_a_query_that_sees_nothing(Q, kw):
    c = Q.Cache([0, 31, 64, 300], 2, 8, "f16", seed=1)
    out, lse, *_ = run(Q, c, new=False, **kw)
    assert (out == 0).all() and torch.isinf(lse).all() and (lse < 0).all()


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("scale", [1e-4, 1e-2, 30.0, 3000.0])
@pytest.mark.parametrize("Hq", [2, 16])
def test_keys_and_values_of_any_size(Q, dtype, scale, Hq):
    """The probabilities' power of two follows the values' scales, the queries' their own size."""
    c = Q.Cache([64, 130, 1000], 2, Hq, dtype, seed=5, scale=scale)
    run(Q, c)


@pytest.mark.parametrize("Hq", [2, 16])
def test_scales_that_grow_and_shrink_from_page_to_page(Q, Hq):
    c = Q.Cache([40 * 32, 33 * 32 + 5], 2, Hq, "f16", seed=6)
    f = torch.exp2(torch.randint(-10, 11, (c.n_pages, 2), generator=c.g).float())
    c.vm[...] = (c.vm.float().nan_to_num(1.0, 1.0, 1.0) * f[:, :, None, None, None]).half()
    c.d["vm"].copy_(c.vm)
    run(Q, c)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_one_key_far_above_the_others(Q, dtype):
    c = Q.Cache([500, 64], 2, 4, dtype, seed=3)
    run(Q, c, q_scale=60.0)


@pytest.mark.parametrize("Hq", [2, 16])
def test_queries_of_zeros_and_of_one_channel(Q, Hq):
    c = Q.Cache([100, 320], 2, Hq, "f16", seed=3)
    q = c.queries(2, Hq)
    q[0] = 0
    q[1] = 0
    q[1, :, 77] = 900.0
    run(Q, c, q=q)


@pytest.mark.parametrize("Hq", [2, 8, 16])
def test_scales_of_scores_at_their_limits(Q, Hq):
    c = Q.Cache([100, 32, 5], 2, Hq, "bf16", seed=9)
    q = torch.zeros(3, Hq, 128, dtype=c.dt)
    q[:, :, 3] = 100.0
    q[1] = 0
    out, lse, *_ = run(Q, c, q=q * 0, sm=2.0e38, new=False)  # all alike
    assert (lse.cpu() - torch.tensor([100.0, 32.0, 5.0]).log()[:, None]).abs().max() < 1e-5
    run(Q, c, q=q, sm=1e-38)
    run(Q, c, q=q, sm=0.0)
    run(Q, c, q=q, sm=-0.02)
    run(Q, c, q=q * 1e-30, sm=1e30)
    run(Q, c, q=q * 1e30, sm=1e-31, cap=20.0)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("H,Hq", [(2, 2), (3, 12), (2, 16)])
def test_append_step_by_step_through_page_ends(Q, dtype, H, Hq):
    c = Q.Cache([0, 30, 31, 60, 63, 95], H, Hq, dtype, seed=11, room=40, max_len=200)
    for i in range(36):
        run(Q, c, append=True, check=i in (0, 1, 2, 3, 33, 34))


def test_append_without_a_page_is_flagged(Q):
    c = Q.Cache([31, 20], 2, 2, "f16", seed=1, room=1)
    c.d["table"].fill_(c.n_pages)
    before = c.d["kc"].clone()
    run(Q, c, append=False, check=True)
    mc = c.mc
    kn = c.rows(2, 2).cuda()
    mc.lib().mc_layer_q4_attn(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), None, None, c.queries(2, 2).cuda(), kn, kn, 1,
                              torch.zeros(2, 2, 128, dtype=c.dt, device="cuda"), None, c.workspace(mc.MC_OP_LAYER_Q4_ATTN, 1))
    assert c.status()[0][0] == 4 and torch.equal(before, c.d["kc"])
    assert torch.equal(c.d["rk"][:, :, 31][0], kn[0]) and torch.equal(c.d["rk"][1, :, 20], kn[1])


def test_bad_pages_and_lengths_are_flagged(Q):
    c = Q.Cache([100, 200], 2, 4, "f16", seed=1, max_len=256)
    good = c.d["table"].clone()
    for bad in (-1, c.n_pages, 2 ** 31 - 1):
        c.d["table"][0, 1] = bad
        run(Q, c, check=False)
        assert c.status()[0][0] == 4
        c.layer.status.zero_()
    c.d["table"].copy_(good)
    for n in ([257, 200], [-3, 200], [2 ** 31 - 1, 0]):
        c.d_lens.copy_(torch.tensor(n))
        c.d["table"].clamp_(min=0)
        run(Q, c, check=False)
        assert c.status()[0][0] == 4
        c.layer.status.zero_()


# ---- selection ---------------------------------------------------------------------------------------------
def select(Q, c, q, budget, sink=0, recent=0, q_pos=None, window=0, docs=None, prefix=None):
    mc = c.mc
    pages = torch.full((c.B, c.H, budget), -9, dtype=torch.int32, device="cuda")
    counts = torch.full((c.B,), -9, dtype=torch.int32, device="cuda")
    opts = mc.ScoreOpts(SM, window=window, doc_start=dev(docs), prefix_len=dev(prefix), q_pos=dev(q_pos))
    mc.lib().mc_layer_q4_select(c.cfg, c.batch, c.layer, opts, mc.PageSelection(budget, sink, recent), q.cuda(), pages, counts,
                                c.workspace(mc.MC_OP_LAYER_Q4_SELECT))
    torch.cuda.synchronize()
    for b in range(c.B):
        for h in range(c.H):
            want = Q.select64(c, q[b, h * c.nq:(h + 1) * c.nq], b, h, budget, sink, recent, q_pos[b] if q_pos else c.lens[b], window,
                              docs[b] if docs else 0, prefix[b] if prefix else 0)
            assert int(counts[b]) == len(want)
            assert pages[b, h].tolist() == want + [-9] * (budget - len(want)), (b, h)
    return pages, counts


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("H,Hq", [(1, 1), (2, 8), (2, 16), (5, 10), (32, 32)])
def test_select(Q, dtype, H, Hq):
    c = Q.Cache([0, 5, 32, 33, 400, 1000, 2500], H, Hq, dtype, seed=H)
    for budget, sink, recent in ((1, 0, 0), (2, 1, 1), (7, 0, 0), (9, 2, 3), (40, 4, 4), (200, 0, 0)):
        select(Q, c, c.queries(c.B, Hq), budget, sink, recent)
    assert c.status()[1] == 0


@pytest.mark.parametrize("kw", [dict(window=300), dict(docs=[0, 70, 400]), dict(window=200, prefix=[40, 40, 40]), dict(q_pos=[10, 500, 2000]),
                                dict(q_pos=[-1, 63, 64])], ids=lambda d: "-".join(d))
def test_select_masks(Q, kw):
    c = Q.Cache([100, 1000, 2500], 2, 8, "bf16", seed=4)
    for budget, sink, recent in ((1, 0, 0), (3, 1, 1), (12, 1, 2)):
        select(Q, c, c.queries(3, 8), budget, sink, recent, **kw)


def test_select_ties_and_numbers_that_are_none(Q):
    c = Q.Cache([3200, 2048], 2, 4, "f16", seed=4)
    select(Q, c, torch.zeros(2, 4, 128, dtype=c.dt), 13)  # all alike: the lowest
    # pages that repeat: ties of the whole sum, resolved by the index
    for h in range(2):
        for s in range(100):
            c.km[c.table[0, s], h] = c.km[c.table[0, s % 3], h]
    # and sums that only 64 bits tell apart
    for s in range(64):
        c.km[c.table[1, s]] = c.km[c.table[1, 0]]
        c.km[c.table[1, s], :, 7, 1] = float(s % 5) * 2.0 ** -24
    c.d["km"].copy_(c.km)
    q = c.queries(2, 4)
    for budget in (1, 5, 34, 67, 99):
        select(Q, c, q, budget)
    q[0, 0, 5] = float("nan")
    select(Q, c, q, 20)


@pytest.mark.parametrize("B,H,n", [(1, 1, 70000), (1, 2, 40000), (2, 8, 9000)])
def test_select_long(Q, B, H, n):
    """Clusters of every size, and more pages than threads."""
    c = Q.Cache([n - 77 * b for b in range(B)], H, 4 * H, "bf16", seed=n)
    for budget in (3, 64, 300):
        select(Q, c, c.queries(B, 4 * H), budget, 1, 2)


def test_select_long_ties(Q):
    """More pages than threads, with sums that are alike, or alike in 32 bits only, on the border of the choice."""
    c = Q.Cache([38000, 25013], 2, 4, "f16", seed=6)
    select(Q, c, torch.zeros(2, 4, 128, dtype=c.dt), 513)  # all alike: the lowest
    for s in range(38000 // 32):
        c.km[c.table[0, s]] = c.km[c.table[0, s % 7]]
    for s in range(25013 // 32):
        c.km[c.table[1, s]] = c.km[c.table[1, 0]]
        c.km[c.table[1, s], :, 7, 1] = float(s % 5) * 2.0 ** -24
    c.d["km"].copy_(c.km)
    q = c.queries(2, 4)
    for budget, sink, recent in ((1, 0, 0), (33, 0, 0), (100, 3, 5), (170, 0, 0), (700, 1, 1), (780, 0, 0), (1186, 0, 0)):
        select(Q, c, q, budget, sink, recent)
    q[1, :, 5] = float("nan")  # no sum is a number: the lowest
    select(Q, c, q, 77)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("H,Hq", [(2, 2), (2, 8), (2, 16), (5, 10)])
def test_attention_over_selected_pages(Q, dtype, H, Hq):
    c = Q.Cache([0, 20, 64, 500, 2000], H, Hq, dtype, seed=21)
    for kw in ({}, dict(window=300, prefix=[33] * 5), dict(docs=[0, 0, 40, 100, 900])):
        for budget in (1, 6, 50):
            q = c.queries(5, Hq)
            pages, counts = select(Q, c, q, budget, min(1, budget - 1), min(2, max(budget - 2, 0)), **kw)
            run(Q, c, q=q, pages=pages, counts=counts.tolist(), cap=30.0, **kw)


def test_lists_of_the_caller(Q):
    """Any ascending list will do, also one whose pages the masks hide in part or altogether; other entries are skipped."""
    c = Q.Cache([400, 330], 2, 4, "f16", seed=2)
    pages = torch.tensor([[[0, 3, 4, 11], [1, 2, 3, 4]], [[0, 9, 99, 99], [4, 5, 99, 99]]], dtype=torch.int32).cuda()
    run(Q, c, pages=pages, counts=[4, 2])
    run(Q, c, pages=pages, counts=[4, 2], window=60, prefix=[3, 40])
    run(Q, c, pages=pages, counts=[0, 1])
    for bad in ([3, 3, 5, 6], [5, 4, 6, 7], [-1, 0, 1, 2], [0, 1, 2, 12], [2 ** 31 - 1, 0, 1, 2]):
        pages[0, 0] = torch.tensor(bad)
        run(Q, c, pages=pages, counts=[4, 2], check=False)
        assert c.status()[0][0] == 4
        c.layer.status.zero_()
    pages[0, 0] = torch.tensor([3, 3, 5, 6])
    q = c.queries(2, 4)
    torch.manual_seed(0)
    out, lse, q, kn, vn = run(Q, c, pages=pages, counts=[4, 2], q=q, check=False)
    o, z, tol, ztol = Q.attn64(c, 0, 0, q[0, :2], SM, k_new=kn[0, 0], v_new=vn[0, 0], pages=[3, 5, 6])
    assert ((out[0, :2].cpu().double() - o).abs() <= tol).all()
    c.layer.status.zero_()
    for n in ([5, 2], [-1, 2]):
        run(Q, c, pages=pages, counts=n, check=False)
        assert c.status()[0][0] == 4
        c.layer.status.zero_()


def test_a_large_batch_and_many_heads(Q):
    c = Q.Cache([(37 * i) % 200 for i in range(300)], 3, 6, "f16", seed=2)
    run(Q, c)
    c = Q.Cache([70, 0, 33], 300, 300, "f16", seed=2)
    run(Q, c)
