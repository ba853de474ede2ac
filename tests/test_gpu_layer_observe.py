"""mc_layer_observe against the definition in 64 bits."""
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


def run(L, lens, J, H=2, Hq=4, ps=16, dtype="f16", acc=False, marks=False, cap=0.0, alibi=False, window=0, docs=None, prefixes=None,
        q_pos=None, sm=SM, seed=0, stream=None, scale=2.5):
    c = L.Cache(lens, H, Hq, ps, dtype, seed=seed, marks=marks, weights=True)
    mc, lib, B = c.mc, c.mc.lib(), c.B
    q = c.queries(B, J, Hq, scale=scale)
    if q_pos is None and marks:
        q_pos = [x - 1 for x in c.q_next]
    slopes = torch.exp2(-8.0 * torch.arange(1, Hq + 1).double() / Hq).float() if alibi else None
    ten = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    opts = mc.ScoreOpts(sm, softcap=cap, alibi_slopes=None if slopes is None else slopes.cuda(), window=window, doc_start=ten(docs),
                        prefix_len=ten(prefixes), q_pos=ten(q_pos))
    w0 = c.w.double()
    ws = c.workspace(mc.MC_OP_LAYER_OBSERVE, J)
    dq = q.cuda()
    torch.cuda.synchronize()
    lib.mc_layer_observe(c.cfg, c.batch, c.layer, opts, dq, mc.MC_LAYER_ACCUMULATE if acc else 0, ws, stream=stream)
    torch.cuda.synchronize()
    words, code = lib.mc_layer_read_status(c.layer, check=False)
    assert code == 0, words
    w, tol = w0.clone(), torch.zeros_like(w0)
    for b, n in enumerate(c.lens):
        last = q_pos[b] if q_pos else n - 1
        t = torch.arange(n)
        for h in range(H):
            k, pos = c.dense_k[b][:, h], c.dense_pos[b][:, h]
            qq = q[b, :, h * c.nq:(h + 1) * c.nq].reshape(-1, 128)  # row j * nq + r
            at = (last - J + 1 + torch.arange(J)).repeat_interleave(c.nq)[:, None]
            s, err = L.scores64(qq, k, pos[None], at, sm, cap, slopes[h * c.nq:(h + 1) * c.nq].repeat(J) if alibi else 0.0)
            ok = L.seen(pos[None].expand_as(s), at, window, docs[b] if docs else 0, prefixes[b] if prefixes else 0) & (at >= 0)
            p, _, rel = L.softmax64(s, err, ok)
            if n:
                pg = c.table[b, t // ps].long()
                w[pg, h, t % ps] = p.sum(0) + (w0[pg, h, t % ps] if acc else 0.0)
                tol[pg, h, t % ps] = (p * (rel[:, None] + (J * c.nq) ** 0.5 * 2 * L.U32)).sum(0) + 2 * L.U32 * w[pg, h, t % ps] + 1e-30
    got = c.d["w"].cpu().double()
    bad = ~((got - w).abs() <= tol)  # (a NaN is bad)
    unused = torch.ones_like(bad)
    for b, n in enumerate(c.lens):
        i = torch.arange(n)
        unused[c.table[b, i // ps].long(), :, i % ps] = False
    assert torch.equal(got[unused], w0[unused])
    assert not bad.any(), (int(bad.sum()), float(((got - w).abs() / tol.clamp(min=1e-30)).max()))
    return c


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("H,Hq,ps,J", [(1, 1, 16, 1), (2, 4, 16, 16), (3, 12, 32, 32), (2, 16, 64, 32), (40, 40, 16, 5), (2, 2, 16, 64),
                                       (1, 4, 64, 24), (2, 8, 32, 40), (1, 1, 16, 256), (2, 4, 16, 65), (1, 8, 16, 17)])
def test_rows_and_lengths(L, H, Hq, ps, J, dtype):
    run(L, [1, 0, 127, 128, 129, 300, 700], J, H=H, Hq=Hq, ps=ps, dtype=dtype)
    run(L, [77, 0, 260], J, H=H, Hq=Hq, ps=ps, dtype=dtype, acc=True, seed=4)


@pytest.mark.parametrize("lens", [[0], [0, 0], [1], [5], [4096], [2000, 3, 1000]])
def test_prompts(L, lens):
    run(L, lens, 32, H=2, Hq=8, ps=16, dtype="bf16")
    run(L, lens, 32, H=2, Hq=8, ps=64, marks=True, acc=True)


@pytest.mark.parametrize("marks", [False, True])
@pytest.mark.parametrize("acc", [False, True])
@pytest.mark.parametrize("window,prefix,doc", [(1, 0, 0), (7, 4, 0), (130, 0, 50), (64, 200, 0), (0, 17, 333), (0, 0, 10 ** 6),
                                               (5, 3, 10 ** 6), (2 ** 31 - 1, 0, 0), (300, 2 ** 31 - 1, 9)])
def test_masks(L, window, prefix, doc, marks, acc):
    run(L, [700, 129, 1, 0, 512], 20, H=2, Hq=8, ps=16, window=window, prefixes=[prefix] * 5, docs=[doc, doc // 2, 0, doc, 5], marks=marks,
        acc=acc, dtype="bf16")
    run(L, [700, 129, 1, 0, 512], 40, H=2, Hq=8, ps=32, window=window, prefixes=[prefix] * 5, marks=marks, acc=acc)


@pytest.mark.parametrize("q_pos", [[-1, 0, 5], [300, 10 ** 6, 2 ** 31 - 2], [40, 100, 255]])
def test_query_positions(L, q_pos):
    run(L, [300, 200, 129], 20, H=2, Hq=8, ps=16, q_pos=q_pos)
    run(L, [300, 200, 129], 20, H=2, Hq=8, ps=16, q_pos=q_pos, window=90, acc=True)


@pytest.mark.parametrize("cap", [0.0, 0.5, 5.0, 50.0, 90.0])
@pytest.mark.parametrize("alibi", [False, True])
def test_cap_and_bias(L, cap, alibi):
    run(L, [900, 65, 2], 16, H=2, Hq=8, ps=32, cap=cap, alibi=alibi, acc=True)
    run(L, [900, 65, 2], 33, H=4, Hq=4, ps=16, dtype="bf16", cap=cap, alibi=alibi, marks=True, sm=3.0, scale=0.1)
    run(L, [900, 65, 2], 64, H=2, Hq=8, ps=16, dtype="bf16", cap=cap, alibi=alibi, sm=-0.2)


@pytest.mark.parametrize("marks", [False, True])
@pytest.mark.parametrize("acc", [False, True])
@pytest.mark.parametrize("window,prefix,doc", [(1, 0, 0), (7, 4, 0), (130, 0, 50), (64, 200, 0), (0, 17, 333), (0, 0, 10 ** 6),
                                               (5, 3, 10 ** 6), (2 ** 31 - 1, 0, 0), (300, 2 ** 31 - 1, 9)])
def test_masks_next_to_a_longer_prompt(L, window, prefix, doc, marks, acc):
    """More than 1024 tokens in one of the sequences: the two launches."""
    run(L, [700, 129, 1, 0, 1100], 20, H=2, Hq=8, ps=16, window=window, prefixes=[prefix] * 5, docs=[doc, doc // 2, 0, doc, 5], marks=marks,
        acc=acc, dtype="bf16")
    run(L, [1030, 129, 1, 0, 512], 40, H=2, Hq=8, ps=32, window=window, prefixes=[prefix] * 5, marks=marks, acc=acc)


@pytest.mark.parametrize("cap", [0.0, 0.5, 50.0, 90.0])
@pytest.mark.parametrize("alibi", [False, True])
def test_cap_bias_and_positions_next_to_a_longer_prompt(L, cap, alibi):
    run(L, [1300, 65, 2], 16, H=2, Hq=8, ps=32, cap=cap, alibi=alibi, acc=True)
    run(L, [1300, 65, 2], 33, H=4, Hq=4, ps=16, dtype="bf16", cap=cap, alibi=alibi, marks=True, sm=3.0, scale=0.1)
    run(L, [65, 1300, 2], 64, H=2, Hq=8, ps=16, dtype="bf16", cap=cap, alibi=alibi, sm=-0.2)
    run(L, [1300, 200, 129], 20, H=2, Hq=8, ps=16, q_pos=[300, 10 ** 6, -1], cap=cap, alibi=alibi, window=90)


@pytest.mark.parametrize("longest", [4200, 2300])
@pytest.mark.parametrize("window,prefix,doc", [(1, 0, 0), (7, 4, 0), (130, 0, 50), (64, 200, 0), (0, 17, 333), (0, 0, 10 ** 6),
                                               (300, 2 ** 31 - 1, 9)])
def test_masks_next_to_a_long_prompt(L, window, prefix, doc, longest):
    """Past what one launch holds (4096 tokens; 2048 where there are more than 128 rows)."""
    J = 20 if longest > 4096 else 40
    for acc, marks in ((False, False), (True, False), (False, True)):
        run(L, [700, 129, 1, 0, longest], J, H=2, Hq=8, ps=16, window=window, prefixes=[prefix] * 5, docs=[doc, doc // 2, 0, doc, 5],
            marks=marks, acc=acc, dtype="bf16", cap=20.0 if acc else 0.0, alibi=marks)


@pytest.mark.parametrize("J", [8, 32, 50])
def test_two_and_four_tiles_per_cta(L, J):
    for lens in ([2000, 1025, 0, 3], [1030, 129], [2048], [4000, 2049, 127, 0], [4096, 100]):
        run(L, lens, J, H=2, Hq=8, ps=64, dtype="bf16", acc=True, cap=30.0 if J == 8 else 0.0)
        run(L, lens[::-1], J, H=1, Hq=2, ps=16, window=700, prefixes=[5] * len(lens), marks=J == 32)
    run(L, [512, 300, 0, 511], J, H=32, Hq=32, ps=16)
    run(L, [512, 257], J, H=32, Hq=32, ps=32, alibi=True)


@pytest.mark.parametrize("tiles", range(1, 9))
def test_every_size_of_a_short_prompt(L, tiles):
    """One to eight tiles of 128 tokens, whole, begun and just begun; rows of each layout."""
    n = 128 * tiles
    for H, Hq, J in ((2, 2, 32), (2, 8, 16), (1, 8, 12), (2, 8, 40)):
        run(L, [n, n - 1, n - 127, max(n - 300, 0)], J, H=H, Hq=Hq, ps=64, dtype="bf16", acc=tiles % 2 == 0, marks=tiles % 3 == 0)


def test_short_prompts_in_two_waves(L):
    run(L, [512, 300, 1, 0, 511, 129, 400, 256], 32, H=8, Hq=32, ps=16, dtype="bf16", cap=30.0)
    run(L, [1024, 0, 1000], 64, H=8, Hq=32, ps=16, alibi=True)


def test_long_many_and_repeatable(L):
    run(L, [20001], 64, H=2, Hq=8, ps=64, dtype="bf16")
    run(L, [70 + 13 * i for i in range(64)], 32, H=2, Hq=2, ps=16)
    run(L, [3] * 512, 4, H=1, Hq=2, ps=16)
    a = run(L, [500, 77, 0, 1300], 32, H=4, Hq=16, seed=5).d["w"]
    b = run(L, [500, 77, 0, 1300], 32, H=4, Hq=16, seed=5, stream=torch.cuda.Stream()).d["w"]
    assert torch.equal(a, b)


def test_bad_pages_are_flagged(L):
    c = L.Cache([300, 50], 2, 4, 16, "f16", weights=True, poison=False)
    mc, lib = c.mc, c.mc.lib()
    q, ws = c.queries(2, 8, 4).cuda(), c.workspace(mc.MC_OP_LAYER_OBSERVE, 8)
    w0 = c.d["w"].clone()
    c.d["table"][0, 2] = 10 ** 6
    c.d["table"][1, 0] = -2
    lib.mc_layer_observe(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), q, 0, ws)
    words, code = lib.mc_layer_read_status(c.layer, check=False)
    assert code == 8 and words[0] == 4
    for page in (int(c.table[0, 2]), int(c.table[1, 0])):
        assert torch.equal(c.d["w"][page], w0[page])  # nothing is written to a page that the table does not name


def test_bad_pages_of_a_long_prompt_are_flagged(L):
    c = L.Cache([4300, 50], 2, 4, 16, "f16", weights=True, poison=False)
    mc, lib = c.mc, c.mc.lib()
    q, ws = c.queries(2, 8, 4).cuda(), c.workspace(mc.MC_OP_LAYER_OBSERVE, 8)
    w0 = c.d["w"].clone()
    c.d["table"][0, 200] = 10 ** 6
    c.d["table"][1, 0] = -2
    lib.mc_layer_observe(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), q, 0, ws)
    words, code = lib.mc_layer_read_status(c.layer, check=False)
    assert code == 8 and words[0] == 4
    for page in (int(c.table[0, 200]), int(c.table[1, 0])):
        assert torch.equal(c.d["w"][page], w0[page])
