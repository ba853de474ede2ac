"""Scores of mc_layer_q4_attn over keys of any size: a query that sees one token has that token's score as its log-sum-exp, so the
score itself is compared with 64 bits, ahead of the rounding that probabilities get."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

SM = 1.0 / math.sqrt(128.0)
U32 = 2.0 ** -24


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2405_14366_b200.build import build_library
    build_library()
    import q4_layer_harness
    return q4_layer_harness


def rescale(c, f):
    """The keys' parameters times f [pages][H][128] (or a number), as binary16 holds them; scales stay positive and below 16000."""
    m = c.km.float().nan_to_num(1.0, 1.0, 1.0) * torch.as_tensor(f, dtype=torch.float32)[..., None]
    m[..., 0] = m[..., 0].abs().clamp(2.0 ** -24, 15990.0)
    m[..., 1] = m[..., 1].clamp(-60000.0, 60000.0)
    c.km[...] = m.half()
    c.d["km"].copy_(c.km)


def compare_scores(Q, c, q, sm, seed=0):
    """Every (sequence, head): one token of a complete page at a time; largest error as a fraction of the bound."""
    mc, g, worst = c.mc, torch.Generator().manual_seed(seed), 0.0
    full = torch.tensor([n // 32 * 32 for n in c.lens])
    for _ in range(6):
        t = (torch.rand(c.B, generator=g) * full).long()
        opts = mc.ScoreOpts(sm, window=1, q_pos=t.int().cuda())
        out, lse = torch.zeros(c.B, c.Hq, 128, dtype=c.dt, device="cuda"), torch.zeros(c.B, c.Hq, device="cuda")
        mc.lib().mc_layer_q4_attn(c.cfg, c.batch, c.layer, opts, None, None, q.cuda(), None, None, 0, out, lse, c.workspace(mc.MC_OP_LAYER_Q4_ATTN))
        got = lse.cpu().double()
        for b in range(c.B):
            for h in range(c.H):
                kc, kz, _, _ = c.values(b, h)
                x = q[b, h * c.nq:(h + 1) * c.nq].double()
                i = int(t[b])
                s = x @ (kc[i] + kz[i]) * sm
                big, top = x.abs().amax(1), c.km[c.table[b, i // 32].long(), h].double()[:, 0].max()
                mass = x.abs() @ (kc[i].abs() + kz[i].abs())
                # sums: 520 units as in the harness; a product next to the largest possible one of its page: 2^-25 of that, codes up to
                # 15; the query's form: 2^-25 of the unit in which its largest number is 2^10
                err = 520 * U32 * mass + 128 * 15 * 2.0 ** -25 * big * top + 2.0 ** -35 * big * (kc[i].abs() + kz[i].abs()).sum()
                # log-sum-exp: the score next to a power of two of at most 15, a logarithm, a product
                tol = err * abs(sm) + 8 * U32 * (s.abs() + 16.0)
                d = (got[b, h * c.nq:(h + 1) * c.nq] - s).abs()
                assert (d <= tol).all(), (b, h, i, float(s.abs().max()), float((d / tol).max()))
                worst = max(worst, float((d / tol).max()))
    assert c.status()[1] == 0
    return worst


HEADS = [(2, 2), (2, 8), (1, 8), (3, 12)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("H,Hq", HEADS)
@pytest.mark.parametrize("bits", [0, -5, -8, -12, -15, -18, 6, 12, 18])
def test_scores_of_small_and_large_keys(Q, dtype, H, Hq, bits):
    """Keys times 2^bits, sm_scale times 2^-bits: the scores of an ordinary layer, whatever the keys' unit is."""
    c = Q.Cache([64, 130, 320, 33], H, Hq, dtype, seed=40 + bits)
    rescale(c, 2.0 ** bits)
    compare_scores(Q, c, c.queries(c.B, Hq), SM * 2.0 ** -bits)


@pytest.mark.parametrize("H,Hq", HEADS)
@pytest.mark.parametrize("bits", [-6, -9, -12, -16, 0, 10])
def test_scores_of_one_channel(Q, H, Hq, bits):
    """Queries of one channel: nothing but that product, its code and its zero."""
    c = Q.Cache([64, 130, 320, 33], H, Hq, "f16", seed=60 + bits)
    rescale(c, 2.0 ** bits)
    q = torch.zeros(c.B, Hq, 128)
    at = torch.randint(0, 128, (c.B, Hq, 1), generator=c.g)
    q.scatter_(2, at, 300.0 * torch.randn(c.B, Hq, 1, generator=c.g))
    compare_scores(Q, c, q.to(c.dt), SM * 2.0 ** -bits)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("H,Hq", HEADS)
def test_scores_of_pages_and_channels_of_all_sizes(Q, dtype, H, Hq):
    """A page's keys 2^-18 to 2^12 of its neighbour's; then channels 2^8 above the others; a query with entries 2^-12 of its largest."""
    c = Q.Cache([640, 330, 1000], H, Hq, dtype, seed=80)
    f = torch.exp2(torch.randint(-18, 13, (c.n_pages, H, 1), generator=c.g).float())
    rescale(c, f)
    q = c.queries(c.B, Hq).float()
    q = (q * torch.exp2(torch.randint(-12, 1, q.shape, generator=c.g).float())).to(c.dt)
    for sm in (SM, SM * 2.0 ** 14):
        compare_scores(Q, c, q, sm)
    f = torch.exp2(8.0 * (torch.rand(c.n_pages, H, 128, generator=c.g) < 0.03).float())
    rescale(c, f)
    compare_scores(Q, c, q, SM)


@pytest.mark.parametrize("Hq", [2, 8, 16])
def test_attention_over_pages_of_all_sizes(Q, Hq):
    """The whole of the attention over such pages, every bound of the definition's own."""
    import test_gpu_layer_q4_attn as A
    for bits in (-14, 0, 9):
        c = Q.Cache([64, 330, 1000], 2, Hq, "bf16", seed=90)
        f = torch.exp2(torch.randint(-8, 9, (c.n_pages, 2, 1), generator=c.g).float() * 0.5 + bits)
        rescale(c, f)
        c.rk[...] = (c.rk.float() * 2.0 ** bits).to(c.dt)
        c.d["rk"].copy_(c.rk)
        q = (torch.randn(c.B, Hq, 128, generator=c.g) * 2.0 ** -bits).to(c.dt)
        A.run(Q, c, q=q, new=False)
        A.run(Q, c, q=q, new=False, cap=20.0)


@pytest.mark.parametrize("Hq", [2, 16])
def test_queries_at_the_ends_of_their_range(Q, Hq):
    """Queries near the largest and the smallest that bfloat16 holds, one of zeros among them."""
    c = Q.Cache([64, 130, 320], 2, Hq, "bf16", seed=70)
    for size in (2.0 ** 120, 2.0 ** 60, 2.0 ** -60, 2.0 ** -110):
        q = torch.randn(c.B, Hq, 128, generator=c.g).clamp(-1.9, 1.9)
        q[0, 0] = 0.0
        q = (q.double() * size).to(c.dt)
        compare_scores(Q, c, q, 4.0 / size)
