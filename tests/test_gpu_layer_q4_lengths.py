"""What the writing calls of a 4-bit layer leave alone when a length is out of range."""
import pytest
import torch

import test_gpu_layer_q4_attn as A

pytestmark = pytest.mark.gpu
SM = A.SM
BAD_METADATA = 4


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2405_14366_b200.build import build_library
    build_library()
    import q4_layer_harness
    return q4_layer_harness


def bits(t):
    return t.view(torch.int16) if t.element_size() == 2 else t


def untouched(c, before, b, pages):
    """Sequence b's pages (the slots `pages` of its block table) and begun page hold what they held."""
    p = c.table[b, :pages].long().cuda()
    for x in ("kc", "km", "vc", "vm"):
        assert torch.equal(bits(c.d[x])[p], bits(before[x])[p]), (b, x)
    for x in ("rk", "rv"):
        assert torch.equal(bits(c.d[x])[b], bits(before[x])[b]), (b, x)


# lengths out of range; 160 is the bound: one above it, and one that would complete a page at the bound's own last slot
LENGTHS = [-1, -(2 ** 31), 161, 191, 2 ** 31 - 1]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("bad", LENGTHS)
@pytest.mark.parametrize("max_len", [160, 159])
def test_append_leaves_a_sequence_of_no_length_alone(Q, dtype, bad, max_len):
    lens = [40, 70, 10]
    c = Q.Cache(lens, 2, 4, dtype, seed=4, room=100, max_len=max_len)
    before = {x: t.clone() for x, t in c.d.items()}
    news = [33, 64, 25]
    k, v = c.rows(sum(news), 2), c.rows(sum(news), 2)
    off = torch.tensor([0, 33, 97, 122], dtype=torch.int32, device="cuda")
    c.d_lens[1] = bad
    c.mc.lib().mc_layer_q4_append(c.cfg, c.batch, c.layer, k.cuda(), v.cuda(), off)
    torch.cuda.synchronize()
    assert c.status()[0][0] == BAD_METADATA
    untouched(c, before, 1, (70 + 100) // 32)
    at = 0
    for b, m in enumerate(news):  # the others get theirs
        if b != 1:
            c.put(b, torch.cat([c.raw[b][0], k[at:at + m]]), torch.cat([c.raw[b][1], v[at:at + m]]))
            p = c.table[b, :(lens[b] + m) // 32].long()
            for x in ("kc", "km", "vc", "vm"):
                assert torch.equal(bits(c.d[x].cpu())[p], bits(getattr(c, x))[p]), (b, x)
        at += m


@pytest.mark.parametrize("H,Hq", [(2, 2), (2, 16)])
@pytest.mark.parametrize("bad", LENGTHS)
@pytest.mark.parametrize("max_len", [160, 159])
@pytest.mark.parametrize("selected", [False, True])
def test_attention_appends_nothing_to_a_sequence_of_no_length(Q, H, Hq, bad, max_len, selected):
    c = Q.Cache([40, 70, 63], H, Hq, "f16", seed=4, room=100, max_len=max_len)
    mc = c.mc
    before = {x: t.clone() for x, t in c.d.items()}
    q, kn, vn = c.queries(3, Hq), c.rows(3, H), c.rows(3, H)
    c.d_lens[1] = bad
    pages = torch.zeros(3, H, 1, dtype=torch.int32, device="cuda") if selected else None
    counts = torch.ones(3, dtype=torch.int32, device="cuda") if selected else None
    out, lse = torch.zeros(3, Hq, 128, dtype=c.dt, device="cuda"), torch.zeros(3, Hq, device="cuda")
    mc.lib().mc_layer_q4_attn(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), pages, counts, q.cuda(), kn.cuda(), vn.cuda(), mc.MC_LAYER_APPEND, out,
                              lse, c.workspace(mc.MC_OP_LAYER_Q4_ATTN, 1))
    torch.cuda.synchronize()
    assert c.status()[0][0] & BAD_METADATA
    untouched(c, before, 1, (70 + 100) // 32)
    assert torch.equal(bits(c.d["rk"].cpu())[0, :, 8], bits(kn)[0]) and torch.equal(bits(c.d["rv"].cpu())[2, :, 31], bits(vn)[2])
    assert not torch.equal(c.d["kc"][int(c.table[2, 1])], before["kc"][int(c.table[2, 1])])  # (its second page is complete now)
