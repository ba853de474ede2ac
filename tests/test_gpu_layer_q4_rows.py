"""mc_layer_q4_append and mc_layer_q4_read: codes and parameters bit for bit against the quantiser in 64 bits, rows of the
begun page untouched, everything else left as it was."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def Q():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2405_14366_b200.build import build_library
    build_library()
    import q4_layer_harness
    return q4_layer_harness


def append(c, news, k, v, stream=None):
    off = torch.tensor([0] + np.cumsum(news).tolist(), dtype=torch.int32, device="cuda")
    c.mc.lib().mc_layer_q4_append(c.cfg, c.batch, c.layer, k, v, off, stream=stream)


def grow(Q, c, news, packed=False, poke=None):
    """Appends news[b] rows to every sequence on the device and on the host."""
    H = c.H
    k, v = [c.rows(m, H) for m in news], [c.rows(m, H) for m in news]
    if poke:
        for x in k + v:
            poke(x)
    dk, dv = torch.cat(k).cuda(), torch.cat(v).cuda()
    if packed:
        qkv = torch.full((len(dk), c.Hq + 2 * H, 128), float("nan"), dtype=c.dt, device="cuda")
        qkv[:, c.Hq:c.Hq + H], qkv[:, c.Hq + H:] = dk, dv
        dk, dv = qkv[:, c.Hq:c.Hq + H], qkv[:, c.Hq + H:]
    append(c, news, dk, dv)
    for b, m in enumerate(news):
        if not m:
            continue
        n = c.lens[b]
        if n + m >= (n // Q.PAGE + 1) * Q.PAGE or not n % Q.PAGE:
            c.raw[b] = [torch.cat([x, y[b]]) for x, y in zip(c.raw[b], (k, v))]
            c.put(b, *c.raw[b])
        else:  # nothing completed: the rows go behind the begun page's
            c.raw[b] = [torch.cat([x, y[b]]) for x, y in zip(c.raw[b], (k, v))]
            c.rk[b, :, n % 32:n % 32 + m], c.rv[b, :, n % 32:n % 32 + m] = k[b].transpose(0, 1), v[b].transpose(0, 1)
        c.lens[b] = n + m
    c.d_lens.copy_(torch.tensor(c.lens, dtype=torch.int32))


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("H,Hq", [(1, 8), (2, 2), (5, 10), (8, 32)])
def test_prompts_chunks_and_single_rows(Q, dtype, H, Hq):
    news = [[1, 31, 32, 33, 64, 0, 200, 5], [31, 1, 32, 0, 1, 7, 40, 28], [1, 1, 1, 31, 95, 25, 3, 0], [64, 0, 1, 1, 1, 1, 1, 1]]
    room = max(sum(x[b] for x in news) for b in range(8))
    c = Q.Cache([0] * 8, H, Hq, dtype, seed=3, room=room, max_len=512, empty=True)
    for i, n in enumerate(news):
        grow(Q, c, n, packed=i % 2 == 1)
        torch.cuda.synchronize()
        assert c.same_as_host() is None, (i, c.same_as_host())
    assert c.status()[1] == 0


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_groups_at_the_edges_of_the_quantiser(Q, dtype):
    """Constant groups, all zeros, ties, tiny and huge numbers, signs, NaN and infinities."""
    dt = torch.float16 if dtype == "f16" else torch.bfloat16

    def poke(x):
        if not len(x):
            return
        g = torch.Generator().manual_seed(len(x))
        r = lambda *s: torch.randint(0, 16, s, generator=g)  # noqa: E731
        n = len(x)
        x[:, 0] = 0.25
        x[:, 1] = 0.0
        x[:, 2] = (r(n, 128) * 0.5 + 0.25 * (r(n, 128) % 2)).to(dt)        # codes' ties: multiples of half a scale
        x[:, 3] = (r(n, 128).double() * 2.0 ** -24).to(dt)                  # subnormal numbers
        x[:, 4] = (x[:, 4].float() * 3e5).clamp(-65504, 65504).to(dt)
        x[:, 5] = torch.tensor(float("nan"), dtype=dt)
        x[n // 2, 6] = float("inf")
        x[n // 3, 6, 5:40] = -float("inf")
        x[n // 3, 7, 3] = float("nan")
        x[:, 7, 100:] = -x[:, 7, 100:].abs()
        x[:, 8] = (x[:, 8].double() * 1e-30).to(dt)
        x[:, 9] = torch.where(r(n, 128) < 8, torch.tensor(60000.0), torch.tensor(1e-6)).to(dt)
        x[:, 10] = (-1.0 + r(n, 128) * 2.0 ** -9).to(dt)
    c = Q.Cache([0, 0], 11, 11, dtype, seed=9, room=400, max_len=512, empty=True)
    for news in ([100, 64], [200, 1], [33, 300]):
        grow(Q, c, news, poke=poke)
        torch.cuda.synchronize()
        assert c.same_as_host() is None, (news, c.same_as_host())


def test_many_ties_of_scales_and_codes(Q):
    """Numbers of few bits: quotients meet ties of the codes and of the scale's rounding all the time."""
    c = Q.Cache([0, 0, 0], 4, 4, "f16", seed=2, room=2048, max_len=2048, empty=True)

    def poke(x):
        g = torch.Generator().manual_seed(len(x))
        e = torch.randint(-12, 13, (len(x), 4, 1), generator=g).double()
        x.copy_((torch.randint(-4096, 4097, x.shape, generator=g).double() * torch.exp2(e - 12)).to(x.dtype))
    grow(Q, c, [2048, 1000, 77], poke=poke)
    torch.cuda.synchronize()
    assert c.same_as_host() is None


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("H,Hq", [(1, 8), (5, 10), (8, 8)])
def test_read(Q, dtype, H, Hq):
    lens = [0, 1, 31, 32, 33, 64, 200, 777]
    c = Q.Cache(lens, H, Hq, dtype, seed=5)
    begin = [0, 0, 5, 0, 31, 32, 17, 100]
    want = [3, 1, 26, 32, 2, 40, 150, 677]  # (some past the end: their rows stay)
    for strided in (False, True):
        rows = sum(want) + 3
        wide = torch.full((rows, 2 * H + 3, 128), 7.0, dtype=c.dt, device="cuda")
        k, v = (wide[:, 1:1 + H], wide[:, 2 + H:2 + 2 * H]) if strided else (torch.full((rows, H, 128), 7.0, dtype=c.dt, device="cuda") for _ in range(2))
        off = torch.tensor([2] + (2 + np.cumsum(want)).tolist(), dtype=torch.int32, device="cuda")
        c.mc.lib().mc_layer_q4_read(c.cfg, c.batch, c.layer, torch.tensor(begin, dtype=torch.int32, device="cuda"), k, v, off)
        torch.cuda.synchronize()
        assert c.status()[1] == 0
        got = [k.cpu(), v.cpu()]
        exp = [torch.full((rows, H, 128), 7.0, dtype=torch.float64) for _ in range(2)]
        at = 2
        for b, n in enumerate(lens):
            m = max(0, min(want[b], n - begin[b]))
            for h in range(H):
                kc, kz, vc, vz = c.values(b, h)
                exp[0][at:at + m, h], exp[1][at:at + m, h] = (kc + kz)[begin[b]:begin[b] + m], (vc + vz)[begin[b]:begin[b] + m]
            at += want[b]
        for g, e in zip(got, exp):
            if dtype == "f16":  # rounded once
                assert torch.equal(g, torch.from_numpy(e.numpy().astype(np.float16)))
            else:  # binary32 in between
                assert ((g.double() - e).abs() <= e.abs() * 2.0 ** -8 * (1 + 2.0 ** -15)).all()
        if strided:
            assert (wide[:, 0] == 7).all() and (wide[:, 1 + H] == 7).all() and (wide[:, 2 + 2 * H:] == 7).all()


def test_read_without_begin_gives_the_whole_prompt_back(Q):
    c = Q.Cache([70, 5], 2, 2, "f16", seed=8)
    k, v = (torch.zeros(75, 2, 128, dtype=c.dt, device="cuda") for _ in range(2))
    off = torch.tensor([0, 70, 75], dtype=torch.int32, device="cuda")
    c.mc.lib().mc_layer_q4_read(c.cfg, c.batch, c.layer, None, k, v, off)
    assert torch.equal(k[64:70].cpu(), c.raw[0][0][64:]) and torch.equal(v[70:].cpu(), c.raw[1][1])
    # off by half a scale at most, and by what scale and value were rounded by
    for x, r in ((k, c.raw[0][0]), (v, c.raw[0][1])):
        d = (x[:64].cpu().double() - r[:64].double()).abs()
        assert float(d.max()) <= float(r.double().abs().max()) * (2 / 30 + 0.01)


def test_bad_offsets_lengths_and_pages_are_flagged_and_never_followed(Q):
    c = Q.Cache([40, 70, 10], 2, 4, "f16", seed=4, room=100, max_len=160)
    before = {x: t.clone() for x, t in c.d.items()}
    k, v = c.rows(90, 2).cuda(), c.rows(90, 2).cuda()
    lib = c.mc.lib()
    bits = lambda t: t.view(torch.int16) if t.element_size() == 2 else t  # noqa: E731
    for off in ([0, 50, 30, 90], [-1, 30, 60, 90], [0, 30, 60, 91], [0, 30, 2 ** 31 - 1, 90]):
        o = torch.tensor(off, dtype=torch.int32, device="cuda")
        lib.mc_layer_q4_append(c.cfg, c.batch, c.layer, k, v, o)
        out = [torch.full_like(k, 3.0) for _ in range(2)]
        lib.mc_layer_q4_read(c.cfg, c.batch, c.layer, None, *out, o)
        assert c.status()[0][0] == 4
        c.layer.status.zero_()
        assert all(torch.equal(bits(c.d[x]), bits(before[x])) for x in before) and (out[0] == 3).all() and (out[1] == 3).all()
    # a page id out of range: that page is not written (read: its rows stay), the others are
    c.d["table"][0, 1] = c.n_pages
    off = torch.tensor([0, 60, 60, 90], dtype=torch.int32, device="cuda")
    lib.mc_layer_q4_append(c.cfg, c.batch, c.layer, k, v, off)
    assert c.status()[0][0] == 4
    c.layer.status.zero_()
    p2, p3 = int(c.table[0, 2]), int(c.table[2, 0])
    assert not torch.equal(c.d["kc"][p2], before["kc"][p2]) and not torch.equal(c.d["kc"][p3], before["kc"][p3])
    p0 = int(c.table[0, 1])
    assert torch.equal(c.d["kc"][p0], before["kc"][p0])
    c.d_lens.copy_(torch.tensor([100, 70, 40]))
    out = [torch.full((110, 2, 128), 3.0, dtype=c.dt, device="cuda") for _ in range(2)]
    lib.mc_layer_q4_read(c.cfg, c.batch, c.layer, None, *out, torch.tensor([0, 100, 100, 110], dtype=torch.int32, device="cuda"))
    assert c.status()[0][0] == 4
    assert (out[0][32:64] == 3).all() and not (out[0][:32] == 3).any() and not (out[0][64:100] == 3).any()
    c.layer.status.zero_()
    # a length over its bound is cut to it, a negative one to nothing; a negative begin reads nothing
    c.d_lens.copy_(torch.tensor([161, -1, 40]))
    lib.mc_layer_q4_read(c.cfg, c.batch, c.layer, None, *out, torch.tensor([0, 0, 100, 110], dtype=torch.int32, device="cuda"))
    assert c.status()[0][0] == 4
    c.layer.status.zero_()
    c.d_lens.copy_(torch.tensor([32, 70, 40]))
    out = [torch.full((110, 2, 128), 3.0, dtype=c.dt, device="cuda") for _ in range(2)]
    lib.mc_layer_q4_read(c.cfg, c.batch, c.layer, torch.tensor([-1, 0, 0], dtype=torch.int32, device="cuda"), *out,
                         torch.tensor([0, 20, 100, 110], dtype=torch.int32, device="cuda"))
    assert c.status()[0][0] == 4 and (out[0][:20] == 3).all()


def test_appended_pages_are_what_the_merge_of_4_bit_layers_reads(Q):
    """Prompts of whole pages through mc_layer_q4_append are, bit for bit, the layers that mc_merge_pair_q4 takes."""
    import gen
    S, H = 96, 4
    c = Q.Cache([0, 0], H, H, "f16", seed=12, room=S, max_len=S, empty=True)
    k, v = c.rows(2 * S, H), c.rows(2 * S, H)
    append(c, [S, S], k.cuda(), v.cuda())
    for x, kind, codes, meta in ((k, "k", "kc", "km"), (v, "v", "vc", "vm")):
        q = gen.quantise_q4(x.view(2, S, H, 128), kind)
        for b in range(2):
            for s in range(S // 32):
                page = int(c.table[b, s])
                assert torch.equal(c.d[codes][page].cpu(), q["codes"][b, 32 * s:32 * s + 32].transpose(0, 1))
                m = q["meta"][b, s] if kind == "k" else q["meta"][b, 32 * s:32 * s + 32].transpose(0, 1)
                assert torch.equal(c.d[meta][page].cpu(), m)
