"""Host-only checks of the mc_layer_* entry points: what they refuse, before anything touches a GPU."""
import ctypes as C

import pytest
import torch

import paper_2405_14366_b200 as mc
from paper_2405_14366_b200 import binding as B
from paper_2405_14366_b200.build import build_library

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    build_library()
    return mc.lib()


def cfg(**kw):
    d = dict(n_kv_heads=8, n_q_heads=32, head_dim=128, page_size=16, dtype=0, retain_mode=0, t=0.6, gamma=0.05, merge_fn=0, cache_bits=0)
    d.update(kw)
    return B._Config(*d.values())


def batch(bt=0x1000, sl=0x2000, batch=2, mpps=4, max_len=64, n_pages=10):
    return B._Batch(bt, sl, batch, mpps, max_len, 0, n_pages)


def layer(k=0x10000, v=0x20000, pos=0x30000, w=0x40000, st=0x50000):
    return B._LayerCache(k, v, pos, w, st)


def opts(slopes=0, doc=0, prefix=0, q_pos=0, sm=0.1, cap=0.0, window=0):
    return B._ScoreOpts(slopes, doc, prefix, q_pos, sm, cap, window, 0)


CFG = [(dict(head_dim=64), 2), (dict(page_size=8), 2), (dict(n_q_heads=12), 2), (dict(dtype=2), 3), (dict(cache_bits=4, page_size=32), 6)]
BATCH = [(dict(batch=-1), 1), (dict(bt=0), 1), (dict(sl=0), 1), (dict(max_len=65), 2), (dict(batch=513), 2), (dict(n_pages=0), 1),
         (dict(n_pages=1 << 40), 2)]
LAYER = [(dict(k=0), 1), (dict(v=0), 1), (dict(st=0), 1), (dict(k=0x10010), 4), (dict(pos=0x30004), 4), (dict(w=0x40004), 4), (dict(st=0x50002), 4)]
OPTS = [(dict(sm=NAN), 1), (dict(sm=INF), 1), (dict(cap=-1.0), 1), (dict(cap=NAN), 1), (dict(cap=INF), 1), (dict(window=-1), 1),
        (dict(slopes=0x1002), 4), (dict(q_pos=0x1001), 4), (dict(doc=0x1001), 4), (dict(prefix=0x1001), 4)]


def attn(lib, c=None, b=None, l=None, o=None, q=0x100000, kn=0x200000, vn=0x300000, flags=0, out=0x400000, lse=0, ws=0x500000, n=1 << 30):
    c, b, l, o = c or cfg(), b or batch(), l or layer(), o or opts()
    return lib._lib.mc_layer_attn(C.byref(c), C.byref(b), C.byref(l), C.byref(o), q, kn, vn, flags, out, lse, ws, n, None)


def test_layer_attn_refusals(lib):
    for kw, code in CFG:
        assert attn(lib, c=cfg(**kw)) == code, kw
    for kw, code in BATCH:
        assert attn(lib, b=batch(**kw)) == code, kw
    for kw, code in LAYER:
        assert attn(lib, l=layer(**kw)) == code, kw
    for kw, code in OPTS:
        assert attn(lib, o=opts(**kw)) == code, kw
    assert attn(lib, q=0) == 1 and attn(lib, out=0) == 1 and attn(lib, kn=0) == 1 and attn(lib, vn=0) == 1
    assert attn(lib, kn=0, vn=0, flags=1) == 1  # nothing to append
    assert attn(lib, l=layer(w=0), flags=2) == 1  # nowhere to gather
    assert attn(lib, flags=4) == 1 and attn(lib, flags=-1) == 1
    assert attn(lib, q=0x100008) == 4 and attn(lib, out=0x400004) == 4 and attn(lib, kn=0x200008) == 4 and attn(lib, lse=0x2) == 4
    assert attn(lib, ws=0) == 1 and attn(lib, ws=0x500080) == 4 and attn(lib, n=16) == 5
    L = lib._lib
    c, b, l, o = cfg(), batch(), layer(), opts()
    for args in ((None, C.byref(b), C.byref(l), C.byref(o)), (C.byref(c), None, C.byref(l), C.byref(o)),
                 (C.byref(c), C.byref(b), None, C.byref(o)), (C.byref(c), C.byref(b), C.byref(l), None)):
        assert L.mc_layer_attn(*args, 0x100000, None, None, 0, 0x400000, None, 0x500000, 1 << 30, None) == 1
    assert L.mc_layer_read_status(None, None, None) == 1


def test_layer_observe_refusals(lib):
    L = lib._lib

    def obs(c=None, b=None, l=None, o=None, q=0x100000, n_obs=32, flags=0, ws=0x500000, n=1 << 30):
        c, b, l, o = c or cfg(), b or batch(), l or layer(), o or opts()
        return L.mc_layer_observe(C.byref(c), C.byref(b), C.byref(l), C.byref(o), q, n_obs, flags, ws, n, None)
    for kw, code in CFG:
        assert obs(c=cfg(**kw)) == code, kw
    for kw, code in BATCH:
        assert obs(b=batch(**kw)) == code, kw
    for kw, code in LAYER + [(dict(w=0), 1)]:
        assert obs(l=layer(**kw)) == code, kw
    for kw, code in OPTS:
        assert obs(o=opts(**kw)) == code, kw
    assert obs(q=0) == 1 and obs(n_obs=0) == 1 and obs(n_obs=-3) == 1 and obs(flags=1) == 1 and obs(flags=4) == 1
    assert obs(n_obs=65) == 2 and obs(c=cfg(n_kv_heads=32), n_obs=257) == 2 and obs(n_obs=1 << 30) == 2
    assert obs(q=0x100008) == 4 and obs(ws=0) == 1 and obs(ws=0x500080) == 4 and obs(n=16) == 5


def test_layer_evict_refusals(lib):
    L = lib._lib

    def ev(c=None, b=None, l=None, o=(0, 100, 4, 10), nl=0x600000, ws=0x500000, n=1 << 30):
        c, b, l, o = c or cfg(), b or batch(), l or layer(), B._EvictOpts(*o, 0)
        return L.mc_layer_evict(C.byref(c), C.byref(b), C.byref(l), C.byref(o), nl, ws, n, None)
    for kw, code in CFG:
        assert ev(c=cfg(**kw)) == code, kw
    for kw, code in BATCH:
        assert ev(b=batch(**kw)) == code, kw
    for kw, code in LAYER + [(dict(w=0), 1), (dict(pos=0), 1)]:
        assert ev(l=layer(**kw)) == code, kw
    for o, code in (((0, 0, 0, 0), 1), ((0, -5, 0, 0), 1), ((0, 10, -1, 0), 1), ((0, 10, 0, -1), 1), ((0, 10, 6, 5), 1),
                    ((0, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1), 1), ((2, 10, 1, 1), 4)):
        assert ev(o=o) == code, o
    assert ev(nl=0) == 1 and ev(nl=0x600002) == 4
    assert ev(nl=0x2000) == 1 and ev(nl=0x2004) == 1 and ev(nl=0x1ffc) == 1  # over the lengths it reads
    assert ev(ws=0) == 1 and ev(ws=0x500080) == 4 and ev(n=16) == 5


def test_refusals_of_sizes_and_scales_past_the_arithmetic(lib):
    """Lengths whose 32-bit token and unit numbers would wrap, scales whose product or quotient is no number, a result
    over an input."""
    L, out = lib._lib, C.c_size_t(0)
    long = [dict(max_len=2 ** 31 - 1, mpps=2 ** 27), dict(max_len=2 ** 30 + 1, mpps=2 ** 27, batch=1),
            dict(batch=512, max_len=2 ** 27, mpps=2 ** 24)]
    for kw in long:
        b, l, e = batch(**kw), layer(), B._EvictOpts(0, 100, 4, 10, 0)
        assert attn(lib, b=b, n=1 << 60) == 2, kw
        assert L.mc_layer_observe(C.byref(cfg()), C.byref(b), C.byref(l), C.byref(opts()), 0x100000, 32, 0, 0x500000, 1 << 60, None) == 2, kw
        assert L.mc_layer_evict(C.byref(cfg()), C.byref(b), C.byref(l), C.byref(e), 0x600000, 0x500000, 1 << 60, None) == 2, kw
        for op, arg in ((2, 0), (2, 3), (3, 32), (4, 0)):
            assert L.mc_layer_workspace_bytes(C.byref(cfg()), C.byref(b), op, arg, C.byref(out)) == 2, kw
    for kw in (dict(sm=1.0, cap=1e-40), dict(cap=2.9e38), dict(sm=2.9e38), dict(sm=-2.9e38), dict(sm=1e20, cap=1e-20)):
        assert attn(lib, o=opts(**kw)) == 1, kw
    for q_pos in (0x600000, 0x600004, 0x5ffffc):  # new_lens over the positions it reads
        o = B._EvictOpts(q_pos, 100, 4, 10, 0)
        assert L.mc_layer_evict(C.byref(cfg()), C.byref(batch()), C.byref(layer()), C.byref(o), 0x600000, 0x500000, 1 << 30, None) == 1


def test_workspace_bytes(lib):
    out = C.c_size_t(0)
    L, c = lib._lib, cfg()

    def need(b, op, arg, c=c):
        code = L.mc_layer_workspace_bytes(C.byref(c), C.byref(b), op, arg, C.byref(out))
        return out.value if code == 0 else -code
    plain = need(batch(), 2, 1)
    assert plain > 0 and plain % 256 == 0
    # gathering weights keeps the scores: 4 bytes per (token, query head), whole units of 64 tokens
    for n, held in ((63, 64), (64, 128), (127, 128), (128, 192)):  # (the step's token counts)
        assert need(batch(max_len=n, mpps=9), 2, 3) - need(batch(max_len=n, mpps=9), 2, 1) == (2 * held + 2) * 32 * 4  # (and the rows' log-sum-exps)
    assert need(batch(), 2, 4) == -1 and need(batch(), 9, 0) == -1 and need(batch(), 0, 0) == -1
    assert need(batch(), 2, 0, cfg(page_size=8)) == -2
    assert need(batch(), 4, 0) >= 2 * 8 * 64 * 4 and need(batch(), 4, 1) == -1
    assert need(batch(), 3, 0) == -1 and need(batch(), 3, 65) == -2 and need(batch(), 3, 64) > need(batch(), 3, 32) > 0
    assert L.mc_layer_workspace_bytes(C.byref(c), None, 2, 0, C.byref(out)) == 1
    assert L.mc_layer_workspace_bytes(C.byref(c), C.byref(batch()), 2, 0, None) == 1


def test_binding_refuses_tensors_of_another_type_or_size():
    c = mc.McConfig(2, 4, 16, "f16")
    k = torch.zeros(3, 2, 16, 128, dtype=torch.float16)
    for bad in (dict(k_pool=k.float()), dict(k_pool=k[:2]), dict(positions=torch.zeros(3, 2, 16)), dict(weights=torch.zeros(2, 2, 16)),
                dict(weights=torch.zeros(3, 2, 32)[:, :, ::2]), dict(v_pool=k.transpose(1, 2))):
        kw = dict(k_pool=k, v_pool=k, status=torch.zeros(4, dtype=torch.int32))
        kw.update(bad)
        with pytest.raises(AssertionError):
            mc.LayerCache(c, **kw).c(3)
    for bad in (dict(alibi_slopes=torch.zeros(3)), dict(doc_start=torch.zeros(2)), dict(q_pos=torch.zeros(1, dtype=torch.int32))):
        with pytest.raises(AssertionError):
            mc.ScoreOpts(0.1, **bad).c(c, 2)


def test_binding_checks_every_call_anew(lib):
    """Against the call's own configuration, and again when a tensor it has seen has become smaller."""
    small, wide = mc.McConfig(2, 4, 16, "f16"), mc.McConfig(4, 8, 16, "f16")
    k = torch.zeros(3, 2, 16, 128, dtype=torch.float16)
    layer = mc.LayerCache(small, k, k.clone(), status=torch.zeros(B.MC_STATUS_WORDS, dtype=torch.int32))
    layer.c(3)
    layer.c(3, small)
    with pytest.raises(AssertionError):
        layer.c(3, wide)
    k.resize_(2, 2, 16, 128)
    with pytest.raises(AssertionError):
        layer.c(3)
    pos = torch.zeros(2, dtype=torch.int32)
    o = mc.ScoreOpts(0.1, q_pos=pos)
    o.c(small, 2)
    pos.resize_(1)
    with pytest.raises(AssertionError):
        o.c(small, 2)


def test_binding_refuses_host_tensors_and_short_block_tables(lib):
    c = mc.McConfig(2, 4, 16, "f16")
    k = torch.zeros(3, 2, 16, 128, dtype=torch.float16)
    layer = mc.LayerCache(c, k, k.clone(), torch.zeros(3, 2, 16, dtype=torch.int32), torch.zeros(3, 2, 16), torch.zeros(B.MC_STATUS_WORDS, dtype=torch.int32))
    lens, ws = torch.tensor([5, 7], dtype=torch.int32), torch.zeros(1 << 20, dtype=torch.uint8)
    q, new = torch.zeros(2, 4, 128, dtype=torch.float16), torch.zeros(2, dtype=torch.int32)
    ok, short = (mc.Batch(torch.zeros(n, 1, dtype=torch.int32), lens, 16, 3) for n in (2, 1))
    for batch in (ok, short):
        with pytest.raises(AssertionError, match="CUDA device" if batch is ok else "block_table"):
            lib.mc_layer_attn(c, batch, layer, mc.ScoreOpts(0.1), q, None, None, 0, q.clone(), None, ws)
        with pytest.raises(AssertionError, match="CUDA device" if batch is ok else "block_table"):
            lib.mc_layer_observe(c, batch, layer, mc.ScoreOpts(0.1), q[:, None], 0, ws)
        with pytest.raises(AssertionError, match="CUDA device" if batch is ok else "block_table"):
            lib.mc_layer_evict(c, batch, layer, mc.EvictOpts(4), new, ws)


def test_positions_and_weights_on_sixteen_byte_boundaries(lib):
    """As the parts of one allocation are: past the alignment check (the workspace is refused next), not at eight bytes."""
    for kw in (dict(pos=0x30010), dict(w=0x40040), dict(pos=0x300f0, w=0x40030)):
        assert attn(lib, l=layer(**kw), n=16) == 5, kw
    for kw in (dict(pos=0x30008), dict(w=0x40008)):
        assert attn(lib, l=layer(**kw), n=16) == 4, kw
