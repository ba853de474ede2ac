"""Host-only checks of the mc_layer_q4_* entry points: what they refuse, before anything touches a GPU."""
import ctypes as C

import pytest
import torch

import paper_2405_14366_b200 as mc
from paper_2405_14366_b200 import binding as B
from paper_2405_14366_b200.build import build_library

NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    build_library()
    return mc.lib()._lib


def cfg(**kw):
    d = dict(n_kv_heads=8, n_q_heads=32, head_dim=128, page_size=32, dtype=0, retain_mode=0, t=0.6, gamma=0.05, merge_fn=0, cache_bits=4)
    d.update(kw)
    return B._Config(*d.values())


def batch(bt=0x1000, sl=0x2000, batch=2, mpps=4, max_len=128, n_pages=10):
    return B._Batch(bt, sl, batch, mpps, max_len, 0, n_pages)


def layer(**kw):
    d = dict(k_codes=0x10000, k_meta=0x20000, v_codes=0x30000, v_meta=0x40000, res_k=0x50000, res_v=0x60000, status=0x70000)
    d.update(kw)
    return B._LayerQ4Cache(*d.values())


def opts(slopes=0, doc=0, prefix=0, q_pos=0, sm=0.1, cap=0.0, window=0):
    return B._ScoreOpts(slopes, doc, prefix, q_pos, sm, cap, window, 0)


CFG = [(dict(head_dim=64), 2), (dict(page_size=16, cache_bits=0), 2), (dict(page_size=64, cache_bits=0), 2), (dict(n_q_heads=12), 2), (dict(dtype=2), 3)]
BATCH = [(dict(batch=-1), 1), (dict(bt=0), 1), (dict(sl=0), 1), (dict(max_len=129), 2), (dict(batch=513), 2), (dict(n_pages=0), 1),
         (dict(n_pages=1 << 40), 2), (dict(max_len=2 ** 30 + 1, mpps=2 ** 26), 2), (dict(batch=512, max_len=2 ** 25, mpps=2 ** 21), 2)]
LAYER = [(dict([(k, 0)]), 1) for k in ("k_codes", "k_meta", "v_codes", "v_meta", "res_k", "res_v", "status")]
LAYER += [(dict([(k, 0x10080)]), 4) for k in ("k_codes", "k_meta", "v_codes", "v_meta", "res_k", "res_v")] + [(dict(status=0x70002), 4)]
OPTS = [(dict(sm=NAN), 1), (dict(sm=INF), 1), (dict(cap=-1.0), 1), (dict(cap=NAN), 1), (dict(window=-1), 1), (dict(q_pos=0x1001), 4),
        (dict(doc=0x1001), 4), (dict(prefix=0x1001), 4)]


def common(call):
    for kw, code in CFG:
        assert call(c=cfg(**kw)) == code, kw
    for kw, code in BATCH:
        assert call(b=batch(**kw)) == code, kw
    for kw, code in LAYER:
        assert call(l=layer(**kw)) == code, kw
    for i in range(3):
        assert call(null=i) == 1


def head(c, b, l, null):
    x = [C.byref(c or cfg()), C.byref(b or batch()), C.byref(l or layer())]
    if null is not None:
        x[null] = None
    return x


@pytest.mark.parametrize("read", [False, True])
def test_rows_refusals(L, read):
    def call(c=None, b=None, l=None, null=None, k=0x100000, v=0x200000, ks=1024, vs=1024, off=0x300000, rows=64, begin=0):
        f = L.mc_layer_q4_read if read else L.mc_layer_q4_append
        return f(*head(c, b, l, null), *([begin] if read else []), k, v, ks, vs, off, rows, None)
    common(call)
    assert call(k=0) == 1 and call(v=0) == 1 and call(off=0) == 1 and call(rows=-1) == 1 and call(rows=1 << 30) == 1
    assert call(ks=1016) == 2 and call(vs=0) == 2 and call(ks=-1024) == 2 and call(vs=(1 << 31) + 8) == 2
    assert call(ks=1028) == 4 and call(k=0x100008) == 4 and call(v=0x200002) == 4 and call(off=0x300002) == 4
    if read:
        assert call(begin=0x1002) == 4
    # nothing to do: no launch
    assert call(rows=0, k=0, v=0) == 0 and call(b=batch(batch=0, bt=0, sl=0)) == 0


def test_select_refusals(L):
    def call(c=None, b=None, l=None, null=None, o=None, keep=(4, 1, 1), q=0x100000, pages=0x200000, counts=0x300000, ws=0x500000, n=1 << 30):
        o = o or opts()
        return L.mc_layer_q4_select(*head(c, b, l, null), C.byref(o), C.byref(B._PageSelection(*keep, 0)), q, pages, counts, ws, n, None)
    common(call)
    for kw, code in OPTS + [(dict(slopes=0x1000), 6), (dict(sm=0.0), 6), (dict(sm=-1.0), 6)]:
        assert call(o=opts(**kw)) == code, kw
    for keep in ((0, 0, 0), (-1, 0, 0), (4, -1, 0), (4, 0, -1), (4, 3, 2), (2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 1)):
        assert call(keep=keep) == 1, keep
    assert call(q=0) == 1 and call(pages=0) == 1 and call(counts=0) == 1
    assert call(q=0x100008) == 4 and call(pages=0x200002) == 4 and call(counts=0x300001) == 4
    assert call(counts=0x2000) == 1 and call(counts=0x2004) == 1 and call(o=opts(q_pos=0x300004)) == 1  # over what it reads
    assert call(ws=0) == 1 and call(ws=0x500080) == 4 and call(n=16) == 5
    assert call(b=batch(max_len=2 ** 19 + 1, mpps=2 ** 16)) == 2
    assert call(b=batch(batch=0, bt=0, sl=0)) == 0
    c, b, l, o = cfg(), batch(), layer(), opts()
    assert L.mc_layer_q4_select(C.byref(c), C.byref(b), C.byref(l), None, C.byref(B._PageSelection(4, 0, 0, 0)), 16, 16, 0x300000, 0x500000, 1 << 30, None) == 1
    assert L.mc_layer_q4_select(C.byref(c), C.byref(b), C.byref(l), C.byref(o), None, 16, 16, 0x300000, 0x500000, 1 << 30, None) == 1


def test_attn_refusals(L):
    def call(c=None, b=None, l=None, null=None, o=None, pages=0, counts=0, stride=0, q=0x100000, kn=0x200000, vn=0x300000, flags=0, out=0x400000,
             lse=0, ws=0x500000, n=1 << 30):
        o = o or opts()
        return L.mc_layer_q4_attn(*head(c, b, l, null), C.byref(o), pages, counts, stride, q, kn, vn, flags, out, lse, ws, n, None)
    common(call)
    for kw, code in OPTS + [(dict(slopes=0x1002), 4)]:
        assert call(o=opts(**kw)) == code, kw
    assert call(q=0) == 1 and call(out=0) == 1 and call(kn=0) == 1 and call(vn=0) == 1 and call(kn=0, vn=0, flags=1) == 1
    assert call(flags=2) == 1 and call(flags=-1) == 1
    assert call(pages=0x600000) == 1 and call(counts=0x600000) == 1 and call(stride=4) == 1 and call(pages=0x600000, counts=0x700000) == 1
    assert call(pages=0x600002, counts=0x700000, stride=4) == 4 and call(pages=0x600000, counts=0x700002, stride=4) == 4
    assert call(q=0x100008) == 4 and call(out=0x400004) == 4 and call(kn=0x200008) == 4 and call(lse=0x2) == 4
    assert call(ws=0) == 1 and call(ws=0x500080) == 4 and call(n=16) == 5
    assert call(b=batch(batch=0, bt=0, sl=0)) == 0
    assert L.mc_layer_q4_read_status(None, None, None) == 1 and L.mc_layer_q4_read_status(C.byref(layer(status=0)), None, (C.c_int32 * 4)()) == 1


def test_workspace_refusals(L):
    out = C.c_size_t(0)

    def call(op, arg=0, c=None, b=None):
        return L.mc_layer_workspace_bytes(C.byref(c or cfg()), C.byref(b or batch(bt=0, sl=0)), op, arg, C.byref(out))
    for op in (5, 6):
        assert call(op) == 0 and out.value % 256 == 0 and out.value > 0
        assert call(op, 2) == 1 and call(op, c=cfg(page_size=16, cache_bits=0)) == 2
        assert call(op, b=batch(batch=513)) == 2 and call(op, b=batch(max_len=2 ** 30 + 1)) == 2 and call(op, b=batch(batch=512, max_len=2 ** 25)) == 2
    assert call(5, 1) == 0 and call(6, 1) == 1 and call(6, b=batch(max_len=2 ** 19 + 1)) == 2 and call(7) == 1


def test_binding_refuses_other_tensors():
    c = mc.McConfig(2, 4, 32, "f16")
    t = torch.zeros(2, 4, dtype=torch.int32)
    b = mc.Batch(t, torch.zeros(2, dtype=torch.int32), 128, 8)
    l = mc.LayerQ4Cache.empty(c, 2, 8, device="cpu")
    lib, off = mc.lib(), torch.zeros(3, dtype=torch.int32)
    k = torch.zeros(10, 2, 128, dtype=torch.float16)
    for bad in (k.float(), k[:, :1], k.transpose(0, 1), torch.zeros(10, 2, 256, dtype=torch.float16)[..., ::2], k[:5],
                torch.zeros(10, 4, 128, dtype=torch.float16)[:, ::2]):
        with pytest.raises(AssertionError):
            lib.mc_layer_q4_append(c, b, l, bad, k, off)
        with pytest.raises(AssertionError):
            lib.mc_layer_q4_read(c, b, l, None, k, bad, off)
    for args in ((k, k, off[:2]), (k, k, off.long()), (k, k, off)):  # the last one: not on a CUDA device
        with pytest.raises(AssertionError):
            lib.mc_layer_q4_append(c, b, l, *args)
    q, ws = torch.zeros(2, 4, 128, dtype=torch.float16), torch.zeros(1 << 20, dtype=torch.uint8)
    pages, counts = torch.zeros(2, 2, 3, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    o = mc.ScoreOpts(0.1)
    for args in ((q[:1], pages, counts), (q, pages[:, :, :2], counts), (q, pages, counts[:1]), (q, pages.long(), counts), (q, pages, counts)):
        with pytest.raises(AssertionError):
            lib.mc_layer_q4_select(c, b, l, o, mc.PageSelection(3), *args, ws)
    out = torch.zeros_like(q)
    for args in ((pages, None, q, None, None), (pages[:1], counts, q, None, None), (None, None, q[:1], None, None), (None, None, q, q, q),
                 (None, None, q, None, None)):
        with pytest.raises(AssertionError):
            lib.mc_layer_q4_attn(c, b, l, o, *args, 0, out, None, ws)
    small = mc.LayerQ4Cache.empty(c, 2, 7, device="cpu")
    with pytest.raises(AssertionError):
        small.c(2, 8)
    with pytest.raises(AssertionError):
        mc.LayerQ4Cache.empty(c, 1, 8, device="cpu").c(2, 8)
