"""The mc_layer_* calls next to other work: behind a kernel that uses tensor memory, from several host threads, and with
other contents in the rows that do not count."""
import math

import numpy as np
import pytest
import torch

import gen
from gen import CONFIGS

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


@pytest.mark.parametrize("lens,Hq,J", [([512, 300], 8, 40), ([700, 1], 2, 128), ([4200, 77], 8, 20)])
@pytest.mark.parametrize("graph", [False, True])
def test_observe_behind_a_prefill_merge(L, lens, Hq, J, graph):
    """Both take tensor memory: the merge in a layer's projection, then the weights of a prompt, without a pause, in turn: the
    bits of calls that find the device idle.  (Short prompts of more than 128 rows, of one and of two tiles per CTA; a long one.)"""
    import mc_harness
    wl = CONFIGS["c1"].scaled("pf", n_kv_heads=8, n_q_heads=8, dtype="bf16", batch=4, seq_len=512, index=68)
    case = {k: v.cuda() for k, v in gen.make_projection_case(wl, 0, 1024, 512).items()}
    zeros = torch.zeros_like(case["k_lm1"]).cpu()
    p = mc_harness.Problem(wl, seq_lens=np.asarray([512, 512, 400, 512], np.int32),
                           tensors={"k_lm1": case["k_lm1"].cpu(), "v_lm1": case["v_lm1"].cpu(), "k_l": zeros, "v_l": zeros.clone()})
    ws_p, pools = p.workspace(0), [p.pools[k] for k in ("k_lm1", "v_lm1", "k_l", "v_l")]
    c = L.Cache(lens, 2, Hq, 16, "bf16", seed=3, weights=True)
    mc, lib = c.mc, c.mc.lib()
    q, ws = c.queries(len(lens), J, Hq).cuda(), c.workspace(mc.MC_OP_LAYER_OBSERVE, J)

    def run(pause, times):
        for i in range(times):
            lib.mc_prefill_merge_pair(p.cfg, p.batch(), case["x"], case["w_k"], case["w_v"], *pools, p.pair, 0.9, i % 2 == 0, ws_p)
            pause()
            lib.mc_layer_observe(c.cfg, c.batch, c.layer, mc.ScoreOpts(SM), q, mc.MC_LAYER_ACCUMULATE if i else 0, ws)
            pause()
    got = []
    for idle in (True, False):
        c.d["w"].zero_()
        p.pair.e_k.zero_()
        torch.cuda.synchronize()
        if idle or not graph:
            run(torch.cuda.synchronize if idle else lambda: None, 20)
        else:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                run(lambda: None, 20)
            g.replay()
        torch.cuda.synchronize()
        assert lib.mc_layer_read_status(c.layer, check=False)[1] == 0
        got.append([c.d["w"].clone(), p.pair.e_k.clone().view(torch.int16)])
    assert all(torch.equal(a, b) for a, b in zip(*got)) and float(got[0][0].sum()) > 0
