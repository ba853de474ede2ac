"""README's decode step of an uncompressed layer, run as it stands there."""
import math
import os
import re

import pytest
import torch

pytestmark = pytest.mark.gpu


def snippet(root):
    with open(os.path.join(root, "README.md")) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    (code,) = [b for b in blocks if "mc.LayerCache(" in b]
    return code


def test_the_layer_snippet_keeps_every_token_it_appends(repo_root):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2405_14366_b200.build import build_library
    build_library()
    import paper_2405_14366_b200 as mc
    lens, H, Hq, ps, n_steps, budget, sink, recent = [1500, 1000, 3], 2, 8, 16, 100, 1024, 4, 64
    g = torch.Generator().manual_seed(1)
    per_seq = max(lens) // ps + 1 + n_steps // ps
    n_pages = len(lens) * per_seq
    table = torch.randperm(n_pages, generator=g).int().view(len(lens), per_seq)
    rows = lambda n: (torch.randn(n, H, 128, generator=g) * 0.1).half()  # noqa: E731
    k_all, v_all = [rows(n + n_steps) for n in lens], [rows(n + n_steps) for n in lens]  # by position
    k_pool, v_pool = (torch.zeros(n_pages, H, ps, 128, dtype=torch.float16, device="cuda") for _ in range(2))
    positions = torch.zeros(n_pages, H, ps, dtype=torch.int32, device="cuda")
    weights = torch.zeros(n_pages, H, ps, device="cuda")
    for b, n in enumerate(lens):
        t = torch.arange(n)
        at = (table[b, t // ps].long().cuda(), slice(None), (t % ps).cuda())
        k_pool[at], v_pool[at] = k_all[b][:n].cuda(), v_all[b][:n].cuda()
        positions[at] = t.int()[:, None].expand(n, H).cuda()
    steps = [((torch.randn(len(lens), Hq, 128, generator=g) * 28).half().cuda(),
              torch.stack([k_all[b][n + i] for b, n in enumerate(lens)]).cuda(), torch.stack([v_all[b][n + i] for b, n in enumerate(lens)]).cuda())
             for i in range(n_steps)]
    space = dict(mc=mc, torch=torch, lib=mc.lib(), cfg=mc.McConfig(H, Hq, ps, "f16"), k_pool=k_pool, v_pool=v_pool, positions=positions,
                 weights=weights, block_table=table.cuda(), seq_lens=torch.tensor(lens, dtype=torch.int32, device="cuda"),
                 max_seq_len=max(lens), n_pages=n_pages, sm_scale=1 / math.sqrt(128.0), steps=steps,
                 sinks=torch.full((len(lens),), sink, dtype=torch.int32, device="cuda"),
                 q_last=(torch.randn(len(lens), 8, Hq, 128, generator=g) * 28).half().cuda(),
                 out=torch.zeros(len(lens), Hq, 128, dtype=torch.float16, device="cuda"), lse=torch.zeros(len(lens), Hq, device="cuda"))
    exec(compile(snippet(repo_root), "README.md", "exec"), space)
    torch.cuda.synchronize()
    assert mc.lib().mc_layer_read_status(space["layer"], check=False)[1] == 0
    held = space["seq_lens"].tolist()
    assert held == [min(n + n_steps, budget) for n in lens]
    for b, n in enumerate(lens):
        t = torch.arange(held[b])
        at = (table[b, t // ps].long(), slice(None), t % ps)
        p, k, v, w = (x.cpu()[at] for x in (positions, k_pool, v_pool, weights))
        for h in range(H):
            have = p[:, h].tolist()
            assert len(set(have)) == len(have)
            guarded = set(range(min(sink, n))) | set(range(max(0, n + n_steps - recent), n + n_steps))
            assert guarded <= set(have)  # the newest tokens are all there
            assert torch.equal(k[:, h], k_all[b][have, h]) and torch.equal(v[:, h], v_all[b][have, h])
            if n + n_steps <= budget:
                assert sorted(have) == list(range(n + n_steps))
            # every step's softmax sums to 1 per query head: with nothing evicted all of it is there
            assert n + n_steps > budget or abs(float(w[:, h].sum()) - (min(8, n) + n_steps) * (Hq // H)) < 1e-3
    assert torch.isfinite(space["lse"]).all() and torch.isfinite(space["out"].float()).all()
