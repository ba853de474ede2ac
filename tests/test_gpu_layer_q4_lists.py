"""Which pages of a caller's list mc_layer_q4_attn attends when the list is not in order."""
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


# a list of the caller's, twelve pages: what is left of it when every entry that is no page, or not above all that count, goes
LISTS = [([5, 4, 5, 6], [5, 6]), ([7, 2, 5, 8], [7, 8]), ([99, 1, 3, 4], [1, 3, 4]), ([4, 99, 3, 7], [4, 7]), ([4, -1, 0, 7], [4, 7]),
         ([2, 2, 2, 2], [2]), ([11, 10, 11, 0], [11]), ([2 ** 31 - 1, -(2 ** 31), 12, 3], [3])]


@pytest.mark.parametrize("H,Hq", [(2, 4), (1, 8)])
@pytest.mark.parametrize("entries,count", LISTS)
def test_no_page_of_a_list_counts_twice(Q, H, Hq, entries, count):
    c = Q.Cache([400, 330], H, Hq, "f16", seed=2)
    pages = torch.tensor([entries, [0, 1, 2, 3]], dtype=torch.int32)[:, None].expand(2, H, 4).contiguous().cuda()
    q = c.queries(2, Hq)
    out, lse, q, kn, vn = A.run(Q, c, pages=pages, counts=[4, 4], q=q, check=False)
    assert c.status()[0][0] == BAD_METADATA
    for h in range(H):
        r = slice(h * c.nq, (h + 1) * c.nq)
        for b, want in ((0, count), (1, [0, 1, 2, 3])):
            o, z, tol, ztol = Q.attn64(c, b, h, q[b, r], SM, k_new=kn[b, h], v_new=vn[b, h], pages=want)
            assert ((out[b, r].cpu().double() - o).abs() <= tol).all(), (b, h)
            assert ((lse[b, r].cpu().double() - z).abs() <= ztol).all(), (b, h)


@pytest.mark.parametrize("Hq", [2, 16])
def test_long_lists_with_entries_out_of_order(Q, Hq):
    """Lists that many warps share: what an entry is measured by lies in another warp's part."""
    n = 40000
    c = Q.Cache([n, 20011], 2, Hq, "bf16", seed=3)
    g = torch.Generator().manual_seed(5)
    full = [x // 32 for x in c.lens]
    width = 700
    lists = torch.zeros(2, 2, width, dtype=torch.int32)
    want = {}
    for b in range(2):
        for h in range(2):
            l = torch.randperm(full[b], generator=g)[:width if full[b] >= width else full[b]].sort().values
            l = torch.cat([l, torch.full((width - len(l),), 2 ** 20)]).int()
            at = torch.randint(0, width, (12,), generator=g)
            l[at] = torch.randint(-3, full[b] + 3, (12,), generator=g).int()
            lists[b, h] = l
            top, keep = -1, []
            for x in l[:min(width, full[b])].tolist():
                if top < x < full[b]:
                    keep.append(x)
                    top = x
            want[b, h] = keep
    q = c.queries(2, Hq)
    out, lse, q, kn, vn = A.run(Q, c, pages=lists.cuda(), counts=[width, min(width, full[1])], q=q, check=False)
    assert c.status()[0][0] == BAD_METADATA
    for (b, h), keep in want.items():
        r = slice(h * c.nq, (h + 1) * c.nq)
        o, z, tol, ztol = Q.attn64(c, b, h, q[b, r], SM, k_new=kn[b, h], v_new=vn[b, h], pages=keep)
        assert ((out[b, r].cpu().double() - o).abs() <= tol).all(), (b, h)
        assert ((lse[b, r].cpu().double() - z).abs() <= ztol).all(), (b, h)
