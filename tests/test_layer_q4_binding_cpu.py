"""Host-only: what the binding passes on for tensors of rows whose stride no element depends on."""
import torch

import paper_2405_14366_b200 as mc
from paper_2405_14366_b200 import binding as B


def test_one_row_has_no_stride():
    """A single row (or none) may come with any stride: the library is given the packed one, which it takes."""
    c = mc.McConfig(2, 4, 32, "f16")
    x = torch.zeros(4096, dtype=torch.float16)
    for step in (1, 130, 260, 259, 512, (1 << 31) + 8):
        for rows in (0, 1):
            assert B._row_stride("k", x.as_strided((rows, 2, 128), (step, 128, 1)), c, rows, -1) == 256, (rows, step)
    assert B._row_stride("k", x.as_strided((3, 2, 128), (512, 128, 1)), c, 3, -1) == 512
