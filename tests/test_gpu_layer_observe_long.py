"""mc_layer_observe where a prompt takes the two launches: every layout of rows, sign of the scale, form of the cap, mask and
query position there, against the definition in 64 bits.  (The rule for one launch or two stands beside the launch.)"""
import pytest
import torch

from test_gpu_layer_observe import L, SM, run  # noqa: F401

pytestmark = pytest.mark.gpu


def two_launches(lens, H, rows):
    """No number of tiles per CTA gives clusters of at most eight CTAs that run in one wave."""
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    tiles, segs, nt = -(-max(lens) // 128), len(lens) * H, 1 if rows <= 128 else 2
    for per in (1, 2, 4):
        cluster = -(-tiles // per)
        if per * nt <= 4 and cluster <= 8 and segs * cluster <= (sms if cluster <= 2 else sms - sms // 8 if cluster <= 4 else sms - sms // 4):
            return False
    return True


def long_run(L, lens, J, H, Hq, **kw):
    assert two_launches(lens, H, J * Hq // H)
    return run(L, lens, J, H=H, Hq=Hq, **kw)


# rows of a group: 20 (laid out four times), 33 and 64 (twice), 100 and 128 (once), 132 and 256 (two row tiles)
ROWS = [(4200, 5, 2, 8), (4200, 33, 2, 2), (4300, 16, 2, 8), (4200, 50, 1, 2), (4097, 16, 1, 8), (2300, 33, 2, 8), (2100, 32, 1, 8)]


@pytest.mark.parametrize("cap", [0.0, 0.5, 5.0, 50.0, 90.0])
@pytest.mark.parametrize("n,J,H,Hq", ROWS)
def test_forms_of_the_cap_and_signs_of_the_scale(L, n, J, H, Hq, cap):
    long_run(L, [n, 65, 2], J, H, Hq, ps=32, cap=cap)
    long_run(L, [77, n, 0], J, H, Hq, ps=16, dtype="bf16", cap=cap, sm=-0.2)
    long_run(L, [n, 129], J, H, Hq, ps=64, dtype="bf16", cap=cap, sm=3.0, scale=0.1, acc=True)
    long_run(L, [n], J, H, Hq, ps=16, cap=cap, sm=-SM, alibi=True)


@pytest.mark.parametrize("cap", [0.0, 0.5, 50.0, 90.0])
@pytest.mark.parametrize("n,J,H,Hq", ROWS)
def test_bias_positions_and_masks(L, n, J, H, Hq, cap):
    long_run(L, [n, 65, 2], J, H, Hq, ps=32, dtype="bf16", cap=cap, alibi=True, acc=True)
    long_run(L, [130, n, 0], J, H, Hq, ps=16, cap=cap, alibi=True, marks=True, window=700, prefixes=[3, 9, 0])
    long_run(L, [n, 300], J, H, Hq, ps=16, dtype="bf16", cap=cap, marks=True, sm=-SM, docs=[n // 2, 10])
    long_run(L, [n, 300], J, H, Hq, ps=64, cap=cap, window=1000, prefixes=[5, 0], docs=[n // 3, 0])


@pytest.mark.parametrize("cap", [0.0, 50.0])
@pytest.mark.parametrize("q_pos", [[-1, 0, 5], [300, 10 ** 6, 2 ** 31 - 2], [4000, 100, 255], [17, 199, 128]])
@pytest.mark.parametrize("n,J,H,Hq", ROWS)
def test_query_positions_before_inside_and_past_the_cache(L, n, J, H, Hq, q_pos, cap):
    """No positions pool: what no query sees keeps no weight, or what it had."""
    long_run(L, [n, 200, 129], J, H, Hq, ps=16, q_pos=q_pos, cap=cap)
    long_run(L, [n, 200, 129], J, H, Hq, ps=32, dtype="bf16", q_pos=q_pos, window=90, prefixes=[2, 0, 0], acc=True, cap=cap)


def test_many_segments_of_short_prompts(L):
    """One wave would not hold their clusters."""
    long_run(L, [600 - 7 * i for i in range(40)], 32, 8, 32, ps=16, dtype="bf16", cap=30.0)
    long_run(L, [300 - i for i in range(80)], 33, 2, 8, ps=32, alibi=True, cap=5.0)
    long_run(L, [130] * 200, 9, 1, 8, ps=64, marks=True, sm=-SM)
