"""How a call of verify_drafts is dealt out: the sizes of the GPU tests reach every loop of its kernels, on the chip's 256 CUs."""
import pytest

from paper_2505_24034_amd import binding
from test_gpu_verify import SIZES
from test_gpu_verify_batch import BATCHES, MASKED

CUS = 256


def _plan(B, K, V, model):
    """chunks a workgroup, workgroups a row, units a workgroup, workgroups a sequence"""
    return binding._load_native().verify_plan(B * (K + 1) + (B * K if model else 0), B, V, CUS)


def test_several_chunks_of_a_workgroup():
    masked = [_plan(*c) for c in MASKED]
    assert all(each >= 2 and groups >= 2 for each, groups, _, _ in masked)
    assert {p[0] for p in masked + [_plan(*c) for c in BATCHES]} == {1, 2, 3, 4}
    # a last workgroup of fewer chunks than the others
    assert any(-(-V // 8192) % p[0] for (_, _, V, _), p in zip(MASKED, masked) if p[1] > 1)


def test_several_units_of_a_workgroup():
    plans = [(_plan(*c), -(-c[2] // 2048)) for c in MASKED + BATCHES]
    assert any(some >= 2 and groups >= 2 for (_, _, some, groups), _ in plans)
    alone = {units for (_, _, _, groups), units in plans if groups == 1 and units <= 4}      # sums that stay in the workgroup
    assert alone >= {2, 3, 4}
    assert any(groups == 1 and units > 4 for (_, _, _, groups), units in plans)
    assert any(groups >= 2 and some == 1 for _, _, some, groups in (_plan(B, K, V, True) for B, K, V in SIZES))


@pytest.mark.parametrize("cus", [1, 64, 256])
def test_everything_is_dealt_out(cus):
    rules = binding._load_native()
    for B in (1, 2, 63, 1000, (1 << 20) - 1):
        for per in (1, 2, 9, 255):
            for V in (1, 2048, 2049, 8193, 128256, (1 << 21) - 1):
                each, row_groups, some, pick_groups = rules.verify_plan(B * per, B, V, cus)
                chunks, units = -(-V // 8192), -(-V // 2048)
                assert 1 <= each <= 4 and (row_groups - 1) * each < chunks <= row_groups * each
                assert 1 <= some <= units and (pick_groups - 1) * some < units <= pick_groups * some
                assert B * pick_groups <= B + 2 * cus                      # all at once, or one a sequence
