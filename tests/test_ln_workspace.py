"""Workgroups that layer norm's gradient plans for few rows, as its workspace shows them."""
import pytest


def _chunks(rows, D, groups=1, n_cu=256):
    import paper_2511_12056_amd as pda
    n = pda.layer_norm_bwd_workspace_bytes(rows, D, groups, n_cu)
    assert n % (groups * 2 * D * 4) == 0
    return n // (groups * 2 * D * 4) or 1


def _at_once(D):
    """Rows of a workgroup."""
    return 16 if D <= 64 else 8 if D <= 128 else 4 if D <= 512 else 1


@pytest.mark.parametrize("D", [1, 7, 64, 65, 100, 128, 129, 256, 500, 512, 513, 1024, 2048, 8192])
def test_no_workgroup_without_rows(D):
    for groups in (1, 2, 7, 300):
        for per in (1, 3, 4, 5, 8, 9, 16, 17, 33, 100, 250, 999, 1000, 4096, 40_000):
            for n_cu in (256, 304, 64, 1):
                c = _chunks(per * groups, D, groups, n_cu)
                assert (c - 1) * _at_once(D) < per, (D, groups, per, n_cu, c)        # the last workgroup's first rows are there


def test_rows_of_one_workgroup_need_no_workspace():
    assert _chunks(16, 64) == _chunks(8, 128) == _chunks(4, 512) == 1
    assert _chunks(17, 64) == _chunks(9, 128) == 2


@pytest.mark.gpu
@pytest.mark.parametrize("rows,D,groups", [(16, 64, 1), (17, 64, 1), (8, 128, 1), (9, 100, 1), (48, 30, 3), (100, 64, 1), (1000, 64, 1), (1000, 128, 2), (5, 4, 1), (70, 128, 7)])
def test_gradients_of_few_rows(rows, D, groups):
    from tests.test_gpu_layer_norm import test_against_the_oracle
    test_against_the_oracle(rows, D, groups, "fp32", "bf16")
