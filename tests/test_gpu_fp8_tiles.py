"""The product of 8-bit matrices through every form of tiles, and with more large tiles than compute units; which form a size takes is held by test_fp8_plan.py."""
import pytest

from tests.test_gpu_fp8 import _check_on_the_gpu, _quantised

pytestmark = pytest.mark.gpu

# M, N, K with more than 256 large tiles: workgroups go from one to the next, with 1 to 12 blocks of K a tile (whole words of four scales and not), rows of the result at multiples of 16 bytes
# and not, whole tiles and ragged ones
MANY = [(20000, 4608, 128), (20001, 4609, 128), (20000, 4616, 256), (19970, 4610, 384), (20000, 4608, 512), (20000, 4602, 640), (20001, 4608, 640), (20000, 4608, 1536),
        (20000, 4609, 1536), (119056, 4608, 1536), (70000, 517, 1100), (260, 80000, 900)]
# and in parts of K, the last of them shorter or not
MANY_PARTS = [(4807, 1564, 19840), (2590, 3352, 21376), (1709, 4947, 20864), (4608, 2048, 19968)]
# the forms for fewer rows in parts of K
PARTS = [(70, 66, 40000), (33, 64, 100000), (130, 140, 16384), (20, 3000, 65536), (257, 256, 24576), (366, 833, 5632), (405, 314, 13568), (472, 842, 9728)]


def _run(M, N, K, kind, block, with_bias, gap):
    """Against 64 bits, into rows that lie `gap` apart, twice to the same bits; a NaN reaches its row and column."""
    import torch
    import paper_2511_12056_amd as pda
    a, sa, b, sb = _quantised(M, N, K, kind, block)
    bias = torch.randn(N, device="cuda") * 30 if with_bias else None
    whole = torch.full((M, N + gap), 7.0, device="cuda", dtype=torch.bfloat16)
    out = whole[:, :N]
    space = torch.full((pda.fp8_matmul_workspace_bytes(M, N, K) + 256,), 0xff, dtype=torch.uint8, device="cuda")
    pda.fp8_matmul(a, sa, b, sb, out, bias=bias, workspace=space)
    _check_on_the_gpu(out, a, sa, b, sb, block, bias)
    assert (whole[:, N:] == 7).all()
    again = torch.full((M, N), 7.0, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(pda.fp8_matmul(a, sa, b, sb, again, bias=bias), out)
    a.view(torch.uint8)[M - 1, K - 1] = 0x7f
    b.view(torch.uint8)[N // 2, 5] = 0x7f
    got = pda.fp8_matmul(a, sa, b, sb, torch.full_like(again, 7.0), bias=bias)
    nan = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    nan[M - 1] = nan[:, N // 2] = True
    assert torch.equal(got.isnan(), nan) and torch.equal(torch.where(nan, 0, got), torch.where(nan, 0, again))
    del a, b, out, whole, again, got, nan
    torch.cuda.empty_cache()


@pytest.mark.parametrize("M,N,K", MANY + MANY_PARTS)
@pytest.mark.parametrize("kind,block,with_bias,gap", [("e4m3", 128, True, 0), ("e5m2", 1, True, 8), ("e4m3", 1, False, 3), ("e5m2", 128, False, 0)])
def test_more_large_tiles_than_compute_units(M, N, K, kind, block, with_bias, gap):
    _run(M, N, K, kind, block, with_bias, gap)


@pytest.mark.parametrize("M,N,K", PARTS)
@pytest.mark.parametrize("kind,block,with_bias,gap", [("e4m3", 128, True, 0), ("e5m2", 1, True, 8), ("e4m3", 1, True, 3), ("e5m2", 128, False, 0)])
def test_parts_of_k_with_few_rows(M, N, K, kind, block, with_bias, gap):
    _run(M, N, K, kind, block, with_bias, gap)
