"""How a product of 8-bit matrices is split over workgroups (host code of the kernel's header, compiled here on its own), and that the GPU tests reach each way."""
import os
import random
import subprocess

import pytest

from tests import test_gpu_fp8, test_gpu_fp8_tiles

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_12056_amd", "csrc")
CLANG = "/opt/rocm/llvm/bin/clang++"
MAIN = r"""
#include "proj_internal.h"
#include <stdio.h>
int main() {
    long long M, N, K;
    int n_cu;
    while (scanf("%lld %lld %lld %d", &M, &N, &K, &n_cu) == 4) {
        const pda::MatmulPlan w = pda::plan_matmul(M, N, K, n_cu);
        const pda::FormSize& s = pda::kForms[w.form];
        printf("%d %d %d %d %d %lld\n", w.form, w.parts, w.part_steps, s.m, s.n, (long long)pda::matmul_workspace_bytes(w, M, N));
    }
}
"""
FEW, MID, MID_WIDE, LARGE = range(4)
CUS = 256


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("no ROCm clang++ here")
    at = tmp_path_factory.mktemp("plan")
    src, exe = at / "plan.cpp", at / "plan"
    src.write_text(MAIN)
    subprocess.run([CLANG, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", CSRC, str(src), "-o", str(exe)], check=True, timeout=120)

    def run(cases, n_cu=CUS):
        text = "\n".join(f"{M} {N} {-(-K // 128) * 128} {n_cu}" for M, N, K in cases)
        out = subprocess.run([str(exe)], input=text, capture_output=True, text=True, check=True, timeout=120).stdout
        return [tuple(int(x) for x in line.split()) for line in out.splitlines()]
    return run


def _tiles(M, N, w):
    return -(-M // w[3]) * -(-N // w[4])


def test_more_large_tiles_than_compute_units(plan):
    for cases, parts in ((test_gpu_fp8_tiles.MANY, False), (test_gpu_fp8_tiles.MANY_PARTS, True)):
        for (M, N, K), w in zip(cases, plan(cases)):
            assert w[0] == LARGE and (w[1] > 1) == parts and _tiles(M, N, w) * w[1] > CUS, (M, N, K, w)
    nk = [-(-K // 128) for _, _, K in test_gpu_fp8_tiles.MANY]
    assert 1 in nk and any(n % 4 for n in nk if n > 4) and any(n % 4 == 0 for n in nk)
    cut = [(-(-K // 128), w) for (_, _, K), w in zip(test_gpu_fp8_tiles.MANY_PARTS, plan(test_gpu_fp8_tiles.MANY_PARTS))]
    assert any(n % w[2] for n, w in cut) and any(n % w[2] == 0 for n, w in cut)


def test_every_form_alone_and_in_parts(plan):
    cases = test_gpu_fp8_tiles.PARTS
    assert {w[0] for w in plan(cases) if w[1] > 1} == {FEW, MID, MID_WIDE}
    assert all(w[1] > 1 for w in plan(cases))
    assert {w[0] for w in plan(test_gpu_fp8.MIDDLE) if w[1] == 1} == {FEW, MID, MID_WIDE, LARGE}
    assert any(w[0] == LARGE and w[1] > 1 for w in plan(test_gpu_fp8.MIDDLE))


@pytest.mark.parametrize("n_cu", [1, 64, 256, 304])
def test_parts_cover_k(plan, n_cu):
    """Nothing left out, nothing empty; ranges begin at words of four scales; the workspace holds the parts' whole tiles and is what the entry point asks for."""
    import paper_2511_12056_amd as pda
    rng = random.Random(n_cu)
    size = lambda most: int(round(most ** rng.random()))               # noqa: E731
    cases = [(size(200000), size(20000), 128 * size(2000)) for _ in range(400)]
    for (M, N, K), w in zip(cases, plan(cases, n_cu)):
        form, parts, steps, m, n, nbytes = w
        nk = K // 128
        assert 1 <= parts <= 32 and (parts - 1) * steps < nk <= parts * steps and (parts == 1 or steps % 4 == 0)
        assert nbytes == (parts * _tiles(M, N, w) * m * n * 4 if parts > 1 else 0) == pda.fp8_matmul_workspace_bytes(M, N, K, n_cu=n_cu)
