"""Cuts of an attention gradient's launch with few query rows, and the runs that they make."""
import os
import subprocess

import pytest

from tests.test_bwd_plan import CLANG, CSRC, plan  # noqa: F401

CLOCK = r"""
#include "attn_internal.h"
#include "train_internal.h"
#include <chrono>
#include <stdio.h>
int main() {
    long long Sq, n_v;
    int BH;
    while (scanf("%d %lld %lld", &BH, &Sq, &n_v) == 3) {
        double best = 1e9;
        volatile int sink = 0;
        for (int rep = 0; rep < 200; ++rep) {
            const auto a = std::chrono::steady_clock::now();
            sink = sink + pda::plan_bwd(Sq, n_v, BH, 128, 256).key_parts;
            const double t = std::chrono::duration<double>(std::chrono::steady_clock::now() - a).count();
            best = t < best ? t : best;
        }
        printf("%.3f\n", best * 1e6);
    }
}
"""


def _time(p):
    *_, end, whole, join, ws = p
    return end + join


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("BH,n_v", [(1, 60_000), (3, 67_576), (24, 9_600), (1, 5_000), (2, 1_025)])
def test_a_single_tile_of_query_rows_does_not_keep_the_query_blocks_whole(plan, BH, n_v, d):  # noqa: F811
    """Key blocks against one tile cannot be cut; the query blocks, which stream every key, still can."""
    rows = (1, 17, 31, 32, 33, 64)
    plans = plan([(BH, Sq, n_v, d, 256) for Sq in rows])
    for Sq, p in zip(rows, plans):
        assert p[6] > 1 and p[5] == BH and (Sq > 32 or p[4] == 1), (Sq, p)
    times = [_time(p) for p in plans]
    assert times == sorted(times), times                     # fewer rows take no longer


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("BH,Sq", [(1, 256), (1, 100), (2, 200), (8, 64), (3, 300)])
def test_one_block_more_than_compute_units(plan, BH, Sq, d):  # noqa: F811
    """A few query blocks end the launch on either side of as many blocks as compute units: the cuts do not become coarser there."""
    query_blocks = BH * -(-Sq // 256)
    fit = (256 - query_blocks) // BH                          # key blocks a head that still make one round
    below, above = plan([(BH, Sq, fit * 256, d, 256), (BH, Sq, fit * 256 + 1, d, 256)])
    assert below[2] + below[3] <= 256 < above[2] + above[3]
    slots = 4 * 256 // query_blocks                           # what the partial sums allow
    assert above[5] == query_blocks and above[6] > min(8, slots - 1), above
    keys = -(-Sq // 32) * 12 + 60                             # the key blocks are a second round now
    assert _time(above) <= _time(below) + keys, (below, above)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("BH,Sq,n_v", [(24, 32, 180_000), (24, 180_000, 226), (1, 17, 4_300_000), (96, 200, 45_000), (2, 2_200_000, 64)])
def test_a_few_long_blocks_among_very_many_short_ones(plan, BH, Sq, n_v, d):  # noqa: F811
    """However many blocks a launch has, the ones that stream the long side do not end it alone: with the long blocks in as many parts as there are places for, a
    launch in which each item goes to the unit that is free first ends within its work over the units and its longest item, and the kernel that adds the parts follows."""
    p, = plan([(BH, Sq, n_v, d, 256)])
    kb, qb, (sk, sq) = p[2], p[3], (-(-Sq // 32), -(-n_v // 32))
    long_keys = sk > sq
    parts = min(16, 4 * 256 // (2 * kb if long_keys else qb))
    parts = min(parts, 2 * 256 // kb) if long_keys else parts             # key blocks: at most two parts a unit in all
    steps = -(-max(sk, sq) // parts)
    key, query = (12 * (steps if long_keys else sk) + 60), (10 * (sq if long_keys else steps) + 60)
    work = kb * (parts if long_keys else 1) * key + qb * (1 if long_keys else parts) * query
    most = work // 256 + max(key, query) + 30 + 4 * 256 * d // 200
    assert kb + qb > 64 * 256 and _time(p) <= most < p[8], (p, most)


def test_planning_takes_microseconds(tmp_path):
    """Every call plans: a long launch is not simulated item by item, and one that is never cut not at all (these took 15 to 90 us: the limits are
    some four times what they take now)."""
    if not os.path.exists(CLANG):
        pytest.skip("no ROCm clang++ here")
    src, exe = tmp_path / "clock.cpp", tmp_path / "clock"
    src.write_text(CLOCK)
    subprocess.run([CLANG, "-std=c++17", "-O2", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", CSRC, str(src), "-o", str(exe)], check=True, timeout=120)
    cases = {(60_000, 8_192, 8_192): 2, (17, 119_056, 119_056): 10, (24, 67_576, 67_576): 10, (25, 120_472, 226): 60}
    out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True, check=True, timeout=60).stdout.split()
    assert len(out) == len(cases)
    for (c, most), us in zip(cases.items(), out):
        assert float(us) <= most, (c, us)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [128, 64])
@pytest.mark.parametrize("size", [(1, 2, 17, 5000, 4990), (1, 1, 1, 3000, 3000), (2, 3, 32, 2100, 2055), (1, 1, 256, 67_576, 67_500)], ids=str)
def test_few_rows_against_many_keys(size, d):
    import torch
    import paper_2511_12056_amd as pda
    from tests.test_gpu_attn_bwd import _forward_call, _near_64_bits
    B, H, Sq, Skv, n_v = size
    x = _forward_call(B, H, Sq, Skv, d, n_v, sum(size))
    got = pda.attn_bwd(*x, *(torch.full_like(t, float("nan")) for t in x[1:4]), d ** -0.5, n_v)
    for b in range(B):
        for h in range(H):
            _near_64_bits([t[b, h] for t in got], *(t[b, h] for t in x[:4]), d ** -0.5, n_v)
