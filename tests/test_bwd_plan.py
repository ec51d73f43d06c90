"""How an attention gradient's launch is cut into work items (host code of the kernel's header, compiled here on its own)."""
import heapq
import os
import random
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2511_12056_amd", "csrc")
CLANG = "/opt/rocm/llvm/bin/clang++"
MAIN = r"""
#include "attn_internal.h"
#include "train_internal.h"
#include <stdio.h>
int main() {
    long long Sq, n_v;
    int BH, d, n_cu;
    while (scanf("%d %lld %lld %d %d", &BH, &Sq, &n_v, &d, &n_cu) == 5) {
        const pda::BwdPlan w = pda::plan_bwd(Sq, n_v, BH, d, n_cu);
        pda::BwdPlan whole = w;
        whole.key_parts = whole.query_parts = 1;
        whole.query_cut = 0;
        printf("%d %d %d %d %d %d %d %lld %lld %lld %lld\n", w.key_per_head, w.query_per_head, w.key_blocks, w.query_blocks, w.key_parts, w.query_cut,
               w.query_parts, (long long)pda::bwd_end(w, Sq, n_v, n_cu), (long long)pda::bwd_end(whole, Sq, n_v, n_cu), (long long)pda::bwd_join_time(w, d),
               (long long)pda::bwd_workspace_bytes(w, BH, Sq, d));
    }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("no ROCm clang++ here")
    at = tmp_path_factory.mktemp("plan")
    src, exe = at / "plan.cpp", at / "plan"
    src.write_text(MAIN)
    subprocess.run([CLANG, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I", CSRC, str(src), "-o", str(exe)],
                   check=True, timeout=120)

    def run(cases):
        out = subprocess.run([str(exe)], input="\n".join(" ".join(map(str, c)) for c in cases), capture_output=True, text=True, check=True, timeout=120)
        return [tuple(int(x) for x in line.split()) for line in out.stdout.splitlines()]
    return run


def _items(Sq, n_v, w):
    """(steps, time) of every work item in the order of the launch, and a check of the ranges that the kernel takes from the plan."""
    kph, qph, kb, qb, kp, qc, qp = w
    sk, sq = -(-Sq // 32), -(-n_v // 32)

    def ranges(n, parts):
        r = [(n * j // parts, n * (j + 1) // parts) for j in range(parts)]
        assert all(a < b for a, b in r) and r[0][0] == 0 and r[-1][1] == n       # nothing empty, nothing left out
        return [b - a for a, b in r]
    items = []
    if kb and sk:
        items += [12 * max(ranges(sk, kp)) + 60] * (kb * kp)
    if qb and sq:
        items += [10 * sq + 60] * (qb - qc)
        if qc:
            items += [10 * max(ranges(sq, qp)) + 60] * (qc * qp)
    return items


def test_plans(plan):
    rng = random.Random(17)
    cases = [(1, 1, 1, 64, 256), (65535, 1, 1, 128, 256), (2, 1024, 1024, 64, 256), (1, 9600, 9600, 128, 256), (24, 16384, 570, 128, 256),
             (24, 9600, 9600, 128, 256), (3, 67576, 67476, 128, 256), (1, 1 << 20, 1 << 20, 128, 256), (1, 2000000000, 3, 64, 256), (1, 3, 2000000000, 64, 256)]
    for n_cu in (256, 256, 304, 64, 1):
        for _ in range(400):
            n = [max(1, int(2 ** rng.uniform(0, 17))) for _ in range(2)]
            cases.append((rng.choice([1, 2, 3, 8, 24, 96, rng.randint(1, 300)]), *n, rng.choice([64, 128]), n_cu))
    for (BH, Sq, n_v, d, n_cu), (*w, end, whole, join, ws) in zip(cases, plan(cases)):
        kph, qph, kb, qb, kp, qc, qp = w
        case = (BH, Sq, n_v, d, n_cu, w)
        assert (kph, qph, kb, qb) == (-(-n_v // 256), -(-Sq // 256), BH * -(-n_v // 256), BH * -(-Sq // 256)), case
        assert 1 <= kp <= 16 and 1 <= qp <= 16 and 0 <= qc <= qb and (qc > 0) == (qp > 1), case
        slots = (kb * kp * 2 if kp > 1 else 0) + qc * (qp if qc else 0)
        assert slots <= 4 * n_cu and (slots == 0) == (join == 0), case
        stat = 256 + (BH * (-(-Sq // 64) * 64) * (16 if d == 64 else 8) + 255) // 256 * 256            # the counter, the statistics
        assert ws == stat + slots * 256 * d * 4, case
        assert end + join <= whole, case                                         # a cut is made where it is expected to pay
        if kb + qb <= n_cu:
            assert kb * kp + qb - qc + qc * qp <= n_cu, case                     # one round
        if kb + qb < 20000:
            free = [0] * n_cu                                                    # the launch, unit by unit
            for t in _items(Sq, n_v, w):
                heapq.heappush(free, heapq.heappop(free) + t)
            assert max(free) == end, case
    forms = [(w[4] > 1, 0 < w[5] < w[3], w[5] == w[3]) for w in plan(cases[:7])]
    assert forms == [(False, False, False), (False, False, False), (True, False, True), (True, False, True), (True, False, False),
                     (False, True, False), (False, True, False)], forms


def test_plans_without_rows_or_keys(plan):
    for c, (*w, end, whole, join, ws) in zip([(3, 0, 5), (3, 700, 0), (3, 0, 0)], plan([(3, 0, 5, 64, 256), (3, 700, 0, 64, 256), (3, 0, 0, 64, 256)])):
        assert w[4:] == [1, 0, 1] and join == 0 and w[2] == c[0] * -(-c[2] // 256) and w[3] == c[0] * -(-c[1] // 256)


def test_workspace_of_the_entry_point(plan):
    import paper_2511_12056_amd as pda
    cases = [(1, 2, 1024, 1024, 64, 1000), (1, 24, 9600, 9600, 128, 9600), (2, 12, 16384, 600, 128, 570), (1, 1, 1, 1, 64, 1), (1, 3, 100, 70, 128, 0)]
    for (B, H, Sq, Skv, d, n_v), p in zip(cases, plan([(c[0] * c[1], c[2], c[5], c[4], 256) for c in cases])):
        assert pda.attn_bwd_workspace_bytes(B, H, Sq, Skv, d, n_v, n_cu=256) == p[-1]
