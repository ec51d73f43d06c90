"""Views of the strided attention gradient: which layouts are taken and which are refused, from their addresses alone."""
import random

import pytest

from tests.test_train_host import _addr, _bwd, _strides, pda  # noqa: F401

ROW = 8 * 64                                                   # elements of a head of 8 rows
APART = "workspace"                                            # what the next check finds to complain of


def _result(pda, word, B=1, H=2, **strides):  # noqa: F811
    other = dict(dq_batch=H * ROW, dq_head=ROW, dkv_batch=H * ROW, dkv_head=ROW)
    assert _bwd(pda, strides=_strides(pda, **{**other, **strides}), B=B, H=H) == 1 and word in pda.last_error(), (B, H, strides, pda.last_error())


@pytest.mark.parametrize("which", ["dq", "dkv"])
def test_results_in_any_order_of_their_axes(pda, which):  # noqa: F811
    name = {"dq": "dq", "dkv": "dk/dv"}[which]
    s = lambda batch, head: {which + "_batch": batch, which + "_head": head}  # noqa: E731
    _result(pda, APART, 3, 4, **s(ROW, 3 * ROW))               # heads outside, batches inside
    _result(pda, APART, 3, 4, **s(ROW + 8, 3 * ROW + 64))
    _result(pda, APART, 2, 2, **s(3 * ROW, 2 * ROW))           # neither inside the other, none shared
    _result(pda, APART, 1, 4, **s(0, ROW))                     # one batch: its stride is not used
    _result(pda, APART, 4, 1, **s(ROW, 0))
    _result(pda, f"batches of {name}", 3, 4, **s(ROW, 2 * ROW))
    _result(pda, f"batches of {name}", 3, 4, **s(ROW - 8, 3 * ROW))
    _result(pda, f"batches of {name}", 2, 3, **s(2 * ROW, ROW))
    _result(pda, f"heads of {name}", 2, 3, **s(9 * ROW, ROW - 8))


def test_results_against_a_list_of_their_blocks(pda):  # noqa: F811
    rng = random.Random(1)
    seen = set()
    for _ in range(600):
        B, H = rng.randint(1, 5), rng.randint(1, 5)
        batch, head = rng.choice([0, 8, ROW // 2, ROW, ROW + 8, 2 * ROW, 3 * ROW, 4 * ROW, 5 * ROW]), rng.choice([0, ROW // 2, ROW, ROW + 16, 2 * ROW, 3 * ROW, 4 * ROW])
        at = sorted(b * batch + h * head for b in range(B) for h in range(H))
        shared = any(y - x < ROW for x, y in zip(at, at[1:]))
        seen.add(shared)
        _result(pda, "of dq overlap" if shared else APART, B, H, dq_batch=batch, dq_head=head)
    assert seen == {False, True}


@pytest.mark.gpu
@pytest.mark.parametrize("d", [128, 64])
def test_heads_outside_batches_inside(d):
    """Tensors kept as [H, B, S, d]."""
    import torch
    import paper_2511_12056_amd as pda
    from tests.test_gpu_attn_bwd import _forward_call
    x = _forward_call(3, 4, 210, 150, d, 140, 8)
    want = pda.attn_bwd(*x, *(torch.empty_like(t) for t in x[1:4]), d ** -0.5, 140)
    outside = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in x]
    grads = [torch.full_like(t.transpose(0, 1).contiguous(), 7.0).transpose(0, 1) for t in x[1:4]]
    got = pda.attn_bwd_strided(*outside, *grads, d ** -0.5, 140)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
