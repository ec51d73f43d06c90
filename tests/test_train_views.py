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


@pytest.mark.parametrize("seed", range(4))
def test_results_against_the_other_tensors(pda, seed):  # noqa: F811
    """Random views in one small arena: refused where a result or the workspace shares a byte with another tensor, and only there."""
    from paper_2511_12056_amd.binding import AttnBwdStrides
    rng = random.Random(seed)
    d, base, counts = 64, 1 << 40, {False: 0, True: 0}
    while min(counts.values()) < 400:
        B, H, Sq, Skv, out_type = rng.randint(1, 3), rng.randint(1, 3), rng.choice([1, 2, 4]), rng.choice([1, 3, 4]), rng.randint(0, 1)
        n = {t: (Sq if t in ("dout", "q", "out", "lse", "dq") else Skv) * (1 if t == "lse" else d) for t in ("dout", "q", "k", "v", "out", "lse", "dq", "dk", "dv")}
        size = {t: 4 if t == "lse" or (t == "out" and not out_type) else 2 for t in n}
        # interleaved along one axis of a common tensor: twelve places a step, each as wide as the widest tensor
        wide = max(n[t] * size[t] for t in n)
        step = 12 * wide
        lie = rng.choice([0.0, 0.15])
        strides, at = {}, {}
        for t in n:
            inner, outer = step, step * (H if rng.random() < 0.8 else H + 1)
            batch, head = (outer, inner) if rng.random() < 0.7 else (inner, step * B)
            if t not in ("dq", "dk", "dv") and rng.random() < 0.2:
                batch = rng.choice([0, batch])
                head = rng.choice([0, head])
            strides[t] = (batch // size[t], head // size[t])
        strides["v"], strides["dv"] = strides["k"], strides["dk"]
        places = rng.sample(range(12), 10)
        for t, place in zip(list(n) + ["ws"], places):
            at[t] = place * wide
            if rng.random() < lie:
                at[t] = rng.choice([rng.choice(places) * wide, max(0, at[t] + rng.choice([-16, 16, 1024, -256]))]) // 16 * 16
        stat = 256 + (B * H * 64 * 16 + 255) // 256 * 256      # the workspace's size at d = 64: one that is in the way of nothing has room elsewhere
        at["ws"] = rng.choice([64 * step, 64 * step, at["ws"] // 256 * 256])
        blocks = {t: [(at[t] + size[t] * (b * strides[t][0] + h * strides[t][1]), n[t] * size[t]) for b in range(B) for h in range(H)] for t in n}
        blocks["ws"] = [(at["ws"], stat)]
        apart = lambda x, y: all(a + m <= b or b + k <= a for a, m in blocks[x] for b, k in blocks[y])  # noqa: E731
        if any(a + m > b for t in ("dq", "dk", "dv") for (a, m), (b, _) in zip(sorted(blocks[t]), sorted(blocks[t])[1:])):
            continue
        results = ["dq", "dk", "dv"]
        shared = [(x, y) for i, x in enumerate(results) for y in [t for t in n if t not in results] + results[:i] if not apart(x, y)]
        shared += [("ws", t) for t in n if not apart("ws", t)]
        st = AttnBwdStrides(*(v for t in ("dout", "q", "k", "out", "lse", "dq", "dk") for v in strides[t]))
        args = {t: base + at[t] for t in n}
        # one byte less than the statistics need: a call whose tensors are apart is refused for that
        rc = _bwd(pda, strides=st, B=B, H=H, Sq=Sq, Skv=Skv, n_v=Skv, d=d, out_type=out_type, ws=base + at["ws"], ws_bytes=stat, **args) if shared else \
            _bwd(pda, strides=st, B=B, H=H, Sq=Sq, Skv=Skv, n_v=Skv, d=d, out_type=out_type, ws=base + at["ws"], ws_bytes=stat - 1, **args)
        assert rc == 1, (rc, pda.last_error())
        counts[bool(shared)] += 1
        if shared:
            words = pda.last_error().split(": ")[-1]
            assert "overlaps" in words, (shared, words)
            x, _, y = words.partition(" overlaps ")
            assert (x.replace("workspace", "ws"), y) in shared, (shared, words)
        else:
            assert "at least" in pda.last_error(), pda.last_error()


@pytest.mark.parametrize("B,H", [(2, 0), (0, 2), (3, 0)])
def test_no_heads_or_batches_share_nothing(pda, B, H):  # noqa: F811
    assert _bwd(pda, strides=_strides(pda, dq_batch=0, dq_head=0, dkv_batch=0, dkv_head=0), B=B, H=H) == 0, pda.last_error()


def test_a_workspace_of_any_size_is_compared(pda):  # noqa: F811
    for size in ((1 << 63) - 1, 1 << 62):
        assert _bwd(pda, ws=256, ws_bytes=size) == 1 and "workspace overlaps dout" in pda.last_error(), pda.last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [128, 64])
def test_views_side_by_side_in_one_tensor(d):
    """All nine tensors interleaved head by head in two allocations, results among inputs."""
    import torch
    import paper_2511_12056_amd as pda
    from tests.test_gpu_attn_bwd import _forward_call
    B, H, S, n_v = 2, 3, 130, 121
    x = _forward_call(B, H, S, S, d, n_v, 4)
    want = pda.attn_bwd(*x, *(torch.empty_like(t) for t in x[1:4]), d ** -0.5, n_v)
    big = torch.full((B, H, 7, S, d), 7.0, device="cuda", dtype=torch.bfloat16)
    flat = torch.full((B, H, S * (d + 1) + 2), 7.0, device="cuda")[:, :, :S * (d + 1)]           # heads start at multiples of 16 bytes
    for i in range(4):
        big[:, :, i] = x[i]
    out, lse = flat[:, :, :S * d].unflatten(2, (S, d)), flat[:, :, S * d:]
    out.copy_(x[4])
    lse.copy_(x[5])
    got = pda.attn_bwd_strided(*(big[:, :, i] for i in range(4)), out, lse, *(big[:, :, i] for i in (4, 5, 6)), d ** -0.5, n_v)
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and all(torch.equal(big[:, :, i], x[i]) for i in range(4))
    with pytest.raises(pda.PdaError, match="dv overlaps v"):
        pda.attn_bwd_strided(*(big[:, :, i] for i in range(4)), out, lse, *(big[:, :, i] for i in (4, 5, 3)), d ** -0.5, n_v)
