"""The workspace of attention gradients whose lengths vary: one buffer for the longest of them."""
import random

import pytest


@pytest.fixture(scope="module")
def pda():
    import paper_2511_12056_amd as pda
    return pda


def test_needs_do_not_grow_with_the_lengths(pda):
    """What a call needs follows from how its launch is cut; a shorter one may be cut where a longer one is not."""
    need = lambda n, S=9600, H=24: pda.attn_bwd_workspace_bytes(1, H, S, S, 128, n, n_cu=256)  # noqa: E731
    assert need(8000) > need(9600) and need(40000, 40000, 3) > need(67576, 67576, 3)


@pytest.mark.parametrize("d", [64, 128])
def test_one_workspace_for_all_lengths(pda, d):
    size, any_len = pda.attn_bwd_workspace_bytes, pda.PDA_ANY_LEN
    rng = random.Random(d)
    for B, H, Sq, Skv in ((1, 24, 9600, 9600), (1, 3, 67576, 67576), (2, 12, 4797, 4797), (1, 1, 9600, 9600), (1, 24, 16384, 600), (1, 2, 40, 70000), (3, 5, 33, 100),
                          (1, 1, 1, 1), (65535, 1, 1, 1), (1, 1, 64, 1), (1, 1, 1, 64), (2, 2, 0, 900), (2, 2, 900, 0)):
        for n_cu in (256, 304, 64, 1):
            bound = size(B, H, Sq, Skv, d, any_len, n_cu)
            assert bound % 256 == 0 and bound <= size(B, H, Sq, Skv, d, 0, n_cu) + 4 * n_cu * 256 * d * 4
            for _ in range(60):
                b, h, sq, skv = rng.randint(1, B), rng.randint(1, H), rng.choice([Sq, rng.randint(0, Sq)]), rng.choice([Skv, rng.randint(0, Skv)])
                n_v = rng.choice([skv, rng.randint(0, skv)])
                assert size(b, h, sq, skv, d, n_v, n_cu) <= bound, (b, h, sq, skv, n_v, n_cu)
                assert size(b, h, sq, skv, d, any_len, n_cu) <= bound
    assert size(0, 3, 8, 8, d, any_len, 256) == 0


def test_any_length_is_no_valid_length(pda):
    """Only the workspace's size is asked for with it."""
    p = 1 << 32
    assert pda.lib.pda_attn_bwd(p, 2 * p, 3 * p, 4 * p, 5 * p, 0, 6 * p, 7 * p, 8 * p, 9 * p, 1, 2, 8, 8, 64, 1.0, pda.PDA_ANY_LEN, None, 0, None) == 1
    assert "kv_valid_len" in pda.last_error()
    with pytest.raises(pda.PdaError, match="kv_valid_len"):
        pda.attn_bwd_workspace_bytes(1, 2, 8, 8, 64, -2, n_cu=256)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
def test_padded_batches_on_one_workspace(d):
    """A loop that keeps one buffer for its padded length: every valid length and every shorter sequence, with the bits of a workspace of its own."""
    import torch
    import paper_2511_12056_amd as pda
    B, H, S = 1, 24, 2600
    ws = pda.attn_bwd_workspace(B, H, S, S, d)
    assert ws.numel() == pda.attn_bwd_workspace_bytes(B, H, S, S, d, pda.PDA_ANY_LEN)
    assert pda.attn_bwd_workspace(B, H, S, S, d, 2500).numel() == pda.attn_bwd_workspace_bytes(B, H, S, S, d, 2500)
    g = torch.Generator(device="cuda").manual_seed(d)
    for h, sq, n_v in ((24, 2600, 2600), (24, 2600, 2300), (24, 2600, 257), (24, 2600, 1), (24, 2600, 0), (24, 700, 500), (3, 2600, 2600), (1, 1, 2600), (1, 2600, 64)):
        q, dout = (torch.randn(B, h, sq, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        k, v = (torch.randn(B, h, S, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
        out, lse = torch.empty(B, h, sq, d, device="cuda"), torch.empty(B, h, sq, device="cuda")
        pda.attn_fwd(q, k, v, out, lse, d ** -0.5, n_v)
        ws.fill_(0xFF)                                          # NaN in every float
        got = pda.attn_bwd(dout, q, k, v, out, lse, *(torch.full_like(t, 7.0) for t in (q, k, v)), d ** -0.5, n_v, workspace=ws)
        want = pda.attn_bwd(dout, q, k, v, out, lse, *(torch.full_like(t, 7.0) for t in (q, k, v)), d ** -0.5, n_v)
        assert all(torch.equal(a, b) and torch.isfinite(a).all() for a, b in zip(got, want)), (h, sq, n_v)
