"""Attention gradient of more query rows than one axis of a launch has threads for."""
import pytest

pytestmark = pytest.mark.gpu


def test_more_rows_than_a_launch_has_threads_for():
    """2^28 rows of 128 elements, 16 threads a row for their statistics; q, dout and out are one tensor of 64 GiB, zero but for its ends."""
    import torch
    import paper_2511_12056_amd as pda
    d, Sq, n_v = 128, (1 << 28) + 300, 5
    if torch.cuda.mem_get_info()[0] < 150 << 30:
        pytest.skip("150 GiB of device memory needed")
    g = torch.Generator(device="cuda").manual_seed(1)
    q, dq = torch.zeros(1, 1, Sq, d, device="cuda", dtype=torch.bfloat16), torch.empty(1, 1, Sq, d, device="cuda", dtype=torch.bfloat16)
    live = torch.cat([torch.arange(40), torch.arange((1 << 28) - 20, (1 << 28) + 20), torch.arange(Sq - 50, Sq)]).cuda()
    q[0, 0, live] = torch.randn(live.numel(), d, generator=g, device="cuda").to(torch.bfloat16)
    k, v = (torch.randn(1, 1, n_v, d, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    lse = torch.full((1, 1, Sq), float(torch.tensor(5.0).log()), device="cuda")
    part = q[:, :, live].contiguous()
    lse[0, 0, live] = torch.logsumexp(torch.mm(part[0, 0].double(), k[0, 0].double().t().contiguous()) * d ** -0.5, -1).float()
    dk, dv = torch.full_like(k, 7.0), torch.full_like(v, 7.0)
    pda.attn_bwd(q, q, k, v, q, lse, dq, dk, dv, d ** -0.5)
    torch.cuda.synchronize()
    want = pda.attn_bwd(part, part, k, v, part, lse[:, :, live].contiguous(), torch.empty_like(part), torch.empty_like(k), torch.empty_like(v), d ** -0.5)
    assert torch.equal(dq[:, :, live], want[0])
    dq[:, :, live] = 0
    assert not any(x.any() for x in dq[0, 0].split(1 << 24))                 # a row without dout gives and gets nothing
    # the same rows' terms, summed in another order in fp32 and rounded once more to bf16: half a step on either side
    for x, w in zip((dk, dv), want[1:]):
        assert ((x.double() - w.double()).abs() <= 2.0 ** -8 * 1.01 * w.double().abs() + 2.0 ** -20 * w.double().abs().max()).all()
    del q, dq, lse
    torch.cuda.empty_cache()                                                 # 130 GiB, for whoever allocates next to torch
