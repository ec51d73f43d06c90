"""Streams that the training operators' wrappers are given, without a GPU."""
import pytest


class _Stream:
    cuda_stream = 1 << 20

    def __init__(self, index):
        import torch
        self.device = torch.device("cuda", index)


def test_streams_of_another_device_are_refused(monkeypatch):
    """A kernel, and the workspace that the wrapper takes for it, would follow the stream to its device, away from the tensors."""
    import torch
    import paper_2511_12056_amd as pda
    from tests.test_train_host import _Elsewhere

    class Here(_Elsewhere):
        device = 0
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    bf16, fp32 = torch.bfloat16, torch.float32
    q, lse = Here(bf16, 1, 2, 8, 64), Here(fp32, 1, 2, 8)
    x, w, s = Here(fp32, 8, 64), Here(fp32, 64), Here(fp32, 8)
    calls = (lambda st: pda.attn_bwd(q, q, q, q, q, lse, q, q, q, 1.0, stream=st), lambda st: pda.attn_bwd_strided(q, q, q, q, q, lse, q, q, q, 1.0, stream=st),
             lambda st: pda.layer_norm_fwd(x, w, w, x, s, s, stream=st), lambda st: pda.layer_norm_bwd(x, x, w, s, s, x, w, w, stream=st),
             lambda st: pda.pack_heads_bwd(q, None, Here(fp32, 1, 8, 2, 64), False, stream=st))
    for call in calls:
        with pytest.raises(ValueError, match="a stream of device 1, the current device is 0"):
            call(_Stream(1))
