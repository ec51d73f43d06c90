"""Strides of the matrices that fp8_quant is given, without a GPU: a kernel that takes other rows than the matrix has reads behind its end."""
import pytest


@pytest.fixture()
def made(monkeypatch):
    """A stand-in for a tensor on device 0 with any strides; asking for its address fails the test."""
    import torch
    from tests.test_train_host import _Elsewhere
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)

    class Made(_Elsewhere):
        device = 0

        def __init__(self, dtype, shape, strides=None):
            super().__init__(dtype, *shape)
            self.strides = _Elsewhere.stride(self) if strides is None else strides

        def stride(self, i=None):
            return self.strides if i is None else self.strides[i]
    return Made


def _results(made, rows, cols, block):
    import torch
    up = lambda n, m: -(-n // m) * m                               # noqa: E731
    out = []
    for r, c in ((rows, cols), (cols, rows)):
        out += [made(torch.float8_e4m3fn, (r, up(c, 128))), made(torch.float8_e8m0fnu, (up(r, block) // block, up(up(c, 128) // 128, 4)))]
    return out


@pytest.mark.parametrize("block", [1, 128])
@pytest.mark.parametrize("rows,cols,strides", [(70, 256, (0, 1)), (300, 200, (0, 1)), (2, 3, (2, 1)), (50, 130, (1, 1)), (129, 128, (127, 1)), (5, 1, (0, 1)), (5, 1, (0, 0))])
def test_rows_that_share_elements_are_refused(made, rows, cols, strides, block):
    """A row repeated (the gradient of a sum over tokens), windows that overlap."""
    import torch
    import paper_2511_12056_amd as pda
    for dtype in (torch.float32, torch.bfloat16):
        q, qs, qt, qts = _results(made, rows, cols, block)
        for args in ((q, qs), (None, None, qt, qts), (q, qs, qt, qts)):
            with pytest.raises(ValueError, match="x: .*stride"):
                pda.fp8_quant(made(dtype, (rows, cols), strides), *args, block_rows=block)


@pytest.mark.parametrize("rows,cols,strides,ldx", [(70, 256, (256, 1), 256), (70, 250, (777, 1), 777), (1, 256, (0, 1), 256), (1, 5, (3, 1), 5), (9, 1, (4, 0), 4), (9, 1, (1, 9), 1)])
def test_rows_that_lie_apart_keep_their_stride(made, monkeypatch, rows, cols, strides, ldx):
    """What the C entry is called with."""
    import torch
    import paper_2511_12056_amd as pda
    from paper_2511_12056_amd import binding
    seen = []

    class Lib:
        @staticmethod
        def pda_fp8_quant(*args):
            seen.append(args[2:5])
            return 0
    monkeypatch.setattr(binding, "lib", Lib)
    monkeypatch.setattr(binding, "_ptr", lambda t: None if t is None else 4096)
    monkeypatch.setattr(binding, "_stream_handle", lambda s: None)
    q, qs, _, _ = _results(made, rows, cols, 1)
    pda.fp8_quant(made(torch.float32, (rows, cols), strides), q, qs)
    assert seen == [(rows, cols, ldx)]
