"""Sizes that no launch of the training operators holds are refused before one is made (addresses are made up, nothing reaches a GPU)."""
import pytest

from tests.test_train_host import _pack, pda  # noqa: F401


@pytest.mark.parametrize("H", [1 << 24, (1 << 30) - 1])
def test_heads_of_the_pack_gradient(pda, H):  # noqa: F811
    """A workgroup a head along one axis of the launch, which has fewer than 2^32 threads; beyond that it would be cut short without an error."""
    assert _pack(pda, H=H, S=1) == 2 and "heads" in pda.last_error(), pda.last_error()
