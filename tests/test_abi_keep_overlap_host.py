"""The choice of tokens refuses lists that share memory with what it reads, without a GPU."""
import pytest

from tests.test_abi_qkv_host import FAKE, SHAPE, binding  # noqa: F401

AT = dict(w=FAKE, lens=FAKE + 10 ** 7, table=FAKE + 2 * 10 ** 7, kept=FAKE + 3 * 10 ** 7, new=FAKE + 4 * 10 ** 7)
SIZE = dict(w=4 * 9 * 2 * 64, lens=4 * 5, table=4 * 5 * 4, kept=4 * 5 * 2 * 100, new=4 * 5)   # bytes


@pytest.mark.parametrize("written,other", [(a, b) for a in ("kept", "new") for b in AT if a != b])
@pytest.mark.parametrize("where", ["same", "its last entry", "the other's last entry"])
def test_select_refuses_shared_memory(binding, written, other, where):  # noqa: F811
    """A list of lengths that is read while the new one is written over it gives some heads the wrong length, and may leave a cluster of CTAs waiting
    for one of its own that has left."""
    at = dict(AT)
    at[written] = at[other] + {"same": 0, "its last entry": 4 - SIZE[written], "the other's last entry": SIZE[other] - 4}[where]
    assert binding.lib.mxkv_select(at["w"], 2, 5, at["lens"], 200, at["table"], 4, 9, 64, 100, 4, 10, at["kept"], at["new"], None) == SHAPE


def test_select_without_a_list(binding):  # noqa: F811
    """keep 0 writes lengths only; these may not be the ones that are read either."""
    assert binding.lib.mxkv_select(AT["w"], 2, 5, AT["lens"], 200, AT["table"], 4, 9, 64, 0, 0, 0, None, AT["lens"], None) == SHAPE
