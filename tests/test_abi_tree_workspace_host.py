"""Workspaces of attention and of trees, without a GPU."""
import pytest

from tests.test_abi_keep_host import masked
from tests.test_abi_qkv_host import FAKE, OK, WORKSPACE, binding  # noqa: F401

CUDA = 6   # a call that would launch, on a machine without a GPU


@pytest.mark.parametrize("n,seqs,mq,ml,qh,heads,dim,need", [
    # one prompt over itself has CTAs enough and joins nothing; half of one over a long history takes two chunks a row
    (1000, 1, 1000, 1000, 32, 8, 128, 0), (4096, 1, 4096, 8192, 32, 8, 128, 0), (512, 1, 512, 8192, 32, 8, 128, 512 * 32 * 2 * 129 * 4),
    (130, 16, 13, 4100, 32, 4, 64, 130 * 32 * 2 * 65 * 4),
])
def test_attention_asks_for_what_it_uses(binding, n, seqs, mq, ml, qh, heads, dim, need):  # noqa: F811
    """Not for what trees can use."""
    assert binding.mxkv_attention_workspace_bytes(n, seqs, mq, ml, qh, heads, dim) == need
    assert binding.mxkv_attention_tree_workspace_bytes(n, seqs, mq, ml, qh, heads, dim) >= need


def test_few_rows_ask_for_the_same(binding):  # noqa: F811
    for args in ((1, 1, 1, 1000, 32, 8, 128), (64, 64, 1, 8192, 32, 8, 128), (12, 1, 12, 1500, 32, 8, 128), (0, 1, 1, 5, 4, 2, 64), (40, 8, 6, 3000, 8, 2, 64)):
        assert binding.mxkv_attention_workspace_bytes(*args) == binding.mxkv_attention_tree_workspace_bytes(*args)
    assert binding.mxkv_attention_tree_workspace_bytes(1, 1, 1, -5, 4, 2, 64) == 0


@pytest.mark.parametrize("n,seqs,mq,ml,qh,heads,dim", [(130, 16, 13, 4100, 32, 4, 64), (512, 1, 512, 8192, 32, 8, 128), (1000, 1, 1000, 1000, 32, 8, 128)])
def test_what_a_tree_takes(binding, n, seqs, mq, ml, qh, heads, dim):  # noqa: F811
    """Anything from the other masks' size up (also where that is nothing); less is refused."""
    if binding.torch.cuda.is_available():
        pytest.skip("accepted calls would launch")
    small = binding.mxkv_attention_workspace_bytes(n, seqs, mq, ml, qh, heads, dim)
    full = binding.mxkv_attention_tree_workspace_bytes(n, seqs, mq, ml, qh, heads, dim)
    assert full > small
    tree = masked("mxkv_attention_tree", ("mask", "words"))
    a = dict(n=n, seqs=seqs, mq=mq, ml=ml, qh=qh, heads=heads, dim=dim, qs=qh * dim, os=qh * dim, width=ml // 64 + 1, words=(mq + 31) // 32, pages=500)
    for size in (small, small + 4, (small + full) // 2, full, full + 1000):
        assert tree(binding.lib, dict(a, ws=FAKE, wsb=size)) == CUDA
    if small:
        assert tree(binding.lib, dict(a, ws=FAKE, wsb=small - 1)) == WORKSPACE and tree(binding.lib, dict(a, ws=None, wsb=full)) == WORKSPACE
    else:
        assert tree(binding.lib, dict(a, ws=None, wsb=0)) == CUDA
    assert tree(binding.lib, dict(a, n=0)) == OK
