"""What the Python binding of the entry points around attention refuses, without a GPU."""
import pytest
import torch


@pytest.fixture(scope="module")
def binding():
    from paper_2603_13180_b200 import build
    build.build_library()
    from paper_2603_13180_b200 import binding as b
    return b


def test_workspaces_lie_in_one_piece(binding):
    """Bytes are counted from the elements, so a tensor with gaps or repeated elements is refused."""
    t = torch.zeros(64, dtype=torch.float32)
    assert binding._workspace(None) == (None, 0)
    assert binding._workspace(t) == (t.data_ptr(), 256) and binding._workspace(t[8:]) == (t.data_ptr() + 32, 224)
    for bad in (t[:1].expand(1 << 20), t[::2], t.view(8, 8).t()):
        with pytest.raises(ValueError):
            binding._workspace(bad)
