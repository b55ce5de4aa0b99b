"""rmsnorm_rope_fwd / rmsnorm_rope_bwd at the ends of their ranges.  Tolerances are those of test_gpu_heads.py."""
import pytest
import torch

from tests import qkv_ref as ref
from tests.test_gpu_heads import close, inputs, mx  # noqa: F401  (mx is the fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("D,rot,pairs", [(64, 64, False), (128, 64, True), (256, 256, False), (48, 16, True)])
@pytest.mark.parametrize("junk", [float("nan"), float("inf"), float("-inf")])
def test_padding_without_an_angle_adds_nothing_to_the_gains(mx, D, rot, pairs, junk):  # noqa: F811
    """Tokens at position -1 whose activations or gradients hold NaN or infinities: NaN for them, and the gains' gradients have
    the bits that the same call gives with ordinary numbers there."""
    T, hq, hk = 50, 6, 2
    q, k, gains, table, pos, g = inputs(T, hq, hk, D, rot, 100, seed=D)
    pos[::3] = -1
    gq, gk = (torch.randn(T, h, D, generator=g).to(torch.bfloat16).cuda() for h in (hq, hk))
    ws = torch.empty(mx.rmsnorm_rope_bwd_workspace_bytes(T, hq, hk, D), dtype=torch.uint8, device="cuda")

    def call():
        outs = [torch.empty_like(gq), torch.empty_like(gk), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")]
        mx.rmsnorm_rope_bwd(q, k, gq, gk, gains[0], gains[1], table, pos, *outs, ws, interleaved=pairs)
        return outs

    clean = call()
    assert bool(clean[2].isfinite().all()) and bool(clean[3].isfinite().all())
    for target in (q, gq, k, gk):
        keep = target[::3].clone()
        target[::3, :, ::5] = junk
        for a, b in zip(call(), clean):
            assert torch.equal(a.view(torch.int32 if a.dtype == torch.float32 else torch.int16),
                               b.view(torch.int32 if b.dtype == torch.float32 else torch.int16))
        target[::3] = keep
    mx.device_bad_indices_reset()
