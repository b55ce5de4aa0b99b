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


# sizes of heads whose squares leave binary32's range, or lose digits in it, among ordinary ones
SIZES = [1.0, 2.0 ** 39, 2.0 ** 41, 2.0 ** 63, 2.0 ** 70, 2.0 ** 100, 2.0 ** 122, 2.0 ** -39, 2.0 ** -41, 2.0 ** -64, 2.0 ** -75, 2.0 ** -100, 2.0 ** -123]


@pytest.mark.parametrize("D,rot,pairs", [(64, 64, False), (128, 128, True), (256, 64, False), (48, 0, False), (16, 16, True)])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
def test_heads_of_any_size(mx, D, rot, pairs, eps):  # noqa: F811
    """Heads from 2^-123 to 2^122 side by side: normalised, and their gradients, as the definitions say."""
    T, hq, hk = 40, 6, 3
    q, k, gains, table, pos, g = inputs(T, hq, hk, D, rot, 100, seed=D)
    outs = [torch.empty(T, h, D, dtype=torch.bfloat16, device="cuda") for h in (hq, hk)]
    size = [torch.tensor(SIZES, device="cuda")[torch.randint(0, len(SIZES), (T, h), generator=g).cuda()][..., None] for h in (hq, hk)]
    x = [(torch.randn(T, h, D, generator=g).cuda().clamp(-4, 4) * s).to(torch.bfloat16) for h, s in zip((hq, hk), size)]
    mx.rmsnorm_rope_fwd(x[0], x[1], gains[0], gains[1], table, pos, *outs, eps=eps, interleaved=pairs)
    for a, gain, y in zip(x, gains, outs):
        u = ref.norm_fwd(a, gain, eps)
        # (what the rounding to bf16 leaves of the smallest results: half of its least step, 2^-134)
        close(y, ref.rotate(u, None if table is None else table.double(), pos, pairs), 2.0 ** -19 * u.abs().amax(-1, keepdim=True) + 2.0 ** -134, "y")
    # gradients of about the square root of the size, so that theirs is about its inverse
    gy = [(torch.randn(T, h, D, generator=g).cuda() * s.sqrt()).to(torch.bfloat16) for h, s in zip((hq, hk), size)]
    dg = [torch.empty(D, device="cuda") for _ in range(2)]
    ws = torch.empty(mx.rmsnorm_rope_bwd_workspace_bytes(T, hq, hk, D), dtype=torch.uint8, device="cuda")
    mx.rmsnorm_rope_bwd(x[0], x[1], gy[0], gy[1], gains[0], gains[1], table, pos, *outs, *dg, ws, eps=eps, interleaved=pairs)
    for a, gradient, gain, dx, got in zip(x, gy, gains, outs, dg):
        du = ref.rotate(gradient.double(), None if table is None else table.double(), pos, pairs, -1.0)
        want, want_g, bound, mags = ref.norm_bwd(a, du, gain, eps)
        close(dx, want, 2.0 ** -18 * bound + 2.0 ** -134, "dx")
        assert bool(((got.double() - want_g).abs() <= (T * a.shape[1] + 116) * 2.0 ** -24 * mags).all()), "dgain"


def test_zeros_beside_heads_of_any_size(mx):  # noqa: F811
    """Heads of zeros stay zero without eps, next to large and tiny ones; an infinity makes its own head NaN only."""
    x = torch.zeros(5, 4, 64, dtype=torch.bfloat16, device="cuda")
    x[:, 1], x[:, 2] = 2.0 ** 120, 2.0 ** -120
    x[3, 3, 7] = float("inf")
    y = torch.empty_like(x)
    mx.rmsnorm_rope_fwd(x, None, None, None, None, None, y, None, eps=0.0)
    assert not bool(y[:, 0].any()) and bool((y[:, 1:3] == 1).all()) and bool(y[3, 3, 7].isnan()) and not bool(y[:3, 3].any())


# sizes of heads whose squares leave binary32's range, or lose digits in it, among ordinary ones
SIZES = [1.0, 2.0 ** 39, 2.0 ** 41, 2.0 ** 63, 2.0 ** 70, 2.0 ** 100, 2.0 ** 122, 2.0 ** -39, 2.0 ** -41, 2.0 ** -64, 2.0 ** -75, 2.0 ** -100, 2.0 ** -123]


@pytest.mark.parametrize("T", [40, 1500])
@pytest.mark.parametrize("D,rot,pairs", [(64, 64, False), (128, 128, True), (256, 64, False), (48, 0, False), (16, 16, True)])
@pytest.mark.parametrize("eps", [0.0, 1e-6])
@pytest.mark.parametrize("in_place", [False, True])
def test_heads_of_any_size(mx, T, D, rot, pairs, eps, in_place):  # noqa: F811
    """Heads from 2^-123 to 2^122 side by side: normalised, and their gradients, as the definitions say."""
    hq, hk = 12, 7
    _, _, gains, table, pos, g = inputs(T, hq, hk, D, rot, 100, seed=D)
    size = [torch.tensor(SIZES, device="cuda")[torch.randint(0, len(SIZES), (T, h), generator=g).cuda()][..., None] for h in (hq, hk)]
    x = [(torch.randn(T, h, D, generator=g).cuda().clamp(-4, 4) * s).to(torch.bfloat16) for h, s in zip((hq, hk), size)]
    kept = [a.clone() for a in x]
    outs = x if in_place else [torch.empty_like(a) for a in x]
    mx.rmsnorm_rope_fwd(x[0], x[1], gains[0], gains[1], table, pos, *outs, eps=eps, interleaved=pairs)
    for a, gain, y in zip(kept, gains, outs):
        u = ref.norm_fwd(a, gain, eps)
        # (what the rounding to bf16 leaves of the smallest results: half of its least step, 2^-134)
        close(y, ref.rotate(u, None if table is None else table.double(), pos, pairs), 2.0 ** -19 * u.abs().amax(-1, keepdim=True) + 2.0 ** -134, "y")
    # gradients of about the square root of the size, so that theirs is about its inverse
    gy = [(torch.randn(T, h, D, generator=g).cuda() * s.sqrt()).to(torch.bfloat16) for h, s in zip((hq, hk), size)]
    given = [a.clone() for a in gy]
    outs = gy if in_place else [torch.empty_like(a) for a in x]
    dg = [torch.empty(D, device="cuda") for _ in range(2)]
    ws = torch.empty(mx.rmsnorm_rope_bwd_workspace_bytes(T, hq, hk, D), dtype=torch.uint8, device="cuda")
    mx.rmsnorm_rope_bwd(kept[0], kept[1], gy[0], gy[1], gains[0], gains[1], table, pos, *outs, *dg, ws, eps=eps, interleaved=pairs)
    for a, gradient, gain, dx, got in zip(kept, given, gains, outs, dg):
        du = ref.rotate(gradient.double(), None if table is None else table.double(), pos, pairs, -1.0)
        want, want_g, bound, mags = ref.norm_bwd(a, du, gain, eps)
        close(dx, want, 2.0 ** -18 * bound + 2.0 ** -134, "dx")
        assert bool(((got.double() - want_g).abs() <= (T * a.shape[1] + 116) * 2.0 ** -24 * mags).all()), "dgain"


def test_zeros_beside_heads_of_any_size(mx):  # noqa: F811
    """Heads of zeros stay zero without eps, next to large and tiny ones; an infinity makes its own head NaN only."""
    x = torch.zeros(5, 4, 64, dtype=torch.bfloat16, device="cuda")
    x[:, 1], x[:, 2] = 2.0 ** 120, 2.0 ** -120
    x[3, 3, 7] = float("inf")
    y = torch.empty_like(x)
    mx.rmsnorm_rope_fwd(x, None, None, None, None, None, y, None, eps=0.0)
    assert not bool(y[:, 0].any()) and bool((y[:, 1:3] == 1).all()) and bool(y[3, 3, 7].isnan()) and not bool(y[:3, 3].any())
