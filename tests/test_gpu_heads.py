"""rmsnorm_rope_fwd / rmsnorm_rope_bwd on the GPU against the definitions in 64 bits.

Tolerances.  Forward: one rounding to bf16 (half a step: 2^-8 of the value) on top of binary32 arithmetic: the sum of squares
of at most 256 terms in four levels, 1/sqrt, three products, the rotation's two products and a sum - fewer than 32 roundings
of 2^-24 each, relative to the larger member of the pair, hence 2^-19 of the head's largest u.
Backward: bf16 again, and fewer than 64 roundings relative to the terms before their cancellation: 2^-18 of `size`.
Gain gradients: a lane adds its items one after another, then fewer than 100 partial sums; each term carries fewer than 16
roundings: (items + 116) 2^-24 of the sum of magnitudes."""
import pytest
import torch

from tests import qkv_ref as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def mx():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2603_13180_b200 import binding
    return binding


def inputs(T, hq, hk, D, rot, rows, seed, extra=3):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, (hq + extra + hk) * D, generator=g) * torch.exp(torch.randn(T, 1, generator=g))
    x[:, :: max(1, (hq * D) // 7)] *= 20
    x = x.to(torch.bfloat16).cuda()
    q, k = x[:, :hq * D].view(T, hq, D), x[:, (hq + extra) * D:].view(T, hk, D)
    gains = [(1 + 0.2 * torch.randn(D, generator=g)).to(torch.bfloat16).cuda() for _ in range(2)]
    table = ref.rope_table(rows, rot).cuda() if rot else None
    pos = torch.randint(0, rows, (T,), generator=g, dtype=torch.int32).cuda()
    return q, k, gains, table, pos, g


SHAPES = [  # T, query heads, key heads, dim, rotated, interleaved pairs
    (1, 1, 1, 64, 64, False), (1, 32, 8, 128, 128, False), (3, 5, 1, 16, 16, True), (7, 3, 2, 32, 16, False),
    (17, 6, 2, 96, 96, False), (17, 6, 2, 96, 48, True), (33, 4, 4, 256, 256, False), (33, 7, 1, 256, 128, True),
    (64, 32, 8, 128, 64, False), (129, 9, 3, 128, 128, True), (200, 2, 2, 208, 32, False), (1000, 32, 4, 64, 32, True),
    (4099, 16, 2, 128, 128, False), (50, 1, 64, 48, 0, False),
]


def close(got, want, size, what):
    err = (got.double() - want).abs()
    tol = 2.0 ** -8 * want.abs() + size
    assert bool((err <= tol).all()), f"{what}: off by {float((err - tol).max()):.3e} over the tolerance"


@pytest.mark.parametrize("T,hq,hk,D,rot,pairs", SHAPES)
def test_forward(mx, T, hq, hk, D, rot, pairs):
    q, k, gains, table, pos, _ = inputs(T, hq, hk, D, rot, 5000, seed=T + D)
    for gq, gk, eps in ((gains[0], gains[1], 1e-6), (None, gains[1], 0.0)):
        qo, ko = torch.full_like(q, 7.0), torch.full((T, hk + 2, D), 7.0, dtype=torch.bfloat16, device="cuda")
        kv = ko[:, 1:hk + 1]    # a strided output between guard heads
        mx.rmsnorm_rope_fwd(q, k, gq, gk, table, pos, qo, kv, eps=eps, interleaved=pairs)
        for x, gain, y in ((q, gq, qo), (k, gk, kv)):
            u = ref.norm_fwd(x, gain, eps)
            want = ref.rotate(u, None if table is None else table.double(), pos, pairs)
            close(y, want, 2.0 ** -19 * u.abs().amax(-1, keepdim=True), "y")
        assert bool((ko[:, 0] == 7).all()) and bool((ko[:, -1] == 7).all())


@pytest.mark.parametrize("T,hq,hk,D,rot,pairs", SHAPES)
def test_backward(mx, T, hq, hk, D, rot, pairs):
    q, k, gains, table, pos, g = inputs(T, hq, hk, D, rot, 5000, seed=T + D + 1)
    gq = (0.01 * torch.randn(T, hq, D, generator=g)).to(torch.bfloat16).cuda()
    gk = (0.01 * torch.randn(T, hk, D, generator=g)).to(torch.bfloat16).cuda()
    ws = torch.empty(mx.rmsnorm_rope_bwd_workspace_bytes(T, hq, hk, D), dtype=torch.uint8, device="cuda")
    for a, b, eps in ((gains[0], gains[1], 1e-6), (None, gains[1], 1e-3)):
        dq, dk = torch.empty_like(gq), torch.empty_like(gk)
        da, db = (torch.full((D,), 9.0, device="cuda") for _ in range(2))
        ws.fill_(0xFF)
        mx.rmsnorm_rope_bwd(q, k, gq, gk, a, b, table, pos, dq, dk, da, db, ws, eps=eps, interleaved=pairs)
        again = [t.clone() for t in (dq, dk, da, db)]
        for x, gy, gain, dx, dg in ((q, gq, a, dq, da), (k, gk, b, dk, db)):
            du = ref.rotate(gy.double(), None if table is None else table.double(), pos, pairs, -1.0)
            want, want_g, size, mags = ref.norm_bwd(x, du, gain, eps)
            close(dx, want, 2.0 ** -18 * size, "dx")
            items = T * x.shape[1]
            assert bool(((dg.double() - want_g).abs() <= (items + 116) * 2.0 ** -24 * mags).all()), "dgain"
        # the same bits again, and dx alone does not depend on whether the gains' gradients are asked for
        mx.rmsnorm_rope_bwd(q, k, gq, gk, a, b, table, pos, dq, dk, da, db, ws, eps=eps, interleaved=pairs)
        assert all(torch.equal(x, y) for x, y in zip(again, (dq, dk, da, db)))
        mx.rmsnorm_rope_bwd(q, k, gq, gk, a, b, table, pos, dq, dk, eps=eps, interleaved=pairs)
        assert torch.equal(again[0], dq) and torch.equal(again[1], dk)


def test_gradient_against_differences(mx):
    """d(sum y w)/dx from the kernel's dx against central differences of the definition in 64 bits."""
    T, hq, hk, D, rot = 5, 2, 1, 64, 32
    q, k, gains, table, pos, g = inputs(T, hq, hk, D, rot, 300, seed=3)
    w = torch.randn(T, hq, D, generator=g).to(torch.bfloat16).cuda()
    dq, dk = torch.empty(T, hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(T, hk, D, dtype=torch.bfloat16, device="cuda")
    mx.rmsnorm_rope_bwd(q, k, w, torch.zeros_like(dk), gains[0], gains[1], table, pos, dq, dk, eps=1e-5, interleaved=True)
    assert not bool(dk.any())
    f = lambda x: (ref.rotate(ref.norm_fwd(x, gains[0], 1e-5), table.double(), pos, True) * w.double()).sum((1, 2))  # noqa: E731
    x, rms = q.double(), q.double().square().mean(-1).sqrt()
    for t, h, d in ((0, 0, 0), (1, 1, 5), (2, 0, 31), (3, 1, 32), (4, 1, 63)):
        step = 1e-5 * rms[t, h]
        up, down = x.clone(), x.clone()
        up[t, h, d] += step
        down[t, h, d] -= step
        want = (f(up)[t] - f(down)[t]) / (2 * step)
        # rounding of dx to bf16, binary32 sums, and the differences' own error of about step^2 / rms^3
        assert abs(float(dq[t, h, d]) - float(want)) <= 2.0 ** -8 * abs(float(want)) + 1e-4 / float(rms[t, h])


def test_rotation_alone_and_in_place(mx):
    T, hq, hk, D, rot = 37, 4, 2, 128, 64
    q, k, gains, table, pos, _ = inputs(T, hq, hk, D, rot, 999, seed=8)
    qo, ko = torch.empty(T, hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(T, hk, D, dtype=torch.bfloat16, device="cuda")
    mx.rmsnorm_rope_fwd(q, k, None, None, table, pos, qo, ko, normalise=False)
    assert torch.equal(qo, ref.rotate(q.float(), table, pos, False).to(torch.bfloat16))   # binary32 operations one by one
    assert torch.equal(ko, ref.rotate(k.float(), table, pos, False).to(torch.bfloat16))
    back = torch.empty_like(qo)
    mx.rmsnorm_rope_bwd(None, None, qo, None, None, None, table, pos, back, None, normalise=False)
    assert torch.equal(back, ref.rotate(qo.float(), table, pos, False, -1.0).to(torch.bfloat16))
    # normalised: written over the inputs, and without positions (row index); keys absent
    want = torch.empty_like(qo)
    mx.rmsnorm_rope_fwd(q, None, gains[0], None, table, None, want, None)
    rows = torch.arange(T, dtype=torch.int32, device="cuda")
    mx.rmsnorm_rope_fwd(q, k, gains[0], gains[1], table, rows, qo, ko)
    assert torch.equal(want, qo)
    mx.rmsnorm_rope_fwd(q, k, gains[0], gains[1], table, rows, q, k)
    assert torch.equal(q, qo) and torch.equal(k, ko)


def test_zero_heads_and_no_tokens(mx):
    q = torch.zeros(3, 2, 64, dtype=torch.bfloat16, device="cuda")
    out = torch.ones_like(q)
    mx.rmsnorm_rope_fwd(q, None, None, None, None, None, out, None, eps=0.0)
    assert not bool(out.any())
    g = torch.ones_like(q)
    dg = torch.ones(64, device="cuda")
    ws = torch.empty(mx.rmsnorm_rope_bwd_workspace_bytes(3, 2, 0, 64), dtype=torch.uint8, device="cuda")
    mx.rmsnorm_rope_bwd(q, None, g, None, None, None, None, None, out, None, dg, None, ws, eps=0.0)
    assert not bool(out.any()) and not bool(dg.any())
    dg.fill_(1)
    mx.rmsnorm_rope_bwd(q[:0], None, g[:0], None, None, None, None, None, out[:0], None, dg, None, None)
    assert not bool(dg.any())
    mx.rmsnorm_rope_fwd(q[:0], None, None, None, None, None, out[:0], None)


def test_backward_on_a_stream_and_captured(mx):
    """The gradients, those of the gains among them, have the same bits on another stream and in a graph that is replayed with new
    inputs in place."""
    T, hq, hk, D, rot = 333, 6, 2, 128, 128
    q, k, gains, table, pos, g = inputs(T, hq, hk, D, rot, 500, seed=4)
    dy = torch.randn(T, hq + hk, D, generator=g).to(torch.bfloat16).cuda()
    ws = torch.empty(mx.rmsnorm_rope_bwd_workspace_bytes(T, hq, hk, D), dtype=torch.uint8, device="cuda")
    outs = [torch.empty_like(dy[:, :hq]), torch.empty_like(dy[:, hq:]), torch.empty(D, device="cuda"), torch.empty(D, device="cuda")]

    def call():
        mx.rmsnorm_rope_bwd(q, k, dy[:, :hq], dy[:, hq:], gains[0], gains[1], table, pos, outs[0], outs[1], outs[2], outs[3], ws)

    def results():
        torch.cuda.synchronize()
        got = [o.clone() for o in outs]
        for o in outs:
            o.fill_(7)
        return got

    call()
    want = results()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        call()
    assert all(torch.equal(a, b) for a, b in zip(results(), want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    graph.replay()
    assert all(torch.equal(a, b) for a, b in zip(results(), want))
    dy.mul_(2)   # exact: every gradient doubles
    graph.replay()
    assert all(torch.equal(a, 2 * b) for a, b in zip(results(), want))


def test_nan_stays_in_its_head(mx):
    """A NaN makes its whole head NaN, forward and backward, and no other."""
    T, hq, hk, D, rot = 9, 6, 2, 64, 32
    q, k, gains, table, pos, g = inputs(T, hq, hk, D, rot, 50, seed=6)
    dy = torch.randn(T, hq, D, generator=g).to(torch.bfloat16).cuda()
    results = []
    for value in (None, float("nan")):
        if value is not None:
            q[4, 3, 40] = value
        qo, ko, dq = torch.empty(T, hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty_like(k.contiguous()), torch.empty_like(dy)
        mx.rmsnorm_rope_fwd(q, k, gains[0], gains[1], table, pos, qo, ko)
        mx.rmsnorm_rope_bwd(q, None, dy, None, gains[0], None, table, pos, dq, None)
        results.append((qo, ko, dq))
    for clean, got in zip(results[0], results[1]):
        if clean.shape[1] == hq:
            assert bool(got[4, 3].isnan().all())
            got[4, 3] = clean[4, 3]
        assert torch.equal(clean, got)


def test_positions_outside_the_table(mx):
    T, hq, hk, D, rot = 9, 3, 1, 64, 64
    q, k, gains, table, _, g = inputs(T, hq, hk, D, rot, 50, seed=2)
    pos = torch.tensor([0, 49, 50, -1, 3, 2 ** 31 - 1, -2 ** 31, 7, 8], dtype=torch.int32, device="cuda")
    bad = torch.tensor([2, 3, 5, 6], device="cuda")
    good = torch.tensor([0, 1, 4, 7, 8], device="cuda")
    mx.device_bad_indices_reset()
    qo, ko = torch.empty(T, hq, D, dtype=torch.bfloat16, device="cuda"), torch.empty(T, hk, D, dtype=torch.bfloat16, device="cuda")
    mx.rmsnorm_rope_fwd(q, k, gains[0], gains[1], table, pos, qo, ko)
    assert mx.device_bad_indices() == 4
    assert bool(qo[bad].isnan().all()) and bool(ko[bad].isnan().all())
    assert bool(qo[good].isfinite().all()) and bool(ko[good].isfinite().all())
    gy = torch.randn(T, hq, D, generator=g).to(torch.bfloat16).cuda()
    dq, dg = torch.empty_like(gy), torch.empty(D, device="cuda")
    ws = torch.empty(mx.rmsnorm_rope_bwd_workspace_bytes(T, hq, 0, D), dtype=torch.uint8, device="cuda")
    mx.rmsnorm_rope_bwd(q, None, gy, None, gains[0], None, table, pos, dq, None, dg, None, ws)
    assert bool(dq[bad].isnan().all()) and bool(dq[good].isfinite().all())
    du = ref.rotate(gy[good].double(), table.double(), pos[good], False, -1.0)
    _, want, _, mags = ref.norm_bwd(q[good], du, gains[0], 1e-6)
    assert bool(((dg.double() - want).abs() <= (T * hq + 116) * 2.0 ** -24 * mags).all())
    mx.device_bad_indices_reset()
    assert mx.device_bad_indices() == 0


def test_more_than_2_31_elements(mx):
    T, hq, D = 140000, 120, 128          # 2.15e9 elements; the last tokens are compared
    q = torch.empty(T, hq, D, dtype=torch.bfloat16, device="cuda")
    q.view(torch.int16).fill_(0x3F00)
    tail = torch.randn(3, hq, D, generator=torch.Generator().manual_seed(1)).to(torch.bfloat16).cuda()
    q[-3:] = tail
    mx.rmsnorm_rope_fwd(q, None, None, None, None, None, q, None, eps=0.0)
    u = ref.norm_fwd(tail, None, 0.0)
    close(q[-3:], u, 2.0 ** -19 * u.abs().amax(-1, keepdim=True), "tail")
    assert bool((q[:1000] == 1).all()) and bool((q[T // 2] == 1).all())
