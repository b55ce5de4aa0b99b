"""Refusals of the entry points around attention, without a GPU: every call fails (or returns) before a launch."""
import pytest
import torch

FAKE = 0x7F0000000000   # never dereferenced


@pytest.fixture(scope="module")
def binding():
    from paper_2603_13180_b200 import build
    build.build_library()
    from paper_2603_13180_b200 import binding as b
    return b


OK, NULL, SHAPE, ALIGN, ENUM, WORKSPACE = range(6)


def rope_fwd(L, **kw):
    a = dict(q=FAKE, qs=512, qh=4, k=FAKE, ks=256, kh=2, T=3, dim=128, norm=1, qg=FAKE, kg=None, eps=1e-6, cs=FAKE, rows=10, rot=128, pairing=0,
             pos=None, qo=FAKE, qos=512, ko=FAKE, kos=256)
    a.update(kw)
    return L.rmsnorm_rope_fwd(*(a[n] for n in ("q", "qs", "qh", "k", "ks", "kh", "T", "dim", "norm", "qg", "kg", "eps", "cs", "rows", "rot",
                                               "pairing", "pos", "qo", "qos", "ko", "kos")), None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=0), OK), (dict(T=-1), SHAPE), (dict(T=2 ** 31), SHAPE), (dict(dim=8), SHAPE), (dict(dim=72), SHAPE), (dict(dim=272), SHAPE),
    (dict(qh=0, kh=0), SHAPE), (dict(qh=-1), SHAPE), (dict(qh=5000, qs=10 ** 6, qos=10 ** 6), SHAPE), (dict(norm=2), ENUM), (dict(norm=0), SHAPE),
    (dict(eps=-1.0), SHAPE), (dict(eps=float("nan")), SHAPE), (dict(rot=8), SHAPE), (dict(rot=144), SHAPE), (dict(rot=24), SHAPE),
    (dict(rows=0), SHAPE), (dict(pairing=2), ENUM), (dict(cs=FAKE + 4), ALIGN), (dict(qg=FAKE + 2), ALIGN), (dict(pos=FAKE + 2), ALIGN),
    (dict(q=None), NULL), (dict(k=None), NULL), (dict(qo=None), NULL), (dict(ko=None), NULL), (dict(qs=511), SHAPE), (dict(qs=516), ALIGN),
    (dict(q=FAKE + 8), ALIGN), (dict(ko=FAKE + 2), ALIGN), (dict(kos=128), SHAPE),
])
def test_rope_forward(binding, kw, status):
    assert rope_fwd(binding.lib, **kw) == status


def rope_bwd(L, ws_bytes, **kw):
    a = dict(q=FAKE, qs=512, qh=4, k=FAKE, ks=256, kh=2, gq=FAKE, gqs=512, gk=FAKE, gks=256, T=3, dim=128, norm=1, qg=FAKE, kg=None, eps=1e-6,
             cs=FAKE, rows=10, rot=128, pairing=0, pos=None, dq=FAKE, dqs=512, dk=FAKE, dks=256, dqg=FAKE, dkg=None, ws=FAKE, wsb=ws_bytes)
    a.update(kw)
    return L.rmsnorm_rope_bwd(*(a[n] for n in ("q", "qs", "qh", "k", "ks", "kh", "gq", "gqs", "gk", "gks", "T", "dim", "norm", "qg", "kg", "eps",
                                               "cs", "rows", "rot", "pairing", "pos", "dq", "dqs", "dk", "dks", "dqg", "dkg", "ws", "wsb")), None)


@pytest.mark.parametrize("kw,status", [
    (dict(T=-1), SHAPE), (dict(dim=40), SHAPE), (dict(norm=0, qg=None), SHAPE), (dict(gq=None), NULL), (dict(dq=None), NULL), (dict(q=None), NULL),
    (dict(ws=None), WORKSPACE), (dict(wsb=16), WORKSPACE), (dict(ws=FAKE + 8), ALIGN), (dict(dqg=FAKE + 2), ALIGN), (dict(gks=260), ALIGN),
    (dict(dqs=100), SHAPE), (dict(pairing=-1), ENUM), (dict(norm=3), ENUM), (dict(T=0, dqg=None), OK),
])
def test_rope_backward(binding, kw, status):
    assert rope_bwd(binding.lib, binding.rmsnorm_rope_bwd_workspace_bytes(3, 4, 2, 128), **kw) == status


def test_rope_workspace_does_not_decrease_with_tokens(binding):
    for hq, hk, dim in ((32, 8, 128), (1, 0, 64), (0, 1, 256), (7, 3, 48)):
        sizes = [binding.rmsnorm_rope_bwd_workspace_bytes(T, hq, hk, dim) for T in (1, 2, 17, 500, 4099, 16384, 10 ** 6)]
        assert sizes[0] > 0 and sizes == sorted(sizes)
    assert binding.rmsnorm_rope_bwd_workspace_bytes(5, 1, 1, 100) == 0


def append(L, **kw):
    a = dict(k=FAKE, ks=256, v=FAKE, vs=256, n=3, heads=2, dim=128, cu=FAKE, seqs=2, lens=FAKE, table=FAKE, width=4, pages=9, page=64, block=16,
             cs=None, rows=0, rot=0, pairing=0, kc=FAKE, ksc=FAKE, vc=FAKE, vsc=FAKE)
    a.update(kw)
    return L.mxkv_append(*(a[n] for n in ("k", "ks", "v", "vs", "n", "heads", "dim", "cu", "seqs", "lens", "table", "width", "pages", "page", "block",
                                          "cs", "rows", "rot", "pairing", "kc", "ksc", "vc", "vsc")), None)


CACHE = [
    (dict(heads=0), SHAPE), (dict(dim=24), SHAPE), (dict(seqs=-1), SHAPE), (dict(width=0), SHAPE), (dict(pages=0), SHAPE),
    (dict(page=8), SHAPE), (dict(page=48), SHAPE), (dict(page=512), SHAPE), (dict(block=8), SHAPE), (dict(block=48), SHAPE),
    (dict(page=32, block=64), SHAPE), (dict(width=2 ** 31 // 64), SHAPE), (dict(pages=2 ** 31 // 2), SHAPE), (dict(cu=None), NULL),
    (dict(lens=None), NULL), (dict(table=None), NULL), (dict(kc=None), NULL), (dict(ksc=None), NULL), (dict(vc=None), NULL), (dict(vsc=None), NULL),
    (dict(cu=FAKE + 2), ALIGN), (dict(lens=FAKE + 1), ALIGN), (dict(table=FAKE + 2), ALIGN), (dict(kc=FAKE + 8), ALIGN), (dict(vc=FAKE + 8), ALIGN),
    (dict(n=-1), SHAPE), (dict(n=2 ** 31), SHAPE), (dict(n=0), OK), (dict(seqs=0), OK),
]


@pytest.mark.parametrize("kw,status", CACHE + [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(ks=255), SHAPE), (dict(vs=260), ALIGN), (dict(v=FAKE + 4), ALIGN),
    (dict(cs=FAKE, rows=10, rot=20), SHAPE), (dict(cs=FAKE, rows=0, rot=64), SHAPE), (dict(cs=FAKE, rows=10, rot=144), SHAPE),
    (dict(cs=FAKE + 8, rows=10, rot=64), ALIGN), (dict(pairing=5), ENUM),
])
def test_append(binding, kw, status):
    assert append(binding.lib, **kw) == status


def attend(L, **kw):
    a = dict(q=FAKE, qs=512, n=3, qh=4, heads=2, dim=128, cu=FAKE, seqs=2, mq=2, lens=FAKE, ml=200, table=FAKE, width=4, pages=9, page=64, block=16,
             kc=FAKE, ksc=FAKE, vc=FAKE, vsc=FAKE, scale=0.1, causal=1, window=0, out=FAKE, os=512, lse=None, ws=None, wsb=0)
    a.update(kw)
    return L.mxkv_attention(*(a[n] for n in ("q", "qs", "n", "qh", "heads", "dim", "cu", "seqs", "mq", "lens", "ml", "table", "width", "pages", "page",
                                             "block", "kc", "ksc", "vc", "vsc", "scale", "causal", "window", "out", "os", "lse", "ws", "wsb")), None)


@pytest.mark.parametrize("kw,status", CACHE + [
    (dict(dim=32), SHAPE), (dict(dim=256), SHAPE), (dict(qh=5), SHAPE), (dict(qh=1), SHAPE), (dict(mq=0), SHAPE), (dict(ml=-1), SHAPE),
    (dict(ml=257), SHAPE), (dict(window=-1), SHAPE), (dict(scale=float("nan")), SHAPE), (dict(causal=2), ENUM), (dict(q=None), NULL),
    (dict(out=None), NULL), (dict(q=FAKE + 8), ALIGN), (dict(os=516), ALIGN), (dict(qs=100), SHAPE), (dict(lse=FAKE + 2), ALIGN),
    (dict(), WORKSPACE), (dict(ws=FAKE, wsb=100), WORKSPACE), (dict(ws=FAKE + 4, wsb=10 ** 9), ALIGN),
])
def test_attention(binding, kw, status):
    assert attend(binding.lib, **kw) == status


def test_attention_workspace(binding):
    f = binding.mxkv_attention_workspace_bytes
    assert f(1, 1, 1, 131072, 32, 8, 128) > 0 and f(1, 1, 1, 16, 32, 8, 128) == 0
    assert f(0, 1, 1, 100, 32, 8, 128) == 0 and f(1, 1, 1, 100, 32, 7, 128) == 0 and f(1, 1, 1, 100, 32, 8, 80) == 0


def test_binding_refuses_other_tensors(binding):
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):      # not on a GPU
        binding.rmsnorm_rope_fwd(q, None, None, None, None, None, q, None)
    for bad in (q.float(), q[0], q.transpose(0, 1), q[..., ::2]):
        with pytest.raises(ValueError):
            binding._heads(bad, "q")
    with pytest.raises(ValueError):
        binding._heads(q, "q_out", q[:1].shape)
    with pytest.raises(ValueError):
        binding._vec(torch.zeros(4, dtype=torch.int64), torch.int32, "positions")
    with pytest.raises(ValueError):
        binding._vec(torch.zeros(4, dtype=torch.int32), torch.int32, "positions", (5,))
    codes, scales = torch.zeros(3, 2, 32, 64, dtype=torch.uint8), torch.zeros(3, 2, 2, dtype=torch.uint8)
    assert binding._cache(codes, scales, codes, scales)[:5] == (3, 2, 32, 64, 16)
    for bad in ((codes, scales, codes[:2], scales), (codes, scales[:, :1], codes, scales), (codes.float(), scales, codes, scales)):
        with pytest.raises(ValueError):
            binding._cache(*bad)
