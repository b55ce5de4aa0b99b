"""Refusals of the cache's further entry points (masks, summed weights, choice, moving), without a GPU: every call fails or returns before a launch."""
import pytest
import torch

from tests.test_abi_qkv_host import ALIGN, CACHE, ENUM, FAKE, NULL, OK, SHAPE, WORKSPACE, binding  # noqa: F401

SIZES = dict(q=FAKE, qs=512, n=3, qh=4, heads=2, dim=128, cu=FAKE, seqs=2, mq=2, lens=FAKE, ml=200, table=FAKE, width=4, pages=9, page=64, block=16,
             kc=FAKE, ksc=FAKE, vc=FAKE, vsc=FAKE, scale=0.1)
HEAD = ("q", "qs", "n", "qh", "heads", "dim", "cu", "seqs", "mq", "lens", "ml", "table", "width", "pages", "page", "block", "kc", "ksc", "vc", "vsc", "scale")
ATTEND = CACHE + [
    (dict(dim=32), SHAPE), (dict(qh=5), SHAPE), (dict(mq=0), SHAPE), (dict(ml=-1), SHAPE), (dict(ml=257), SHAPE), (dict(scale=float("nan")), SHAPE),
    (dict(q=None), NULL), (dict(q=FAKE + 8), ALIGN), (dict(qs=100), SHAPE), (dict(page=2 ** 31 - 1), SHAPE), (dict(block=2 ** 31 - 1), SHAPE),
    (dict(heads=-2), SHAPE),
]
OUT = [(dict(out=None), NULL), (dict(os=516), ALIGN), (dict(lse=FAKE + 2), ALIGN), (dict(), WORKSPACE), (dict(ws=FAKE, wsb=100), WORKSPACE),
       (dict(ws=FAKE + 4, wsb=10 ** 9), ALIGN)]


def masked(entry, middle):
    def call(L, kw):
        a = dict(SIZES, window=50, sinks=4, mask=FAKE, words=1, out=FAKE, os=512, lse=None, ws=None, wsb=0)
        a.update(kw)
        return getattr(L, entry)(*(a[n] for n in HEAD + middle + ("out", "os", "lse", "ws", "wsb")), None)
    return call


@pytest.mark.parametrize("kw,status", [x for x in ATTEND + OUT] + [
    (dict(window=0), SHAPE), (dict(window=-1), SHAPE), (dict(window=2 ** 31), SHAPE), (dict(sinks=-1), SHAPE), (dict(sinks=2 ** 31), SHAPE),
])
def test_sinks(binding, kw, status):  # noqa: F811
    kw = dict(kw) if "window" in kw else dict(kw, window=150)
    assert masked("mxkv_attention_sinks", ("window", "sinks"))(binding.lib, kw) == status


@pytest.mark.parametrize("kw,status", ATTEND + OUT + [
    (dict(words=0), SHAPE), (dict(words=-1), SHAPE), (dict(words=2 ** 31), SHAPE), (dict(mask=None), NULL), (dict(mask=FAKE + 2), ALIGN),
    (dict(mask=None, n=0), OK),
])
def test_tree(binding, kw, status):  # noqa: F811
    assert masked("mxkv_attention_tree", ("mask", "words"))(binding.lib, kw) == status


@pytest.mark.parametrize("kw,status", [x for x in ATTEND if x[0] not in (dict(n=0), dict(vc=None), dict(vsc=None), dict(vc=FAKE + 8))] + [
    (dict(causal=2), ENUM), (dict(window=-1), SHAPE), (dict(sinks=-1), SHAPE), (dict(sinks=3), SHAPE), (dict(sinks=3, window=9, causal=0), SHAPE),
    (dict(window=2 ** 31), SHAPE), (dict(lse=None), NULL), (dict(lse=FAKE + 1), ALIGN), (dict(sums=None), NULL), (dict(sums=FAKE + 2), ALIGN),
    (dict(earlier=FAKE + 2), ALIGN), (dict(ml=0), OK), (dict(n=2 ** 30, qh=8), SHAPE),
])
def test_weights(binding, kw, status):  # noqa: F811
    a = dict(SIZES, causal=1, window=0, sinks=0, lse=FAKE, earlier=None, sums=FAKE)
    a.update(kw)
    if "qh" in kw and kw["qh"] == 8:
        a.update(qs=8 * 128, heads=2)
    names = [n for n in HEAD if n not in ("vc", "vsc")] + ["causal", "window", "sinks", "lse", "earlier", "sums"]
    assert binding.lib.mxkv_attention_weights(*(a[n] for n in names), None) == status


@pytest.mark.parametrize("kw,status", [
    (dict(heads=0), SHAPE), (dict(seqs=-1), SHAPE), (dict(seqs=0), OK), (dict(width=0), SHAPE), (dict(pages=0), SHAPE), (dict(page=48), SHAPE),
    (dict(page=512), SHAPE), (dict(ml=-1), SHAPE), (dict(ml=257), SHAPE), (dict(keep=-1), SHAPE), (dict(keep=2 ** 31), SHAPE), (dict(sinks=-1), SHAPE),
    (dict(recent=-1), SHAPE), (dict(sinks=60, recent=41), SHAPE), (dict(sinks=2 ** 62, recent=2 ** 62), SHAPE), (dict(w=None), NULL), (dict(lens=None), NULL),
    (dict(table=None), NULL), (dict(kept=None), NULL), (dict(new=None), NULL), (dict(w=FAKE + 2), ALIGN), (dict(kept=FAKE + 2), ALIGN),
    (dict(new=FAKE + 1), ALIGN), (dict(seqs=2 ** 28, heads=4000), SHAPE),
])
def test_select(binding, kw, status):  # noqa: F811
    a = dict(w=FAKE, heads=2, seqs=2, lens=FAKE, ml=200, table=FAKE, width=4, pages=9, page=64, keep=100, sinks=4, recent=10, kept=FAKE, new=FAKE)
    a.update(kw)
    assert binding.lib.mxkv_select(*(a[n] for n in ("w", "heads", "seqs", "lens", "ml", "table", "width", "pages", "page", "keep", "sinks", "recent", "kept",
                                                    "new")), None) == status


@pytest.mark.parametrize("kw,status", [x for x in CACHE if "n" not in x[0]] + [
    (dict(dim=96), SHAPE), (dict(kept_heads=0), SHAPE), (dict(kept_heads=3), SHAPE), (dict(n=-1), SHAPE), (dict(n=2 ** 31), SHAPE), (dict(n=0), OK),
    (dict(kept=None), NULL), (dict(kept=FAKE + 2), ALIGN), (dict(first=FAKE + 2), ALIGN), (dict(sums=FAKE + 2), ALIGN), (dict(), WORKSPACE),
    (dict(ws=FAKE, wsb=16), WORKSPACE), (dict(ws=FAKE + 4, wsb=10 ** 9), ALIGN), (dict(out=FAKE, ws=FAKE, wsb=16), WORKSPACE), (dict(out=FAKE + 64, ow=0), SHAPE),
    (dict(out=FAKE + 66, ow=4), ALIGN), (dict(out=FAKE + 64, ow=2 ** 31), SHAPE), (dict(seqs=2 ** 29), SHAPE), (dict(pages=2 ** 24), SHAPE), (dict(pages=2 ** 24 - 1), WORKSPACE),
])
def test_compact(binding, kw, status):  # noqa: F811
    a = dict(kept=FAKE, kept_heads=2, n=100, first=None, cu=FAKE, lens=FAKE, heads=2, dim=128, seqs=2, table=FAKE, width=4, out=None, ow=0, pages=9, page=64,
             block=16, kc=FAKE, ksc=FAKE, vc=FAKE, vsc=FAKE, sums=None, ws=None, wsb=0)
    a.update(kw)
    assert binding.lib.mxkv_compact(*(a[n] for n in ("kept", "kept_heads", "n", "first", "cu", "lens", "heads", "dim", "seqs", "table", "width", "out", "ow",
                                                     "pages", "page", "block", "kc", "ksc", "vc", "vsc", "sums", "ws", "wsb")), None) == status


def test_compact_workspace(binding):  # noqa: F811
    f = binding.mxkv_compact_workspace_bytes
    assert f(2, 2, 100) >= 4 * 4 * 2 * 2 and f(1, 1, 1) > 0 and f(3, 2, 1000) >= f(2, 2, 1000) >= f(2, 1, 1000) >= f(2, 1, 10)
    assert f(0, 2, 100) == 0 and f(1, 0, 5) == 0 and f(1, 1, 0) == 0 and f(1, 1, 2 ** 31) == 0


def test_binding_refuses_other_tensors(binding):  # noqa: F811
    codes = torch.zeros(3, 2, 32, 64, dtype=torch.uint8)
    assert binding._weights(None, "earlier", codes.shape) is None
    for bad in (torch.zeros(3, 2, 32, dtype=torch.float64), torch.zeros(3, 2, 16), torch.zeros(3, 32, 2).transpose(1, 2)):
        with pytest.raises(ValueError):
            binding._weights(bad, "weights", codes.shape)
    q = torch.zeros(2, 4, 64, dtype=torch.bfloat16)
    for call in (lambda: binding.mxkv_select(torch.zeros(3, 2, 32), q, q, q, q, 5), lambda: binding.mxkv_attention_tree(*[q] * 9, 1, 1, 1.0, q)):
        with pytest.raises(ValueError):      # not on a GPU
            call()


def test_lists_of_choice_and_move(binding):  # noqa: F811
    """Every list's type, shape and layout is looked at, whichever way the check takes."""
    good = dict(kept=torch.zeros(3, 2, 5, dtype=torch.int32), new_lens=torch.zeros(3, dtype=torch.int32), kv_lens=torch.zeros(3, dtype=torch.int32),
                page_table=torch.zeros(3, 4, dtype=torch.int32))
    assert binding._kept_lists(**good, s=3) == tuple(t.data_ptr() for t in good.values())
    wide = torch.zeros(3, 2, 10, dtype=torch.int32)
    for name, bad in (("kept", good["kept"].long()), ("kept", good["kept"][:2]), ("kept", wide[..., ::2]), ("new_lens", good["new_lens"][:2]),
                      ("new_lens", torch.zeros(3, 1, dtype=torch.int32)), ("kv_lens", torch.zeros(6, dtype=torch.int32)[::2]),
                      ("kv_lens", good["kv_lens"].float()), ("page_table", good["page_table"].long()), ("page_table", torch.zeros(4, 3, dtype=torch.int32).t())):
        with pytest.raises(ValueError):
            binding._kept_lists(**dict(good, **{name: bad}), s=3)
