"""Refusals and sizes of the decoding operators: on the host, before anything is launched (no GPU)."""
import ctypes as C

import pytest

from decode_reference import cache_shape

FAKE = 4096            # a "device pointer" that nothing may touch
OK, NULL, SHAPE, DTYPE, WORKSPACE, UNSUPPORTED = 0, 1, 2, 3, 4, 6


@pytest.fixture(scope="module")
def lib():
    import paper_2506_05229_amd as P
    return P.load_library()


def cfg(heads="1b", of="bf16", **kw):
    import paper_2506_05229_amd as P
    c = P.ArmtConfig.from_shape(cache_shape(heads, of))
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def cache(**kw):
    from paper_2506_05229_amd.binding import ArmtKvCache
    c = ArmtKvCache(k=FAKE, v=FAKE, pages=FAKE, lens=FAKE, row_start=FAKE, n_seqs=2, n_pages=9, page_len=64, max_pages=4, page_stride=0)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


CACHE = [(dict(k=None), NULL), (dict(v=None), NULL), (dict(pages=None), NULL), (dict(lens=None), NULL), (dict(row_start=None), NULL),
         (dict(n_seqs=0), SHAPE), (dict(n_seqs=65537), SHAPE), (dict(n_pages=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(page_len=0), SHAPE),
         (dict(page_len=8), UNSUPPORTED), (dict(page_len=48), UNSUPPORTED), (dict(page_len=8192), UNSUPPORTED),
         (dict(page_stride=8 * 64 * 64 - 8), SHAPE), (dict(page_stride=8 * 64 * 64 + 4), UNSUPPORTED), (dict(k=FAKE + 8), UNSUPPORTED), (dict(v=FAKE + 2), UNSUPPORTED)]
CONFIG = [(dict(dtype=7), DTYPE), (dict(n_kv_heads=5), SHAPE), (dict(head_dim=32), SHAPE), (dict(n_kv_heads=2), UNSUPPORTED)]


@pytest.mark.parametrize("kw,status", CACHE)
def test_cache_refusals(lib, kw, status):
    c, k = cfg(), cache(**kw)
    assert lib.armt_kv_append(C.byref(c), C.byref(k), FAKE, 48 * 64, 5, None, FAKE, None) == status
    assert lib.armt_kv_attention(C.byref(c), C.byref(k), FAKE, 5, 3, None, FAKE, FAKE, 1 << 40, None) == status


@pytest.mark.parametrize("kw,status", CONFIG)
def test_configuration_refusals(lib, kw, status):
    c, k = cfg(**kw), cache()
    assert lib.armt_kv_append(C.byref(c), C.byref(k), FAKE, 48 * 64, 5, None, FAKE, None) == status
    assert lib.armt_kv_attention(C.byref(c), C.byref(k), FAKE, 5, 3, None, FAKE, FAKE, 1 << 40, None) == status
    assert lib.armt_kv_attention_workspace_bytes(C.byref(c), 2, 4, 64, 5, 3) == 0


def test_fp32_head_sizes(lib):
    for dim, status in ((18, UNSUPPORTED), (132, UNSUPPORTED)):
        c = cfg("tiny", "f32", head_dim=dim, d_model=4 * dim)
        assert lib.armt_kv_append(C.byref(c), C.byref(cache()), FAKE, 4096, 5, None, FAKE, None) == status


def test_append_refusals(lib):
    c, k = cfg(), cache()
    call = lambda qkv=FAKE, ld=48 * 64, n=5, out=FAKE + (1 << 20): lib.armt_kv_append(C.byref(c), C.byref(k), qkv, ld, n, None, out, None)  # noqa: E731
    assert lib.armt_kv_append(None, C.byref(k), FAKE, 48 * 64, 5, None, FAKE, None) == NULL
    assert lib.armt_kv_append(C.byref(c), None, FAKE, 48 * 64, 5, None, FAKE, None) == NULL
    assert call(qkv=None) == NULL and call(out=None) == NULL
    assert call(n=0) == SHAPE and call(ld=48 * 64 - 8) == SHAPE
    assert call(ld=48 * 64 + 4) == UNSUPPORTED and call(qkv=FAKE + 4) == UNSUPPORTED and call(out=FAKE + (1 << 20) + 8) == UNSUPPORTED and call(out=FAKE + 4096) == SHAPE


def test_attention_refusals(lib):
    c, k = cfg(), cache()
    need = lib.armt_kv_attention_workspace_bytes(C.byref(c), 2, 4, 64, 5, 3)
    assert need >= 256

    def call(q=FAKE, n=5, rows=3, tree=None, out=FAKE + (1 << 20), ws=FAKE, size=need):
        return lib.armt_kv_attention(C.byref(c), C.byref(k), q, n, rows, tree, out, ws, size, None)

    assert call(q=None) == NULL and call(out=None) == NULL
    assert call(n=0) == SHAPE and call(rows=0) == SHAPE and call(rows=65, tree=FAKE, size=1 << 40) == SHAPE
    assert call(q=FAKE + 8) == UNSUPPORTED and call(out=FAKE + (1 << 20) + 4) == UNSUPPORTED and call(out=FAKE + 64) == SHAPE
    assert call(ws=None) == WORKSPACE and call(ws=FAKE + 128) == WORKSPACE and call(size=need - 1) == WORKSPACE
    assert call(rows=2 ** 31 - 1, size=1 << 62) == UNSUPPORTED


def test_attention_workspace(lib):
    c = cfg()
    size = lambda *a: lib.armt_kv_attention_workspace_bytes(C.byref(c), *a)  # noqa: E731
    assert all(size(*a) == 0 for a in ((0, 4, 64, 1, 1), (2, 0, 64, 1, 1), (2, 4, 0, 1, 1), (2, 4, 64, 0, 1), (2, 4, 64, 1, 0), (65537, 4, 64, 1, 1)))
    assert 0 < size(1, 1, 16, 1, 1) <= 1 << 16                                    # keys of one step: nothing is cut
    assert size(1, 1, 16, 1, 1) <= size(1, 16384, 64, 1, 1) < 64 << 20 and size(256, 16384, 64, 256 * 64, 64) < 2 << 30


def test_beam_select_refusals(lib):
    need = lib.armt_beam_select_workspace_bytes(2, 3, 1000, 6)
    assert need > 0
    assert all(lib.armt_beam_select_workspace_bytes(*a) == 0 for a in ((0, 3, 9, 1), (2, 0, 9, 1), (2, 3, 0, 1), (2, 3, 9, 0), (2, 3, 9, 28), (2, 3, 999, 65),
                                                                      (1, 3, 2 ** 31 - 1, 6), (2 ** 24, 1, 9, 1)))

    def call(x=FAKE, ld=1000, s=FAKE, n=2, beams=3, vocab=1000, n_out=6, o=(2 * FAKE, 3 * FAKE, 4 * FAKE), ws=FAKE, size=need):
        return lib.armt_beam_select(x, ld, s, n, beams, vocab, n_out, *o, ws, size, None)

    assert call(x=None) == NULL and call(s=None) == NULL
    assert all(call(o=tuple(None if i == j else (2 + i) * FAKE for i in range(3))) == NULL for j in range(3))
    assert call(n=0) == SHAPE and call(beams=0) == SHAPE and call(vocab=0) == SHAPE and call(n_out=0) == SHAPE and call(ld=999) == SHAPE
    assert call(vocab=1, n_out=4) == SHAPE
    assert call(n_out=65) == UNSUPPORTED and call(beams=2 ** 22) == UNSUPPORTED
    assert call(ws=None) == WORKSPACE and call(ws=FAKE + 64) == WORKSPACE and call(size=need - 1) == WORKSPACE
    assert all(call(o=tuple(FAKE if i == j else (2 + i) * FAKE for i in range(3))) == SHAPE for j in range(3))


def test_beam_reorder_refusals(lib):
    from paper_2506_05229_amd.binding import ArmtBeamState

    def call(*states, parents=FAKE, n=2, beams=4, count=None):
        c = (ArmtBeamState * max(1, len(states)))()
        for s, (src, dst, size, *strides) in zip(c, states):
            s.src, s.dst, s.row_bytes = src, dst, size
            s.src_stride, s.dst_stride = strides if strides else (0, 0)
        return lib.armt_beam_reorder(parents, n, beams, c if states else None, len(states) if count is None else count, None)

    far = 1 << 20
    fine = (FAKE, FAKE + far, 100)
    assert call(fine, parents=None) == NULL and call() == NULL
    assert call((None, FAKE, 100)) == NULL and call((FAKE, None, 100)) == NULL
    assert call(fine, n=0) == SHAPE and call(fine, beams=0) == SHAPE and call(fine, count=0) == SHAPE
    assert call(fine, beams=65) == UNSUPPORTED and call(*[fine] * 9) == UNSUPPORTED
    assert call((FAKE, FAKE + far, 0)) == SHAPE and call((FAKE, FAKE + far, 100, 99, 100)) == SHAPE and call((FAKE, FAKE + far, 100, 100, 64)) == SHAPE
    assert call((FAKE, FAKE + 100, 100)) == SHAPE                              # shifted by a row
    assert call((FAKE, FAKE, 100, 100, 200)) == SHAPE                          # in place, other strides
    assert call((FAKE, FAKE, 100), (FAKE, FAKE, 100)) == SHAPE                 # written twice
    assert call((FAKE, FAKE + far, 100), (FAKE + far, FAKE + 2 * far, 100)) == SHAPE      # what one writes another reads
    assert call((FAKE, FAKE, 100, 200, 200), (FAKE + 60, FAKE + 60, 100, 200, 200)) == SHAPE
    assert call((FAKE, FAKE + far, 1 << 40)) == SHAPE or call((FAKE, FAKE + far, 1 << 40)) == UNSUPPORTED


def test_selection_of_the_reference_itself():
    """The float64 selection against a sort of all continuations."""
    import math

    import torch
    from decode_reference import beam_select
    gen = torch.Generator().manual_seed(0)
    logits, scores = torch.randn(6, 40, generator=gen), -torch.rand(2, 3, generator=gen)
    total = (scores.double().view(-1, 1) + torch.log_softmax(logits.double(), 1)).view(2, -1)
    best, at = torch.sort(total, descending=True, stable=True)
    s, p, t = beam_select(logits, scores, 7)
    assert torch.allclose(s, best[:, :7], rtol=0, atol=1e-14) and torch.equal(p * 40 + t, at[:, :7].int())
    s, p, t = beam_select(torch.full((3, 4), -math.inf), scores[:1], 5)
    assert (s == -math.inf).all() and (p * 4 + t).tolist() == [[0, 1, 2, 3, 4]]
