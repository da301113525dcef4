"""Selection and reordering of a beam search against float64 and plain indexing."""
import math

import numpy as np
import pytest
import torch

from decode_reference import beam_select

pytestmark = pytest.mark.gpu


def check(logits, scores, n_out, device_logits=None):
    import paper_2506_05229_amd as P
    got = [t.cpu() for t in P.beam_select(logits.cuda() if device_logits is None else device_logits, scores.cuda(), n_out)]
    want = beam_select(logits, scores, n_out)
    assert torch.equal(got[1], want[1]) and torch.equal(got[2], want[2]), (got, want)
    # log of a sum in fp32: vocab / 256 additions per lane at most, exponentials of 3 half steps; the score is rounded once
    u, finite = 2.0 ** -24, want[0].isfinite()
    assert torch.equal(got[0].double()[~finite], want[0][~finite])
    err = (got[0].double() - want[0]).abs()[finite]
    assert (err <= u * want[0].abs()[finite] + (logits.shape[1] / 256 + 16) * u).all(), float(err.max())
    return got


@pytest.mark.parametrize("n,beams,vocab,n_out", [(1, 1, 1, 1), (1, 1, 7, 7), (2, 3, 5, 15), (1, 4, 128256, 8), (3, 5, 1003, 10), (2, 16, 4099, 32),
                                                 (1, 64, 300, 64), (5, 2, 2048, 1), (2, 1, 70001, 64), (70, 7, 513, 14)])
@pytest.mark.parametrize("kind", ["normal", "banned", "flat", "rising", "dead"])
def test_select(n, beams, vocab, n_out, kind):
    gen = torch.Generator().manual_seed(vocab + beams)
    logits = 3.0 * torch.randn(n * beams, vocab, generator=gen)
    scores = -4.0 * torch.rand(n, beams, generator=gen)
    if kind == "banned":                                     # nearly everything, as under a grammar
        logits[torch.rand(n * beams, vocab, generator=gen) < 0.97] = -math.inf
    elif kind == "flat":                                     # ties everywhere: the lowest indices
        logits.fill_(0.25)
        logits[:, vocab // 2] = -0.0
        scores.fill_(-1.0)
    elif kind == "rising":
        logits = torch.linspace(-5, 5, vocab).expand(n * beams, vocab) + 1e-3 * torch.arange(n * beams)[:, None]
        logits = logits.contiguous()
    elif kind == "dead":                                     # the first step of a search: one live beam; one sequence without any
        scores[:, 1:] = -math.inf
        scores[-1] = -math.inf
        if n > 1:
            scores[0, 0] = float("nan")
    check(logits, scores, n_out)


def test_select_values_that_are_not_finite():
    gen = torch.Generator().manual_seed(1)
    logits = torch.randn(12, 400, generator=gen)
    logits[0, ::3] = float("nan")
    logits[1] = float("nan")
    logits[2, 5], logits[2, 300] = math.inf, math.inf
    logits[3] = -math.inf
    logits[4] = -math.inf
    logits[4, 399] = -80.0
    logits[5] = -3.4e38
    logits[6, 10] = 3.4e38
    scores = -torch.rand(3, 4, generator=gen)
    scores[2, 3] = math.inf
    check(logits, scores, 9)


def test_select_rows_apart_and_unaligned():
    gen = torch.Generator().manual_seed(2)
    wide = torch.randn(6, 1031, generator=gen)
    check(wide[:, 3:1002].contiguous(), -torch.rand(2, 3, generator=gen), 6, device_logits=wide.cuda()[:, 3:1002])


def test_equal_beams_tie_to_the_lowest():
    gen = torch.Generator().manual_seed(3)
    row = torch.randn(1, 3000, generator=gen)
    got = check(row.repeat(4, 1), torch.full((1, 4), -2.0), 12)
    assert got[1][0].tolist() == [0, 1, 2, 3] * 3


def test_scores_in_place():
    import ctypes as C

    import paper_2506_05229_amd as P
    lib = P.load_library()
    gen = torch.Generator().manual_seed(6)
    x, scores = torch.randn(10, 700, generator=gen).cuda(), (-torch.rand(2, 5, generator=gen)).cuda()
    want = P.beam_select(x, scores, 5)
    parents, tokens = torch.empty(2, 5, dtype=torch.int32, device="cuda"), torch.empty(2, 5, dtype=torch.int32, device="cuda")
    need = lib.armt_beam_select_workspace_bytes(2, 5, 700, 5)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    call = lambda n_out, out: lib.armt_beam_select(x.data_ptr(), 700, scores.data_ptr(), 2, 5, 700, n_out, out, parents.data_ptr(),  # noqa: E731
                                                   tokens.data_ptr(), ws.data_ptr(), need, C.c_void_p(torch.cuda.current_stream().cuda_stream))
    assert call(4, scores.data_ptr()) == 2 and call(5, scores.data_ptr() + 4) == 2
    assert call(5, scores.data_ptr()) == 0
    torch.cuda.synchronize()
    assert torch.equal(scores, want[0]) and torch.equal(parents, want[1]) and torch.equal(tokens, want[2])


def test_select_and_reorder_replay_from_a_graph():
    import paper_2506_05229_amd as P
    gen = torch.Generator().manual_seed(4)
    inputs = [(torch.randn(8, 5000, generator=gen).cuda(), (-torch.rand(2, 4, generator=gen)).cuda()) for _ in range(4)]
    state = torch.randn(8, 6, 50, generator=gen).cuda()
    logits, scores = inputs[0][0].clone(), inputs[0][1].clone()
    P.beam_reorder(P.beam_select(logits, scores, 4)[1], [state])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = P.beam_select(logits, scores, 4)
        moved = P.beam_reorder(got[1], [state])
    for x, s in inputs:
        logits.copy_(x)
        scores.copy_(s)
        want = P.beam_select(x, s, 4)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert torch.equal(moved[0], P.beam_reorder(want[1], [state])[0])


# ------------------------------------------------------------------------------------------------ reorder
def plain(parents, t):
    n, beams = parents.shape
    at = (torch.arange(n)[:, None] * beams + parents.clamp(0, beams - 1)).view(-1)
    return t.reshape(n * beams, -1)[at].view(t.shape)


@pytest.mark.parametrize("beams", [1, 2, 4, 5, 8, 13, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("in_place", [False, True])
def test_reorder(beams, in_place):
    import paper_2506_05229_amd as P
    n = 3
    gen = torch.Generator().manual_seed(beams)
    parents = torch.randint(0, beams, (n, beams), generator=gen, dtype=torch.int32)
    parents[0] = torch.arange(beams)                         # everybody stays
    parents[1, -1], parents[1, 0] = beams + 3, -2            # clamped
    states = [torch.randn(n * beams, 2, 64, 33, generator=gen), torch.randn(n, beams, 77, generator=gen),
              torch.randint(0, 999, (n * beams, 5), generator=gen, dtype=torch.int32), torch.randn(n * beams, 4096, generator=gen).bfloat16()]
    want = [plain(parents, t) for t in states]
    dev = [t.cuda() for t in states]
    out = P.beam_reorder(parents.cuda(), dev, out=dev if in_place else None)
    torch.cuda.synchronize()
    for o, w, d, t in zip(out, want, dev, states):
        assert torch.equal(o.cpu(), w)
        assert in_place or torch.equal(d.cpu(), t)


@pytest.mark.parametrize("dtype,cols", [(torch.bfloat16, 131), (torch.uint8, 37), (torch.float64, 3), (torch.bool, 1)])
def test_reorder_odd_rows(dtype, cols):
    """Rows of two-byte and one-byte multiples, and rows further apart than they are long, between another state's rows."""
    import paper_2506_05229_amd as P
    gen = torch.Generator().manual_seed(cols)
    parents = torch.randint(0, 6, (2, 6), generator=gen, dtype=torch.int32)
    t = torch.randint(0, 2, (12, cols + 9), generator=gen).to(dtype)
    dev = t.cuda()
    P.beam_reorder(parents.cuda(), [dev[:, :cols], dev[:, cols + 2:]], out=[dev[:, :cols], dev[:, cols + 2:]])
    want = t.clone()
    want[:, :cols], want[:, cols + 2:] = plain(parents, t[:, :cols]), plain(parents, t[:, cols + 2:])
    assert torch.equal(dev.cpu(), want)


def test_a_search_step_by_step():
    """Append, attend, select and reorder as a search uses them: every beam's cache and scores follow its tokens.  The 'model' is one attention layer with
    random projections; the beams are compared with runs of each final token sequence from the start, in float64 on the host."""
    import paper_2506_05229_amd as P
    from decode_reference import cache_shape, rotate
    shape, vocab, beams, steps, ctx, page = cache_shape("tiny", "f32"), 50, 4, 5, 21, 16
    H, Hkv, dh = shape.n_heads, shape.n_kv_heads, shape.head_dim
    gen = torch.Generator().manual_seed(8)
    emb, proj = torch.randn(vocab, 64, generator=gen), 0.1 * torch.randn(64, (H + 2 * Hkv) * dh, generator=gen)
    head = 0.3 * torch.randn(H * dh, vocab, generator=gen)
    prompt = torch.randint(0, vocab, (2, ctx), generator=gen)
    n, per = 2 * beams, 2                                    # beams of two sequences, two pages each
    k, v = (torch.zeros(n * per, Hkv, page, dh, device="cuda") for _ in range(2))
    pages = torch.arange(n * per, dtype=torch.int32, device="cuda").view(n, per)
    cache = P.KvCache(shape, k, v)
    de, dp, dh_ = emb.cuda(), proj.cuda(), head.cuda()
    zero, tok = torch.zeros(n, dtype=torch.int32, device="cuda"), prompt.repeat_interleave(beams, 0).cuda()
    rows = torch.arange(0, n * ctx + 1, ctx, dtype=torch.int32, device="cuda")
    q = cache.append((de[tok.reshape(-1)] @ dp).contiguous(), pages, zero, rows)
    h = cache.attend(q, pages, zero, rows, ctx).view(n, ctx, -1)[:, -1]
    scores = torch.full((2, beams), -math.inf, device="cuda")
    scores[:, 0] = 0.0
    one = torch.arange(n + 1, dtype=torch.int32, device="cuda")
    history = torch.zeros(n, steps, dtype=torch.int32, device="cuda")
    for t in range(steps):
        scores, parents, tokens = P.beam_select((h @ dh_).contiguous(), scores, beams)
        P.beam_reorder(parents, [k.view(n, -1), v.view(n, -1), history], out=[k.view(n, -1), v.view(n, -1), history])
        history[:, t] = tokens.view(-1)
        if t + 1 < steps:
            lens = torch.full((n,), ctx + t, dtype=torch.int32, device="cuda")
            q = cache.append((de[tokens.view(-1).long()] @ dp).contiguous(), pages, lens, one)
            h = cache.attend(q, pages, lens, one, 1)
    torch.cuda.synchronize()

    def run(tokens):                                          # log-probability of the tokens behind the prompt
        x = (emb.double()[tokens] @ proj.double()).view(len(tokens), H + 2 * Hkv, dh)
        r = rotate(x[:, :H + Hkv], torch.arange(len(tokens)), 500000.0)
        total = 0.0
        for i in range(ctx - 1, len(tokens) - 1):
            o = [torch.softmax(r[:i + 1, H + g * Hkv // H] @ r[i, g] / math.sqrt(dh), 0) @ x[:i + 1, H + Hkv + g * Hkv // H] for g in range(H)]
            total += float(torch.log_softmax(torch.cat(o) @ head.double(), 0)[tokens[i + 1]])
        return total

    got, hist = scores.cpu().double(), history.cpu().view(2, beams, steps)
    for s in range(2):
        assert len({tuple(b.tolist()) for b in hist[s]}) == beams and (got[s].diff() <= 0).all()
        for b in range(beams):
            want = run(torch.cat([prompt[s], hist[s, b].long()]))
            # five steps of fp32 attention and products over at most 128 terms of size ~ 1: 128 u each, amplified by the head's norm (~ 3)
            assert abs(float(got[s, b]) - want) < 5 * 3 * 128 * 2.0 ** -24 * 8, (s, b)
