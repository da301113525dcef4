"""The operators of token-by-token decoding, measured alone: keys and values into a paged cache, attention of drafted tokens over
that cache, the selection of a beam search, and the reordering of its states.

A case is a dict of plain values; `op` names the operator:

  append   rows of q | k | v as the fused projection leaves them: q and k rotated to their positions, k and v written to the cache's pages
  attend   attention of every sequence's new rows (one token, a chain of tokens, a tree of drafted tokens) over its cached keys
  select   the n_out best continuations of every sequence over its beams and the vocabulary, from logits and running scores
  reorder  the beams' states (memory matrices, normalisers, token histories) gathered from the beams they continue

`heads`, `kv_heads` and `head_dim` are those of the repository's shapes.  Every operator is computed either in its plain form
(`own` false) or by the framework (`own` true)."""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

# heads, KV heads, head_dim of the repository's models
HEADS = {"tiny": (4, 2, 32), "160m": (12, 12, 64), "1b": (32, 8, 64), "3b": (24, 8, 128), "8b": (32, 8, 128)}
THETA = 500000.0
VOCAB = 128256
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # one decoding step of a few requests: the smallest calls, where latency counts
        dict(name="append_token_1b", op="append", model="1b", dtype="bf16", seqs=8, rows=1, ragged=False, context=1040, page=64, tree=False),
        # a tree of drafts in the fp32 configuration
        dict(name="append_tree_tiny_f32", op="append", model="tiny", dtype="f32", seqs=5, rows=13, ragged=True, context=72, page=16, tree=True),
        # prompts of many requests, ragged, behind a far context
        dict(name="append_prompts_3b", op="append", model="3b", dtype="bf16", seqs=24, rows=700, ragged=True, context=120000, page=64, tree=False),
        # one request, one token, one segment's worth of keys
        dict(name="attend_token_1b", op="attend", model="1b", dtype="bf16", seqs=1, rows=1, ragged=False, context=1040, page=64, tree=False),
        # a serving batch of uneven lengths, one token each
        dict(name="attend_batch_1b", op="attend", model="1b", dtype="bf16", seqs=48, rows=1, ragged=True, context=9000, page=64, tree=False),
        # few requests over very long contexts
        dict(name="attend_long_1b", op="attend", model="1b", dtype="bf16", seqs=3, rows=1, ragged=False, context=131072, page=64, tree=False),
        # trees of drafted tokens over contexts of uneven length
        dict(name="attend_tree_3b", op="attend", model="3b", dtype="bf16", seqs=16, rows=48, ragged=True, context=5000, page=32, tree=True),
        # small trees in fp32
        dict(name="attend_tree_tiny_f32", op="attend", model="tiny", dtype="f32", seqs=9, rows=7, ragged=True, context=600, page=16, tree=True),
        # one request, four beams, the whole vocabulary
        dict(name="select_one", op="select", seqs=1, beams=4, vocab=VOCAB, n_out=8, banned=0.0, dead=False),
        # many requests, an odd vocabulary, banned tokens, the first step of some of them (one live beam)
        dict(name="select_batch", op="select", seqs=24, beams=8, vocab=100003, n_out=16, banned=0.3, dead=True),
        # memory states of the 1b model: 16 layers of 2048 x 384
        dict(name="reorder_memory_1b", op="reorder", seqs=2, beams=4, layers=16, d_model=2048, phi=384, history=1024, dtype="f32"),
        # the fp32 configuration's states
        dict(name="reorder_tiny", op="reorder", seqs=3, beams=5, layers=4, d_model=128, phi=192, history=77, dtype="f32"),
    ]


def _log_int(rng, lo, hi):
    """An integer spread evenly over the logarithm of [lo, hi]."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the same ranges; costs at most what the largest listed one does."""
    op = rng.choice(["append", "attend", "attend", "attend", "select", "reorder"])
    if op == "select":
        vocab, beams = _log_int(rng, 1000, VOCAB), rng.randint(1, 16)
        seqs = _log_int(rng, 1, max(1, min(64, 19_000_000 // (vocab * beams))))
        return dict(op=op, seqs=seqs, beams=beams, vocab=vocab, n_out=rng.randint(beams, 2 * beams), banned=rng.choice([0.0, 0.3]),
                    dead=rng.random() < 0.5)
    if op == "reorder":
        layers, d_model, phi = rng.choice([(4, 128, 192), (12, 768, 384), (16, 2048, 384)])
        beams = rng.randint(2, 16)
        most = max(1, 100_000_000 // (layers * d_model * phi * beams))
        return dict(op=op, seqs=_log_int(rng, 1, min(16, most)), beams=min(beams, max(2, 100_000_000 // (layers * d_model * phi))),
                    layers=layers, d_model=d_model, phi=phi, history=_log_int(rng, 1, 4096), dtype=rng.choice(["f32", "bf16"]))
    model = rng.choice(["tiny", "160m", "1b", "1b", "3b", "8b"])
    dtype = "f32" if model == "tiny" else rng.choice(["bf16", "bf16", "bf16", "f32"])
    heads, kv_heads, dh = HEADS[model]
    page, tree = rng.choice([16, 32, 64, 128]), rng.random() < 0.5
    if op == "append":
        rows = rng.randint(2, 64) if tree else _log_int(rng, 1, 900)
        most = max(1, 50_000_000 // (rows * (heads + 2 * kv_heads) * dh))
        return dict(op=op, model=model, dtype=dtype, seqs=_log_int(rng, 1, min(64, most)), rows=rows, ragged=rng.random() < 0.7,
                    context=_log_int(rng, 1, 100000), page=page, tree=tree)
    rows = rng.randint(2, 64) if tree else rng.choice([1, 1, _log_int(rng, 2, 300)])
    context = _log_int(rng, 1, 40000)
    per_key = kv_heads * dh * (2 if dtype == "bf16" else 4) / 2 + heads * rows * 4          # cache and the plain form's scores
    most = max(1, int(180_000_000 // (per_key * (context + rows))))
    return dict(op=op, model=model, dtype=dtype, seqs=_log_int(rng, 1, min(64, most)), rows=rows, ragged=rng.random() < 0.7,
                context=context, page=page, tree=tree)


# ------------------------------------------------------------------------------------------------ inputs
def _sequences(case):
    """Rows and cached keys per sequence, which belong to the case.  Ragged: rows from one on, contexts from a quarter of the longest
    on, the first one whole."""
    n, rows, ctx = case["seqs"], np.full(case["seqs"], case["rows"]), np.full(case["seqs"], case["context"])
    rng = np.random.default_rng([n, case["rows"], case["context"]])
    if case["ragged"] and n > 1:
        rows[1:] = rng.integers(1, case["rows"] + 1, n - 1)
        ctx[1:] = rng.integers(case["context"] // 4, case["context"] + 1, n - 1)
    return rows, ctx


def _trees(rows, rng):
    """Per row the bits of the drafts that it sees (itself and its ancestors), and its depth."""
    masks, depths = [], []
    for n in rows:
        m, d = [], []
        for i in range(n):
            parent = int(rng.integers(max(0, i - 8), i)) if i else -1
            m.append((1 << i) | (m[parent] if i else 0))
            d.append(d[parent] + 1 if i else 0)
        masks += m
        depths += d
    return np.array(masks, dtype=np.uint64).view(np.int64), np.array(depths, dtype=np.int64)


def _cache_inputs(case, seed):
    rng = np.random.default_rng(seed)
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    heads, kv_heads, dh = HEADS[case["model"]]
    dt, page = DTYPES[case["dtype"]], case["page"]
    rows, ctx = _sequences(case)
    if case["op"] == "append" and case["context"] > 8 * page * 16:      # only the pages that are written have to exist: the far ones are others'
        first = ctx // page
    else:
        first = np.zeros_like(ctx)
    last = (ctx + rows + page - 1) // page
    need = int((last - first).sum())
    n_pages = need + 3
    order = rng.permutation(n_pages)[:need]
    pages = np.full((case["seqs"], int(last.max())), -1, dtype=np.int32)
    at = 0
    for s in range(case["seqs"]):
        pages[s, first[s]:last[s]] = order[at:at + last[s] - first[s]]
        at += last[s] - first[s]
    row_start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    masks, depths = _trees(rows, rng) if case["tree"] else (None, None)
    seq = np.repeat(np.arange(case["seqs"]), rows)
    inside = np.arange(len(seq)) - row_start[seq]
    positions = ctx[seq] + (depths if case["tree"] else inside)
    dev = lambda a: torch.from_numpy(np.ascontiguousarray(a)).cuda()  # noqa: E731
    normal = lambda *dims, std=1.0: torch.randn(dims, generator=gen, device="cuda").mul_(std).to(dt)  # noqa: E731
    s = dict(case=case, pages=dev(pages), lens=dev(ctx.astype(np.int32)), row_start=dev(row_start), max_rows=int(rows.max()),
             max_keys=int((ctx + rows).max()), tree=dev(masks) if case["tree"] else None, positions=dev(positions.astype(np.int32)),
             n_rows=int(rows.sum()), k=normal(n_pages, kv_heads, page, dh), v=normal(n_pages, kv_heads, page, dh))
    if case["op"] == "append":
        s["qkv"] = normal(s["n_rows"], (heads + 2 * kv_heads) * dh)
        s["q_out"] = torch.empty(s["n_rows"], heads * dh, device="cuda", dtype=dt)
    else:       # scores of a trained model spread over a few units
        s["q"] = normal(s["n_rows"], heads * dh, std=2.0)
        s["out"] = torch.empty(s["n_rows"], heads * dh, device="cuda", dtype=dt)
    return s


def _handle(case, k, v):
    import armt_synth as S
    import paper_2506_05229_amd as P
    heads, kv_heads, dh = HEADS[case["model"]]
    shape = S.get_shape("tiny").replace(n_heads=heads, n_kv_heads=kv_heads, head_dim=dh, d_model=heads * dh, d_ff=512, seg_len=64,
                                        n_mem=16, dtype=case["dtype"], rope_theta=THETA)
    return P.KvCache(shape, k, v)


def _reorder_dims(case):
    lead = (case["seqs"] * case["beams"], case["layers"])
    return [lead + (case["d_model"], case["phi"]), lead + (case["phi"],), (lead[0], case["history"])]


def prepare(case, seed):
    if case["op"] in ("append", "attend"):
        s = _cache_inputs(case, seed)
        s["cache"] = _handle(case, s["k"], s["v"]) if own else None
        return s
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    n = case["seqs"] * case["beams"]
    if case["op"] == "select":
        logits = torch.randn(n, case["vocab"], generator=gen, device="cuda").mul_(3.0)
        if case["banned"]:
            logits.masked_fill_(torch.rand(n, case["vocab"], generator=gen, device="cuda") < case["banned"], -math.inf)
        scores = torch.rand(case["seqs"], case["beams"], generator=gen, device="cuda").mul_(-6.0)
        if case["dead"]:
            scores[::3, 1:] = -math.inf
        return dict(case=case, logits=logits, scores=scores)
    A, z, history = _reorder_dims(case)
    dt = DTYPES[case["dtype"]]
    states = [torch.randn(A, generator=gen, device="cuda").to(dt), torch.rand(z, generator=gen, device="cuda"),
              torch.randint(0, VOCAB, history, generator=gen, device="cuda", dtype=torch.int32)]
    parents = torch.randint(0, case["beams"], (case["seqs"], case["beams"]), generator=gen, device="cuda", dtype=torch.int32)
    return dict(case=case, states=states, parents=parents, out=[torch.empty_like(t) for t in states])


# ------------------------------------------------------------------------------------------------ one pass
def run(s):
    return {"append": _append, "attend": _attend, "select": _select, "reorder": _reorder}[s["case"]["op"]](s)


def _row_owner(s):
    """Sequence of every row and the row's number inside it."""
    r = torch.arange(s["n_rows"], device="cuda")
    seq = (r[:, None] >= s["row_start"][None, 1:]).sum(1)
    return seq, r - s["row_start"][seq]


def _append(s):
    if own:
        s["cache"].append(s["qkv"], s["pages"], s["lens"], s["row_start"], s["positions"], out=s["q_out"])
        return s["q_out"], s["k"], s["v"]
    heads, kv_heads, dh = HEADS[s["case"]["model"]]
    page = s["case"]["page"]
    x = s["qkv"].view(s["n_rows"], heads + 2 * kv_heads, dh)
    freq = THETA ** (torch.arange(dh // 2, device="cuda", dtype=torch.float64) * (-2.0 / dh))
    angle = s["positions"].double()[:, None] * freq
    c, sn = angle.cos().float()[:, None], angle.sin().float()[:, None]
    rot = x[:, :heads + kv_heads].float()
    a, b = rot[..., :dh // 2], rot[..., dh // 2:]
    rot = torch.cat([a * c - b * sn, b * c + a * sn], -1).to(x.dtype)
    seq, inside = _row_owner(s)
    slot = s["lens"][seq] + inside
    where = s["pages"][seq, slot // page].long()
    s["k"][where, :, slot % page] = rot[:, heads:]
    s["v"][where, :, slot % page] = x[:, heads + kv_heads:]
    return rot[:, :heads].reshape(s["n_rows"], -1), s["k"], s["v"]


def _attend(s):
    if own:
        return s["cache"].attend(s["q"], s["pages"], s["lens"], s["row_start"], s["max_rows"], tree=s["tree"], out=s["out"])
    heads, kv_heads, dh = HEADS[s["case"]["model"]]
    page, n, group = s["case"]["page"], s["case"]["seqs"], heads // kv_heads
    t = torch.arange(s["max_keys"], device="cuda")
    where = s["pages"][:, t // page].clamp(min=0).long()
    k = s["k"][where, :, t % page].float().permute(0, 2, 3, 1).contiguous()             # [n, kv, dh, keys]
    v = s["v"][where, :, t % page].float().transpose(1, 2).contiguous()                 # [n, kv, keys, dh]
    i = torch.arange(s["max_rows"], device="cuda")
    row = (s["row_start"][:-1, None] + i).clamp(max=s["n_rows"] - 1)
    q = s["q"][row].float().view(n, s["max_rows"], kv_heads, group, dh).permute(0, 2, 1, 3, 4)
    score = torch.matmul(q.reshape(n, kv_heads, -1, dh), k) * dh ** -0.5
    draft = t - s["lens"][:, None]                                                      # [n, keys]: which draft a key is, negative: context
    rows = s["row_start"].diff()[:, None]
    bits = s["tree"][row][:, :, None] >> draft.clamp(0, 63)[:, None] & 1 if s["tree"] is not None else (draft[:, None] <= i[:, None])
    sees = ((draft < 0)[:, None] | (bits != 0)) & (draft < rows)[:, None]               # [n, rows, keys]
    sees = sees[:, None, :, None].expand(n, kv_heads, s["max_rows"], group, s["max_keys"]).reshape(score.shape)
    score = score.masked_fill(~sees, -math.inf)
    top = score.amax(-1, keepdim=True)
    p = (score - torch.where(top == -math.inf, 0.0, top)).exp()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, v) / torch.where(total == 0, 1.0, total)
    o = o.view(n, kv_heads, s["max_rows"], group, dh).permute(0, 2, 1, 3, 4).reshape(n, s["max_rows"], heads * dh)
    seq, inside = _row_owner(s)
    return o[seq, inside].to(s["q"].dtype)


def _select(s):
    c = s["case"]
    if own:
        import paper_2506_05229_amd as P
        return P.beam_select(s["logits"], s["scores"], c["n_out"])
    x = s["logits"].double()
    x = torch.where(x.isnan(), -math.inf, x).clamp(max=torch.finfo(torch.float32).max)
    top = x.amax(-1, keepdim=True)
    x = x - torch.where(top == -math.inf, 0.0, top)
    x = x - x.exp().sum(-1, keepdim=True).log().clamp(min=-1e300)
    total = (s["scores"].double().view(-1, 1) + x).view(c["seqs"], -1)
    best, at = torch.sort(total, dim=-1, descending=True, stable=True)
    at = at[:, :c["n_out"]]
    return best[:, :c["n_out"]].float(), (at // c["vocab"]).int(), (at % c["vocab"]).int()


def _reorder(s):
    c = s["case"]
    if own:
        import paper_2506_05229_amd as P
        return P.beam_reorder(s["parents"], s["states"], out=s["out"])
    first = torch.arange(c["seqs"], device="cuda")[:, None] * c["beams"]
    at = (first + s["parents"]).view(-1)
    return [t[at] for t in s["states"]]


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["op"] in ("append", "attend"):
        heads, kv_heads, dh = HEADS[case["model"]]
        size = 2 if case["dtype"] == "bf16" else 4
        per_seq, ctx = _sequences(case)
        rows = int(per_seq.sum())
        if case["op"] == "append":
            return {"bytes": 2 * rows * (heads + 2 * kv_heads) * dh * size, "flops": 3 * rows * (heads + kv_heads) * dh}
        pairs = float((per_seq * (ctx + (per_seq + 1) / 2)).sum())
        return {"bytes": 2 * int((ctx + per_seq).sum()) * kv_heads * dh * size + 2 * rows * heads * dh * size, "flops": 4 * pairs * heads * dh}
    n = case["seqs"] * case["beams"]
    if case["op"] == "select":
        return {"bytes": n * case["vocab"] * 4 + case["seqs"] * case["n_out"] * 12, "flops": 4 * n * case["vocab"]}
    sizes = (2 if case["dtype"] == "bf16" else 4, 4, 4)
    row = sum(math.prod(d[1:]) * b for d, b in zip(_reorder_dims(case), sizes))
    met = case["beams"] * (1 - (1 - 1 / case["beams"]) ** case["beams"])                # distinct parents among the beams of a sequence
    return {"bytes": case["seqs"] * (case["beams"] + met) * row, "flops": 0}


# ------------------------------------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    if case["op"] == "append":
        return _append_exact(_cache_inputs(case, seed))
    if case["op"] == "attend":
        return _attend_exact(_cache_inputs(case, seed))
    s = prepare(case, seed)
    return _select_exact(s) if case["op"] == "select" else _reorder_exact(s)


def _append_exact(s):
    c = s["case"]
    heads, kv_heads, dh = HEADS[c["model"]]
    x = torch.view_as_complex(torch.stack(s["qkv"].double().view(-1, heads + 2 * kv_heads, 2, dh // 2).unbind(2), -1).contiguous())
    turn = s["positions"].double()[:, None] * torch.exp(-math.log(THETA) * 2 / dh * torch.arange(dh // 2, device="cuda", dtype=torch.float64))
    rot = x[:, :heads + kv_heads] * torch.polar(torch.ones_like(turn), turn)[:, None]
    rot = torch.cat([rot.real, rot.imag], -1)
    k, v = s["k"].double(), s["v"].double()
    plain = s["qkv"].double().view(-1, heads + 2 * kv_heads, dh)[:, heads + kv_heads:]
    start, lens, pages = s["row_start"].tolist(), s["lens"].tolist(), s["pages"].cpu()
    for n in range(c["seqs"]):
        slots = torch.arange(lens[n], lens[n] + start[n + 1] - start[n])
        where, off = pages[n, slots // c["page"]].long().cuda(), (slots % c["page"]).cuda()
        k[where, :, off] = rot[start[n]:start[n + 1], heads:]
        v[where, :, off] = plain[start[n]:start[n + 1]]
    return rot[:, :heads].reshape(s["n_rows"], -1), k, v


def _attend_exact(s):
    c = s["case"]
    heads, kv_heads, dh = HEADS[c["model"]]
    start, lens = s["row_start"].tolist(), s["lens"].tolist()
    out = torch.empty(s["n_rows"], heads, dh, device="cuda", dtype=torch.float64)
    for n in range(c["seqs"]):
        rows, keys = start[n + 1] - start[n], lens[n] + start[n + 1] - start[n]
        used = s["pages"][n, :-(-keys // c["page"])].long()
        k = s["k"][used].double().transpose(0, 1).reshape(kv_heads, -1, dh)[:, :keys]
        v = s["v"][used].double().transpose(0, 1).reshape(kv_heads, -1, dh)[:, :keys]
        q = s["q"][start[n]:start[n + 1]].double().view(rows, heads, dh)
        hidden = torch.zeros(rows, keys, device="cuda", dtype=torch.bool)
        if s["tree"] is None:
            hidden[:, lens[n]:] = torch.ones(rows, rows, device="cuda").triu(1).bool()
        else:
            hidden[:, lens[n]:] = ((s["tree"][start[n]:start[n + 1], None] >> torch.arange(rows, device="cuda")) & 1) == 0
        for h in range(heads):
            score = q[:, h] @ k[h * kv_heads // heads].T / math.sqrt(dh)
            out[start[n]:start[n + 1], h] = torch.softmax(score.masked_fill(hidden, -math.inf), -1) @ v[h * kv_heads // heads]
    return out.view(s["n_rows"], -1)


def _select_exact(s):
    c = s["case"]
    best, parent, token = [], [], []
    for n in range(c["seqs"]):
        rows = s["logits"][n * c["beams"]:(n + 1) * c["beams"]].double()
        total = (s["scores"][n].double()[:, None] + rows - torch.logsumexp(rows, -1, keepdim=True)).flatten()
        edge = torch.topk(total, c["n_out"]).values[-1]
        near = torch.nonzero(total >= edge).flatten().tolist()
        order = sorted(zip(total[near].tolist(), near), key=lambda p: (-p[0], p[1]))[:c["n_out"]]
        best.append([p[0] for p in order])
        parent.append([p[1] // c["vocab"] for p in order])
        token.append([p[1] % c["vocab"] for p in order])
    as_int = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return torch.tensor(best, dtype=torch.float64), as_int(parent), as_int(token)


def _reorder_exact(s):
    c = s["case"]
    parents = s["parents"].tolist()
    out = []
    for t in s["states"]:
        rows = [t[n * c["beams"] + p] for n in range(c["seqs"]) for p in parents[n]]
        out.append(torch.stack(rows).double() if t.is_floating_point() else torch.stack(rows))
    return out
