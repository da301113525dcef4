"""Plain float64 forms of the decoding operators and the problems their tests share."""
import math

import numpy as np
import torch

import armt_synth as S

HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}      # half a step relative to the value
HEADS = {"tiny": (4, 2, 32), "narrow": (6, 3, 20), "wide": (4, 1, 100), "160m": (12, 12, 64), "1b": (32, 8, 64), "3b": (24, 8, 128), "8b": (32, 8, 128),
         "one": (8, 1, 64),
         "mini": (3, 1, 4), "eight": (2, 2, 8), "twelve": (4, 2, 12)}


def cache_shape(heads, dtype, theta=500000.0):
    H, Hkv, dh = HEADS[heads]
    return S.get_shape("tiny").replace(n_heads=H, n_kv_heads=Hkv, head_dim=dh, d_model=H * dh, d_ff=512, seg_len=64, n_mem=16, dtype=dtype,
                                       rope_theta=theta)


def torch_type(dtype):
    return torch.bfloat16 if dtype == "bf16" else torch.float32


class Problem:
    """A cache whose unused places hold NaN, sequences of given lengths over scattered pages, and rows on top of them."""

    def __init__(self, heads, dtype, page, lens, rows, seed=0, spare_rows=0, pool_pages=1, fill=float("nan"), extra_pages=2):
        self.heads, self.dt, self.page, self.lens, self.rows = heads, torch_type(dtype), page, list(lens), list(rows)
        self.H, self.Hkv, self.dh = HEADS[heads]
        self.shape = cache_shape(heads, dtype)
        rng = np.random.default_rng(seed)
        gen = torch.Generator().manual_seed(seed)
        self.gen = gen
        n = len(self.lens)
        counts = [-(-(l + r) // page) for l, r in zip(lens, rows)]
        n_pages = sum(counts) + extra_pages
        order = rng.permutation(n_pages)
        pages = np.full((n, max(max(counts), 1) + 1), -1, dtype=np.int32)
        at = 0
        for s, c in enumerate(counts):
            pages[s, :c] = order[at:at + c]
            at += c
        self.pages = torch.from_numpy(pages)
        self.row_start = torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32)
        self.n_rows = int(self.row_start[-1]) + spare_rows
        pool = torch.full((n_pages, pool_pages, self.Hkv, page, self.dh), fill, dtype=self.dt)
        self.k_pool, self.v_pool = pool, pool.clone()
        self.k, self.v = self.k_pool[:, pool_pages - 1], self.v_pool[:, pool_pages - 1]
        for s in range(n):                                   # the context
            for t in range(self.lens[s]):
                p = int(pages[s, t // page])
                self.k[p, :, t % page] = torch.randn(self.Hkv, self.dh, generator=gen).to(self.dt)
                self.v[p, :, t % page] = torch.randn(self.Hkv, self.dh, generator=gen).to(self.dt)

    def own_keys(self):
        """Random keys and values for the call's own rows, written where armt_kv_append would."""
        for s, r in enumerate(self.rows):
            for i in range(r):
                t = self.lens[s] + i
                p = int(self.pages[s, t // self.page])
                self.k[p, :, t % self.page] = torch.randn(self.Hkv, self.dh, generator=self.gen).to(self.dt)
                self.v[p, :, t % self.page] = torch.randn(self.Hkv, self.dh, generator=self.gen).to(self.dt)

    def queries(self, std=2.0):
        return (std * torch.randn(self.n_rows, self.H * self.dh, generator=self.gen)).to(self.dt)

    def trees(self, seed=1):
        rng = np.random.default_rng(seed)
        words = np.zeros(self.n_rows, dtype=np.uint64)
        for s, r in enumerate(self.rows):
            for i in range(r):
                at = int(self.row_start[s]) + i
                words[at] = np.uint64(1 << i)
                if i:
                    words[at] |= words[int(self.row_start[s]) + int(rng.integers(0, i))]
        return torch.from_numpy(words.view(np.int64))

    def on_gpu(self):
        import paper_2506_05229_amd as P
        self.kd, self.vd = self.k_pool.cuda()[:, -1], self.v_pool.cuda()[:, -1]
        self.args = (self.pages.cuda(), torch.tensor(self.lens, dtype=torch.int32).cuda(), self.row_start.cuda())
        return P.KvCache(self.shape, self.kd, self.vd)

    def keys_of(self, s):
        """k, v [keys, Hkv, dh] of a sequence in float64, and which of them exist."""
        n = self.lens[s] + self.rows[s]
        t = torch.arange(min(n, self.pages.shape[1] * self.page))
        page = self.pages[s, t // self.page].long()
        have = (page >= 0) & (page < self.k.shape[0])
        page = page.clamp(0, self.k.shape[0] - 1)
        return self.k[page, :, t % self.page].double(), self.v[page, :, t % self.page].double(), have

    def attend(self, q, tree=None, max_rows=None, called=None):
        """Output, and a bound of the kernel's rounding, per element (rows that nobody owns: NaN).  called: the max_rows of the call.

        The bound counts half steps.  Output: one of its type.  Second product in bf16: every probability rounded once, so at most a half step of
        sum p |v|, or twice (the rest of the first rounding) for few keys or rows: a half step of a half step.  In fp32, with u = 2^-24: a score of dh products is off by (dh + 4) u sum |q k| / sqrt(dh), the exponential by
        3 u, sums over n keys by (n + 8) u; each moves the result by at most twice that share of sum p |v|."""
        H, Hkv, dh, u = self.H, self.Hkv, self.dh, 2.0 ** -24
        called = called or max_rows or max(self.rows)
        out = torch.full((self.n_rows, H, dh), float("nan"), dtype=torch.float64)
        tol = torch.zeros_like(out)
        for s in range(len(self.lens)):
            k, v, have = self.keys_of(s)
            half = HALF_STEP[self.dt]
            half_p = 0 if self.dt == torch.float32 else half * half if min(self.rows[s], called) * H // Hkv <= 64 or len(have) <= 512 else half
            for i in range(self.rows[s] if max_rows is None else min(self.rows[s], max_rows)):
                r = int(self.row_start[s]) + i
                see = have.clone()
                for j in range(len(have) - self.lens[s]):
                    ok = (int(tree[r]) >> j) & 1 if tree is not None else j <= i
                    see[self.lens[s] + j] &= bool(ok)
                kk, vv = k[see], v[see]
                for h in range(H):
                    qq = q[r].double().view(H, dh)[h]
                    if len(kk) == 0:
                        out[r, h] = 0
                        continue
                    sc = kk[:, h * Hkv // H] @ qq / math.sqrt(dh)
                    p = torch.softmax(sc, 0)
                    out[r, h] = p @ vv[:, h * Hkv // H]
                    spread = p @ vv[:, h * Hkv // H].abs()
                    off = (kk[:, h * Hkv // H].abs() @ qq.abs()).max() / math.sqrt(dh) * (dh + 4) * u + (len(kk) + 11) * u
                    tol[r, h] = half * out[r, h].abs() + spread * (2 * off + half_p) * 1.02
        return out.view(self.n_rows, -1), tol.view(self.n_rows, -1)


def rotate(x, positions, theta):
    """R(p) x for x [n, heads, dh] in float64."""
    half = x.shape[-1] // 2
    ang = positions.double()[:, None] * theta ** (-torch.arange(half, dtype=torch.float64) / half)
    c, s = ang.cos()[:, None], ang.sin()[:, None]
    a, b = x[..., :half].double(), x[..., half:].double()
    return torch.cat([a * c - b * s, b * c + a * s], -1)


def beam_select(logits, scores, n_out):
    """float64 selection: (scores, parents, tokens)."""
    n, beams = scores.shape
    vocab = logits.shape[1]
    x = logits.double().clone()
    x[x.isnan()] = -math.inf
    x = x.clamp(max=float(np.finfo(np.float32).max))
    out = ([], [], [])
    for s in range(n):
        cand = []
        for b in range(beams):
            row, before = x[s * beams + b], float(scores[s, b])
            top = float(row.max())
            if not math.isfinite(before) or top == -math.inf:
                cand += [(math.inf, b * vocab + t) for t in range(min(n_out, vocab))]
                continue
            lse = math.log(float((row - top).exp().sum()))
            order = np.lexsort((np.arange(vocab), -row.numpy()))[:n_out]
            cand += [(-(before + ((float(row[t]) - top) - lse)), b * vocab + int(t)) for t in order]
        cand = sorted(cand)[:n_out]
        out[0].append([-c[0] for c in cand])
        out[1].append([c[1] // vocab for c in cand])
        out[2].append([c[1] % vocab for c in cand])
    return torch.tensor(out[0], dtype=torch.float64), torch.tensor(out[1], dtype=torch.int32), torch.tensor(out[2], dtype=torch.int32)
