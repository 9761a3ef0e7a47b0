"""Plain 64-bit references of the attention calls, and inputs whose unused places hold NaN."""
import random

import torch

DEV = "cuda"


def offsets(lengths):
    out = [0]
    for a in lengths:
        out.append(out[-1] + a)
    return out


def ints(values):
    return torch.tensor(values, dtype=torch.int32, device=DEV)


def random_tree(rng, n):
    kind = rng.choice(["chain", "binary", "random", "roots"])
    return [i - 1 if kind == "chain" else (i - 1) // 2 if kind == "binary" else -1 if kind == "roots" else rng.randint(-1, i - 1)
            for i in range(n)]


def ancestors(tree, i):
    """Node i and what is above it; a parent that does not come before its child counts as none."""
    seen = []
    while i >= 0:
        seen.append(i)
        i = tree[i] if tree[i] < i else -1
    return seen


def attend(q, k, v, visible, scale):
    """One row in 64 bits: (output, sum of weights times |v|, largest sum |q_i k_i| * scale)."""
    if not visible:
        z = torch.zeros(v.shape[1], dtype=torch.float64, device=v.device)
        return z, z, 0.0
    q, k, v = q.double(), k[visible].double(), v[visible].double()
    s = (k @ q) * scale
    w = torch.exp(s - s.max())
    w = w / w.sum()
    return w @ v, w @ v.abs(), float((k.abs() @ q.abs()).max()) * scale


def tolerance(dtype, dim, n_keys, mean_abs, ref, s_abs):
    """How far a row may be off.  Scores are sums of `dim` products in binary32: each is off by at most (dim + 4) 2^-23
    s_abs (products and sums, the scaling by log2 e, the subtraction of the maximum; a step of 2^-23, as the tensor cores
    need not round to nearest).  An exponential is off by 2^-21 of itself besides, a weight that enters the product in
    bfloat16 by 2^-8 (half a step), a sum of n_keys terms by n_keys 2^-23.  These act on the numerator (bounded by the mean
    of |v|) and on the denominator alike, and the output is rounded once: 2^-8 or 2^-24 of its value."""
    weight = (dim + 4) * 2.0 ** -23 * s_abs + 2.0 ** -21 + n_keys * 2.0 ** -23
    rounding = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    out = 2.0 ** -8 if dtype == torch.bfloat16 else 2.0 ** -23
    return (2 * weight + rounding) * 1.01 * mean_abs + out * ref.abs() + 1e-30


def check_rows(got, rows, dtype, what=""):
    """rows: list of (token, head, q, k, v, visible keys, scale)."""
    for token, head, q, k, v, visible, scale in rows:
        ref, mean_abs, s_abs = attend(q, k, v, visible, scale)
        tol = tolerance(dtype, q.shape[0], len(visible), mean_abs, ref, s_abs)
        err = (got[token, head].double() - ref).abs()
        assert bool((err <= tol).all()), (what, token, head, float((err / tol).max()), float(err.max()))


class Batch:
    """Sequences over a paged cache whose places outside the sequences hold NaN."""

    def __init__(self, seed, dtype, heads, kv_heads, dim, page, contexts, trees, layers=1, layer=0, extra_pages=3, spare=0):
        from paper_2608_15018_b200 import binding
        rng = random.Random(seed)
        gen = torch.Generator(device=DEV).manual_seed(seed)
        self.dtype, self.heads, self.kv_heads, self.dim, self.page, self.layer = dtype, heads, kv_heads, dim, page, layer
        self.contexts, self.trees, self.scale = contexts, trees, dim ** -0.5
        total = [c + len(t) for c, t in zip(contexts, trees)]
        need = [max(1, (a + page - 1) // page) for a in total]
        n_pages = sum(need) + extra_pages
        order = rng.sample(range(n_pages), n_pages)
        shape = (layers, n_pages, kv_heads, page, dim)
        k = torch.full(shape, float("nan"), dtype=dtype, device=DEV)
        v = torch.full(shape, float("nan"), dtype=dtype, device=DEV)
        self.k_rows, self.v_rows, self.tables, at = [], [], [], 0
        for a, n in zip(total, need):
            pages = order[at:at + n]
            at += n
            self.tables.append(pages)
            kk = torch.randn((a, kv_heads, dim), generator=gen, device=DEV).to(dtype)
            vv = torch.randn((a, kv_heads, dim), generator=gen, device=DEV).to(dtype)
            if a:
                idx = torch.arange(a, device=DEV)
                pg = torch.tensor(pages, device=DEV)[idx // page]
                k[layer, pg, :, idx % page] = kk
                v[layer, pg, :, idx % page] = vv
            self.k_rows.append(kk)
            self.v_rows.append(vv)
        width = max(need) + spare
        self.page_table = ints([t + [n_pages + 7] * (width - len(t)) for t in self.tables])
        self.cache = binding.KVCache(k, v)
        self.context = ints(contexts)
        self.starts = offsets([len(t) for t in trees])
        self.seq_start = ints(self.starts)
        self.parent = ints([p for t in trees for p in t]) if self.starts[-1] else torch.zeros(0, dtype=torch.int32, device=DEV)
        self.q = (2 * torch.randn((self.starts[-1], heads, dim), generator=gen, device=DEV)).to(dtype)

    def visible(self, s, i, chain=False):
        c = self.contexts[s]
        nodes = range(i + 1) if chain else ancestors(self.trees[s], i)
        return list(range(c)) + [c + x for x in sorted(nodes)]

    def check(self, got, rng=None, most=200, chain=False, what=""):
        rows = []
        for s, tree in enumerate(self.trees):
            for i in range(len(tree)):
                for h in range(self.heads):
                    g = h * self.kv_heads // self.heads
                    t = self.starts[s] + i
                    rows.append((t, h, self.q[t, h], self.k_rows[s][:, g], self.v_rows[s][:, g], (s, i), self.scale))
        if len(rows) > most:
            rows = (rng or random.Random(0)).sample(rows, most)
        rows = [(t, h, q, k, v, self.visible(*x, chain=chain), sc) for t, h, q, k, v, x, sc in rows]
        check_rows(got, rows, self.dtype, what)
        assert bool(torch.isfinite(got[:self.starts[-1]].float()).all()), what
