"""The work around the verified layer: attention of prompts and draft trees, and the key/value cache under both.

A target model that is verified layer by layer runs its attention between the MoE layers.  A prompt is attended to as a
whole (``prompt_attention``) and its keys and values are written to a paged cache (``kv_write``).  Every verification step
then attends with a tree of drafted tokens to the committed context and to each token's ancestors (``tree_attention``),
and commits the accepted path by moving its keys and values to the end of the context (``kv_commit``).  Sequences that
share a prefix are forked by copying pages (``kv_copy_pages``).

A case is a dict of plain values; ``op`` names the entry point.  Lengths that differ from sequence to sequence are made
from ``mix`` alone, so that a case's work is known without its inputs.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
LARGEST_FLOPS = 2.21e12      # the largest listed case, in bf16
LARGEST_BYTES = 1.1e9


def listed():
    return [
        # plain decoding: one new token of one sequence, 16 heads of their own keys; all of it latency
        dict(name="tree-one-token", op="tree", type="bf16", heads=16, kv_heads=16, dim=128, page=64, seqs=1, lo=700, hi=700,
             nodes=1, mix=0),
        # a batch of 12 sequences of very different lengths, each verifying a tree of up to 64 tokens, 4 query heads to a
        # key head (the head layout of the Mixtral-shaped stack, the largest tree of the DeepSeek-shaped one)
        dict(name="tree-batch-ragged", op="tree", type="bf16", heads=32, kv_heads=8, dim=128, page=64, seqs=12, lo=2100, hi=30000,
             nodes=64, mix=3),
        # the tree of the Qwen1.5-MoE-shaped stack in binary32, with small pages and odd contexts
        dict(name="tree-f32", op="tree", type="f32", heads=16, kv_heads=16, dim=128, page=16, seqs=3, lo=301, hi=2500, nodes=16,
             mix=1),
        # a packed batch of prompts of different lengths, odd ones among them
        dict(name="prompt-packed", op="prompt", type="bf16", heads=16, kv_heads=16, dim=128, seqs=17, lo=21, hi=4000, mix=2),
        # one long prompt, 4 query heads to a key head
        dict(name="prompt-long", op="prompt", type="bf16", heads=32, kv_heads=8, dim=128, seqs=1, lo=16384, hi=16384, mix=0),
        # binary32, narrow heads, short prompts
        dict(name="prompt-f32", op="prompt", type="f32", heads=8, kv_heads=2, dim=64, seqs=5, lo=40, hi=700, mix=4),
        # the keys and values of a tree of 16 drafted tokens into the cache: a few hundred kilobytes, all latency
        dict(name="write-tree", op="write", type="bf16", heads=16, kv_heads=16, dim=128, page=64, seqs=1, lo=16, hi=16, mix=0),
        # those of a packed batch of prompts
        dict(name="write-prompts", op="write", type="bf16", heads=32, kv_heads=8, dim=128, page=32, seqs=24, lo=100, hi=4000,
             mix=5),
        # one accepted path over the 16 layers of the OLMoE-shaped stack
        dict(name="commit-one", op="commit", type="bf16", heads=16, kv_heads=16, dim=128, page=64, seqs=1, lo=1500, hi=1500,
             nodes=16, layers=16, mix=0),
        # the paths of 48 sequences over 32 layers
        dict(name="commit-batch", op="commit", type="bf16", heads=32, kv_heads=8, dim=128, page=32, seqs=48, lo=5, hi=200,
             nodes=64, layers=32, mix=6),
        # a fork: the last, half filled page of one sequence, in all 16 layers
        dict(name="copy-fork", op="copy", type="bf16", heads=16, kv_heads=16, dim=128, page=64, pairs=1, pages=8, layers=16,
             mix=0),
        # moving many pages together (compacting the pool)
        dict(name="copy-many", op="copy", type="bf16", heads=32, kv_heads=8, dim=128, page=64, pairs=260, pages=600, layers=8,
             mix=7),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the listed ranges: any entry point, type, head layout, page size and mix of lengths."""
    op = rng.choice(["tree", "tree", "tree", "prompt", "prompt", "prompt", "write", "commit", "copy"])
    heads, kv_heads, dim = rng.choice([(16, 16, 128), (32, 8, 128), (32, 4, 128), (8, 2, 64), (64, 8, 64), (16, 16, 64),
                                       (28, 4, 128), (9, 3, 64), (8, 1, 128)])
    case = dict(op=op, type=rng.choice(["bf16", "bf16", "bf16", "f32"]), heads=heads, kv_heads=kv_heads, dim=dim,
                mix=rng.randint(0, 10 ** 6))
    if op == "prompt":
        top = _log_int(rng, 2, 16000)
        case.update(seqs=_log_int(rng, 1, 24), lo=rng.choice([1, max(1, top // 3), top]), hi=top)
    elif op == "tree":
        top = _log_int(rng, 2, 32000)
        case.update(page=rng.choice([16, 32, 64, 128]), seqs=_log_int(rng, 1, 32), lo=rng.choice([1, max(1, top // 3), top]),
                    hi=top, nodes=_log_int(rng, 1, 64))
    elif op == "write":
        top = _log_int(rng, 1, 4000)
        case.update(page=rng.choice([16, 32, 64, 128]), seqs=_log_int(rng, 1, 32), lo=rng.choice([1, top]), hi=top)
    elif op == "commit":
        top = _log_int(rng, 1, 400)
        case.update(page=rng.choice([16, 32, 64, 128]), seqs=_log_int(rng, 1, 48), lo=rng.choice([1, top]), hi=top,
                    nodes=rng.randint(1, 64), layers=_log_int(rng, 1, 32))
    else:
        pairs = _log_int(rng, 1, 200)
        case.update(page=rng.choice([16, 32, 64, 128]), pairs=pairs, pages=2 * pairs + rng.randint(0, 60),
                    layers=_log_int(rng, 1, 16))
    while True:                                     # no dearer than the largest listed case
        w = work(case)
        share = 1 / 24 if case["type"] == "f32" else 1.0
        if w["flops"] <= LARGEST_FLOPS * share and max(w["bytes"], _held(case) / 2) <= LARGEST_BYTES:
            return case
        if op == "copy":
            case["layers"] = max(1, case["layers"] // 2)
            case["pairs"] = max(1, case["pairs"] * 3 // 4)
            case["pages"] = 2 * case["pairs"] + 5
        elif op == "commit" and case["layers"] > 4:
            case["layers"] //= 2
        elif case["seqs"] > 1:
            case["seqs"] -= max(1, case["seqs"] // 4)
        else:
            case["hi"] = max(1, case["hi"] * 3 // 4)
            case["lo"] = min(case["lo"], case["hi"])


# ---- lengths, trees and paths of a case, from its plain values alone ------------------------------------------------

def _lengths(case):
    rng = random.Random(1000 + case["mix"])
    return [_log_int(rng, case["lo"], case["hi"]) for _ in range(case["seqs"])]


def _trees(case):
    """Per sequence the parent of every drafted token (-1: a child of the context's last token).  About a third of the
    trees are chains, the others branch twice as a breadth-first tree or at random."""
    rng = random.Random(2000 + case["mix"])
    trees = []
    for s in range(case["seqs"]):
        n = case["nodes"] if s == 0 else rng.randint(max(1, case["nodes"] // 2), case["nodes"])
        kind = rng.choice(["chain", "binary", "random"])
        trees.append([i - 1 if kind == "chain" else (i - 2) // 2 if kind == "binary" and i > 1 else -1 if i == 0 or kind == "binary"
                      else rng.randint(-1, i - 1) for i in range(n)])
    return trees


def _paths(case):
    """Accepted tokens per sequence: the first j drafted ones where they are, then ones from further back in the tree (so
    that committing twice moves the same values twice)."""
    rng = random.Random(3000 + case["mix"])
    paths = []
    for s in range(case["seqs"]):
        n = case["nodes"]
        take = rng.randint(1, max(1, min(n // 2, 9)))
        stay = rng.randint(0, take - 1) if n > 1 else take
        rest = sorted(rng.sample(range(take, n), take - stay)) if n - take >= take - stay else []
        paths.append(list(range(stay)) + rest)
    return paths


def _pairs(case):
    ids = random.Random(4000 + case["mix"]).sample(range(case["pages"]), 2 * case["pairs"])
    return list(zip(ids[:case["pairs"]], ids[case["pairs"]:]))


def _slots(case):
    """Positions that each sequence has room for."""
    n = _lengths(case)
    return [a + case.get("nodes", 0) for a in n]


def _n_pages(case):
    if case["op"] == "copy":
        return case["pages"]
    return sum((a + case["page"] - 1) // case["page"] for a in _slots(case)) + 3


def _held(case):
    """Bytes that the state holds."""
    size = 4 if case["type"] == "f32" else 2
    if case["op"] == "prompt":
        return 2 * size * case["dim"] * (case["heads"] + case["kv_heads"]) * sum(_lengths(case))
    return 2 * size * case["dim"] * case["kv_heads"] * case["page"] * case.get("layers", 1) * _n_pages(case)


def work(case):
    size = 4 if case["type"] == "f32" else 2
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]
    row = 2 * size * hk * d                                  # a token's key and value
    if case["op"] == "prompt":
        n = _lengths(case)
        return dict(bytes=sum(n) * (row + 2 * size * hq * d), flops=4 * hq * d * sum(a * (a + 1) // 2 for a in n))
    if case["op"] == "tree":
        nbytes = flops = 0
        for a, tree in zip(_lengths(case), _trees(case)):
            depth = []
            for p in tree:
                depth.append(1 + (depth[p] if p >= 0 else 0))
            nbytes += (a + len(tree)) * row + 2 * size * hq * d * len(tree)
            flops += 4 * hq * d * sum(a + x for x in depth)
        return dict(bytes=nbytes, flops=flops)
    if case["op"] == "write":
        return dict(bytes=2 * row * sum(_lengths(case)), flops=0)
    if case["op"] == "commit":
        moved = sum(sum(i != p for i, p in enumerate(path)) for path in _paths(case))
        return dict(bytes=2 * row * case["layers"] * moved + 64 * case["seqs"], flops=0)
    return dict(bytes=2 * row * case["page"] * case["layers"] * case["pairs"], flops=0)


# ---- inputs ---------------------------------------------------------------------------------------------------------

def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _offsets(lengths):
    out = [0]
    for a in lengths:
        out.append(out[-1] + a)
    return out


def _inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    dtype = TYPES[case["type"]]
    hq, hk, d = case["heads"], case["kv_heads"], case["dim"]

    def normal(*shape):
        return torch.randn(shape, generator=gen, device="cuda", dtype=dtype)

    s = dict(case=case, scale=1.0 / math.sqrt(d))
    if case["op"] == "prompt":
        n = _lengths(case)
        # one projection's output: queries, keys and values of a token side by side, as the model has them
        qkv = normal(sum(n), (hq + 2 * hk) * d)
        qkv[:, :hq * d] *= 2
        s["q"] = qkv[:, :hq * d].unflatten(1, (hq, d))
        s["k"] = qkv[:, hq * d:(hq + hk) * d].unflatten(1, (hk, d))
        s["v"] = qkv[:, (hq + hk) * d:].unflatten(1, (hk, d))
        s["starts"] = _offsets(n)
        s["seq_start"] = _ints(s["starts"])
        return s
    layers, page, n_pages = case.get("layers", 1), case["page"], _n_pages(case)
    s["k_pool"] = normal(layers, n_pages, hk, page, d)
    s["v_pool"] = normal(layers, n_pages, hk, page, d)
    if case["op"] == "copy":
        s["pairs"] = _pairs(case)
        return s
    # every sequence's pages lie anywhere in the pool; places of the table that no page fills hold 0
    order = random.Random(int(seed) * 7 + case["mix"]).sample(range(n_pages), n_pages)
    need = [(a + page - 1) // page for a in _slots(case)]
    s["tables"], at = [], 0
    for a in need:
        s["tables"].append(order[at:at + a])
        at += a
    s["page_table"] = _ints([t + [0] * (max(need) - len(t)) for t in s["tables"]])
    if case["op"] == "write":
        n = _lengths(case)
        s["starts"], s["first"] = _offsets(n), [0] * len(n)
        s["k_new"], s["v_new"] = normal(sum(n), hk, d), normal(sum(n), hk, d)
        s["first_dev"] = _ints(s["first"])
        s["seq_start"] = _ints(s["starts"])
        return s
    s["contexts"] = _lengths(case)
    s["context"] = _ints(s["contexts"])
    if case["op"] == "commit":
        s["paths"] = _paths(case)
        most = max(1, max(len(p) for p in s["paths"]))
        s["path"] = _ints([p + [0] * (most - len(p)) for p in s["paths"]])
        s["n_path"] = _ints([len(p) for p in s["paths"]])
        return s
    s["trees"] = _trees(case)
    s["starts"] = _offsets([len(t) for t in s["trees"]])
    s["seq_start"] = _ints(s["starts"])
    s["parent"] = _ints([p for t in s["trees"] for p in t])
    s["q"] = 2 * normal(s["starts"][-1], hq, d)
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    if "k_pool" in s:
        layers, n_pages, hk, page, d = s["k_pool"].shape
        # flat positions of the plain form's indexing, as a program that indexes would keep them
        s["flat"] = [torch.tensor([p * page + i for p in t for i in range(page)], dtype=torch.int64, device="cuda")
                     for t in s.get("tables", [])]
        if case["op"] == "commit":
            src = [(s["flat"][j][c + p], s["flat"][j][c + i]) for j, (c, path) in enumerate(zip(s["contexts"], s["paths"]))
                   for i, p in enumerate(path) if i != p]
            s["from"] = torch.stack([a for a, _ in src]) if src else None
            s["to"] = torch.stack([b for _, b in src]) if src else None
        if case["op"] == "copy":
            s["from"] = torch.tensor([a for a, _ in s["pairs"]], device="cuda")
            s["to"] = torch.tensor([b for _, b in s["pairs"]], device="cuda")
        if case["op"] == "tree":
            # which drafted tokens every drafted token sees: itself and its ancestors
            s["sees"] = []
            for tree in s["trees"]:
                m = torch.zeros(len(tree), len(tree), dtype=torch.bool)
                for i, p in enumerate(tree):
                    if p >= 0:
                        m[i] = m[p]
                    m[i, i] = True
                s["sees"].append(m.cuda())
        if own:
            from paper_2608_15018_b200 import binding
            s["cache"] = binding.KVCache(s["k_pool"], s["v_pool"])
    return s


# ---- one pass -------------------------------------------------------------------------------------------------------

def _softmax_rows(scores, seen):
    if seen is not None:
        scores = scores.masked_fill(~seen, float("-inf"))
    e = torch.exp(scores - scores.amax(dim=-1, keepdim=True))
    return e / e.sum(dim=-1, keepdim=True)


def _plain_prompt(s):
    q, k, v = s["q"], s["k"], s["v"]
    hq, hk = q.shape[1], k.shape[1]
    out = torch.empty(q.shape, dtype=q.dtype, device=q.device)
    for a, b in zip(s["starts"], s["starts"][1:]):
        kk, vv = k[a:b].float().transpose(0, 1), v[a:b].float().transpose(0, 1)
        for c in range(a, b, 2048):
            e = min(c + 2048, b)
            seen = torch.arange(e - a, device=q.device) <= torch.arange(c - a, e - a, device=q.device)[:, None]
            for h in range(hk):
                g = slice(h * hq // hk, (h + 1) * hq // hk)
                qq = q[c:e, g].float().transpose(0, 1)
                p = _softmax_rows(torch.matmul(qq, kk[h, :e - a].T) * s["scale"], seen)
                out[c:e, g] = torch.matmul(p, vv[h, :e - a]).transpose(0, 1).to(q.dtype)
    return out


def _rows(pool, flat, n):
    """Keys or values of the first n positions of a sequence: [kv heads][n][dim] in binary32."""
    page = pool.shape[2]
    return pool[flat[:n] // page, :, flat[:n] % page].float().transpose(0, 1)


def _plain_tree(s):
    q = s["q"]
    hq, hk = q.shape[1], s["k_pool"].shape[2]
    out = torch.empty_like(q)
    for j, (a, b) in enumerate(zip(s["starts"], s["starts"][1:])):
        n, c = b - a, s["contexts"][j]
        k, v = _rows(s["k_pool"][0], s["flat"][j], c + n), _rows(s["v_pool"][0], s["flat"][j], c + n)
        seen = torch.cat([torch.ones(n, c, dtype=torch.bool, device=q.device), s["sees"][j]], dim=1)
        qq = q[a:b].float().reshape(n, hk, hq // hk, -1).permute(1, 2, 0, 3)
        p = _softmax_rows(torch.matmul(qq, k[:, None].transpose(2, 3)) * s["scale"], seen)
        out[a:b] = torch.matmul(p, v[:, None]).permute(2, 0, 1, 3).reshape(n, hq, -1).to(q.dtype)
    return out


def _plain_write(s):
    page = s["k_pool"].shape[3]
    for j, (a, b) in enumerate(zip(s["starts"], s["starts"][1:])):
        at = s["flat"][j][s["first"][j]:s["first"][j] + b - a]
        s["k_pool"][0, at // page, :, at % page] = s["k_new"][a:b]
        s["v_pool"][0, at // page, :, at % page] = s["v_new"][a:b]


def _plain_commit(s):
    page = s["k_pool"].shape[3]
    if s["from"] is not None:
        for pool in (s["k_pool"], s["v_pool"]):
            pool[:, s["to"] // page, :, s["to"] % page] = pool[:, s["from"] // page, :, s["from"] % page]
    return s["context"] + s["n_path"]


def _plain_copy(s):
    for pool in (s["k_pool"], s["v_pool"]):
        pool[:, s["to"]] = pool[:, s["from"]]


def run(state):
    s = state
    op = s["case"]["op"]
    if own:
        from paper_2608_15018_b200 import binding
        if op == "prompt":
            return binding.prompt_attention(s["q"], s["k"], s["v"], s["seq_start"], scale=s["scale"])
        if op == "tree":
            return binding.tree_attention(s["q"], s["cache"], 0, s["page_table"], s["context"], s["seq_start"], s["parent"],
                                          scale=s["scale"])
        if op == "write":
            binding.kv_write(s["cache"], 0, s["k_new"], s["v_new"], s["page_table"], s["first_dev"], s["seq_start"])
        elif op == "commit":
            return s["k_pool"], s["v_pool"], binding.kv_commit(s["cache"], s["page_table"], s["context"], s["path"], s["n_path"])
        else:
            binding.kv_copy_pages(s["cache"], s["pairs"])
        return s["k_pool"], s["v_pool"]
    if op == "prompt":
        return _plain_prompt(s)
    if op == "tree":
        return _plain_tree(s)
    if op == "commit":
        length = _plain_commit(s)
        return s["k_pool"], s["v_pool"], length
    (_plain_write if op == "write" else _plain_copy)(s)
    return s["k_pool"], s["v_pool"]


# ---- the definition in 64 bits --------------------------------------------------------------------------------------

def _attend64(q, k, v, scale, visible):
    """q [n][d], k, v [m][d] in 64 bits; visible [n][m] or None."""
    x = (q @ k.T) * scale
    if visible is not None:
        x = torch.where(visible, x, torch.full_like(x, -math.inf))
    top = x.max(dim=1, keepdim=True).values
    w = (x - top).exp_()
    return (w @ v) / w.sum(dim=1, keepdim=True)


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "prompt":
        q, k, v = s["q"], s["k"], s["v"]
        group = q.shape[1] // k.shape[1]
        out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
        for a, b in zip(s["starts"], s["starts"][1:]):
            for h in range(q.shape[1]):
                kk, vv = k[a:b, h // group].double(), v[a:b, h // group].double()
                for c in range(0, b - a, 1024):
                    e = min(c + 1024, b - a)
                    visible = torch.ones(e - c, e, dtype=torch.bool, device=q.device).tril(c)
                    out[a + c:a + e, h] = _attend64(q[a + c:a + e, h].double(), kk[:e], vv[:e], s["scale"], visible)
        return out
    page = case["page"]
    if op == "tree":
        q = s["q"]
        group = q.shape[1] // case["kv_heads"]
        out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
        for j, (a, b) in enumerate(zip(s["starts"], s["starts"][1:])):
            c, tree = s["contexts"][j], s["trees"][j]
            rows = [[i < c for i in range(c + b - a)] for _ in tree]
            for i in range(len(tree)):
                x = i
                while x >= 0:
                    rows[i][c + x] = True
                    x = tree[x]
            visible = torch.tensor(rows, device=q.device)
            used = s["tables"][j]
            for h in range(case["kv_heads"]):
                k = s["k_pool"][0, used, h].reshape(-1, case["dim"])[:c + b - a].double()
                v = s["v_pool"][0, used, h].reshape(-1, case["dim"])[:c + b - a].double()
                for g in range(group):
                    out[a:b, h * group + g] = _attend64(q[a:b, h * group + g].double(), k, v, s["scale"], visible)
        return out
    k, v = s["k_pool"].clone(), s["v_pool"].clone()
    if op == "write":
        for j, (a, b) in enumerate(zip(s["starts"], s["starts"][1:])):
            for i in range(0, b - a, page):
                n = min(page, b - a - i)
                where = s["tables"][j][i // page]
                k[0, where, :, :n] = s["k_new"][a + i:a + i + n].transpose(0, 1)
                v[0, where, :, :n] = s["v_new"][a + i:a + i + n].transpose(0, 1)
        return k, v
    if op == "commit":
        for j, path in enumerate(s["paths"]):
            for i, p in enumerate(path):
                there, here = s["contexts"][j] + i, s["contexts"][j] + p
                for new, old in ((k, s["k_pool"]), (v, s["v_pool"])):
                    new[:, s["tables"][j][there // page], :, there % page] = old[:, s["tables"][j][here // page], :, here % page]
        return k, v, torch.tensor([c + len(p) for c, p in zip(s["contexts"], s["paths"])], dtype=torch.int32, device="cuda")
    for a, b in s["pairs"]:
        k[:, b] = s["k_pool"][:, a]
        v[:, b] = s["v_pool"][:, a]
    return k, v
