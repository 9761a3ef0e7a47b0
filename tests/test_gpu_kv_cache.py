"""Writing, committing and copying in the paged cache, bit by bit against plain indexing, and the calls run together."""
import random

import pytest
import torch

from paper_2608_15018_b200 import binding
from tests.attn_util import DEV, ancestors, check_rows, ints, offsets, random_tree

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]


def pool(dtype, layers, n_pages, heads, page, dim, seed=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    k = torch.randn((layers, n_pages, heads, page, dim), generator=gen, device=DEV).to(dtype)
    v = torch.randn((layers, n_pages, heads, page, dim), generator=gen, device=DEV).to(dtype)
    return binding.KVCache(k, v), k.clone(), v.clone()


def same(cache, k, v):
    as_bits = torch.int16 if cache.dtype == torch.bfloat16 else torch.int32
    return torch.equal(cache.k.view(as_bits), k.view(as_bits)) and torch.equal(cache.v.view(as_bits), v.view(as_bits))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page,heads,dim", [(16, 1, 64), (32, 3, 128), (64, 16, 128), (128, 8, 64)])
def test_write(dtype, page, heads, dim):
    rng = random.Random(page)
    lengths = [0, 1, 7, 200, 0, page, 33]
    first = [5, 0, page - 3, 11, 2, 0, page]
    need = [(a + b + page - 1) // page for a, b in zip(first, lengths)]
    cache, k, v = pool(dtype, 3, sum(need) + 2, heads, page, dim)
    order = rng.sample(range(cache.n_pages), cache.n_pages)
    starts, at, tables = offsets(lengths), 0, []
    for n in need:
        tables.append(order[at:at + n] + [-1] * (max(need) - n))
        at += n
    gen = torch.Generator(device=DEV).manual_seed(1)
    wide = torch.randn((sum(lengths) + 4, 2 * heads * dim + 64), generator=gen, device=DEV).to(dtype)
    wide[3] = float("nan")                                       # bits are moved, whatever they mean
    nk, nv = wide[:, :heads * dim].unflatten(1, (heads, dim)), wide[:, heads * dim:2 * heads * dim].unflatten(1, (heads, dim))
    binding.kv_write(cache, 1, nk, nv, ints(tables), ints(first), ints(starts))
    for s, (a, b) in enumerate(zip(starts, starts[1:])):
        for i in range(b - a):
            p = first[s] + i
            k[1, tables[s][p // page], :, p % page] = nk[a + i]
            v[1, tables[s][p // page], :, p % page] = nv[a + i]
    assert same(cache, k, v)


@pytest.mark.parametrize("n_seq", [31, 33, 1000, 40000])
def test_write_of_many_sequences(n_seq):
    """Many of them empty, some at the same offset."""
    rng = random.Random(n_seq)
    lengths = [rng.choice([0, 0, 1, 3]) for _ in range(n_seq)]
    cache, k, v = pool(torch.bfloat16, 1, n_seq + 1, 1, 16, 64)
    new = torch.randn((sum(lengths), 1, 64), device=DEV).bfloat16()
    table = torch.randperm(n_seq, device=DEV).to(torch.int32).view(n_seq, 1).contiguous()
    binding.kv_write(cache, 0, new, new, table, torch.full((n_seq,), 5, dtype=torch.int32, device=DEV), ints(offsets(lengths)))
    owner = torch.repeat_interleave(torch.arange(n_seq, device=DEV), torch.tensor(lengths, device=DEV))
    place = 5 + torch.arange(sum(lengths), device=DEV) - torch.tensor(offsets(lengths), device=DEV)[owner]
    for x in (k, v):
        x[0, table[owner, 0].long(), 0, place] = new[:, 0]
    assert same(cache, k, v)


@pytest.mark.parametrize("dtype", TYPES)
def test_write_leaves_out_what_has_no_place(dtype):
    cache, k, v = pool(dtype, 1, 6, 2, 16, 64)
    new = torch.ones((60, 2, 64), dtype=dtype, device=DEV)
    table = ints([[1, -1, 3], [2 ** 31 - 1, 6, 4], [-2 ** 31, 0, 5]])
    binding.kv_write(cache, 0, new, new, table, ints([8, 30, -4]), ints([0, 30, 50, 60]))
    for s, first, n, pages in ((0, 8, 30, [1, None, 3]), (1, 30, 20, [None, None, 4]), (2, -4, 10, [None, 0, 5])):
        for p in range(first, first + n):
            if 0 <= p < 48 and pages[p // 16] is not None:
                k[0, pages[p // 16], :, p % 16] = 1
                v[0, pages[p // 16], :, p % 16] = 1
    assert same(cache, k, v)
    binding.kv_write(cache, 0, new, new, table, ints([2 ** 31 - 1, -2 ** 31, 48]), ints([-5, 2 ** 31 - 1, 20, 60]))
    binding.kv_write(cache, 0, new, new, table, ints([47, 100, 100]), ints([60, 90, 20, 0]))
    assert same(cache, k, v)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page,heads,dim,layers", [(16, 1, 64, 1), (32, 3, 128, 4), (64, 16, 128, 2)])
def test_commit(dtype, page, heads, dim, layers):
    """Ascending paths whose targets are other rows' sources, any order, a node named twice, empty and full paths."""
    rng = random.Random(page)
    paths = [[], [0], [1, 3, 4, 9], [5, 2, 2, 0, 1, 1], list(range(63, -1, -1)), sorted(rng.sample(range(64), 40)), [0, 1, 2, 3],
             [-1, 3, 200, 5]]
    contexts = [0, 15, page - 2, 7, 100, 33, 64, 3]
    most = 64
    width = (max(contexts) + 64 + page - 1) // page
    cache, k, v = pool(dtype, layers, width * len(paths) + 1, heads, page, dim)
    order = rng.sample(range(cache.n_pages), cache.n_pages)
    tables = [order[width * s:width * (s + 1)] for s in range(len(paths))]
    tables[6][64 // page] = cache.n_pages                        # a page that is not there
    ok, ov = k.clone(), v.clone()
    for s, (c, path) in enumerate(zip(contexts, paths)):
        for i, node in enumerate(path):
            src, dst = c + node, c + i
            if node < 0 or src >= width * page:
                continue
            ps, pd = tables[s][src // page], tables[s][dst // page]
            if ps < cache.n_pages and pd < cache.n_pages:
                k[:, pd, :, dst % page] = ok[:, ps, :, src % page]
                v[:, pd, :, dst % page] = ov[:, ps, :, src % page]
    path = ints([p + [0] * (most - len(p)) for p in paths])
    new = binding.kv_commit(cache, ints(tables), ints(contexts), path, ints([len(p) for p in paths]))
    assert same(cache, k, v)
    assert new.tolist() == [c + len(p) for c, p in zip(contexts, paths)]


@pytest.mark.parametrize("dtype", TYPES)
def test_commit_brings_lengths_into_range(dtype):
    cache, k, v = pool(dtype, 1, 4, 1, 16, 64)
    table = ints([[0, 1], [2, 3]])
    new = binding.kv_commit(cache, table, ints([10 ** 9, -3]), ints([[1, 2], [4, 5]]), ints([2, 2]))
    assert same(cache, k, v) and new.tolist() == [10 ** 9 + 2, -1]
    new = binding.kv_commit(cache, table, ints([0, 4]), ints([[1, 2], [1, 0]]), ints([-7, 10 ** 6]))
    for x, y in ((k, k.clone()), (v, v.clone())):
        x[0, 2, :, 4], x[0, 2, :, 5] = y[0, 2, :, 5], y[0, 2, :, 4]
    assert same(cache, k, v) and new.tolist() == [0, 6]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page,heads,dim,layers,pairs", [(16, 1, 64, 1, 1), (128, 3, 128, 3, 7), (32, 2, 64, 2, 700)])
def test_copy_pages(dtype, page, heads, dim, layers, pairs):
    rng = random.Random(pairs)
    cache, k, v = pool(dtype, layers, 2 * pairs + 3, heads, page, dim)
    ids = rng.sample(range(cache.n_pages), 2 * pairs)
    todo = list(zip(ids[:pairs], ids[pairs:]))
    if pairs > 2:
        todo[1] = (todo[0][0], todo[1][1])                       # one source, two copies
    binding.kv_copy_pages(cache, todo)
    for a, b in todo:
        k[:, b], v[:, b] = k[:, a], v[:, a]
    assert same(cache, k, v)
    with pytest.raises(binding.S2MoEError):
        binding.kv_copy_pages(cache, [(todo[0][0], todo[0][1]), (todo[0][1], ids[1] if pairs > 1 else todo[0][0])])
    assert same(cache, k, v)


@pytest.mark.parametrize("dtype", TYPES)
def test_prompt_fork_draft_commit(dtype):
    """A prompt, two forks of it, three verification steps each with trees and accepted paths, the pool compacted in
    between: every step's attention against the keys and values that the sequence really has."""
    rng = random.Random(4)
    gen = torch.Generator(device=DEV).manual_seed(4)
    heads, kv_heads, dim, page, layers = 8, 2, 64, 16, 2
    pages = binding.PagePool(60, page)
    cache = binding.KVCache.empty(layers, 60, kv_heads, page, dim, dtype)
    cache.k.fill_(float("nan"))
    cache.v.fill_(float("nan"))

    def rows(n, h):
        return torch.randn((n, h, dim), generator=gen, device=DEV).to(dtype)

    def table(seqs):
        lists = [pages.pages(s) for s in seqs]
        return ints([x + [0] * (max(map(len, lists)) - len(x)) for x in lists])

    prompt = 45
    a, filler = pages.open(), pages.open()
    pages.reserve(filler, 0, 20 * page)                          # lies in front of what comes later, and goes away
    assert pages.reserve(a, 0, prompt) == []
    true = {a: [(rows(prompt, kv_heads), rows(prompt, kv_heads)) for _ in range(layers)]}
    q = rows(prompt, heads)
    for layer in range(layers):
        k, v = true[a][layer]
        out = binding.prompt_attention(q, k, v, ints([0, prompt]))
        check_rows(out, [(i, h, q[i, h], k[:, h // 4], v[:, h // 4], list(range(i + 1)), dim ** -0.5)
                         for i in range(0, prompt, 7) for h in range(heads)], dtype)
        binding.kv_write(cache, layer, k, v, table([a]), ints([0]), ints([0, prompt]))
    b = pages.fork(a)
    true[b] = list(true[a])
    length = {a: prompt, b: prompt}
    for step in range(3):
        seqs = [b, a] if step % 2 else [a, b]
        trees = [random_tree(rng, n) for n in (9, 16)]
        copies = [c for s, t in zip(seqs, trees) for c in pages.reserve(s, length[s], length[s] + len(t))]
        binding.kv_copy_pages(cache, copies)
        assert step or len(copies) == 1                           # the second owner of the half filled page stays on it
        starts = offsets([len(t) for t in trees])
        ctx, tab = ints([length[s] for s in seqs]), table(seqs)
        parent = ints([p for t in trees for p in t])
        drafted = [(rows(starts[-1], kv_heads), rows(starts[-1], kv_heads)) for _ in range(layers)]
        q = rows(starts[-1], heads)
        for layer in range(layers):
            k, v = drafted[layer]
            binding.kv_write(cache, layer, k, v, tab, ctx, ints(starts))
            out = binding.tree_attention(q, cache, layer, tab, ctx, ints(starts), parent)
            checks = []
            for j, s in enumerate(seqs):
                kk = torch.cat([true[s][layer][0], k[starts[j]:starts[j + 1]]])
                vv = torch.cat([true[s][layer][1], v[starts[j]:starts[j + 1]]])
                for i in range(len(trees[j])):
                    keys = list(range(length[s])) + [length[s] + x for x in sorted(ancestors(trees[j], i))]
                    checks += [(starts[j] + i, h, q[starts[j] + i, h], kk[:, h // 4], vv[:, h // 4], keys, dim ** -0.5) for h in range(heads)]
            check_rows(out, checks, dtype, step)
        paths = [sorted(ancestors(t, rng.randrange(len(t)))) for t in trees]
        most = max(map(len, paths))
        new = binding.kv_commit(cache, tab, ctx, ints([p + [0] * (most - len(p)) for p in paths]), ints([len(p) for p in paths]))
        for j, s in enumerate(seqs):
            true[s] = [(torch.cat([tk, k[starts[j]:][paths[j]]]), torch.cat([tv, v[starts[j]:][paths[j]]]))
                       for (tk, tv), (k, v) in zip(true[s], drafted)]
            length[s] += len(paths[j])
            pages.truncate(s, length[s])
        assert new.tolist() == [length[s] for s in seqs]
        if step == 1:
            pages.free(filler)
            moves = pages.compact()
            assert moves
            binding.kv_copy_pages(cache, moves)
    assert binding.attention_status() == 0
