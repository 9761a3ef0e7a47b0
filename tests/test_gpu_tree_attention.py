"""Attention of drafted trees over a paged cache against a plain 64-bit computation, row by row."""
import random

import pytest
import torch

from paper_2608_15018_b200 import binding
from tests.attn_util import DEV, Batch, check_rows, ints, random_tree

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]


def run(b, **kw):
    kw.setdefault("parent", b.parent)
    out = binding.tree_attention(b.q, b.cache, b.layer, b.page_table, b.context, b.seq_start, **kw)
    assert binding.attention_status() == 0
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 64), (16, 16, 128), (32, 8, 128), (9, 3, 64), (28, 4, 128), (64, 1, 64), (40, 1, 128)])
@pytest.mark.parametrize("page", [16, 128])
def test_one_tree(dtype, heads, kv_heads, dim, page):
    rng = random.Random(heads * dim + page)
    for context, nodes in ((0, 1), (1, 1), (127, 1), (128, 3), (63, 2), (700, 16), (513, 64)):
        b = Batch(context + nodes, dtype, heads, kv_heads, dim, page, [context], [random_tree(rng, nodes)])
        b.check(run(b), rng, 60, what=(context, nodes))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("page", [16, 32, 64])
def test_ragged_batch(dtype, page):
    rng = random.Random(page)
    contexts = [0, 5, 1200, 64, 33, 4097, 128, 0, 999]
    trees = [random_tree(rng, n) for n in (1, 64, 17, 0, 33, 8, 2, 0, 64)]
    b = Batch(7, dtype, 8, 2, 128, page, contexts, trees, layers=3, layer=1, spare=2)
    b.check(run(b), rng, 400)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_sequences(dtype):
    rng = random.Random(11)
    contexts = [rng.choice([0, 1, 15, 16, 300, 2000]) for _ in range(75)]
    trees = [random_tree(rng, rng.choice([0, 1, 1, 4, 20])) for _ in contexts]
    b = Batch(3, dtype, 4, 4, 64, 16, contexts, trees)
    b.check(run(b), rng, 300)


@pytest.mark.parametrize("dtype", TYPES)
def test_long_context_is_split_and_joined(dtype):
    rng = random.Random(5)
    b = Batch(9, dtype, 4, 1, 128, 64, [60001, 3], [random_tree(rng, 6), random_tree(rng, 3)])
    b.check(run(b), rng, 40)


@pytest.mark.parametrize("dtype", TYPES)
def test_chains_without_parents_of_any_length(dtype):
    b = Batch(13, dtype, 8, 2, 64, 32, [100, 0, 17], [[0] * 150, [0] * 70, [0]])
    b.check(run(b, parent=None), random.Random(1), 300, chain=True)


@pytest.mark.parametrize("dtype", TYPES)
def test_tokens_are_the_last_nodes_of_their_tree(dtype):
    """A draft that adds a level: the tree's other nodes are in the cache already."""
    rng = random.Random(17)
    trees = [random_tree(rng, n) for n in (64, 9, 5)]
    b = Batch(19, dtype, 8, 8, 128, 64, [300, 0, 65], trees)
    last = [3, 9, 0]
    starts = ints([0, 3, 12, 12])
    whole = b.q
    b.q = torch.cat([whole[b.starts[s + 1] - n:b.starts[s + 1]] for s, n in enumerate(last)])
    out = binding.tree_attention(b.q, b.cache, 0, b.page_table, b.context, starts, b.parent, b.seq_start)
    full = binding.tree_attention(whole, b.cache, 0, b.page_table, b.context, b.seq_start, b.parent)
    rows, t = [], 0
    for s, n in enumerate(last):
        for i in range(len(trees[s]) - n, len(trees[s])):
            for h in range(8):
                rows.append((t, h, b.q[t, h], b.k_rows[s][:, h], b.v_rows[s][:, h], b.visible(s, i), b.scale))
            t += 1
    check_rows(out, rows, dtype)
    assert torch.isfinite(full.float()).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_parents_that_do_not_come_before_their_child_count_as_none(dtype):
    tree = [0, 5, 1, -7, 3, 2 ** 31 - 1, 4]
    b = Batch(23, dtype, 4, 2, 64, 16, [40], [tree])
    clean = [-1, -1, 1, -1, 3, -1, 4]
    out = run(b)
    b.trees = [clean]
    b.check(out)


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_no_sequence_stay_as_they_were(dtype):
    rng = random.Random(3)
    b = Batch(29, dtype, 4, 2, 64, 16, [40, 10], [random_tree(rng, 5), random_tree(rng, 4)])
    pad = torch.full((6, 4, 64), float("nan"), dtype=dtype, device=DEV)
    q = torch.cat([b.q, pad])
    out = torch.full((15, 4, 64), 7.0, dtype=dtype, device=DEV)
    parent = torch.cat([b.parent, ints([2 ** 30] * 6)])
    got = binding.tree_attention(q, b.cache, 0, b.page_table, b.context, b.seq_start, parent, out=out)
    assert got is out and bool((out[9:] == 7.0).all())
    b.check(out)
    same = binding.tree_attention(q[:9], b.cache, 0, b.page_table, b.context, b.seq_start, b.parent)
    assert torch.equal(same, out[:9])


@pytest.mark.parametrize("dtype", TYPES)
def test_queries_that_are_part_of_a_wider_tensor(dtype):
    rng = random.Random(31)
    b = Batch(37, dtype, 4, 2, 128, 64, [333], [random_tree(rng, 12)])
    wide = torch.full((12, 4 * 128 + 256), float("nan"), dtype=dtype, device=DEV)
    wide[:, :512] = b.q.flatten(1)
    want = run(b)
    b.q = wide[:, :512].unflatten(1, (4, 128))
    assert torch.equal(run(b), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("context", [50, 3000])
def test_values_and_keys_that_a_row_does_not_see_have_no_part_in_it(dtype, context):
    """Infinite and NaN keys and values of one branch reach the rows of that branch only."""
    tree = [-1, 0, 0, 1, 2, 2, 4]                              # node 2 and below: 2, 4, 5, 6
    b = Batch(41, dtype, 4, 2, 64, 16, [context], [tree])
    clean = run(b)
    for bad in (float("nan"), float("inf"), -float("inf")):
        for where in ("k", "v"):
            pool = getattr(b.cache, where)
            at = context + 2
            keep = pool[0, b.tables[0][at // 16], :, at % 16].clone()
            pool[0, b.tables[0][at // 16], :, at % 16] = bad
            out = run(b)
            pool[0, b.tables[0][at // 16], :, at % 16] = keep
            # two results of one row, each off by at most 2^-8 (|result| + mean of |v|), and that mean below 2
            off = (out[[0, 1, 3]].float() - clean[[0, 1, 3]].float()).abs()
            assert bool((off <= 2.0 ** -7 * clean[[0, 1, 3]].float().abs() + 2.0 ** -6).all())
            assert torch.isfinite(out[[0, 1, 3]].float()).all()
            if where == "v" or bad != bad:
                assert not torch.isfinite(out[[2, 4, 5, 6]].float()).any()


@pytest.mark.parametrize("dtype", TYPES)
def test_scores_of_minus_infinity_and_rows_that_see_nothing(dtype):
    b = Batch(43, dtype, 2, 2, 64, 16, [20], [[-1, 0, 1]])
    table = b.page_table.clone()
    table[:] = -1                                              # no page of the sequence exists
    out = binding.tree_attention(b.q, b.cache, 0, table, b.context, b.seq_start, b.parent)
    assert bool((out == 0).all())
    b.q[:] = -1                                                # every score minus infinity: 0 / 0
    for pages in b.tables[0]:
        b.cache.k[0, pages] = float("inf")
    assert bool(torch.isnan(run(b)).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("context", [40, 2100])
def test_keys_on_pages_outside_the_cache_are_left_out(dtype, context):
    rng = random.Random(47)
    b = Batch(53, dtype, 4, 2, 128, 16, [context], [random_tree(rng, 9)])
    gone = [1, len(b.tables[0]) - 2]
    for bad in (-1, b.cache.n_pages, 2 ** 31 - 1, -2 ** 31):
        table = b.page_table.clone()
        table[0, gone] = bad
        out = binding.tree_attention(b.q, b.cache, 0, table, b.context, b.seq_start, b.parent)
        rows = []
        for i in range(9):
            keys = [x for x in b.visible(0, i) if x // 16 not in gone]
            rows += [(i, h, b.q[i, h], b.k_rows[0][:, h // 2], b.v_rows[0][:, h // 2], keys, b.scale) for h in range(4)]
        check_rows(out, rows, dtype, bad)


@pytest.mark.parametrize("dtype", TYPES)
def test_lengths_out_of_range_read_nothing_outside(dtype):
    """Contexts and offsets beyond the arrays are brought into range; too many nodes or tokens give NaN."""
    b = Batch(59, dtype, 2, 1, 64, 16, [30], [[-1] * 3])
    args = (b.page_table, ints([10 ** 9]), ints([0, 3]), b.parent)
    out = binding.tree_attention(b.q, b.cache, 0, *args)        # the context fills the table, the nodes lie behind it
    assert out.shape == b.q.shape
    assert bool((binding.tree_attention(b.q, b.cache, 0, b.page_table, ints([-5]), ints([3, 0]), b.parent, out=torch.full_like(b.q, 2)) == 2).all())
    binding.tree_attention(b.q, b.cache, 0, b.page_table, b.context, ints([-4, 2 ** 31 - 1]), b.parent)
    many = Batch(61, dtype, 2, 1, 64, 16, [30, 10], [list(range(-1, 64)), [-1, 0]])
    out = run(many)
    assert bool(torch.isnan(out[:65]).all()) and bool(torch.isfinite(out[65:].float()).all())
    more = binding.tree_attention(b.q, b.cache, 0, b.page_table, b.context, ints([0, 3]), b.parent[:2].contiguous(), ints([0, 2]))
    assert bool(torch.isnan(more).all())
    assert binding.attention_status() == 0


@pytest.mark.parametrize("dtype", TYPES)
def test_captured_calls_follow_lengths_and_do_not_share_workspaces(dtype):
    rng = random.Random(67)
    b = Batch(71, dtype, 8, 8, 128, 64, [3000, 900], [random_tree(rng, 16), random_tree(rng, 5)])
    c = Batch(73, dtype, 8, 8, 128, 64, [2500, 10], [random_tree(rng, 9), random_tree(rng, 64)])
    want_b, want_c = run(b), run(c)
    out_b, out_c = torch.empty_like(want_b), torch.empty_like(want_c)
    graphs = []
    for x, out in ((b, out_b), (c, out_c)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            binding.tree_attention(x.q, x.cache, 0, x.page_table, x.context, x.seq_start, x.parent, out=out)
        graphs.append(g)
    streams = [torch.cuda.Stream() for _ in graphs]
    for _ in range(20):
        out_b.zero_()
        out_c.zero_()
        torch.cuda.synchronize()
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out_b, want_b) and torch.equal(out_c, want_c)
    b.context.copy_(ints([1111, 17]))                           # another length, the same graph
    graphs[0].replay()
    torch.cuda.synchronize()
    now = binding.tree_attention(b.q, b.cache, 0, b.page_table, b.context, b.seq_start, b.parent)
    assert torch.equal(out_b, now) and not torch.equal(out_b, want_b)


def test_on_a_stream_of_its_own():
    rng = random.Random(79)
    b = Batch(83, torch.bfloat16, 8, 2, 128, 64, [5000], [random_tree(rng, 16)])
    want = run(b)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    outs = [binding.tree_attention(b.q, b.cache, 0, b.page_table, b.context, b.seq_start, b.parent, stream=s,
                                   out=torch.empty_like(want)) for _ in range(8)]
    junk = [torch.full((1 << 22,), float("nan"), device=DEV) for _ in range(4)]      # would land in a workspace given back early
    torch.cuda.synchronize()
    assert len(junk) == 4 and all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("heads,kv_heads,nodes,contexts", [
    (16, 16, 16, [32000]), (8, 1, 8, [20000, 7]), (16, 16, 8, [8000] * 8), (32, 8, 64, [3000, 9000, 100]), (16, 4, 1, [700] * 40)])
@pytest.mark.parametrize("dim", [64, 128])
def test_every_run_gives_the_same_bits(heads, kv_heads, nodes, contexts, dim):
    """Work is cut by lengths alone, so runs do not differ; a tile taken from another place than its own would show."""
    rng = random.Random(97)
    b = Batch(101, torch.bfloat16, heads, kv_heads, dim, 64, contexts, [random_tree(rng, nodes) for _ in contexts])
    want = run(b)
    b.check(want, rng, 30)
    outs = [binding.tree_attention(b.q, b.cache, 0, b.page_table, b.context, b.seq_start, b.parent) for _ in range(40)]
    assert binding.attention_status() == 0
    assert all(torch.equal(o, want) for o in outs)


@pytest.mark.parametrize("dtype", TYPES)
def test_hundreds_of_sequences(dtype):
    rng = random.Random(103)
    contexts = [rng.choice([0, 3, 40, 130, 600]) for _ in range(333)]
    b = Batch(107, dtype, 32, 8, 64, 32, contexts, [random_tree(rng, rng.choice([0, 1, 1, 2, 17])) for _ in contexts])
    b.check(run(b), rng, 300)


def test_more_work_than_is_counted_is_refused():
    """Refused by its sizes, before anything is read: 2^20 tokens over 2^28 positions."""
    b = Batch(109, torch.bfloat16, 8, 4, 64, 16, [10], [[-1]])
    p = b.q.data_ptr()
    lib = binding.load_library()
    rc = lib.s2moe_tree_attention(b.cache._ref, 0, 1, 1 << 20, 8, p, 512, p, 1 << 24, p, p, 1 << 20, None, None, 0.1, p, p, 1 << 40, None)
    assert rc == binding.ERANGE
