"""Causal attention over packed prompts against a plain 64-bit computation, row by row."""
import random

import pytest
import torch

from paper_2608_15018_b200 import binding
from tests.attn_util import DEV, check_rows, ints, offsets

pytestmark = pytest.mark.gpu
TYPES = [torch.bfloat16, torch.float32]


def inputs(seed, dtype, heads, kv_heads, dim, lengths, tail=0):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    n = sum(lengths) + tail
    wide = torch.randn((n, (heads + 2 * kv_heads) * dim), generator=gen, device=DEV)
    wide[:, :heads * dim] *= 2
    wide = wide.to(dtype)
    if tail:
        wide[sum(lengths):] = float("nan")
    q, k, v = wide.split([heads * dim, kv_heads * dim, kv_heads * dim], dim=1)
    return q.unflatten(1, (heads, dim)), k.unflatten(1, (kv_heads, dim)), v.unflatten(1, (kv_heads, dim)), ints(offsets(lengths))


def check(out, q, k, v, lengths, dtype, rng, most=150, first=0):
    heads, group, rows = q.shape[1], q.shape[1] // k.shape[1], []
    starts = [first + x for x in offsets(lengths)]
    want = [(s, i) for s, n in enumerate(lengths) for i in range(n)]
    ends = [(s, i) for s, n in enumerate(lengths) for i in {0, n - 1} if n]
    for s, i in rng.sample(want, min(most, len(want))) + rng.sample(ends, min(40, len(ends))):
        a, b = starts[s], starts[s + 1]
        h = rng.randrange(heads)
        rows.append((a + i, h, q[a + i, h], k[a:b, h // group], v[a:b, h // group], list(range(i + 1)), q.shape[2] ** -0.5))
    check_rows(out, rows, dtype)
    assert bool(torch.isfinite(out[starts[0]:starts[-1]].float()).all())


def run(*args, **kw):
    out = binding.prompt_attention(*args, **kw)
    assert binding.attention_status() == 0
    return out


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 64), (16, 16, 128), (32, 8, 128), (9, 3, 64), (28, 4, 128), (64, 1, 64), (40, 1, 128)])
def test_single_prompts(dtype, heads, kv_heads, dim):
    rng = random.Random(heads + dim)
    for n in (1, 2, 63, 64, 65, 127, 128, 129, 255, 256, 257, 500):
        q, k, v, starts = inputs(n, dtype, heads, kv_heads, dim, [n])
        check(run(q, k, v, starts), q, k, v, [n], dtype, rng, 40)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 128), (8, 2, 64), (7, 1, 128)])
def test_packed_prompts(dtype, heads, kv_heads, dim):
    rng = random.Random(heads)
    lengths = [1, 0, 130, 64, 7, 0, 900, 256, 1, 333, 0]
    q, k, v, starts = inputs(3, dtype, heads, kv_heads, dim, lengths)
    check(run(q, k, v, starts), q, k, v, lengths, dtype, rng, 300)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_short_prompts(dtype):
    rng = random.Random(1)
    lengths = [rng.choice([0, 1, 2, 5, 40, 140]) for _ in range(90)]
    q, k, v, starts = inputs(5, dtype, 4, 2, 64, lengths)
    check(run(q, k, v, starts), q, k, v, lengths, dtype, rng, 300)


@pytest.mark.parametrize("dtype,n", [(torch.bfloat16, 9001), (torch.float32, 2777)])
def test_long_prompt(dtype, n):
    rng = random.Random(2)
    q, k, v, starts = inputs(7, dtype, 4, 2, 128, [n])
    check(run(q, k, v, starts), q, k, v, [n], dtype, rng, 120)


@pytest.mark.parametrize("dtype", TYPES)
def test_tokens_of_no_sequence(dtype):
    """Tokens before the first and behind the last sequence hold NaN; their rows of the output stay as they were."""
    rng = random.Random(3)
    lengths = [70, 130, 5]
    q, k, v, starts = inputs(11, dtype, 4, 2, 64, lengths, tail=90)
    out = torch.full((295, 4, 64), 3.0, dtype=dtype, device=DEV)
    assert run(q, k, v, starts, out=out) is out
    check(out, q, k, v, lengths, dtype, rng)
    assert bool((out[205:] == 3.0).all())
    later = run(q, k, v, starts[1:].contiguous(), out=torch.full_like(out, 3.0))
    assert bool((later[:70] == 3.0).all()) and torch.equal(later[70:205], out[70:205])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [100, 700])
def test_later_tokens_have_no_part_whatever_they_hold(dtype, n):
    q, k, v, starts = inputs(13, dtype, 4, 2, 64, [n])
    clean = run(q, k, v, starts)
    for at in (n - 1, n // 2, 1):
        for bad in (float("nan"), float("inf"), -float("inf")):
            for x in (k, v):
                keep = x[at].clone()
                x[at] = bad
                out = run(q, k, v, starts)
                x[at] = keep
                # two results of one row, each off by at most 2^-8 (|result| + mean of |v|), and that mean below 2
                near = (out[:at].float() - clean[:at].float()).abs() <= 2.0 ** -6 * clean[:at].float().abs() + 2.0 ** -6
                assert bool(near.all()), (at, bad)
                if bad != bad:
                    assert not bool(torch.isfinite(out[at:].float()).any())


@pytest.mark.parametrize("dtype", TYPES)
def test_offsets_out_of_range_read_nothing_outside(dtype):
    q, k, v, _ = inputs(17, dtype, 2, 1, 64, [50])
    want = run(q, k, v, ints([0, 50]))
    assert torch.equal(run(q, k, v, ints([-9, 2 ** 31 - 1])), want)
    out = torch.full((50, 2, 64), 5.0, dtype=dtype, device=DEV)
    run(q, k, v, ints([40, 20, 10 ** 9, 3]), out=out)
    assert bool((out[:20] == 5.0).all())
    assert torch.equal(run(q, k, v, ints([0]), out=torch.full_like(out, 5.0)), torch.full_like(out, 5.0))


@pytest.mark.parametrize("dtype", TYPES)
def test_scale_and_captured_call(dtype):
    rng = random.Random(5)
    q, k, v, starts = inputs(19, dtype, 4, 2, 128, [300, 40])
    want = run(q, k, v, starts, scale=0.0)
    i = 299                                                    # scale 0: the mean of the values
    ref = v[:i + 1].double().mean(0).repeat_interleave(2, dim=0)
    assert bool(((want[i].double() - ref).abs() <= 2.0 ** -7 * v[:i + 1].double().abs().mean(0).repeat_interleave(2, dim=0)).all())
    out = torch.empty((340, 4, 128), dtype=dtype, device=DEV)
    plain = run(q, k, v, starts)
    check(plain, q, k, v, [300, 40], dtype, rng)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        binding.prompt_attention(q, k, v, starts, out=out)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, plain)
    starts.copy_(ints([0, 10, 333]))                            # other lengths, the same graph
    g.replay()
    torch.cuda.synchronize()
    check(out, q, k, v, [10, 323], dtype, rng)


@pytest.mark.parametrize("dtype,n", [(torch.bfloat16, 140000), (torch.float32, 20000)])
def test_very_many_sequences(dtype, n):
    """More items than a million: prompts of one token, whose output is their value."""
    gen = torch.Generator(device=DEV).manual_seed(23)
    q, k = (torch.randn((n, 8, 64), generator=gen, device=DEV).to(dtype) for _ in range(2))
    v = torch.randn((n, 8, 64), generator=gen, device=DEV).to(dtype)
    out = run(q, k, v, torch.arange(n + 1, dtype=torch.int32, device=DEV))
    assert torch.equal(out, v)


@pytest.mark.parametrize("heads,kv_heads,dim", [(16, 16, 128), (32, 8, 64)])
def test_every_run_gives_the_same_bits(heads, kv_heads, dim):
    lengths = [1500, 3, 700, 129, 2500, 64]
    q, k, v, starts = inputs(29, torch.bfloat16, heads, kv_heads, dim, lengths)
    want = run(q, k, v, starts)
    outs = [binding.prompt_attention(q, k, v, starts) for _ in range(40)]
    assert binding.attention_status() == 0
    assert all(torch.equal(o, want) for o in outs)
