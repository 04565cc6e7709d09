"""Long key ranges, where a mean over thousands of values hides any one of them: keys that alone decide a row's output, at the borders of tiles, pages and parts and of what a row sees; log-sum-exps of every row."""
import pytest
import torch

import paper_2605_29233_amd as bb
from kv_oracle import DEV, PAGE, TYPES, attention, check, gen, ints, limit, rnd, shared, starts
from test_attention_ops import branches, inputs, run, run_plan, run_shared, run_shared_plan

STRONG = 16.0           # of a decisive key and its query: a score of 32 (dim 64) or 22.6 (dim 128) where all others have 0, of 16384 keys with e^22.6 = 6.7e9


def probes(n, m, at, dim, dtype, seed):
    """Queries, keys and values of two heads on one: row i looks along its own direction, in which only key at[i] lies (None: no key); that key's values are i + 2, the others' within 1."""
    assert n <= dim
    q, k = torch.zeros(n, 2, dim, dtype=TYPES[dtype]), torch.zeros(m, 1, dim, dtype=TYPES[dtype])
    v = (torch.rand(m, 1, dim, generator=gen(seed)) * 2 - 1).to(TYPES[dtype])
    for i, j in enumerate(at):
        q[i, :, i] = STRONG
        if j is not None:
            k[j, 0, i] = STRONG
            v[j] = i + 2
    return q, k, v


def decided(out, n, m, block, at):
    """What the rows must show without any oracle: their key's value where they see it (off by its share, roundings and the others' weights: below a quarter), far less where they do not."""
    for i, j in enumerate(at):
        if j is not None and j < limit(n, m, block, i):
            assert (out[i].float() - (i + 2)).abs().max() < 0.25, (i, j)
        else:
            assert out[i].float().abs().max() < 1.25, (i, j)


def borders(n, m, block):
    """For n rows each: the last key they see, the first that they do not, and keys at the ends of tiles, halves and parts."""
    last = [max(limit(n, m, block, i) - 1, 0) for i in range(n)]
    yield [j if j not in last[:i] else None for i, j in enumerate(last)]
    past = [limit(n, m, block, i) for i in range(n)]
    yield [j if j < m and j not in past[:i] else None for i, j in enumerate(past)]
    tiles = -(-m // 64)
    edges = sorted({x for t in {tiles * p // parts for parts in (1, 2, 3, 7, 32) for p in range(parts + 1)} | {1, 2, 3} for x in (64 * t - 33, 64 * t - 32, 64 * t - 1, 64 * t) if 0 <= x < m} | {m - 1})
    pick = torch.randperm(len(edges), generator=gen(m + n)).tolist()
    for a in range(0, len(edges), n):
        part = [edges[x] for x in pick[a:a + n]]
        yield part + [None] * (n - len(part))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("block", [0, 1, 32])
@pytest.mark.parametrize("n,m,dim", [(12, 3000, 64), (60, 4097, 64), (16, 8190, 128), (100, 8190, 128), (64, 16384, 64)])
def test_one_key_decides(n, m, dim, block, dtype):
    """(values of up to 101 take 7 bits: exact in both types)"""
    for case, at in enumerate(borders(n, m, block)):
        q, k, v = probes(n, m, at, dim, dtype, case)
        out, lse = run(q, k, v, [n], [m], block)
        decided(out, n, m, block, at)
        if case < 3:
            want = attention(q, k, v, [n], [m], block, dim ** -0.5)
            check(out, lse, want, q.dtype)
            for plan in ((1, 1), (2, 3), (1, 7), (2, 32)):
                out, lse = run_plan(q, k, v, [n], [m], block, *plan)
                decided(out, n, m, block, at)
                check(out, lse, want, q.dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("block", [0, 1])
@pytest.mark.parametrize("n,prefix,own", [(8, 8129, 300), (40, 4096, 130), (40, 8190, 64)])
def test_one_key_of_a_prefix_or_of_its_own_decides(n, prefix, own, block):
    """Two branches on a shared prefix: a row's key is at the borders of pages and parts of the prefix, or of the second branch's own keys."""
    dim, m = 64, prefix + own
    rows, lens = [n, n], [own, own]
    tiles = -(-prefix // 64)
    edges = sorted({x for t in {tiles * p // parts for parts in (1, 3, 24, 32) for p in range(parts + 1)} | {1, 2} for x in (64 * t - 1, 64 * t) if 0 <= x < prefix} | {prefix - 1, prefix, m - 1} |
                   {prefix + x for x in (31, 32, 63, 64, own - n, own - n + 1) if x < own})
    pick = torch.randperm(len(edges), generator=gen(prefix)).tolist()
    for case, a in enumerate(range(0, len(edges), n)):
        at = [edges[x] for x in pick[a:a + n]]
        _, k, v, op, pp = branches(case, rows, lens, [prefix], 2, 1, dim, "bf16")
        k = torch.where(torch.isnan(k), k, 0.0)
        v = v.clamp(-1, 1)
        q = torch.zeros(2 * n, 2, dim, dtype=k.dtype)
        for i, j in enumerate(at):
            page, place = (pp[0, j // PAGE], j % PAGE) if j < prefix else (op[1, (j - prefix) // PAGE], (j - prefix) % PAGE)
            q[i, :, i] = q[n + i, :, i] = STRONG
            k[page, 0, place, i] = STRONG
            v[page, 0, place] = i + 2
        want = shared(q, rows, k, v, op, lens, pp, [prefix], [0, 2], block, dim ** -0.5)

        def one(got):
            check(*got, want, k.dtype)
            for b in (0, 1):
                of_own = [None if j is None or (j >= prefix and b == 0) else j for j in at]
                for i, j in enumerate(of_own):
                    seen = j is not None and (j < prefix or j - prefix < limit(n, own, block, i))
                    x = got[0][b * n + i].float()
                    assert (x - (i + 2)).abs().max() < 0.25 if seen else x.abs().max() < 1.25, (b, i, j)

        one(run_shared(q, rows, k, v, op, lens, pp, [prefix], [0, 2], block))
        for plan in ((1, 1, 0), (2, 3, 0), (1, 2, 24), (2, 1, 32)):
            one(run_shared_plan(q, rows, k, v, op, lens, pp, [prefix], [0, 2], block, *plan))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("block", [0, 1, 32])
def test_log_sum_exp_of_every_row_of_a_long_prompt(block, dtype):
    """2049 tokens, against 64 bits on the device; tolerance as kv_oracle.rows_of has it."""
    n, heads, dim = 2049, 3, 128
    q, k, v = inputs(1, [n], [n], heads, 1, dim, dtype)
    _, lse = run(q, k, v, [n], None, block)
    see = torch.tensor([limit(n, n, block, i) for i in range(n)], device=DEV)
    dk = k[:, 0].to(DEV).double().t().contiguous()
    for h in range(heads):
        dq = q[:, h].to(DEV).double()
        s = (dq @ dk * dim ** -0.5).masked_fill(torch.arange(n, device=DEV) >= see[:, None], float("-inf"))
        want, top = torch.logsumexp(s, 1), s.amax(1)
        e = dim * 2.0 ** -24 * (dq.abs() @ dk.abs()).amax(1) * dim ** -0.5 + 2.0 ** -23 * 1.45 * 2 * s.masked_fill(torch.isinf(s), 0).abs().amax(1) + 2.0 ** -21 + n * 2.0 ** -24
        assert ((lse[:, h].double() - want).abs() <= e + 2.0 ** -22 * (want.abs() + top.abs() + 1)).all()


@pytest.mark.gpu
def test_a_page_that_is_not_there_leaves_the_others():
    """A prefix of four full pages of which one is not in the cache gives what the three others give, named by a table without it."""
    rows, own, groups = [2, 3], [100, 130], [0, 2]
    q, k, v, op, pp = branches(21, rows, own, [256], 4, 2, 64, "bf16")
    for i, bad in enumerate((-1, k.shape[0], 2 ** 31 - 1, -2 ** 31)):
        gone, left = pp.clone(), torch.cat((pp[:, :i], pp[:, i + 1:]), 1)
        gone[0, i] = bad
        want = shared(q, rows, k, v, op, own, left, [192], groups, 0, 0.125)
        check(*run_shared(q, rows, k, v, op, own, gone, [256], groups), want, q.dtype)
        check(*run_shared(q, rows, k, v, op, own, left, [192], groups), want, q.dtype)
