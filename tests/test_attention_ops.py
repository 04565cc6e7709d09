"""Attention over packed prompts and attention of branches that share a prefix, against their definitions in 64 bits, row by row: types, heads, lengths, masks, rows that
see nothing, pages that end inside a tile, values that must not be read, strides, streams, graphs and refusals.  Tolerances: kv_oracle.rows_of."""
import os
import re

import pytest
import torch

import paper_2605_29233_amd as bb
from paper_2605_29233_amd import BBError, binding
from kv_oracle import DEV, PAGE, TYPES, attention, check, gen, ints, rnd, shared, starts

HEADS = [(4, 4, 64), (6, 2, 128), (7, 1, 64), (3, 3, 128)]
LENGTHS = [([1], None), ([64], None), ([65, 0, 1, 127], None), ([33, 40], [97, 40]), ([130], [64]), ([5, 3, 0, 2], [0, 200, 9, 2]), ([257], None), ([1, 1, 1], [300, 1, 129])]


def inputs(seed, ql, kl, heads, kv_heads, dim, dtype, scale=1.0):
    return (rnd(seed, sum(ql), heads, dim, dtype=dtype, scale=scale), rnd(seed + 1, sum(kl), kv_heads, dim, dtype=dtype), rnd(seed + 2, sum(kl), kv_heads, dim, dtype=dtype))


def run(q, k, v, ql, kl, block, scale=None, want_lse=True):
    lse = torch.full(q.shape[:2], 7.0, device=DEV) if want_lse else None
    out = torch.full(q.shape, 9.0, dtype=q.dtype, device=DEV)
    r = bb.attention(q.to(DEV), k.to(DEV), v.to(DEV), starts(ql).to(DEV), None if kl is None else starts(kl).to(DEV), block=block, scale=scale, out=out, lse=lse)
    assert r is out
    return out, lse


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("block", [0, 1, 5, 32, 1000])
@pytest.mark.parametrize("ql,kl", LENGTHS)
@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
def test_attention_equals_the_definition(heads, kv_heads, dim, ql, kl, block, dtype):
    q, k, v = inputs(len(ql) + dim, ql, kl or ql, heads, kv_heads, dim, dtype, 2.0)
    out, lse = run(q, k, v, ql, kl, block)
    check(out, lse, attention(q, k, v, ql, kl or ql, block, dim ** -0.5), q.dtype)
    again, l2 = run(q, k, v, ql, kl, block)
    assert torch.equal(out, again) and torch.equal(lse, l2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(2, 2, 128), (28, 4, 128), (1, 1, 64)])
def test_longer_prompts(heads, kv_heads, dim, dtype):
    """Some of the rows of longer sequences, causal and not (the others are compared with a product of matrices elsewhere)."""
    for n, m, block in ((700, 700, 1), (513, 1400, 32), (40, 3000, 0), (1, 4097, 1)):
        q, k, v = inputs(n, [n], [m], heads, kv_heads, dim, dtype)
        out, lse = run(q, k, v, [n], [m], block)
        pick = sorted({0, 1, 31, 32, 63, 127, 128, 300, n // 2, n - 2, n - 1} & set(range(n)))
        for i in pick:
            seen = m if block == 0 else min(m, ((m - n + i) // block + 1) * block)
            want = attention(q[i:i + 1], k[:seen], v[:seen], [1], [seen], 0, dim ** -0.5)
            check(out[i:i + 1], lse[i:i + 1], want, q.dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("block", [0, 1, 32])
def test_every_row_of_a_long_prompt(block):
    """2049 tokens against the definition as products of matrices in 64 bits on the device: every row, tolerance as for one row with the largest of its terms."""
    n, heads, dim = 2049, 3, 128
    q, k, v = inputs(1, [n], [n], heads, 1, dim, "bf16")
    out, _ = run(q, k, v, [n], None, block)
    see = torch.tensor([n if block == 0 else min(n, (i // block + 1) * block) for i in range(n)], device=DEV)
    for h in range(heads):
        s = q[:, h].to(DEV).double() @ k[:, 0].to(DEV).double().t().contiguous() * dim ** -0.5
        s = s.masked_fill(torch.arange(n, device=DEV) >= see[:, None], float("-inf"))
        p = torch.softmax(s, 1)
        want, mean = p @ v[:, 0].to(DEV).double(), p @ v[:, 0].to(DEV).double().abs()
        e = dim * 2.0 ** -24 * (q[:, h].to(DEV).double().abs() @ k[:, 0].to(DEV).double().abs().t().contiguous()).amax(1) * dim ** -0.5
        e = e + 2.0 ** -22 * 1.45 * s.masked_fill(torch.isinf(s), 0).abs().amax(1) + 2.0 ** -21 + n * 2.0 ** -24
        slack = 2.0 ** -8 * mean + 2 * e[:, None] * mean
        off = (out[:, h].double() - want).abs()
        assert (off <= slack + 2.0 ** -8 * (want.abs() + slack)).all()


@pytest.mark.gpu
def test_strides_scale_and_what_is_left_alone():
    """Parts of one projection's output, heads first, padded heads; tokens behind the last sequence, before the first and between two stay as they were."""
    ql = [70, 9]
    for dim, heads, kv in ((64, 4, 2), (128, 2, 1)):
        x = rnd(3, 100, heads + 2 * kv, dim)
        q, k, v = x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:]
        want = attention(q[:79], k[:79], v[:79], ql, ql, 1, 0.3)
        d = x.to(DEV)
        out, lse = torch.full((100, heads, dim), 9.0, dtype=x.dtype, device=DEV), torch.full((100, heads), 9.0, device=DEV)
        parts = d[:, :heads], d[:, heads:heads + kv], d[:, heads + kv:]
        bb.attention(*parts, starts(ql).to(DEV), block=1, scale=0.3, out=out, lse=lse)
        check(out[:79], lse[:79], want, x.dtype)
        assert (out[79:] == 9).all() and (lse[79:] == 9).all()
        first = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in parts]
        wide = torch.full((heads, 100, dim + 8), 9.0, dtype=x.dtype, device=DEV)
        o2 = wide[:, :, :dim].transpose(0, 1)
        bb.attention(*first, starts(ql).to(DEV), block=1, scale=0.3, out=o2)
        assert torch.equal(o2[:79], out[:79]) and (o2[79:] == 9).all() and (wide[:, :, dim:] == 9).all()
        # sequences that begin later and leave a gap (starts as given, keys elsewhere)
        qs, ks = ints([10, 80, 80]).to(DEV), ints([0, 70, 70]).to(DEV)
        o3 = torch.full((100, heads, dim), 9.0, dtype=x.dtype, device=DEV)
        bb.attention(torch.cat((parts[0][:10], parts[0][:90])), parts[1], parts[2], qs, ks, block=1, scale=0.3, out=o3)
        assert torch.equal(o3[10:80], out[:70]) and (o3[:10] == 9).all() and (o3[80:] == 9).all()


@pytest.mark.gpu
def test_starts_outside_are_bounded():
    q, k, v = inputs(5, [40], [40], 2, 2, 64, "bf16")
    out = torch.full(q.shape, 9.0, dtype=q.dtype, device=DEV)
    for s in ([-5, 40], [0, 1000], [0, 2 ** 31 - 1], [-2 ** 31, 2 ** 31 - 1]):
        bb.attention(q.to(DEV), k.to(DEV), v.to(DEV), ints(s).to(DEV), block=1, out=out.fill_(9.0))
        check(out, None, attention(q, k, v, [40], [40], 1, 0.125), q.dtype)
    bb.attention(q.to(DEV), k.to(DEV), v.to(DEV), ints([30, 20, 10]).to(DEV), block=1, out=out.fill_(9.0))
    assert (out == 9).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_a_query_does_not_see_does_not_reach_it(bad, dim, dtype):
    """A right-padded prompt: keys and values from token 75 on are garbage, causal rows before it are as without it, rows behind it see it."""
    n, at = 140, 75
    q, k, v = inputs(7, [n], [n], 2, 1, dim, dtype)
    k2, v2 = k.clone(), v.clone()
    k2[at:] = bad
    v2[at:] = bad
    out, lse = run(q, k, v, [n], None, 1)
    got, l2 = run(q, k2, v2, [n], None, 1)
    assert torch.equal(got[:at], out[:at]) and torch.equal(lse[:at], l2[:at])
    # a value alone: rows that see it get it, in its own element only
    v3 = v.clone()
    v3[at, 0, 3] = bad
    got, _ = run(q, k, v3, [n], None, 1)
    hit = torch.zeros(n, 2, dim, dtype=torch.bool)
    hit[at:, :, 3] = True
    assert torch.equal(got.cpu()[~hit], out.cpu()[~hit])
    assert torch.isnan(got.cpu()[hit]).all() if bad != bad else (got.cpu()[hit] == bad).all()
    # both infinities seen: a NaN
    v3[at + 1, 0, 3] = -bad
    if bad == bad:
        got, _ = run(q, k, v3, [n], None, 1)
        assert (got[at, :, 3] == bad).all() and torch.isnan(got[at + 1:, :, 3]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_extreme_scores(dtype):
    """Scores far apart and large: the largest takes all; equal ones share; infinite ones as the definition has it."""
    q, k, v = inputs(9, [70], [200], 2, 2, 64, dtype)
    for factor in (0.0, 30.0, 200.0):
        out, lse = run(q * factor, k, v, [70], [200], 0)
        check(out, lse, attention(q * factor, k, v, [70], [200], 0, 0.125), q.dtype)
    q2 = q.clone()
    q2[3, 0] = float("nan")
    q2[4, 1, 0] = float("inf")
    out, _ = run(q2, k, v, [70], [200], 0)
    base, _ = run(q, k, v, [70], [200], 0)
    assert torch.isnan(out[3, 0]).all() and torch.isnan(out[4, 1]).all()
    keep = torch.ones(70, 2, dtype=torch.bool)
    keep[3, 0] = keep[4, 1] = False
    assert torch.equal(out.cpu()[keep], base.cpu()[keep])
    k2 = k.clone()
    k2[:, 0] = 0
    k2[100, 0, 0] = float("-inf")           # scores of -inf and +inf by the sign of q
    out, _ = run(q, k2, v, [70], [200], 0)
    plus = q[:, 0, 0] < 0
    assert torch.isnan(out.cpu()[plus, 0]).all() and torch.isfinite(out.cpu()[~plus, 0]).all()


def paged(seed, lens, width, pages_left, kv_heads, dim, dtype, n_pages, token_major=False):
    """A cache whose unused tokens are NaN, and the tables of `lens` (pages dealt from pages_left)."""
    table = torch.full((len(lens), width), -7, dtype=torch.int32)
    for i, n in enumerate(lens):
        for j in range(-(-n // PAGE)):
            table[i, j] = pages_left.pop()
    return table


def branches(seed, rows, own, prefixes, heads, kv_heads, dim, dtype, spare=3, token_major=False):
    n_pages = sum(-(-n // PAGE) for n in own + prefixes) + spare
    left = torch.randperm(n_pages, generator=gen(seed)).tolist()
    op = paged(seed, own, max([-(-n // PAGE) for n in own] + [1]) + 1, left, kv_heads, dim, dtype, n_pages)
    pp = paged(seed, prefixes, max([-(-n // PAGE) for n in prefixes] + [1]) + 1, left, kv_heads, dim, dtype, n_pages)
    k, v = (torch.full((n_pages, kv_heads, PAGE, dim), float("nan"), dtype=TYPES[dtype]) for _ in range(2))
    for s, c in ((seed + 1, k), (seed + 2, v)):
        x = rnd(s, n_pages, kv_heads, PAGE, dim, dtype=dtype)
        for table, lens in ((op, own), (pp, prefixes)):
            for i, n in enumerate(lens):
                for j in range(0, n, PAGE):
                    c[table[i, j // PAGE], :, :min(PAGE, n - j)] = x[table[i, j // PAGE], :, :min(PAGE, n - j)]
    q = rnd(seed + 3, sum(rows), heads, dim, dtype=dtype, scale=2.0)
    return q, k, v, op, pp


def on_device(c, token_major):
    c = c.to(DEV)
    return c.transpose(1, 2).contiguous().transpose(1, 2) if token_major else c


def run_shared(q, rows, k, v, op, own, pp=None, prefixes=None, groups=None, block=0, scale=None, token_major=False):
    out, lse = torch.full(q.shape, 9.0, dtype=q.dtype, device=DEV), torch.full(q.shape[:2], 9.0, device=DEV)
    prefix = () if pp is None else (pp.to(DEV), ints(prefixes).to(DEV), ints(groups).to(DEV))
    r = bb.shared_attention(q.to(DEV), starts(rows).to(DEV), on_device(k, token_major), on_device(v, token_major), op.to(DEV), ints(own).to(DEV), *prefix, block=block, scale=scale, out=out, lse=lse)
    assert r is out
    return out, lse


BRANCHES = [
    ([1], [1], [1], [0, 1]),
    ([1, 1, 1, 1], [5, 64, 65, 130], [200], [0, 4]),
    ([8, 16, 32], [20, 16, 70], [64], [0, 3]),
    ([3, 0, 5, 2, 1], [10, 4, 5, 0, 65], [129, 1], [0, 2, 4]),              # a branch outside every group, one without rows, one without keys
    ([2, 4, 1, 1], [1, 9, 64, 3], [0, 63], [0, 2, 4]),                      # an empty prefix; more rows than own keys
    ([40, 33], [100, 33], [300, 17], [0, 1, 2]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("block", [0, 1, 32])
@pytest.mark.parametrize("rows,own,prefixes,groups", BRANCHES)
@pytest.mark.parametrize("heads,kv_heads,dim", HEADS)
def test_shared_attention_equals_the_definition(heads, kv_heads, dim, rows, own, prefixes, groups, block, dtype):
    q, k, v, op, pp = branches(dim + len(rows), rows, own, prefixes, heads, kv_heads, dim, dtype)
    want = shared(q, rows, k, v, op, own, pp, prefixes, groups, block, dim ** -0.5)
    out, lse = run_shared(q, rows, k, v, op, own, pp, prefixes, groups, block, token_major=block == 1)
    check(out, lse, want, q.dtype)
    again, l2 = run_shared(q, rows, k, v, op, own, pp, prefixes, groups, block)
    assert torch.equal(out, again) and torch.equal(lse, l2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("block", [0, 1])
def test_pages_without_a_prefix(block, dtype):
    rows, own = [1, 3, 70], [700, 3, 129]
    q, k, v, op, _ = branches(5, rows, own, [], 4, 2, 128, dtype)
    want = shared(q, rows, k, v, op, own, [], [], [0], block, 128 ** -0.5)
    check(*run_shared(q, rows, k, v, op, own, block=block), want, q.dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 64), (28, 4, 128), (32, 32, 128)])
def test_many_branches_on_a_long_prefix(heads, kv_heads, dim):
    """24 continuations, a token each, of 2500 shared tokens, and two groups of them."""
    for prefixes, groups in (([2500], [0, 24]), ([700, 2001], [0, 9, 24])):
        rows, own = [1] * 24, [(37 * i) % 90 + 1 for i in range(24)]
        q, k, v, op, pp = branches(11, rows, own, prefixes, heads, kv_heads, dim, "bf16")
        out, lse = run_shared(q, rows, k, v, op, own, pp, prefixes, groups, 1)
        some = [0, heads // 2, heads - 1]
        for h in some:
            g = h // (heads // kv_heads)
            want = shared(q[:, h:h + 1], rows, k[:, g:g + 1], v[:, g:g + 1], op, own, pp, prefixes, groups, 1, dim ** -0.5)
            check(out[:, h:h + 1], lse[:, h:h + 1], want, q.dtype)


@pytest.mark.gpu
def test_pages_and_lengths_that_do_not_exist():
    """Pages outside the cache count as not there, lengths beyond the table as the table's, negative ones as none; nothing outside is read."""
    rows, own, prefixes, groups = [2, 3], [100, 130], [200], [0, 2]
    q, k, v, op, pp = branches(21, rows, own, prefixes, 4, 2, 64, "bf16")
    n = k.shape[0]
    for i, bad in enumerate((-1, n, 2 ** 31 - 1, -2 ** 31)):
        p2, o2 = pp.clone(), op.clone()
        p2[0, i % 4] = bad
        kp = [j for j in range(4) if j != i % 4]
        # the same without that page: the oracle leaves it out
        want = shared(q, rows, k, v, o2, own, p2, prefixes, groups, 0, 0.125)
        check(*run_shared(q, rows, k, v, o2, own, p2, prefixes, groups), want, q.dtype)
        assert len(kp) == 3
    none = torch.full_like(pp, -1)
    want = shared(q, rows, k, v, op, own, none, prefixes, groups, 0, 0.125)
    check(*run_shared(q, rows, k, v, op, own, none, prefixes, groups), want, q.dtype)
    # no key at all: zeros, not a NaN
    out, lse = run_shared(q, rows, k, v, torch.full_like(op, -1), own, none, prefixes, groups)
    assert (out == 0).all() and (lse == float("-inf")).all()
    out, lse = run_shared(q, rows, k, v, op, [-5, -2 ** 31], pp, [-1], groups)
    assert (out == 0).all() and (lse == float("-inf")).all()
    # a table of two full pages and a length beyond it
    full = torch.randn(n, 2, PAGE, 64, generator=gen(3)).to(torch.bfloat16)
    want = shared(q, rows, full, full, op[:, :2], [128, 128], pp, prefixes, groups, 0, 0.125)
    check(*run_shared(q, rows, full, full, op[:, :2], [2 ** 31 - 1, 1000], pp, prefixes, groups), want, q.dtype)


@pytest.mark.gpu
def test_cache_and_queries_beyond_32_bits():
    """Pages 2^31 elements apart, query rows 2^31 elements apart."""
    far = torch.empty(3 * (1 << 31), dtype=torch.bfloat16, device=DEV)
    k = far.as_strided((3, 1, 64, 64), (1 << 31, 4096, 64, 1))[:3]
    v = far[8192:].as_strided((3, 1, 64, 64), (1 << 31, 4096, 64, 1))
    x = rnd(1, 3, 1, 64, 64), rnd(2, 3, 1, 64, 64)
    k.copy_(x[0])
    v.copy_(x[1])
    q = rnd(3, 2, 1, 64)
    fq = far[16384:].as_strided((2, 1, 64), (1 << 31, 64, 1))
    fo = far[32768:].as_strided((2, 1, 64), (1 << 31, 64, 1))
    fq.copy_(q)
    op = ints([[2, 0], [1, -1]])
    own = [100, 30]
    with pytest.raises(BBError):            # (the cache's strides and the output's interleave in a way that is not looked into)
        bb.shared_attention(fq, starts([1, 1]).to(DEV), k, v, op.to(DEV), ints(own).to(DEV), out=fo)
    out = bb.shared_attention(fq, starts([1, 1]).to(DEV), k, v, op.to(DEV), ints(own).to(DEV))
    check(out, None, shared(q, [1, 1], x[0], x[1], op, own, [], [], [0], 0, 0.125), q.dtype)
    # packed keys: 2^31 elements from the first to the last
    packed = far[:(1 << 31) + 64 * 300].view(-1, 64)
    rows = packed.shape[0]
    kk, vv = rnd(4, 280, 1, 64), rnd(5, 280, 1, 64)
    keys = packed[:, None]
    keys[rows - 290:rows - 10] = kk.to(DEV)
    vals = torch.zeros(rows, 1, 64, dtype=torch.bfloat16, device=DEV)
    vals[rows - 290:rows - 10] = vv.to(DEV)
    out = bb.attention(q.to(DEV), keys, vals, ints([0, 2]).to(DEV), ints([rows - 290, rows - 10]).to(DEV), block=1)
    check(out, None, attention(q, kk, vv, [2], [280], 1, 0.125), q.dtype)


@pytest.mark.gpu
def test_a_prompt_then_token_by_token_equals_the_whole():
    """As a program uses them: a prompt's rows turned and appended to the cache, attention over it, then tokens one at a time of three branches that share it; every token's
    output against the definition on the whole sequence of its branch."""
    heads, kv, dim, prompt, steps, nb = 6, 2, 64, 100, 5, 3
    n_pages = 2 + nb
    kc, vc = (torch.zeros(n_pages, kv, PAGE, dim, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    f = bb.rope_frequencies(dim, device=DEV)
    x = rnd(1, prompt, heads + 2 * kv, dim).to(DEV)
    pos = torch.arange(prompt, dtype=torch.int32, device=DEV)
    q = bb.rope_append(x[:, :heads], x[:, heads:heads + kv], x[:, heads + kv:], pos, f, kc, vc, pos, q_out=torch.empty(prompt, heads, dim, dtype=x.dtype, device=DEV))
    keys, vals = (c[:2].transpose(1, 2).reshape(-1, kv, dim)[:prompt] for c in (kc, vc))
    assert torch.equal(vals, x[:, heads + kv:])
    out = bb.attention(q, keys.contiguous(), vals.contiguous(), starts([prompt]).to(DEV), block=1)
    check(out, None, attention(q.cpu(), keys.cpu(), vals.cpu(), [prompt], [prompt], 1, dim ** -0.5), x.dtype)
    own = ints([[2], [3], [4]]).to(DEV)
    prefix = ints([[0, 1]]).to(DEV), ints([prompt]).to(DEV), ints([0, nb]).to(DEV)
    for s in range(steps):
        y = rnd(10 + s, nb, heads + 2 * kv, dim).to(DEV)
        slots = ints([(2 + b) * PAGE + s for b in range(nb)]).to(DEV)
        p = torch.full((nb,), prompt + s, dtype=torch.int32, device=DEV)
        q = bb.rope_append(y[:, :heads], y[:, heads:heads + kv], y[:, heads + kv:], p, f, kc, vc, slots)
        lens = [s + 1] * nb
        out = bb.shared_attention(q, starts([1] * nb).to(DEV), kc, vc, own, ints(lens).to(DEV), *prefix, block=1)
        want = shared(q.cpu(), [1] * nb, kc.cpu(), vc.cpu(), own.cpu(), lens, prefix[0].cpu(), [prompt], [0, nb], 1, dim ** -0.5)
        check(out, None, want, x.dtype)


@pytest.mark.gpu
def test_captured_and_replayed_with_other_lengths():
    """Both calls in one graph; between replays the lengths, tables and inputs change and eager calls of the same run; every replay equals the eager result."""
    rows, own, prefixes, groups = [1, 2, 1], [60, 64, 1], [150], [0, 3]
    q, k, v, op, pp = branches(31, rows, own, prefixes, 4, 2, 64, "bf16")
    k, v = (torch.nan_to_num(c).to(DEV) for c in (k, v))
    d = dict(q=q.to(DEV), qs=starts(rows).to(DEV), op=op.to(DEV), own=ints(own).to(DEV), pp=pp.to(DEV), pl=ints(prefixes).to(DEV), gs=ints(groups).to(DEV))
    x = rnd(32, 90, 4, 64).to(DEV)
    ps = ints([0, 50, 90]).to(DEV)

    def both():
        return (bb.shared_attention(d["q"], d["qs"], k, v, d["op"], d["own"], d["pp"], d["pl"], d["gs"], block=1), bb.attention(x, x[:, :2], x[:, 2:], ps, block=1))

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        got = both()
    for n, (lens, prefix, cut) in enumerate((([60, 64, 1], 150, 50), ([3, 64, 64], 128, 1), ([0, 0, 0], 0, 90), ([64, 1, 33], 191, 0))):
        d["own"].copy_(ints(lens))
        d["pl"].copy_(ints([prefix]))
        ps.copy_(ints([0, cut, 90]))
        d["q"].copy_(rnd(40 + n, *q.shape))
        g.replay()
        torch.cuda.synchronize()
        a, b = (t.clone() for t in got)
        e = both()
        torch.cuda.synchronize()
        assert torch.equal(a, e[0]) and torch.equal(b, e[1]), n


@pytest.mark.gpu
def test_two_streams_at_once():
    q, k, v = inputs(41, [300], [300], 8, 2, 128, "bf16")
    d = [t.to(DEV) for t in (q, k, v)]
    s = starts([300]).to(DEV)
    want = bb.attention(*d, s, block=1)
    rows, own, prefixes, groups = [1] * 8, [50] * 8, [900], [0, 8]
    b = branches(43, rows, own, prefixes, 8, 2, 128, "bf16")
    bd = [t.to(DEV) for t in b]
    tail = starts(rows).to(DEV), ints(own).to(DEV), ints(prefixes).to(DEV), ints(groups).to(DEV)

    def second(stream=None):
        return bb.shared_attention(bd[0], tail[0], bd[1], bd[2], bd[3], tail[1], bd[4], tail[2], tail[3], block=1, stream=stream)

    want2 = second()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for _ in range(6):
        outs.append((bb.attention(*d, s, block=1, stream=streams[0]), second(streams[1])))
        outs.append((bb.attention(*d, s, block=1, stream=streams[1]), second(streams[0])))
    torch.cuda.synchronize()
    for a, c in outs:
        assert torch.equal(a, want) and torch.equal(c, want2)


@pytest.mark.gpu
def test_nothing_to_do():
    e = torch.empty(0, 4, 64, dtype=torch.bfloat16, device=DEV)
    x = rnd(1, 5, 4, 64).to(DEV)
    assert bb.attention(e, x, x, ints([0]).to(DEV)).shape == (0, 4, 64)
    out = torch.full_like(x, 9.0)
    bb.attention(x, e, e, ints([0, 3]).to(DEV), ints([0, 0]).to(DEV), out=out)
    assert (out[:3] == 0).all() and (out[3:] == 9).all()
    bb.attention(x, x, x, ints([0]).to(DEV), out=out.fill_(9))
    assert (out == 9).all()


def test_argument_structs_are_packed_as_the_header_has_them():
    """Every field has eight bytes, and the doubles stand where the binding packs them."""
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "blockbatch.h")).read()
    for name, packed in (("rope", binding.ROPE_ARGS), ("rope_append", binding.ROPE_APPEND_ARGS), ("attention", binding.ATTENTION_ARGS), ("shared_attention", binding.SHARED_ATTENTION_ARGS)):
        body = re.search(r"typedef struct \{([^}]*)\} bb_%s_args;" % name, header).group(1)
        kinds = ""
        for field in body.split(";"):
            for _ in field.split(",") if field.strip() else ():
                kinds += "d" if re.search(r"\bdouble (?!\*)", field) and "*" not in field else "q"
        packed_kinds = "".join(int(n or 1) * c for n, c in re.findall(r"(\d*)([qd])", packed.format))
        assert kinds == packed_kinds, name
        assert packed.size == 8 * len(kinds)


def heads_of(t):
    return t.data_ptr(), t.stride(0), t.stride(1)


def run_plan(q, k, v, ql, kl, block, halves, parts):
    """bb_attention with a plan of the test's choice."""
    d = [t.to(DEV) for t in (q, k, v)]
    qs, ks = starts(ql).to(DEV), starts(kl).to(DEV)
    out, lse = torch.full(q.shape, 9.0, dtype=q.dtype, device=DEV), torch.full(q.shape[:2], 9.0, device=DEV)
    tokens, heads, dim = q.shape
    args = binding.ATTENTION_ARGS.pack(*(x for t in d for x in heads_of(t)), qs.data_ptr(), ks.data_ptr(), len(ql), tokens, k.shape[0], heads, k.shape[1], dim,
                                       {torch.bfloat16: 1, torch.float16: 2}[q.dtype], block, dim ** -0.5, *heads_of(out), lse.data_ptr())
    ws = torch.full((parts * tokens * heads * (dim * 4 + 8) + 512,), 255, dtype=torch.uint8, device=DEV)       # (NaN wherever nothing is written)
    assert bb.load_library().bb_debug_attention(args, halves, parts, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
    torch.cuda.synchronize()
    return out, lse


def run_shared_plan(q, rows, k, v, op, own, pp, prefixes, groups, block, halves, own_parts, prefix_parts):
    d = [t.to(DEV) for t in (q, k, v, op, pp, ints(own), ints(prefixes), ints(groups), starts(rows))]
    dq, dk, dv, do, dp, ol, pl, gs, qs = d
    out, lse = torch.full(q.shape, 9.0, dtype=q.dtype, device=DEV), torch.full(q.shape[:2], 9.0, device=DEV)
    tokens, heads, dim = q.shape

    def cache(t):
        return t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)

    args = binding.SHARED_ATTENTION_ARGS.pack(*heads_of(dq), qs.data_ptr(), len(rows), tokens, *cache(dk), *cache(dv), k.shape[0], do.data_ptr(), do.stride(0), do.shape[1], ol.data_ptr(),
                                              dp.data_ptr(), dp.stride(0), dp.shape[1], pl.data_ptr(), gs.data_ptr(), len(prefixes), heads, k.shape[1], dim,
                                              {torch.bfloat16: 1, torch.float16: 2}[q.dtype], block, dim ** -0.5, *heads_of(out), lse.data_ptr())
    ws = torch.full(((own_parts + prefix_parts) * tokens * heads * (dim * 4 + 8) + 512,), 255, dtype=torch.uint8, device=DEV)
    rc = bb.load_library().bb_debug_shared_attention(args, halves, own_parts, prefix_parts, ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
    assert rc == 0
    torch.cuda.synchronize()
    return out, lse


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(6, 2, 128), (7, 1, 64)])
@pytest.mark.parametrize("block", [0, 1, 32])
@pytest.mark.parametrize("ql,kl", [([130, 0, 33, 1, 5], [130, 7, 300, 70, 2]), ([9, 60], [700, 33]), ([300], [641])])
def test_every_plan_of_packed_sequences(ql, kl, block, heads, kv_heads, dim, dtype):
    """One and two halves, the keys in one part up to more than there are tiles: each against the definition."""
    q, k, v = inputs(dim + block, ql, kl, heads, kv_heads, dim, dtype, 2.0)
    want = attention(q, k, v, ql, kl, block, dim ** -0.5)
    for halves in (1, 2):
        for parts in (1, 2, 3, 7, 32):
            check(*run_plan(q, k, v, ql, kl, block, halves, parts), want, q.dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(6, 2, 128), (7, 1, 64)])
@pytest.mark.parametrize("block", [0, 1])
@pytest.mark.parametrize("rows,own,prefixes,groups", BRANCHES + [([1, 2], [4500, 70], [5000], [0, 2]), ([50, 40], [100, 64], [4480, 130], [0, 1, 2])])
def test_every_plan_of_shared_prefixes(rows, own, prefixes, groups, block, heads, kv_heads, dim, dtype):
    """Prefixes taken by every branch, or by the group in one part and in many; own keys in one and many; a page that is not there among them."""
    q, k, v, op, pp = branches(dim + len(rows), rows, own, prefixes, heads, kv_heads, dim, dtype)
    pp = pp.clone()
    if prefixes[0] > 128:
        pp[0, 1] = k.shape[0]
    want = shared(q, rows, k, v, op, own, pp, prefixes, groups, block, dim ** -0.5)
    for halves in (1, 2):
        for own_parts, prefix_parts in ((1, 0), (3, 0), (32, 0), (1, 1), (2, 3), (1, 32)):
            check(*run_shared_plan(q, rows, k, v, op, own, pp, prefixes, groups, block, halves, own_parts, prefix_parts), want, q.dtype)


def many(n, seed):
    """Lengths of n sequences: tokens by ones and twos, some empty, a few of more than a tile, the first and the last among them."""
    g = torch.Generator().manual_seed(seed)
    lens = torch.randint(0, 3, (n,), generator=g)
    lens[torch.randint(0, n, (6,), generator=g)] = 131
    lens[0], lens[-1] = 140, 133
    return lens.tolist()


@pytest.mark.gpu
@pytest.mark.parametrize("heads,kv_heads", [(4, 2), (1, 1)])
@pytest.mark.parametrize("n", [64, 65, 72, 511, 513, 576, 577, 1100, 3000])
def test_many_sequences(n, heads, kv_heads):
    """More sequences than a wave has lanes, and than it looks over at once; in one part and in parts that are joined."""
    ql = many(n, n)
    kl = [m + 3 * (i % 2) for i, m in enumerate(ql)]
    q, k, v = inputs(n, ql, kl, heads, kv_heads, 64, "bf16", 2.0)
    want = attention(q, k, v, ql, kl, 1, 0.125)
    check(*run(q, k, v, ql, kl, 1, 0.125), want, q.dtype)
    for parts in (3, 7):
        check(*run_plan(q, k, v, ql, kl, 1, 1, parts), want, q.dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [64, 65, 127, 128, 129, 600, 4100])
def test_many_groups(n):
    """Groups of none to three branches, some branches outside the first and the last; prefixes once a group, and again by every branch."""
    g = torch.Generator().manual_seed(n)
    edges = [2]
    for c in torch.randint(0, 4, (n,), generator=g).tolist():
        edges.append(edges[-1] + c)
    branches_n = edges[-1] + 3
    rows = torch.randint(0, 3, (branches_n,), generator=g).tolist()
    own = torch.randint(1, 9, (branches_n,), generator=g).tolist()
    prefixes = torch.randint(0, 70, (n,), generator=g).tolist()
    q, k, v, op, pp = branches(n, rows, own, prefixes, 2, 1, 64, "bf16")
    want = shared(q, rows, k, v, op, own, pp, prefixes, edges, 1, 0.125)
    check(*run_shared(q, rows, k, v, op, own, pp, prefixes, edges, 1), want, q.dtype)
    for plan in ((1, 1, 0), (1, 1, 1), (2, 2, 0)):
        check(*run_shared_plan(q, rows, k, v, op, own, pp, prefixes, edges, 1, *plan), want, q.dtype)


@pytest.mark.gpu
def test_starts_of_many_that_do_not_ascend():
    """Garbage among thousands of starts, lengths and groups: nothing out of range is read or written, and what lies outside stays as it is."""
    g = torch.Generator().manual_seed(3)
    n, tokens = 2000, 300
    q, k = (torch.zeros(tokens, 2, 64, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    room = torch.full((tokens + 20, 2, 64), 9.0, dtype=torch.bfloat16, device=DEV)
    c = torch.zeros(4, 2, PAGE, 64, dtype=torch.bfloat16, device=DEV)

    def noise(*shape):
        return torch.randint(-2 ** 31, 2 ** 31 - 1, shape, generator=g).to(torch.int32)

    for qs in (noise(n + 1), noise(n + 1) % 400, torch.tensor([0, 2 ** 30] * (n // 2) + [0], dtype=torch.int32)):
        qs = qs.to(DEV)
        bb.attention(q, k, k, qs, noise(n + 1).to(DEV), block=1, out=room[10:-10])
        bb.shared_attention(q, qs, c, c, noise(n, 2).to(DEV), noise(n).to(DEV), noise(700, 3).to(DEV), noise(700).to(DEV), (noise(701) % 2500).to(DEV), block=1, out=room[10:-10])
        torch.cuda.synchronize()
        assert (room[:10] == 9).all() and (room[-10:] == 9).all()


@pytest.mark.gpu
@pytest.mark.parametrize("n,at", [(140, 75), (140, 66), (140, 69), (140, 94), (9, 4), (300, 250)])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf")])
def test_unseen_values_under_every_plan(bad, dim, n, at):
    """Garbage behind token `at` of a causal prompt, and one value that later rows do see, in tiles of few and of many rows."""
    q, k, v = inputs(7, [n], [n], 2, 1, dim, "bf16")
    k2, v2 = k.clone(), v.clone()
    k2[at:], v2[at:] = bad, bad
    v3 = v.clone()
    v3[at, 0, 3] = bad
    hit = torch.zeros(n, 2, dim, dtype=torch.bool)
    hit[at:, :, 3] = True
    for halves in (1, 2):
        for parts in (1, 3):
            out, _ = run_plan(q, k, v, [n], [n], 1, halves, parts)
            got, _ = run_plan(q, k2, v2, [n], [n], 1, halves, parts)
            assert torch.equal(got[:at], out[:at])
            got, _ = run_plan(q, k, v3, [n], [n], 1, halves, parts)
            assert torch.equal(got.cpu()[~hit], out.cpu()[~hit])
            assert torch.isnan(got.cpu()[hit]).all() if bad != bad else (got.cpu()[hit] == bad).all()


def test_c_entries_refuse_before_touching_a_device():
    """Every call below is refused on the host (the pointers are never followed)."""
    lib = bb.load_library()
    p = 1 << 20
    good = dict(q=p, qt=256, qh=64, k=2 * p, kt=128, kh=64, v=3 * p, vt=128, vh=64, qs=4 * p, ks=5 * p, n=2, qn=8, kn=9, heads=4, kv=2, dim=64, type=1, block=1, scale=0.1, o=6 * p,
                ot=256, oh=64, lse=0)

    def call(**kw):
        return lib.bb_attention(binding.ATTENTION_ARGS.pack(*dict(good, **kw).values()), None, 0, None)

    assert call(qn=0) == 0 and call(n=0) == 0 and lib.bb_attention(None, None, 0, None) == -1 and lib.bb_attention_workspace_bytes(None) == 0
    for bad in (dict(q=0), dict(q=p + 2), dict(qt=250), dict(qh=4), dict(k=0), dict(k=2 * p + 8), dict(kt=1 << 24), dict(v=0), dict(vh=65), dict(qs=0), dict(ks=0),
                dict(qs=4 * p + 1), dict(n=-1), dict(qn=-1), dict(kn=-1), dict(qn=1 << 31), dict(n=1 << 33), dict(heads=3), dict(heads=0), dict(kv=0), dict(heads=4096, kv=2), dict(dim=96),
                dict(dim=0), dict(type=0), dict(type=7), dict(block=-1), dict(block=1 << 31), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")),
                dict(scale=1e39), dict(scale=1e-60), dict(lse=p + 4), dict(lse=2 * p), dict(n=1 << 24), dict(heads=1024, kv=4, qn=(1 << 20) + 1), dict(heads=1024, kv=1024, qn=1 << 24), dict(o=0), dict(ot=128), dict(oh=0), dict(o=p), dict(o=2 * p), dict(o=3 * p + 128), dict(lse=6), dict(qt=-8), dict(qt=1 << 50)):
        assert call(**bad) == -1, bad
    args = binding.ATTENTION_ARGS.pack(*good.values())
    for halves, parts in ((0, 1), (3, 1), (1, 0), (1, 33), (1, -1)):
        assert lib.bb_debug_attention(args, halves, parts, None, 0, None) == -1
    assert lib.bb_debug_attention(args, 1, 2, None, 0, None) == -3
    # work that wants its keys in parts wants a workspace for them
    large = dict(good, qn=16, kn=100000, n=1, k=1 << 32, v=1 << 33)
    args = binding.ATTENTION_ARGS.pack(*large.values())
    need = lib.bb_attention_workspace_bytes(args)
    assert need > 0 and lib.bb_attention(args, None, 0, None) == -3 and lib.bb_attention(args, 256 * p, need - 1, None) == -3
    assert lib.bb_attention(args, None, need, None) == -1 and lib.bb_attention(args, 256 * p + 128, need, None) == -1
    good = dict(q=p, qt=256, qh=64, qs=4 * p, n=2, qn=8, k=16 * p, kp=8192, kh=4096, kt=64, v=32 * p, vp=8192, vh=4096, vt=64, pages=4, own=5 * p, old=3, ow=3, lens=6 * p, pre=7 * p, pld=3,
                pw=3, pl=8 * p, gs=9 * p, g=1, heads=4, kv=2, dim=64, type=1, block=1, scale=0.1, o=10 * p, ot=256, oh=64, lse=0)

    def call(**kw):
        return lib.bb_shared_attention(binding.SHARED_ATTENTION_ARGS.pack(*dict(good, **kw).values()), None, 0, None)

    assert call(qn=0) == 0 and call(n=0) == 0 and lib.bb_shared_attention(None, None, 0, None) == -1 and lib.bb_shared_attention_workspace_bytes(None) == 0
    for bad in (dict(q=0), dict(qs=0), dict(k=0), dict(k=16 * p + 2), dict(kp=100), dict(kt=1 << 24), dict(v=0), dict(pages=0), dict(pages=1 << 26), dict(own=0), dict(own=5 * p + 2),
                dict(old=-1), dict(ow=-1), dict(ow=1 << 33), dict(lens=0), dict(pre=0), dict(pld=-1, g=2), dict(pw=-1), dict(pl=0), dict(gs=0), dict(g=-1), dict(heads=5), dict(dim=32),
                dict(type=0), dict(block=-2), dict(scale=0.0), dict(o=0), dict(o=16 * p), dict(o=p), dict(ot=64), dict(o=10 * p + 2)):
        assert call(**bad) == -1, bad


def test_python_refuses_cpu_tensors():
    x = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(BBError, match="GPU"):
        bb.attention(x, x, x, ints([0, 3]))
    c = torch.zeros(2, 4, 64, 64, dtype=torch.bfloat16)
    with pytest.raises(BBError, match="GPU"):
        bb.shared_attention(x, ints([0, 3]), c, c, ints([[0]]), ints([3]))


@pytest.mark.gpu
def test_python_refuses_on_the_device():
    x = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device=DEV)
    s = ints([0, 3]).to(DEV)
    c = torch.zeros(2, 4, 64, 64, dtype=torch.bfloat16, device=DEV)
    op, ol = ints([[0]]).to(DEV), ints([3]).to(DEV)
    bad = [lambda: bb.attention(x.float(), x.float(), x.float(), s), lambda: bb.attention(x, x.half(), x, s), lambda: bb.attention(x, x[:, :3], x[:, :3], s), lambda: bb.attention(x, x, x[:2], s),
           lambda: bb.attention(x, x, x, s.long()), lambda: bb.attention(x, x, x, s, s[:1]), lambda: bb.attention(x, x, x, s, out=x), lambda: bb.attention(x, x, x, s, out=x[:2]),
           lambda: bb.attention(x, x, x, s, lse=torch.zeros(4, 3, device=DEV)), lambda: bb.attention(x[:, :, :32], x[:, :, :32], x[:, :, :32], s), lambda: bb.attention(x, x, x, s, block=-1),
           lambda: bb.attention(x, x, x, s, scale=0.0), lambda: bb.attention(x[0], x, x, s), lambda: bb.attention(x, x, x, s.cpu()),
           lambda: bb.shared_attention(x, s, c, c[:, :2], op, ol), lambda: bb.shared_attention(x, s, c[0], c[0], op, ol), lambda: bb.shared_attention(x, s, c, c, op[0], ol),
           lambda: bb.shared_attention(x, s, c, c, op, ol.long()), lambda: bb.shared_attention(x, s, c, c, op, ol, op, ol), lambda: bb.shared_attention(x, s, c, c, op, ol, group_starts=ints([0, 1]).to(DEV)),
           lambda: bb.shared_attention(x, s, c[:, :, :32], c[:, :, :32], op, ol), lambda: bb.shared_attention(x, s, c, c, op, ol, out=x),
           lambda: bb.attention(x, x, x, s[0]), lambda: bb.attention(x, x, x, s, s[0]), lambda: bb.attention(x, x, x, s, block=1.5), lambda: bb.attention(x, x, x, s, block=1 << 70),
           lambda: bb.attention(x, x, x, s, scale="1"), lambda: bb.shared_attention(x, s[0], c, c, op, ol), lambda: bb.shared_attention(x, s, c, c, op, ol[0]),
           lambda: bb.shared_attention(x, s, c, c, op, ol, op, ol, s[0]), lambda: bb.shared_attention(x, s, c, c, op, ol, block="1")]
    for i, call in enumerate(bad):
        with pytest.raises(BBError):
            call()
            print("not refused:", i)
