"""Attention where fp32 exponents run short of places: finite scores from thousands to 2^100, with scores that are exact in fp32, so that what the softmax has to give is known whatever their size."""
import pytest
import torch

import paper_2605_29233_amd as bb
from kv_oracle import DEV, PAGE, TYPES, close, gen, ints, rnd, starts
from test_attention_ops import run_plan, run_shared_plan

KEYS = 200


def exact_scores(p, scale, order, dtype, dim, n, seed):
    """(q [n][1][dim], k [KEYS][1][dim], s in 64 bits [n][KEYS]): s = f (2^p + 2^c j) scale with whole numbers j below 128 and c = max(p - 23, 0), so that s / scale needs no more than fp32's 24 bits; in
    products of powers of two, 16 of 2^(p - 4) and, in another sixteen of a head's elements, 2^c by j.  f is a row's own: 1, -1, 0 and smaller powers of two."""
    c = max(p - 23, 0)
    a = (p - 4) // 2
    j = torch.randint(0, 128, (KEYS,), generator=gen(seed)).double()
    if order:
        j = j.sort(descending=order == "falling").values
    f = torch.tensor([1.0, -1.0, 0.0, 2.0 ** -4, 2.0 ** -9, -2.0 ** -6, 1.0])[torch.arange(n) % 7].double()
    q, k = torch.zeros(n, dim).double(), torch.zeros(KEYS, dim).double()
    q[:, :16], q[:, 40] = 2.0 ** a * f[:, None], 2.0 ** c * f
    k[:, :16], k[:, 40] = 2.0 ** (p - 4 - a), j
    t = TYPES[dtype]
    s = f[:, None] * (2.0 ** p + 2.0 ** c * j) * scale
    assert torch.equal((s / scale).float().double() * scale, s) and torch.equal((q @ k.t()) * scale, s)
    assert torch.equal(q.to(t).double(), q) and torch.equal(k.to(t).double(), k)
    return q.to(t)[:, None], k.to(t)[:, None], s


def weighed(s, v, dtype):
    """softmax(s) v and its logarithm, and what they may be off by.  Scores are exact.  A weight's exponent is the difference to the largest, rounded to fp32 and multiplied by a scale that is rounded twice
    (2^-22 of it, and no weight is left 104 below), or the difference of products rounded to 2^-24 of scores of up to 1024 / log2(e) at most, twice where parts are joined: below 2^-22 * 710 and 2^-21 of its
    own; weights are rounded to the operands' type, fp16 below 2^-14 to 2^-25; sums of KEYS terms in fp32."""
    t = torch.finfo(dtype)
    top = s.amax(1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(1, keepdim=True)
    mean = (p @ v.abs()) / total
    e = 2.0 ** -22 * 104 + 2.0 ** -22 * top.abs().clamp(max=710) + 2.0 ** -21 + KEYS * 2.0 ** -24
    slack = (t.eps / 2 + 2 * e) * mean
    if dtype is torch.float16:
        slack = slack + 2.0 ** -25 * v.abs().sum(0) / total
    lse = (top + torch.log(total))[:, 0]
    return p @ v / total, slack, lse, e[:, 0] + 2.0 ** -22 * (lse.abs() + top[:, 0].abs() + 1)


SIZES = [(14, 0.125), (14, 1.0), (20, 0.125), (27, 0.125), (30, 0.125), (30, 2.0 ** -6), (32, 0.125), (34, 0.125), (34, 1.0)]


def check(out, lse, want, dtype):
    close(out[:, 0], want[0], want[1], dtype)
    close(lse[:, 0], want[2], want[3], torch.float32)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,p,scale", [(d, *x) for d in ("bf16", "fp16") for x in SIZES] + [("bf16", 60, 0.125), ("bf16", 100, 0.125)])
@pytest.mark.parametrize("order", ["", "rising", "falling"])
@pytest.mark.parametrize("dim", [64, 128])
def test_large_scores(dim, order, dtype, p, scale):
    """Largest keys share by what lies between them, however large they are: few rows and many, under every kind of plan."""
    v = rnd(2, KEYS, 1, dim, dtype=dtype)
    for n in (9, 70):
        q, k, s = exact_scores(p, scale, order, dtype, dim, n, p)
        want = weighed(s, v[:, 0].double(), TYPES[dtype])
        lse = torch.zeros(n, 1, device=DEV)
        out = bb.attention(q.to(DEV), k.to(DEV), v.to(DEV), starts([n]).to(DEV), starts([KEYS]).to(DEV), scale=scale, lse=lse)
        check(out, lse, want, v.dtype)
        if scale == 0.125 and dim == 64:
            for halves in (1, 2):
                for parts in (1, 3):
                    check(*run_plan(q, k, v, [n], [KEYS], 0, halves, parts), want, v.dtype)
            cache = [torch.cat((x, x[:56])).view(4, PAGE, 1, dim).transpose(1, 2).contiguous() for x in (k, v)]
            for plan in ((1, 1, 0), (2, 2, 0), (1, 1, 2)):        # two pages shared, 72 keys of the branch's own
                got = run_shared_plan(q, [n], *cache, ints([[2, 3]]), [KEYS - 128], ints([[0, 1]]), [128], [0, 1], 0, *plan)
                check(*got, want, v.dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n", [7, 60])
def test_large_operands_pick_the_largest(n, dtype):
    """Elements of 6000 to 9000 of either sign: scores of some 10^8, of which one leads by far more than sums in fp32 can be off by: its value, and nothing else."""
    dim, seen = 64, 0
    for seed in range(20):
        q, k = ((torch.rand(m, dim, generator=gen(10 * seed + i)) * 3000 + 6000) * (torch.randint(0, 2, (m, dim), generator=gen(10 * seed + i + 2)) * 2 - 1) for i, m in ((0, n), (1, KEYS)))
        q, k = q.to(TYPES[dtype]), k.to(TYPES[dtype])
        v = rnd(seed, KEYS, 1, dim, dtype=dtype)
        s = q.double() @ k.double().t()
        best = s.topk(2, dim=1)
        off = dim * 2.0 ** -24 * (q.double().abs() @ k.double().abs().t()).amax(1)
        clear = (best.values[:, 0] - best.values[:, 1] - 2 * off) * 0.125 > 110       # (e^-104 is below fp32's smallest)
        seen += int(clear.sum())
        lse = torch.zeros(n, 1, device=DEV)
        out = bb.attention(q[:, None].to(DEV), k[:, None].to(DEV), v.to(DEV), starts([n]).to(DEV), starts([KEYS]).to(DEV), lse=lse)
        assert torch.isfinite(out).all()
        assert torch.equal(out.cpu()[clear], v[best.indices[:, 0]][clear])
        assert ((lse.cpu()[:, 0].double() - best.values[:, 0] * 0.125).abs() <= off * 0.125 + 2.0 ** -21 * best.values[:, 0].abs())[clear].all()
    assert seen > 10 * n


@pytest.mark.gpu
@pytest.mark.parametrize("n", [5, 60])
def test_values_up_to_the_documented_limit(n):
    """bf16 values just below 2^120 / keys, on scores that the running maximum does not follow (weights of 2^7.93): their mean, not an infinity."""
    keys, dim, t = 256, 64, torch.bfloat16
    q, k = torch.zeros(n, 1, dim, dtype=t), torch.zeros(keys, 1, dim, dtype=t)
    q[:, :, 0], k[64:, :, 0] = 1, 44                    # (44 / 8 log2(e) = 7.93)
    v = (rnd(1, keys, 1, dim).double().abs().clamp(0.25, 1.0) * 2.0 ** 112 * (1 - 2.0 ** -8)).to(t)
    assert float(v.double().max()) < 2.0 ** 120 / keys
    s = (q[:, 0].double() @ k[:, 0].double().t()) * 0.125
    want = weighed(s, v[:, 0].double(), t)
    for halves in (1, 2):
        for parts in (1, 2, 4):
            got = run_plan(q, k, v, [n], [keys], 0, halves, parts)
            check(*got, want, t)


@pytest.mark.gpu
@pytest.mark.parametrize("n", [5, 60])
@pytest.mark.parametrize("rise", [680, 1112, 2048])
def test_large_values_that_later_scores_leave_behind(n, rise):
    """64 values of 2^113 (below 2^120 / keys), then one key whose score is 2^122 to 2^369 of weight higher, of value 2^-20: nothing of the first is left but what its weight gives (at 2^-126, 2^-7 of them would)."""
    keys, dim, t = 65, 64, torch.bfloat16
    q, k = torch.zeros(n, 1, dim, dtype=t), torch.zeros(keys, 1, dim, dtype=t)
    q[:, :, 0], k[64, :, 0] = 1, rise
    v = torch.full((keys, 1, dim), 2.0 ** -20, dtype=t)
    v[:64] = 2.0 ** 113
    s = (q[:, 0].double() @ k[:, 0].double().t()) * 0.125
    want = weighed(s, v[:, 0].double(), t)
    for halves in (1, 2):
        for parts in (1, 2):
            check(*run_plan(q, k, v, [n], [keys], 0, halves, parts), want, t)
    v[3, 0, 7] = float("inf")
    out, _ = run_plan(q, k, v, [n], [keys], 0, 1, 1)
    assert not torch.isfinite(out[:, :, 7]).any() and torch.isfinite(out[:, :, :7]).all()
