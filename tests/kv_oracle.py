"""What the tests of the operators around K,V compare with: the definitions in 64 bits on the CPU, and how far fp32 sums and 16-bit weights may be from them."""
import torch

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
DEV = "cuda:0"
PAGE = 64


def gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def rnd(seed, *shape, dtype="bf16", scale=1.0):
    return (torch.randn(*shape, generator=gen(seed)) * scale).to(TYPES[dtype])


def starts(lens):
    s = [0]
    for n in lens:
        s.append(s[-1] + n)
    return torch.tensor(s, dtype=torch.int32)


def ints(values):
    return torch.tensor(values, dtype=torch.int32)


def turned(x, positions, freqs, interleaved, magnitude=1.0):
    """(rotated rows in 64 bits, what the fp32 chain may be off before the last rounding).

    cos and sin: the angle in turns is rounded to fp32 below half a turn (2^-26 turns, 2 pi 2^-26 < 1.6 * 2^-24), sine and cosine are taken within 4 units of 2^-24,
    multiplied by the magnitude (2^-24), and by an element (2^-24); the sum is rounded once more (2^-24): below 9 * 2^-24 of (|a| + |b|) * magnitude, 2^-20 allows 16."""
    x, rot = x.double(), 2 * len(freqs)
    angle = positions.double()[:, None, None] * freqs
    c, s = torch.cos(angle) * magnitude, torch.sin(angle) * magnitude
    at = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    a, b = x[..., at[0]], x[..., at[1]]
    y, slack = x.clone(), torch.zeros_like(x)
    y[..., at[0]], y[..., at[1]] = a * c - b * s, a * s + b * c
    slack[..., at[0]] = slack[..., at[1]] = 2.0 ** -20 * (a.abs() + b.abs()) * abs(magnitude)
    return y, slack


def close(got, want, slack, dtype):
    """got is want, off by slack at most, rounded to its type (half a step; the smallest subnormal below that)."""
    t = torch.finfo(dtype)
    got = got.detach().cpu().double()
    assert got.shape == want.shape
    nan = torch.isnan(want)
    assert torch.equal(torch.isnan(got), nan), "NaN in other places"
    inf = torch.isinf(want)
    assert torch.equal(got[inf], want[inf]), "infinities in other places"
    ok = ~nan & ~inf
    room = (slack + t.eps / 2 * (want.abs() + slack) + t.smallest_normal * t.eps)[ok]
    off = (got - want).abs()[ok]
    assert (off <= room).all(), f"off by {(off / room).max().item():.3f} of what is allowed"


def limit(n, m, block, i):
    p = m - n + i
    return m if block == 0 else 0 if p < 0 else min(m, (p // block + 1) * block)


def rows_of(q, k, v, seen, dtype, scale):
    """Queries [n][dim] of one head on the first seen[i] of its keys: (out, log-sum-exp, slack of out, slack of lse), 64 bits.

    With weights p_j = exp(s_j - max) and A = sum p |v| / sum p: a weight is rounded to the operands' type (eps / 2 of it; fp16 below 2^-14: 2^-25), its score
    is a sum of D products in fp32 (D 2^-24 sum |q k|), then scaled, subtracted and exponentiated in fp32 (arguments t = s log2(e): 2^-23 |t| + 2^-21), the sums over m
    weights are fp32 (m 2^-24).  A relative error e of every weight moves the quotient by 2 e A at most, of the numerator alone by e A."""
    n, d = q.shape
    m = k.shape[0]
    out, slack = torch.zeros(n, d).double(), torch.zeros(n, d).double()
    lse, sl = torch.full((n,), float("-inf")).double(), torch.zeros(n).double()
    if n == 0 or m == 0:
        return out, lse, slack, sl
    see = torch.arange(m) < torch.as_tensor(seen)[:, None]
    s = torch.where(see, (q @ k.t()) * scale, float("-inf"))
    top = s.amax(1, keepdim=True)
    p = torch.where(see, torch.exp(s - torch.where(see.any(1, keepdim=True), top, 0.0)), 0.0)
    total = p.sum(1, keepdim=True)
    some = see.any(1)
    if torch.isfinite(v).all():
        o = p @ v
    else:
        o = torch.stack([torch.where((see[i] & (p[i] != 0))[:, None], p[i][:, None] * v, 0.0).sum(0) for i in range(n)])
    av = torch.nan_to_num(v.abs(), nan=0.0, posinf=0.0)
    mean = (p @ av) / total
    # (weights that are 0 in 64 bits too move nothing)
    score = torch.where(p > 0, d * 2.0 ** -24 * ((q.abs() @ k.abs().t()) * scale) + 2.0 ** -23 * 1.45 * (s.abs() + top.abs()), 0.0)
    e = score.amax(1, keepdim=True) + 2.0 ** -21 + m * 2.0 ** -24
    t = torch.finfo(dtype)
    room = (t.eps / 2) * mean + 2 * e * mean
    if dtype is torch.float16:
        room = room + 2.0 ** -25 * (see.double() @ av) / total
    l = (top + torch.log(total))[:, 0]
    out[some], slack[some], lse[some] = (o / total)[some], room[some], l[some]
    sl[some] = (e[:, 0] + 2.0 ** -22 * (l.abs() + top[:, 0].abs() + 1))[some]
    return out, lse, slack, sl


def attention(q, k, v, ql, kl, block, scale):
    """Packed sequences, row by row: (out, lse, slack of out, slack of lse); tokens outside every sequence NaN."""
    tokens, heads, dim = q.shape
    each = heads // k.shape[1]
    dtype = q.dtype
    q, k, v = q.double(), k.double(), v.double()
    out, so = torch.full((tokens, heads, dim), float("nan")).double(), torch.zeros(tokens, heads, dim).double()
    lse, sl = torch.full((tokens, heads), float("nan")).double(), torch.zeros(tokens, heads).double()
    q0 = k0 = 0
    for n, m in zip(ql, kl):
        seen = [limit(n, m, block, i) for i in range(n)]
        for h in range(heads):
            at, g = slice(q0, q0 + n), h // each
            out[at, h], lse[at, h], so[at, h], sl[at, h] = rows_of(q[at, h], k[k0:k0 + m, g], v[k0:k0 + m, g], seen, dtype, scale)
        q0, k0 = q0 + n, k0 + m
    return out, lse, so, sl


def of_pages(cache, table, n):
    """[tokens][kv heads][dim] of the first n tokens in a table's pages; those in pages that the cache has not are left out."""
    parts = []
    for j in range(0, n, PAGE):
        page = int(table[j // PAGE])
        if 0 <= page < cache.shape[0]:
            parts.append(cache[page].transpose(0, 1)[:min(PAGE, n - j)])
    return torch.cat(parts) if parts else cache.new_zeros(0, cache.shape[1], cache.shape[3])


def shared(q, rows, k_cache, v_cache, own_pages, own_lens, prefix_pages, prefix_lens, group_starts, block, scale):
    """As attention(), for branches over a paged cache (own pages all inside it)."""
    tokens, heads, dim = q.shape
    each = heads // k_cache.shape[1]
    dtype = q.dtype
    out, so = torch.full((tokens, heads, dim), float("nan")).double(), torch.zeros(tokens, heads, dim).double()
    lse, sl = torch.full((tokens, heads), float("nan")).double(), torch.zeros(tokens, heads).double()
    at = 0
    for b, n in enumerate(rows):
        k, v = (of_pages(c, own_pages[b], own_lens[b]).double() for c in (k_cache, v_cache))
        kp = vp = k[:0]
        for g in range(len(prefix_lens)):
            if group_starts[g] <= b < group_starts[g + 1]:
                kp, vp = (of_pages(c, prefix_pages[g], prefix_lens[g]).double() for c in (k_cache, v_cache))
                break
        seen = [kp.shape[0] + limit(n, own_lens[b], block, i) for i in range(n)]
        ka, va = torch.cat((kp, k)), torch.cat((vp, v))
        for h in range(heads):
            rows_at, g = slice(at, at + n), h // each
            out[rows_at, h], lse[rows_at, h], so[rows_at, h], sl[rows_at, h] = rows_of(q[rows_at, h].double(), ka[:, g], va[:, g], seen, dtype, scale)
        at += n
    return out, lse, so, sl


def check(got, lse, want, dtype):
    """Outputs against what attention() or shared() gives; tokens that are no query's are not compared."""
    out, l, so, sl = want
    mine = ~torch.isnan(l)
    close(got.cpu()[mine], out[mine], so[mine], dtype)
    if lse is not None:
        close(lse.cpu()[mine], l[mine], sl[mine], torch.float32)
