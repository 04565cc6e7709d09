"""Performance cases of the operators around K,V: rotary positions (with the rows' way into a paged cache), attention over packed
prompts, and attention of branches that share a prefix, over a paged cache.

  rope              pairs (x_a, x_b) of a head turned by position * f_j: (x_a cos - x_b sin, x_a sin + x_b cos); pair j is elements
                    (j, j + rot/2) ("half") or (2j, 2j + 1) ("interleaved") of the head's first `rot`, the rest stays as it is
  rope_append       the same, with the turned keys and the values written to slots (page * 64 + place in the page) of a paged cache
  attention         per packed sequence of n queries and m keys: softmax(scale q k^T) v over the keys that a query sees.  Query i stands
                    at key position p = m - n + i and sees all keys (block 0), or those before the end of its block, j < (p / block + 1) *
                    block (block 1: causal); one that sees none gives 0, and -inf as its log-sum-exp
  shared_attention  per branch of n queries: the same over the group's prefix, which all its branches' queries see whole, and the branch's own
                    keys, seen as above; both in pages of 64 tokens, [page][kv head][token][head_dim]

Heads and widths are those of `workload/configs.py` (4 x 64; 32 x 128; 28 on 4 x 128), lengths those of its workloads and generic ones.
"""
import math

import torch

own = False

_DEVICE = "cuda:0"
_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
_PAGE = 64
_BASE = 10000.0
_TRAINED, _LOW, _HIGH = 4096, 1.0, 4.0          # of the frequencies scaled for long contexts
_SCORES = 1 << 28                               # scores that the plain forms hold at once


def _rope(name, tokens, heads, kv_heads, dim, dtype, rot=None, interleaved=False, start=0, factor=1.0, cache=True):
    return {"name": name, "op": "rope_append" if cache else "rope", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "dim": dim, "type": dtype,
            "rot": rot or dim, "interleaved": interleaved, "start": start, "factor": factor}


def _prompt(name, q_lens, heads, kv_heads, dim, dtype, block, k_lens=None, lse=False):
    return {"name": name, "op": "attention", "q_lens": _text(q_lens), "k_lens": _text(k_lens or q_lens), "heads": heads, "kv_heads": kv_heads,
            "dim": dim, "type": dtype, "block": block, "lse": lse}


def _shared(name, rows, own_lens, prefixes, heads, kv_heads, dim, dtype, block, lse=False):
    """rows, own_lens: of every branch, the groups' branches one after the other, equally many a group."""
    return {"name": name, "op": "shared_attention", "rows": _text(rows), "own": _text(own_lens), "prefixes": _text(prefixes), "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "type": dtype, "block": block, "lse": lse}


def _text(values):
    return ",".join(map(str, values))


def _ints(text):
    return [int(x) for x in text.split(",")]


def listed():
    return [
        # one token on its way into the cache: latency
        _rope("rope_token", 1, 32, 32, 128, "bf16", start=700),
        # the packed rows of a block step, grouped heads; neighbouring elements are the pairs, half of the head is turned
        _rope("rope_step", 112, 28, 4, 128, "fp16", rot=64, interleaved=True, start=1024),
        # fp32 heads of the tiny model, an odd number of tokens, no cache
        _rope("rope_odd", 1013, 4, 4, 64, "fp32", rot=48, cache=False),
        # a refresh of long rows far beyond the trained context, frequencies scaled
        _rope("rope_far", 20480, 32, 32, 128, "bf16", start=100000, factor=16.0),
        # the tiny model's prompt: latency
        _prompt("prompt_tiny", [64], 4, 4, 64, "bf16", 1),
        # a request's initial forward, every token seen by every other
        _prompt("prompt_init", [768], 32, 32, 128, "bf16", 0),
        # sixteen prompts of different lengths packed, blocks of 32 that see what is before them and themselves
        _prompt("prompt_ragged", [258, 1008, 511, 640, 333, 897, 770, 260, 1, 965, 402, 575, 689, 316, 823, 448], 28, 4, 128, "fp16", 32, lse=True),
        # 500 new tokens of three conversations behind long contexts
        _prompt("prompt_context", [211, 37, 252], 28, 4, 128, "bf16", 1, k_lens=[5120, 2049, 8190]),
        # a whole long prompt, causal
        _prompt("prompt_long", [16384], 32, 32, 128, "bf16", 1),
        # a block step of the headline workload: four branches, 120 rows, windows in the middle of the generation
        _shared("shared_step", [8, 16, 32, 64], [104, 112, 128, 128], [512], 32, 32, 128, "bf16", 0),
        # its long form: 240 rows against 4096 shared and up to 1024 own tokens
        _shared("shared_long", [16, 32, 64, 128], [400, 417, 512, 640], [4096], 32, 32, 128, "fp16", 0, lse=True),
        # sixty-four continuations of one long document, a token each
        _shared("shared_tokens", [1] * 64, [(i * 37) % 501 + 1 for i in range(64)], [16381], 28, 4, 128, "bf16", 1),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _size(rng, lo, hi, unit):
    """Over the logarithm of the range; half of them multiples of `unit`."""
    v = _log(rng, lo, hi)
    return max(lo, v // unit * unit) if rng.random() < 0.5 else v


_HEADS = [(4, 4, 64), (32, 32, 128), (28, 4, 128), (16, 2, 64), (5, 1, 128)]


def draw(rng):
    op = rng.choice(["rope", "rope_append", "attention", "attention", "shared_attention", "shared_attention"])
    heads, kv_heads, dim = rng.choice(_HEADS)
    if op.startswith("rope"):
        dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        rot = rng.choice([dim, dim, dim // 2, 2 * rng.randint(1, dim // 2)])
        while True:
            tokens = _size(rng, 1, 24576, 16)
            if tokens * (heads + 2 * kv_heads) * dim * _BYTES[dtype] <= 20480 * 96 * 128 * 2:
                break
        c = _rope("", tokens, heads, kv_heads, dim, dtype, rot, rng.random() < 0.5, _log(rng, 1, 1 << 20), rng.choice([1.0, 1.0, 4.0, 32.0]), op == "rope_append")
    elif op == "attention":
        while True:
            n = _log(rng, 1, 32)
            top = _size(rng, 1, 16384, 64)
            q = [rng.randint((top + 3) // 4, top) for _ in range(n)]
            k = [x + _log(rng, 1, 8192) for x in q] if rng.random() < 0.3 else q
            if sum(a * b for a, b in zip(q, k)) * heads * dim <= 16384 * 16384 * 32 * 128 // 2 and max(k) <= 16384:
                break
        c = _prompt("", q, heads, kv_heads, dim, rng.choice(["bf16", "fp16"]), rng.choice([0, 1, 1, 32, rng.randint(2, 200)]), k, rng.random() < 0.3)
    else:
        while True:
            groups, branches = _log(rng, 1, 16), _log(rng, 1, 64)
            n = groups * branches
            most = rng.choice([1, 1, _log(rng, 2, 128)])
            rows = [rng.randint((most + 3) // 4, most) for _ in range(n)]
            top = _log(rng, 1, 2048)
            lens = [r + rng.randint(0, top) for r in rows]
            prefixes = [_size(rng, 1, 32768, _PAGE) for _ in range(groups)]
            pairs = sum(r * (lens[i] + prefixes[i // branches]) for i, r in enumerate(rows))
            if n <= 256 and pairs * heads * dim <= 240 * 4800 * 32 * 128 and (sum(lens) + sum(prefixes)) * kv_heads * dim <= 6000 * 32 * 128:
                break
        c = _shared("", rows, lens, prefixes, heads, kv_heads, dim, rng.choice(["bf16", "fp16"]), rng.choice([0, 0, 1, 32]), rng.random() < 0.3)
    del c["name"]
    return c


def _gen(seed):
    return torch.Generator(device=_DEVICE).manual_seed(seed)


def _projected(g, rows, heads, kv_heads, dim, dtype):
    """Queries, keys and values of rows as the three column ranges of one projection's output: normal values, a few channels of queries and
    keys larger, as trained models have them, so that scores spread over some ten units."""
    x = torch.randn(rows, heads + 2 * kv_heads, dim, generator=g, device=_DEVICE)
    big = torch.where(torch.rand(heads + kv_heads, dim, generator=g, device=_DEVICE) < 1 / 32, 3.0, 1.0)
    x[:, :heads + kv_heads] *= big
    x = x.to(dtype)
    return x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]


def _starts(lens):
    s = [0]
    for n in lens:
        s.append(s[-1] + n)
    return s


def _device_ints(values):
    return torch.tensor(values, dtype=torch.int32, device=_DEVICE)


def _frequencies(case):
    """f_j = base^(-2j / rot); with a factor, those that turn less than `low` times over the trained context are divided by it, those that turn more
    than `high` times stay, linear between."""
    f = _BASE ** (-torch.arange(0, case["rot"], 2, dtype=torch.float64) / case["rot"])
    if case["factor"] != 1:
        keep = ((_TRAINED * f / (2 * math.pi) - _LOW) / (_HIGH - _LOW)).clamp(0, 1)
        f = f * keep + f / case["factor"] * (1 - keep)
    return f.to(_DEVICE)


def _magnitude(case):
    return 0.1 * math.log(case["factor"]) + 1.0


def _tables(g, *lens):
    """Pages of 64 tokens for every length, in no order: (number of pages, a table per list of lengths, with a row per length)."""
    need = [[-(-n // _PAGE) for n in x] for x in lens]
    pages = sum(map(sum, need))
    order = torch.randperm(pages, generator=g, device=_DEVICE).int()
    tables, at = [], 0
    for x in need:
        t = torch.full((len(x), max(x)), -1, dtype=torch.int32, device=_DEVICE)
        for i, n in enumerate(x):
            t[i, :n] = order[at:at + n]
            at += n
        tables.append(t)
    return (pages, *tables)


def _inputs(case, seed):
    g, t = _gen(seed), _TYPES[case["type"]]
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    if case["op"] in ("rope", "rope_append"):
        n = case["tokens"]
        q, k, v = _projected(g, n, heads, kv_heads, dim, t)
        s = {"q": q, "k": k, "v": v, "positions": torch.arange(case["start"], case["start"] + n, dtype=torch.int32, device=_DEVICE)}
        if case["op"] == "rope_append":
            pages, table = _tables(g, [n])
            s["pages"] = pages
            s["slots"] = (table[0, :, None] * _PAGE + torch.arange(_PAGE, dtype=torch.int32, device=_DEVICE)).view(-1)[:n].contiguous()
        return s
    if case["op"] == "attention":
        ql, kl = _ints(case["q_lens"]), _ints(case["k_lens"])
        q, k, v = _projected(g, sum(ql), heads, kv_heads, dim, t)
        s = {"ql": ql, "kl": kl, "q": q, "k": k, "v": v, "q_starts": _device_ints(_starts(ql)), "k_starts": None}
        if ql != kl:
            _, s["k"], s["v"] = _projected(g, sum(kl), heads, kv_heads, dim, t)
            s["k_starts"] = _device_ints(_starts(kl))
        return s
    rows, lens, prefixes = _ints(case["rows"]), _ints(case["own"]), _ints(case["prefixes"])
    pages, prefix_pages, own_pages = _tables(g, prefixes, lens)
    _, k, v = _projected(g, pages * _PAGE, 1, kv_heads, dim, t)
    cache = [x.reshape(pages, _PAGE, kv_heads, dim).transpose(1, 2).contiguous() for x in (k, v)]
    groups, branches = len(prefixes), len(rows) // len(prefixes)
    return {"rows": rows, "lens": lens, "prefixes": prefixes, "q": _projected(g, sum(rows), heads, kv_heads, dim, t)[0], "k_cache": cache[0], "v_cache": cache[1],
            "q_starts": _device_ints(_starts(rows)), "own_pages": own_pages, "own_lens": _device_ints(lens),
            "prefix_pages": prefix_pages, "prefix_lens": _device_ints(prefixes),
            "group_starts": _device_ints([i * branches for i in range(groups + 1)])}


def prepare(case, seed):
    s, t = _inputs(case, seed), _TYPES[case["type"]]
    s.update(case={k: v for k, v in case.items() if k != "name"}, type=t)
    if case["op"] in ("rope", "rope_append"):
        s["freqs"], s["magnitude"] = _frequencies(case), _magnitude(case)
        s["q_out"] = torch.empty(s["q"].shape, dtype=t, device=_DEVICE)
        if case["op"] == "rope":
            s["k_out"] = torch.empty(s["k"].shape, dtype=t, device=_DEVICE)
        else:
            s["k_cache"], s["v_cache"] = (torch.zeros(s["pages"], case["kv_heads"], _PAGE, case["dim"], dtype=t, device=_DEVICE) for _ in range(2))
        return s
    s["out"] = torch.empty(s["q"].shape, dtype=t, device=_DEVICE)
    s["lse"] = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=_DEVICE) if case["lse"] else None
    return s


# ---- the plain forms ------------------------------------------------------------------------------------------------------------------

def _turned(x, s):
    """Rows of heads turned by their positions: angles in 64 bits, the rest in 32."""
    rot, inter = s["case"]["rot"], s["case"]["interleaved"]
    angle = s["positions"].double()[:, None] * s["freqs"]
    c, n = ((f(angle) * s["magnitude"]).float()[:, None] for f in (torch.cos, torch.sin))
    y = x.float()
    a, b = (y[..., 0:rot:2], y[..., 1:rot:2]) if inter else (y[..., :rot // 2], y[..., rot // 2:rot])
    a, b = a * c - b * n, a * n + b * c
    turned = torch.stack((a, b), -1).flatten(-2) if inter else torch.cat((a, b), -1)
    return torch.cat((turned, y[..., rot:]), -1).to(s["type"])


def _seen(n, m, block, at):
    """Of queries at .. of n, how many of the m keys each sees."""
    if block == 0:
        return torch.full((len(at),), m, dtype=torch.long, device=_DEVICE)
    p = torch.arange(at.start, at.stop, device=_DEVICE) + (m - n)
    return ((torch.div(p, block, rounding_mode="floor") + 1) * block).clamp(0, m)


def _heads_first(x, kv_heads):
    """[tokens][heads][dim] -> fp32 [kv head][tokens * heads of it][dim]."""
    n, h, d = x.shape
    return x.float().view(n, kv_heads, h // kv_heads, d).transpose(0, 1).reshape(kv_heads, -1, d)


def _scores(q, k, scale, seen, each):
    """q [kv head][rows * each][dim], k [kv head][keys][dim], keys seen per row -> scores, -inf where unseen."""
    x = torch.bmm(q, k.transpose(1, 2).contiguous()) * scale
    hidden = torch.arange(k.shape[1], device=_DEVICE) >= seen.repeat_interleave(each)[:, None]
    return x.masked_fill_(hidden, float("-inf"))


def _weighed(x, v, lse):
    """Softmax over the last axis of x, rows without a key zero, times v; x is used up."""
    top = x.amax(2, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = x.sub_(top).exp_()
    total = p.sum(2, keepdim=True)
    out = torch.bmm(p, v) / torch.where(total == 0, torch.ones_like(total), total)
    return out, (total.log() + top)[..., 0] if lse else None


def _tokens_first(x, n, kv_heads):
    """[kv head][rows * each](...) -> [rows][heads](...)."""
    return x.view(kv_heads, n, -1, *x.shape[2:]).transpose(0, 1).reshape(n, -1, *x.shape[2:])


def _plain_attention(s):
    c, scale = s["case"], s["q"].shape[2] ** -0.5
    kv_heads = c["kv_heads"]
    out, lse, q0, k0 = [], [], 0, 0
    for n, m in zip(s["ql"], s["kl"]):
        k, v = (_heads_first(s[x][k0:k0 + m], kv_heads) for x in "kv")
        step = max(1, _SCORES // (m * c["heads"]))
        for r in range(0, n, step):
            at = range(r, min(r + step, n))
            x = _scores(_heads_first(s["q"][q0 + at.start:q0 + at.stop], kv_heads), k, scale, _seen(n, m, c["block"], at), c["heads"] // kv_heads)
            o, l = _weighed(x, v, c["lse"])
            out.append(_tokens_first(o, len(at), kv_heads).to(s["type"]))
            if c["lse"]:
                lse.append(_tokens_first(l, len(at), kv_heads))
        q0, k0 = q0 + n, k0 + m
    return torch.cat(out), torch.cat(lse) if c["lse"] else None


def _paged(cache, table, n):
    """fp32 [kv head][n][dim] of the pages that a table's row names."""
    pages = table[:-(-n // _PAGE)].long()
    return cache[pages].float().transpose(0, 1).reshape(cache.shape[1], -1, cache.shape[3])[:, :n]


def _plain_shared(s):
    c, scale, kv_heads = s["case"], s["q"].shape[2] ** -0.5, s["case"]["kv_heads"]
    each, branches = c["heads"] // kv_heads, len(s["rows"]) // len(s["prefixes"])
    out, lse, at = [], [], 0
    for b, (n, m) in enumerate(zip(s["rows"], s["lens"])):
        if b % branches == 0:
            g = b // branches
            prefix = s["prefixes"][g]
            kp, vp = (_paged(s[x], s["prefix_pages"][g], prefix) for x in ("k_cache", "v_cache"))
        k, v = (torch.cat((p, _paged(s[x], s["own_pages"][b], m)), 1) for x, p in (("k_cache", kp), ("v_cache", vp)))
        x = _scores(_heads_first(s["q"][at:at + n], kv_heads), k, scale, prefix + _seen(n, m, c["block"], range(n)), each)
        o, l = _weighed(x, v, c["lse"])
        out.append(_tokens_first(o, n, kv_heads).to(s["type"]))
        if c["lse"]:
            lse.append(_tokens_first(l, n, kv_heads))
        at += n
    return torch.cat(out), torch.cat(lse) if c["lse"] else None


def _plain(s):
    op = s["case"]["op"]
    if op == "rope":
        return {"q": _turned(s["q"], s), "k": _turned(s["k"], s)}
    if op == "rope_append":
        page, place = (s["slots"] // _PAGE).long(), (s["slots"] % _PAGE).long()
        s["k_cache"][page, :, place] = _turned(s["k"], s)
        s["v_cache"][page, :, place] = s["v"]
        return {"q": _turned(s["q"], s), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    out, lse = _plain_attention(s) if op == "attention" else _plain_shared(s)
    return {"out": out} if lse is None else {"out": out, "lse": lse}


# ---- the framework's calls ------------------------------------------------------------------------------------------------------------

def _own(s):
    import paper_2605_29233_amd as bb
    c = s["case"]
    op = c["op"]
    if op == "rope":
        bb.rope(s["q"], s["k"], s["positions"], s["freqs"], interleaved=c["interleaved"], magnitude=s["magnitude"], q_out=s["q_out"], k_out=s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if op == "rope_append":
        bb.rope_append(s["q"], s["k"], s["v"], s["positions"], s["freqs"], s["k_cache"], s["v_cache"], s["slots"], interleaved=c["interleaved"],
                       magnitude=s["magnitude"], q_out=s["q_out"])
        return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if op == "attention":
        bb.attention(s["q"], s["k"], s["v"], s["q_starts"], s["k_starts"], block=c["block"], out=s["out"], lse=s["lse"])
    else:
        bb.shared_attention(s["q"], s["q_starts"], s["k_cache"], s["v_cache"], s["own_pages"], s["own_lens"], s["prefix_pages"], s["prefix_lens"],
                            s["group_starts"], block=c["block"], out=s["out"], lse=s["lse"])
    return {"out": s["out"]} if s["lse"] is None else {"out": s["out"], "lse": s["lse"]}


def run(state):
    return _own(state) if own else _plain(state)


def _pairs(n, m, block):
    """Query-key pairs of n queries on m keys."""
    if block == 0:
        return n * m
    return sum(max(0, min(m, ((m - n + i) // block + 1) * block)) for i in range(n))


def work(case):
    b, dim, heads, kv_heads = _BYTES[case["type"]], case["dim"], case["heads"], case["kv_heads"]
    if case["op"] in ("rope", "rope_append"):
        append = case["op"] == "rope_append"
        e = case["tokens"] * (heads + kv_heads) * dim
        return {"bytes": 2 * b * (e + append * case["tokens"] * kv_heads * dim) + case["tokens"] * (8 if append else 4) + case["rot"] * 4,
                "flops": 3 * case["tokens"] * (heads + kv_heads) * case["rot"]}
    if case["op"] == "attention":
        ql, kl = _ints(case["q_lens"]), _ints(case["k_lens"])
        rows, keys, pairs = sum(ql), sum(kl), sum(_pairs(n, m, case["block"]) for n, m in zip(ql, kl))
    else:
        rl, ol, pl = _ints(case["rows"]), _ints(case["own"]), _ints(case["prefixes"])
        each = len(rl) // len(pl)
        rows, keys = sum(rl), sum(ol) + sum(pl)
        pairs = sum(_pairs(n, m, case["block"]) + n * pl[i // each] for i, (n, m) in enumerate(zip(rl, ol)))
    return {"bytes": 2 * b * dim * (rows * heads + keys * kv_heads) + (4 * rows * heads if case["lse"] else 0), "flops": 4 * dim * heads * pairs}


# ---- the definitions in 64 bits -------------------------------------------------------------------------------------------------------

def _exact_rope(case, s):
    t = torch.complex128
    f = torch.tensor([math.exp(-2 * j / case["rot"] * math.log(_BASE)) for j in range(case["rot"] // 2)], dtype=torch.float64)
    if case["factor"] != 1:
        for j in range(len(f)):
            turns = _TRAINED * float(f[j]) / (2 * math.pi)
            part = min(1.0, max(0.0, (turns - _LOW) / (_HIGH - _LOW)))
            f[j] *= part + (1 - part) / case["factor"]
    angle = torch.outer(s["positions"].double(), f.to(_DEVICE))
    turn = torch.polar(torch.full_like(angle, _magnitude(case)), angle)[:, None]

    def turned(x):
        x, rot = x.double(), case["rot"]
        shape = (*x.shape[:2], rot // 2, 2)
        first = x[..., :rot].reshape(shape) if case["interleaved"] else x[..., :rot].reshape(*x.shape[:2], 2, rot // 2).transpose(2, 3)
        z = torch.view_as_real(torch.view_as_complex(first.contiguous()).to(t) * turn)
        z = z if case["interleaved"] else z.transpose(2, 3)
        return torch.cat((z.reshape(*x.shape[:2], rot), x[..., rot:]), 2)

    if case["op"] == "rope":
        return {"q": turned(s["q"]), "k": turned(s["k"])}
    out = {"q": turned(s["q"])}
    for name, x in (("k_cache", turned(s["k"])), ("v_cache", s["v"].double())):
        flat = torch.zeros(s["pages"] * _PAGE, *x.shape[1:], dtype=torch.float64, device=_DEVICE)
        flat.index_copy_(0, s["slots"].long(), x)
        out[name] = flat.view(s["pages"], _PAGE, *x.shape[1:]).permute(0, 2, 1, 3).contiguous()
    return out


def _exact_head(q, k, v, limits):
    """One head's queries on its keys, those below each query's limit, a piece of the queries at a time."""
    out, lse = torch.zeros_like(q), torch.full((len(q),), float("-inf"), dtype=torch.float64, device=_DEVICE)
    step = max(1, (1 << 26) // max(1, len(k)))
    column = torch.arange(len(k), device=_DEVICE)
    kt = k.t().contiguous()
    for r in range(0, len(q), step):
        limit = limits[r:r + step]
        x = torch.mm(q[r:r + step], kt).div_(math.sqrt(q.shape[1]))
        x = torch.where(column < limit[:, None], x, float("-inf"))
        l = torch.logsumexp(x, 1)
        lse[r:r + step] = l
        p = torch.where(limit[:, None] > 0, torch.exp(x - l[:, None]), 0.0)
        out[r:r + step] = torch.mm(p, v)
    return out, lse


def _limits(n, m, block, shift=0):
    return torch.tensor([shift + (m if block == 0 else max(0, min(m, ((m - n + i) // block + 1) * block))) for i in range(n)], device=_DEVICE)


def _exact_sequences(case, q, sequences):
    """sequences: (first query row, queries, keys [m][kv heads][dim], values, limits)."""
    out = torch.zeros(q.shape, dtype=torch.float64, device=_DEVICE)
    lse = torch.zeros(q.shape[:2], dtype=torch.float64, device=_DEVICE)
    each = case["heads"] // case["kv_heads"]
    for at, n, k, v, limits in sequences:
        for h in range(case["heads"]):
            kh, vh = k[:, h // each].double().contiguous(), v[:, h // each].double().contiguous()
            out[at:at + n, h], lse[at:at + n, h] = _exact_head(q[at:at + n, h].double().contiguous(), kh, vh, limits)
    return {"out": out, "lse": lse} if case["lse"] else {"out": out}


def exact(case, seed):
    s, block = _inputs(case, seed), case["block"] if "block" in case else 0
    if case["op"] in ("rope", "rope_append"):
        return _exact_rope(case, s)
    if case["op"] == "attention":
        qs, ks = _starts(s["ql"]), _starts(s["kl"])
        return _exact_sequences(case, s["q"], [(qs[i], n, s["k"][ks[i]:ks[i + 1]], s["v"][ks[i]:ks[i + 1]], _limits(n, m, block))
                                               for i, (n, m) in enumerate(zip(s["ql"], s["kl"]))])

    def row_of(cache, table, n):
        """The n rows that a table's row names, one token at a time by its page and place."""
        j = torch.arange(n, device=_DEVICE)
        return cache.permute(0, 2, 1, 3)[table[j // _PAGE].long(), j % _PAGE]

    sequences, at, each = [], 0, len(s["rows"]) // len(s["prefixes"])
    for b, (n, m) in enumerate(zip(s["rows"], s["lens"])):
        g = b // each
        p = s["prefixes"][g]
        k, v = (torch.cat((row_of(s[x], s["prefix_pages"][g], p), row_of(s[x], s["own_pages"][b], m))) for x in ("k_cache", "v_cache"))
        sequences.append((at, n, k, v, _limits(n, m, block, p)))
        at += n
    return _exact_sequences(case, s["q"], sequences)
