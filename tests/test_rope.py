"""Rotary positions against their formula in 64 bits: both pairings, part of the head, far and negative positions, strides, in place, into a paged cache;
what they refuse and what they leave alone.  Tolerances: kv_oracle.turned."""
import math

import pytest
import torch

import paper_2605_29233_amd as bb
from paper_2605_29233_amd import BBError, binding
from kv_oracle import DEV, PAGE, TYPES, close, gen, ints, rnd, turned


def freqs_of(rot, base=10000.0):
    return base ** (-torch.arange(0, rot, 2, dtype=torch.float64) / max(rot, 1))


@pytest.mark.parametrize("rot", [2, 48, 64, 128])
def test_frequencies(rot):
    """Host only: plain, divided, and by parts, against the formula."""
    f = freqs_of(rot, 500.0)
    assert torch.allclose(bb.rope_frequencies(rot, 500.0, device="cpu"), f, rtol=1e-14, atol=0)
    assert torch.allclose(bb.rope_frequencies(rot, 500.0, factor=8.0, device="cpu"), f / 8, rtol=1e-14, atol=0)
    got = bb.rope_frequencies(rot, 500.0, factor=8.0, context=4096, low=1.0, high=4.0, device="cpu")
    for j in range(rot // 2):
        turns = 4096 * f[j].item() / (2 * math.pi)
        keep = min(1.0, max(0.0, (turns - 1) / 3))
        want = f[j].item() * (keep + (1 - keep) / 8)
        assert abs(got[j].item() - want) <= 1e-14 * want
        assert abs(got[j] - f[j] / (1 if turns >= 4 else 8)) <= 1e-14 * f[j] or 1 < turns < 4


def test_frequencies_refuse():
    for bad in (dict(rot=0), dict(rot=3), dict(rot=2048), dict(rot=64, base=0.0), dict(rot=64, base=float("inf")), dict(rot=64, factor=0.0), dict(rot=64, context=-1),
                dict(rot=64, context=100, low=4.0, high=4.0), dict(rot=64, factor=float("nan"))):
        with pytest.raises(BBError):
            bb.rope_frequencies(device="cpu", **bad)


CASES = [(1, 1, 1, 2, 2), (3, 2, 1, 64, 64), (5, 4, 4, 64, 48), (7, 28, 4, 128, 64), (2, 3, 0, 128, 128), (130, 2, 2, 80, 34), (9, 5, 1, 7, 6), (4, 2, 1, 1024, 1024), (3, 1, 1, 64, 0),
         (33, 32, 32, 128, 128)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("tokens,heads,kv_heads,dim,rot", CASES)
def test_rope_equals_the_formula(tokens, heads, kv_heads, dim, rot, interleaved, dtype):
    t = TYPES[dtype]
    x = rnd(tokens + dim, tokens, heads + 2 * kv_heads, dim, dtype=dtype, scale=2.0)
    q, k = x[:, :heads], x[:, heads:heads + kv_heads]
    pos = torch.randint(-50, 1 << 20, (tokens,), generator=gen(3), dtype=torch.int32)
    f = freqs_of(rot)
    d = x.to(DEV)
    dq, dk = d[:, :heads], d[:, heads:heads + kv_heads]
    qo, ko = torch.empty(q.shape, dtype=t, device=DEV), torch.empty(k.shape, dtype=t, device=DEV)
    args = pos.to(DEV), f.to(DEV), interleaved
    r = bb.rope(dq, dk if kv_heads else None, *args, magnitude=1.25, q_out=qo, k_out=ko if kv_heads else None)
    assert r[0] is qo
    wq, wk = turned(q, pos, f, interleaved, 1.25), turned(k, pos, f, interleaved, 1.25)
    close(qo, *wq, t)
    if kv_heads:
        close(ko, *wk, t)
    assert torch.equal(d.cpu(), x)
    # in place, inside the projection's output: what is not q or k stays
    if kv_heads:
        bb.rope(dq, dk, *args, magnitude=1.25)
    else:
        bb.rope(dq, None, *args, magnitude=1.25)
    assert torch.equal(dq, qo) and (not kv_heads or torch.equal(dk, ko)) and torch.equal(d[:, heads + kv_heads:].cpu(), x[:, heads + kv_heads:])
    # heads first, and rows at an odd element
    hq = q.to(DEV).transpose(0, 1).contiguous().transpose(0, 1)
    base = torch.full((tokens, heads * dim + 3), 7.0, dtype=t, device=DEV)
    odd = base[:, 1:1 + heads * dim].unflatten(1, (heads, dim))
    bb.rope(hq, None, *args, magnitude=1.25, q_out=odd)
    assert torch.equal(odd, qo) and (base[:, 0] == 7).all() and (base[:, 1 + heads * dim:] == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_positions_at_the_ends_of_their_type(interleaved):
    pos = ints([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 1 << 24, (1 << 24) + 1])
    x = rnd(1, len(pos), 3, 64, dtype="fp32")
    f = freqs_of(64)
    q, _ = bb.rope(x.to(DEV), None, pos.to(DEV), f.to(DEV), interleaved=interleaved)
    close(q, *turned(x, pos, f, interleaved), torch.float32)
    assert torch.equal(q[0].cpu(), x[0])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("tokens,heads,kv_heads,dim,rot", [(1, 32, 32, 128, 128), (70, 4, 2, 64, 32), (131, 28, 4, 128, 128), (5, 3, 1, 24, 10), (3, 0, 2, 64, 64)])
@pytest.mark.parametrize("token_major", [False, True])
def test_append_writes_slots_and_nothing_else(tokens, heads, kv_heads, dim, rot, dtype, token_major):
    t, pages = TYPES[dtype], tokens // 50 + 3
    q, k, v = (rnd(s, tokens, h, dim, dtype=dtype) for s, h in ((1, heads), (2, kv_heads), (3, kv_heads)))
    pos = torch.randint(0, 5000, (tokens,), generator=gen(4), dtype=torch.int32)
    slots = torch.randperm(pages * PAGE, generator=gen(5))[:tokens].int()
    out_of = [i for i in range(tokens) if i % 7 == 3]
    for n, i in enumerate(out_of):
        slots[i] = (-1, pages * PAGE, 2 ** 31 - 1, -2 ** 31)[n % 4]
    shape = (pages, PAGE, kv_heads, dim) if token_major else (pages, kv_heads, PAGE, dim)
    kc, vc = (torch.full(shape, 5.0, dtype=t, device=DEV) for _ in range(2))
    if token_major:
        kc, vc = kc.transpose(1, 2), vc.transpose(1, 2)
    f = freqs_of(rot)
    dq = q.to(DEV)
    r = bb.rope_append(dq, k.to(DEV), v.to(DEV), pos.to(DEV), f.to(DEV), kc, vc, slots.to(DEV), interleaved=True)
    assert r is dq
    close(r, *turned(q, pos, f, True), t)
    wk, slack = turned(k, pos, f, True)
    kept = [i for i in range(tokens) if i not in out_of]
    at = slots[kept].long()
    close(kc.cpu()[at // PAGE, :, at % PAGE], wk[kept], slack[kept], t)
    assert torch.equal(vc.cpu()[at // PAGE, :, at % PAGE], v[kept])
    for c in (kc.cpu(), vc.cpu()):
        c[at // PAGE, :, at % PAGE] = 5
        assert (c == 5).all()


@pytest.mark.gpu
def test_cache_beyond_32_bits():
    """Pages 2^31 elements apart."""
    far = torch.empty(2 * (1 << 31) + 2 * 64 * 64, dtype=torch.bfloat16, device=DEV)
    kc = far.as_strided((3, 1, 64, 64), (1 << 31, 4096, 64, 1))
    vc = torch.zeros(3, 1, 64, 64, dtype=torch.bfloat16, device=DEV)
    k = rnd(1, 2, 1, 64)
    pos, f = ints([3, 9]), freqs_of(64)
    bb.rope_append(torch.empty(2, 0, 64, dtype=torch.bfloat16, device=DEV), k.to(DEV), k.to(DEV), pos.to(DEV), f.to(DEV), kc, vc, ints([2 * 64 + 5, 63]).to(DEV))
    w, s = turned(k, pos, f, False)
    close(kc[2, :, 5][None], w[:1], s[:1], torch.bfloat16)
    close(kc[0, :, 63][None], w[1:], s[1:], torch.bfloat16)


@pytest.mark.gpu
def test_more_tokens_than_a_launch_takes():
    """A workgroup for every token, and more of them than a launch has: rows on both sides of the border, and the last."""
    tokens, heads, kv_heads, dim = (1 << 20) + 3, 40, 8, 64
    q = torch.zeros(tokens, heads, dim, dtype=torch.bfloat16, device=DEV)
    kv = torch.zeros(tokens, 2 * kv_heads, dim, dtype=torch.bfloat16, device=DEV)
    cache = torch.zeros(2, tokens // PAGE + 1, kv_heads, PAGE, dim, dtype=torch.bfloat16, device=DEV)
    at = torch.tensor([0, 1, (1 << 20) - 1, 1 << 20, tokens - 1])
    x, y = rnd(1, len(at), heads, dim), rnd(2, len(at), 2 * kv_heads, dim)
    q[at.to(DEV)], kv[at.to(DEV)] = x.to(DEV), y.to(DEV)
    pos = torch.arange(tokens, dtype=torch.int32).flip(0)
    slots = torch.arange(tokens, dtype=torch.int32) ^ 1                     # (an odd number of tokens: the last one's slot is one further)
    f = freqs_of(dim)
    wq, wk = turned(x, pos[at], f, False), turned(y[:, :kv_heads], pos[at], f, False)
    k0 = kv[:, :kv_heads].clone()
    bb.rope_append(q, k0, kv[:, kv_heads:], pos.to(DEV), f.to(DEV), cache[0], cache[1], slots.to(DEV))
    close(q[at.to(DEV)], *wq, torch.bfloat16)
    s = slots[at].long().to(DEV)
    close(cache[0][s // PAGE, :, s % PAGE], *wk, torch.bfloat16)
    assert torch.equal(cache[1][s // PAGE, :, s % PAGE].cpu(), y[:, kv_heads:])
    r, k = bb.rope(q, k0, (-pos).to(DEV), f.to(DEV))                        # back, in place
    w = turned(x, pos[at], f, False)
    assert r is q and k is k0 and float((r[at.to(DEV)].cpu().double() - x.double()).abs().max()) <= float(2 ** -6 * w[0].abs().max())
    assert float(q[7].abs().max()) == 0


@pytest.mark.gpu
def test_not_a_number_stays_in_its_pair():
    x = rnd(1, 2, 2, 64, dtype="fp16")
    x[0, 1, 5], x[1, 0, 40] = float("nan"), float("inf")
    pos, f = ints([2, 3]), freqs_of(32)
    q, _ = bb.rope(x.to(DEV), None, pos.to(DEV), f.to(DEV))
    bad = torch.zeros_like(x, dtype=torch.bool)
    bad[0, 1, 5] = bad[0, 1, 21] = bad[1, 0, 40] = True
    assert torch.equal(~torch.isfinite(q.cpu()), bad)


@pytest.mark.gpu
def test_no_tokens_and_another_stream():
    f = freqs_of(64).to(DEV)
    e = torch.empty(0, 4, 64, device=DEV)
    q, k = bb.rope(e, e[:, :2], ints([]).to(DEV), f)
    assert q.shape == (0, 4, 64)
    s = torch.cuda.Stream()
    x = rnd(1, 3, 4, 64, dtype="fp32")
    d, pos = x.to(DEV), ints([1, 2, 3])
    dp = pos.to(DEV)
    s.wait_stream(torch.cuda.current_stream())
    q, _ = bb.rope(d, None, dp, f, stream=s)
    s.synchronize()
    close(q, *turned(x, pos, freqs_of(64), False), torch.float32)


def test_c_entry_refuses_before_touching_a_device():
    """Every call below is refused on the host (the pointers are never followed)."""
    lib = bb.load_library()
    p = 1 << 20
    good = dict(q=p, qt=256, qh=64, qo=2 * p, qot=256, qoh=64, nq=4, k=3 * p, kt=128, kh=64, ko=4 * p, kot=128, koh=64, nk=2, pos=5 * p, f=6 * p, rot=64, il=0, mag=1.0, n=8, dim=64, type=1)

    def call(**kw):
        return lib.bb_rope(binding.ROPE_ARGS.pack(*dict(good, **kw).values()), None)

    assert call(n=0) == 0 and call(nq=0, nk=0) == 0 and lib.bb_rope(None, None) == -1 and lib.bb_rope_append(None, None) == -1
    for bad in (dict(q=0), dict(q=p + 1), dict(qo=0), dict(k=0), dict(ko=4 * p + 1), dict(pos=0), dict(pos=5 * p + 2), dict(f=0), dict(f=6 * p + 4), dict(rot=63), dict(rot=66),
                dict(rot=-2), dict(dim=0), dict(dim=2048, rot=64), dict(type=3), dict(type=-1), dict(n=-1), dict(n=1 << 40), dict(nq=-1), dict(nk=5000), dict(nq=1 << 32), dict(mag=float("nan")),
                dict(mag=float("inf")), dict(mag=1e39), dict(qt=-1), dict(qt=1 << 45), dict(qt=1 << 62), dict(qot=0), dict(qot=100), dict(qoh=32), dict(qo=p + 2), dict(qo=p, qot=512),
                dict(ko=2 * p), dict(ko=p), dict(qo=3 * p), dict(rot=1 << 33), dict(dim=1 << 32), dict(type=1 << 32)):
        assert call(**bad) == -1, bad
    good = dict(q=p, qt=256, qh=64, qo=2 * p, qot=256, qoh=64, nq=4, k=3 * p, kt=128, kh=64, v=4 * p, vt=128, vh=64, nk=2, pos=5 * p, f=6 * p, rot=64, il=0, mag=1.0, slots=7 * p,
                kc=16 * p, kcp=8192, kch=4096, kct=64, vc=32 * p, vcp=8192, vch=4096, vct=64, pages=4, n=8, dim=64, type=1)

    def call(**kw):
        return lib.bb_rope_append(binding.ROPE_APPEND_ARGS.pack(*dict(good, **kw).values()), None)

    assert call(n=0) == 0
    for bad in (dict(slots=0), dict(slots=7 * p + 1), dict(kc=0), dict(vc=0), dict(v=0), dict(pages=0), dict(pages=1 << 26), dict(pages=1 << 33), dict(nk=0), dict(kcp=4096), dict(kct=32),
                dict(vch=64), dict(vc=16 * p), dict(kc=4 * p), dict(qo=16 * p), dict(kc=16 * p + 1), dict(qo=3 * p), dict(kcp=-8192)):
        assert call(**bad) == -1, bad


def test_python_refuses():
    x = torch.zeros(3, 4, 64, dtype=torch.bfloat16)
    with pytest.raises(BBError, match="GPU"):
        bb.rope(x, None, ints([1, 2, 3]), freqs_of(64))


@pytest.mark.gpu
def test_python_refuses_on_the_device():
    x = torch.zeros(3, 4, 64, dtype=torch.bfloat16, device=DEV)
    pos, f = ints([1, 2, 3]).to(DEV), freqs_of(64).to(DEV)
    c = torch.zeros(2, 4, 64, 64, dtype=torch.bfloat16, device=DEV)
    bad = [lambda: bb.rope(x[0], None, pos, f), lambda: bb.rope(x.int(), None, pos, f), lambda: bb.rope(x, None, pos.long(), f), lambda: bb.rope(x, None, pos[:2], f),
           lambda: bb.rope(x, None, pos, f.float()), lambda: bb.rope(x, x.float(), pos, f), lambda: bb.rope(x, None, pos, f, q_out=x[:2]), lambda: bb.rope(x, None, pos, f, k_out=x),
           lambda: bb.rope(x, None, pos, freqs_of(66).to(DEV)), lambda: bb.rope(x.transpose(1, 2).contiguous().transpose(1, 2), None, pos, f),
           lambda: bb.rope(x, x, pos, f), lambda: bb.rope(x[:, :, :32], None, pos, f[:16], q_out=x[:, :, 16:48]),
           lambda: bb.rope_append(x, x.clone(), x, pos, f, c, c, pos), lambda: bb.rope_append(x, x.clone(), x, pos, f, c, c[:, :2], pos),
           lambda: bb.rope_append(x, x.clone(), x, pos, f, c, c.float(), pos), lambda: bb.rope_append(x, x.clone(), x, pos, f, c, c.clone(), pos.long()),
           lambda: bb.rope(x.expand(3, 4, 64), None, pos, f, q_out=x[:1].expand(3, 4, 64)),
           lambda: bb.rope(x, None, pos, f[0]), lambda: bb.rope(x, None, pos[0], f), lambda: bb.rope(x, None, pos, f, magnitude="1"), lambda: bb.rope(x, None, pos, f, interleaved=0.5),
           lambda: bb.rope_append(x, x.clone(), x, pos, f[0], c, c.clone(), pos), lambda: bb.rope_append(x, x.clone(), x, pos, f, c[0, 0, 0, 0], c.clone(), pos)]
    for i, call in enumerate(bad):
        with pytest.raises(BBError):
            call()
            print("not refused:", i)
