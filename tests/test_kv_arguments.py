"""Calls of the operators around K,V that their documentation allows or rules out and that need no large tensors: sizes of workspaces, numbers that no field holds, tensors that autograd looks after."""
import pytest
import torch

import paper_2605_29233_amd as bb
from paper_2605_29233_amd import BBError, binding
from kv_oracle import DEV, PAGE, ints, rnd, starts

P = 1 << 20
PACKED = dict(q=P, qt=256, qh=64, k=2 * P, kt=128, kh=64, v=3 * P, vt=128, vh=64, qs=4 * P, ks=5 * P, n=1, qn=16, kn=100000, heads=4, kv=2, dim=64, type=1, block=1, scale=0.1, o=6 * P, ot=256,
              oh=64, lse=0)
PAGED = dict(q=P, qt=256, qh=64, qs=4 * P, n=2, qn=8, k=16 * P, kp=8192, kh=4096, kt=64, v=32 * P, vp=8192, vh=4096, vt=64, pages=4, own=5 * P, old=3, ow=300, lens=6 * P, pre=7 * P, pld=3, pw=500,
             pl=8 * P, gs=9 * P, g=1, heads=4, kv=2, dim=64, type=1, block=1, scale=0.1, o=10 * P, ot=256, oh=64, lse=0)


@pytest.mark.parametrize("struct,good,size", [(binding.ATTENTION_ARGS, PACKED, "bb_attention_workspace_bytes"), (binding.SHARED_ATTENTION_ARGS, PAGED, "bb_shared_attention_workspace_bytes")])
def test_workspace_bytes_look_at_sizes_alone(struct, good, size):
    """A caller may ask with nothing but the sizes filled in."""
    size = getattr(bb.load_library(), size)
    sizes = ("n", "qn", "kn", "ow", "pw", "g", "heads", "kv", "dim", "type")
    need = size(struct.pack(*good.values()))
    assert need > 0
    assert size(struct.pack(*{k: v if k in sizes else 0 for k, v in good.items()}.values())) == need
    for other in (dict(block=-1), dict(block=1 << 40), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf"))):
        assert size(struct.pack(*dict(good, **other).values())) == need, other
    for bad in (dict(n=-1), dict(qn=-1), dict(heads=3), dict(heads=0), dict(kv=0), dict(dim=96), dict(type=0), dict(type=7)):
        assert size(struct.pack(*dict(good, **bad).values())) == 0, bad


def operands():
    """Of every operator around K,V: (call, its float inputs, its outputs), by names of the call's arguments."""
    def x(seed, *shape):
        return rnd(seed, *shape).to(DEV)

    pos, f, s = ints([1, 2, 3]).to(DEV), bb.rope_frequencies(64, device=DEV), starts([3]).to(DEV)
    table, lens, slots = ints([[1]]).to(DEV), ints([3]).to(DEV), ints([5, 6, 7]).to(DEV)
    return [
        (bb.rope, dict(positions=pos, freqs=f), dict(q=x(1, 3, 4, 64), k=x(2, 3, 2, 64)), dict(q_out=x(3, 3, 4, 64), k_out=x(4, 3, 2, 64))),
        (bb.rope_append, dict(positions=pos, freqs=f, slots=slots), dict(q=x(1, 3, 4, 64), k=x(2, 3, 2, 64), v=x(5, 3, 2, 64)),
         dict(k_cache=x(6, 2, 2, PAGE, 64), v_cache=x(7, 2, 2, PAGE, 64), q_out=x(3, 3, 4, 64))),
        (bb.attention, dict(q_starts=s), dict(q=x(1, 3, 4, 64), k=x(2, 3, 2, 64), v=x(5, 3, 2, 64)), dict(out=x(3, 3, 4, 64), lse=torch.zeros(3, 4, device=DEV))),
        (bb.shared_attention, dict(q_starts=s, own_pages=table, own_lens=lens), dict(q=x(1, 3, 4, 64), k_cache=x(6, 2, 2, PAGE, 64), v_cache=x(7, 2, 2, PAGE, 64)),
         dict(out=x(3, 3, 4, 64), lse=torch.zeros(3, 4, device=DEV))),
    ]


@pytest.mark.gpu
def test_tensors_that_require_a_gradient_are_refused():
    """There is no backward pass: with gradients recorded such a tensor, read or written, is refused and stays as it is; without, or detached, the call runs."""
    for call, others, inputs, outputs in operands():
        for name, t in {**inputs, **outputs}.items():
            leaf = t.clone().requires_grad_()
            for graded in (leaf, leaf * 1):             # (one that autograd would refuse to overwrite, and one that it would let be)
                args = {**others, **inputs, **outputs, name: graded}
                before = [a.detach().clone() for a in (*inputs.values(), *outputs.values())]
                with pytest.raises(BBError, match=f"{name}.*gradient"):
                    call(**args)
                assert all(torch.equal(a, b) for a, b in zip((*inputs.values(), *outputs.values()), before))
                with torch.no_grad():
                    call(**args)
            call(**{**others, **inputs, **outputs, name: leaf.detach()})


@pytest.mark.gpu
def test_outputs_count_as_written():
    """What a call writes has another version afterwards, in place or not, so that autograd finds a tensor changed that it kept; what it reads has not.  Inference tensors, which have none, are taken too."""
    for call, others, inputs, outputs in operands():
        seen = {n: t._version for n, t in {**inputs, **outputs}.items()}
        call(**others, **inputs, **outputs)
        assert all(t._version == seen[n] for n, t in inputs.items())
        assert all(t._version > seen[n] for n, t in outputs.items())
        with torch.inference_mode():
            call(**others, **inputs, **{n: t.clone() for n, t in outputs.items()})
    call, others, inputs, _ = operands()[0]
    q, k = (inputs[n].float() for n in "qk")
    seen = q._version, k._version
    call(q, k, **others)
    assert q._version > seen[0] and k._version > seen[1]
    # a product that has kept q: its gradient would be taken with the turned rows
    w = torch.ones_like(q, requires_grad=True)
    y = (q * w).sum()
    call(q, None, **others)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


@pytest.mark.gpu
def test_head_of_no_elements_and_numbers_that_no_field_holds():
    x, s = rnd(1, 3, 4, 64).to(DEV), starts([3]).to(DEV)
    c, table, lens = rnd(2, 2, 4, PAGE, 64).to(DEV), ints([[1]]).to(DEV), ints([3]).to(DEV)
    pos, f = ints([1, 2, 3]).to(DEV), bb.rope_frequencies(64, device=DEV)
    e, ec = x[:, :, :0], c[:, :, :, :0]
    huge = 10 ** 400
    for call in (lambda: bb.attention(e, e, e, s), lambda: bb.shared_attention(e, s, ec, ec, table, lens), lambda: bb.attention(x, x, x, s, scale=huge),
                 lambda: bb.shared_attention(x, s, c, c, table, lens, scale=huge), lambda: bb.rope(x.clone(), None, pos, f, magnitude=huge),
                 lambda: bb.rope_append(x.clone(), x, x, pos, f, c.clone(), c.clone(), pos, magnitude=huge), lambda: bb.rope(e, None, pos, f[:0])):
        with pytest.raises(BBError):
            call()


def test_frequencies_of_more_pairs_than_a_head_has():
    """2^32 + 64 elements are not 64 (the C entry's int)."""
    for rot in (2 ** 32 + 64, 1026, 2 ** 80):
        with pytest.raises(BBError):
            bb.rope_frequencies(rot, device="cpu")


@pytest.mark.gpu
def test_rope_captured_and_replayed_with_other_positions_and_slots():
    """Both calls in one graph; positions, slots and rows change between replays, eager calls of the same run between them; every replay equals the eager result, and slots of earlier ones stay."""
    x, f = rnd(1, 9, 8, 64).to(DEV), bb.rope_frequencies(64, device=DEV)
    pos, slots = ints(range(9)).to(DEV), ints(range(9)).to(DEV)
    cache = torch.zeros(2, 3, 2, PAGE, 64, dtype=x.dtype, device=DEV)
    q2, k2, q3 = (torch.empty(9, h, 64, dtype=x.dtype, device=DEV) for h in (4, 2, 4))

    def both(cache, q2, k2, q3):
        bb.rope(x[:, :4], x[:, 4:6], pos, f, q_out=q2, k_out=k2)
        bb.rope_append(x[:, :4], x[:, 4:6], x[:, 6:], pos, f, cache[0], cache[1], slots, interleaved=True, q_out=q3)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both(torch.zeros_like(cache), q2, k2, q3)
    torch.cuda.current_stream().wait_stream(side)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both(cache, q2, k2, q3)
    other = [torch.zeros_like(cache), torch.empty_like(q2), torch.empty_like(k2), torch.empty_like(q3)]
    for n in range(4):
        x.copy_(rnd(10 + n, 9, 8, 64))
        pos.copy_(torch.randint(-9, 1 << 20, (9,), generator=torch.Generator().manual_seed(n)))
        slots.copy_(torch.randperm(3 * PAGE, generator=torch.Generator().manual_seed(n))[:9])
        g.replay()
        both(*other)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip((cache, q2, k2, q3), other)), n
    assert (cache != 0).any()
