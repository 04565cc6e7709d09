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
