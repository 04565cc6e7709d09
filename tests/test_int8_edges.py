"""The 8-bit integer operators at the edges of their ranges: gates so negative that exp(-gate) leaves fp32.

The references and tolerances are those of tests/test_int8_ops.py: codes equal the formula's in 64 bits, a scale is one fp32 rounding of it."""
import pytest
import torch

import paper_2605_29233_amd as bb
from test_int8_ops import DEV, TYPES, check_swiglu, gen, rnd, strided


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cols", [1, 7, 8, 43, 700, 4096, 12289, 40001])
def test_swiglu_of_very_negative_gates(cols, dtype):
    """SiLU(-89) is 2e-37, a normal fp32, and times a large `up` anything: rows made of such gates alone, beside ordinary values that are smaller, as large
    or larger, and rows whose values lie below fp32 (scale 0, the formula's codes) or are all zero."""
    t = TYPES[dtype]
    large = 1e4 if dtype == "fp16" else 1e30
    low = -(87.0 + 63.0 * torch.rand(10, cols, generator=gen(cols)))
    gate, up = rnd(70 + cols, 10, cols, dtype, 2.0), rnd(71 + cols, 10, cols, dtype)
    few = torch.rand(10, cols, generator=gen(72 + cols)) < 0.1
    few[:, cols // 2] = True
    gate[0], up[0] = low[0].to(t), (up[0].float() * large).to(t)
    gate[1], up[1] = -88.0, min(large, 1e5)
    gate[2], up[2] = -89.0, large
    gate[3], up[3] = torch.where(few[3], low[3].to(t), gate[3]), torch.where(few[3], (up[3].float() * large).to(t), up[3])
    gate[4] = torch.where(few[4], low[4].to(t), gate[4])
    if dtype != "fp16":                     # ordinary values of about 1e-8, 1e-7 and 1e-9 beside -89 times 1e30: 2e-7
        for row, by in ((5, 1e-8), (6, 1e-7), (7, 1e-9)):
            gate[row], up[row] = torch.where(few[row], torch.tensor(-89.0, dtype=t), gate[row]), torch.where(few[row], torch.tensor(1e30, dtype=t), (up[row].float() * by).to(t))
        gate[9], up[9] = -89.0, 1e38
    gate[8], up[8] = -1000.0, large         # (exp(1000) leaves 64 bits too)
    y = gate.double() / (1 + torch.exp(-gate.double())) * up.double()
    assert (y[:3] != 0).all() and (y[8] == 0).all()
    q, s = bb.swiglu_quantize(gate.to(DEV), up.to(DEV))
    check_swiglu(q, s, gate, up)
    q2, s2 = bb.swiglu_quantize(strided(gate, 5, 1), strided(up, 2, 1))
    assert torch.equal(q, q2) and torch.equal(s, s2)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_swiglu_of_the_lowest_gates_and_of_infinities(dtype):
    """The type's lowest value as a mask gives zeros; -inf is NaN by the formula, as is a zero of SiLU times an infinity."""
    t, cols = TYPES[dtype], 48
    gate, up = rnd(80, 6, cols, dtype), rnd(81, 6, cols, dtype)
    gate[0] = torch.finfo(t).min
    gate[1, 5:40] = torch.finfo(t).min
    gate[2, 7] = float("-inf")
    gate[3, 7], up[3, 7] = -1e4, float("inf")
    gate[4], up[4] = -300.0, 1e38           # 1e-90: the scale rounds to 0
    check_swiglu(*bb.swiglu_quantize(gate.to(DEV), up.to(DEV)), gate, up)
