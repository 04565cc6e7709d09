"""Performance cases of the 8-bit operators: rows of activations or weights quantised to int8 with a scale each (plainly, out
of an RMSNorm with the residual's addition, or out of SwiGLU), and the int8 product with a scale per token and per channel.

  quantize_rows     q[r][c] = rint(127 x[r][c] / max_c |x[r]|), scale[r] = max_c |x[r]| / 127
  rmsnorm_quantize  h = x + residual (rounded to its type), y = h / sqrt(mean h^2 + eps) * gain, y's rows quantised
  swiglu_quantize   y = gate / (1 + exp(-gate)) * up, y's rows quantised
  gemm_int8         C[m][n] = (sum_k A[m][k] W[n][k]) a_scale[m] w_scale[n] + bias[n]

Sizes are those of `workload/configs.py` (widths 4096, 3584, 12288, 18944 and the tiny model's 256 and 688; the rows of block
steps, refreshes and many requests) and generic ones around them.  A quantised row is returned as the values that its codes
stand for, in the type of the operator's input, beside its scale.
"""
import torch

own = False

_DEVICE = "cuda:0"
_TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
_BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
_EPS = 1e-5


def _rows(name, op, rows, cols, dtype, residual=False):
    c = {"name": name, "op": op, "rows": rows, "cols": cols, "type": dtype}
    return dict(c, residual=residual) if op == "rmsnorm_quantize" else c


def _gemm(name, m, n, k, dtype, bias=False, pad=16):
    return {"name": name, "op": "gemm_int8", "m": m, "n": n, "k": k, "type": dtype, "bias": bias, "pad": pad}


def listed():
    return [
        # weights of a gate/up matrix made 8-bit per output channel, as a model is loaded
        _rows("quantize_weights", "quantize_rows", 24576, 4096, "bf16"),
        # an attention output on its way into the output projection: odd rows and columns
        _rows("quantize_odd", "quantize_rows", 173, 1001, "fp32"),
        # one token through one norm: latency
        _rows("norm_token", "rmsnorm_quantize", 1, 4096, "bf16", residual=True),
        # the packed rows of a block step with four branches, on the fp32 residual stream
        _rows("norm_step", "rmsnorm_quantize", 120, 4096, "fp32", residual=True),
        # a refresh of four long rows
        _rows("norm_refresh", "rmsnorm_quantize", 20480, 4096, "bf16", residual=True),
        # a block step of the wide feed-forward
        _rows("swiglu_step", "swiglu_quantize", 112, 18944, "fp16"),
        # many requests at once
        _rows("swiglu_many", "swiglu_quantize", 6143, 12288, "bf16"),
        # one token through a feed-forward's first product: every weight read once
        _gemm("gemm_token", 1, 24576, 4096, "bf16"),
        # a block step of the tiny model with a padded k range, fp32 out
        _gemm("gemm_tiny", 56, 256, 688, "fp32"),
        # a block step's down projection
        _gemm("gemm_step", 120, 4096, 12288, "fp32"),
        # ragged rows, columns that no tile divides, a bias
        _gemm("gemm_ragged", 1402, 4610, 3592, "fp16", bias=True),
        # a refresh's gate/up product
        _gemm("gemm_refresh", 8192, 24576, 4096, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def _size(rng, lo, hi, unit):
    """Over the logarithm of the range; half of them multiples of `unit`."""
    v = _log(rng, lo, hi)
    return max(lo, v // unit * unit) if rng.random() < 0.5 else v


def draw(rng):
    op = rng.choice(["quantize_rows", "rmsnorm_quantize", "swiglu_quantize", "gemm_int8", "gemm_int8", "gemm_int8"])
    dtype = rng.choice(["bf16", "bf16", "fp16", "fp32"])
    if op == "gemm_int8":
        while True:
            m, n, k = _size(rng, 1, 8192, 8), _size(rng, 32, 24576, 64), _size(rng, 32, 18944, 64)
            if m * n * k <= 8192 * 24576 * 4096 and n * k <= 24576 * 4096:
                break
        c = _gemm("", m, n, k, dtype, rng.random() < 0.3, 16 if rng.random() < 0.75 else 1)
    else:
        while True:
            rows, cols = _size(rng, 1, 24576, 16), _size(rng, 32, 18944, 64)
            if rows * cols * (2 if dtype == "fp32" else 1) <= 20480 * 4096:
                break
        c = _rows("", op, rows, cols, dtype, rng.random() < 0.75)
    del c["name"]
    return c


def _gen(seed):
    return torch.Generator(device=_DEVICE).manual_seed(seed)


def _activations(g, rows, cols, dtype):
    """Normal values; of the channels every 64th or so is some ten times as large, as in a trained model's activations."""
    x = torch.randn(rows, cols, generator=g, device=_DEVICE)
    x *= torch.where(torch.rand(cols, generator=g, device=_DEVICE) < 1 / 64, 12.0, 1.0)
    return x.to(dtype)


def _codes(g, rows, cols, pad):
    """Codes of normal rows, their largest value 127, with a row stride of whole `pad` bytes."""
    stride = -(-cols // pad) * pad
    q = torch.empty(rows, stride, dtype=torch.int8, device=_DEVICE)[:, :cols]
    q.copy_((torch.randn(rows, cols, generator=g, device=_DEVICE) * 34).round_().clamp_(-127, 127))
    q[:, :1] = 127
    return q


def _inputs(case, seed):
    g, t, op = _gen(seed), _TYPES[case["type"]], case["op"]
    if op == "gemm_int8":
        m, n, k = case["m"], case["n"], case["k"]
        s = {"a": _codes(g, m, k, case["pad"]), "w": _codes(g, n, k, case["pad"]),
             "a_scale": torch.rand(m, generator=g, device=_DEVICE) * 0.05 + 0.01,
             "w_scale": torch.rand(n, generator=g, device=_DEVICE) * 0.0005 + 0.0004}
        s["bias"] = torch.randn(n, generator=g, device=_DEVICE) if case["bias"] else None
        return s
    rows, cols = case["rows"], case["cols"]
    if op == "swiglu_quantize":             # the two halves of one product's output
        gu = torch.randn(rows, 2 * cols, generator=g, device=_DEVICE).mul_(1.5).to(t)
        return {"gate": gu[:, :cols], "up": gu[:, cols:]}
    s = {"x": _activations(g, rows, cols, t)}
    if op == "rmsnorm_quantize":
        s["gain"] = (torch.randn(cols, generator=g, device=_DEVICE) * 0.2 + 1.0).to(t)
        s["residual"] = _activations(g, rows, cols, t).mul_(3) if case["residual"] else None
    return s


def prepare(case, seed):
    s = dict(_inputs(case, seed), op=case["op"], type=_TYPES[case["type"]])
    if case["op"] == "gemm_int8":
        s["out"] = torch.empty(case["m"], case["n"], dtype=s["type"], device=_DEVICE)
    else:
        rows, cols = case["rows"], case["cols"]
        s["q"] = torch.empty(rows, -(-cols // 16) * 16, dtype=torch.int8, device=_DEVICE)[:, :cols]
        s["scale"] = torch.empty(rows, dtype=torch.float32, device=_DEVICE)
        s["values"] = torch.empty(rows, cols, dtype=s["type"], device=_DEVICE)
        if case["op"] == "rmsnorm_quantize" and case["residual"]:
            s["h"] = torch.empty(rows, cols, dtype=s["type"], device=_DEVICE)
    return s


def _quantized(y, dtype):
    """Rows of y, in 64 bits, as int8 codes with a scale: the values they stand for and the scales (codes next to a border want 64 bits)."""
    top = y.abs().amax(1, keepdim=True)
    q = torch.round(127 * y / top)
    scale = (top / 127).float()
    return {"values": (q.float() * scale).to(dtype), "scale": scale[:, 0]}


def _plain(s):
    op = s["op"]
    if op == "gemm_int8":
        c = (s["a"].float() @ s["w"].float().t()) * s["a_scale"][:, None] * s["w_scale"]
        return (c if s["bias"] is None else c + s["bias"]).to(s["type"])
    if op == "quantize_rows":
        return _quantized(s["x"].double(), s["type"])
    if op == "swiglu_quantize":
        g = s["gate"].double()
        return _quantized(g / (1 + torch.exp(-g)) * s["up"].double(), s["type"])
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["type"])
    d = h.double()
    out = _quantized(d / torch.sqrt(d.square().mean(1, keepdim=True) + _EPS) * s["gain"].double(), s["type"])
    return out if s["residual"] is None else dict(out, h=h)


def _own(s):
    import paper_2605_29233_amd as bb
    op = s["op"]
    if op == "gemm_int8":
        return bb.gemm_int8(s["a"], s["a_scale"], s["w"], s["w_scale"], bias=s["bias"], out=s["out"])
    if op == "quantize_rows":
        bb.quantize_rows(s["x"], out=s["q"], scale=s["scale"])
    elif op == "swiglu_quantize":
        bb.swiglu_quantize(s["gate"], s["up"], out=s["q"], scale=s["scale"])
    else:
        bb.rmsnorm_quantize(s["x"], s["gain"], _EPS, residual=s["residual"], residual_out=s.get("h"), out=s["q"], scale=s["scale"])
    torch.mul(s["q"], s["scale"][:, None], out=s["values"])
    r = {"values": s["values"], "scale": s["scale"]}
    return dict(r, h=s["h"]) if "h" in s else r


def run(state):
    return _own(state) if own else _plain(state)


def work(case):
    b = _BYTES[case["type"]]
    if case["op"] == "gemm_int8":
        m, n, k = case["m"], case["n"], case["k"]
        return {"bytes": m * k + n * k + 4 * (m + n) + (4 * n if case["bias"] else 0) + b * m * n, "flops": 2 * m * n * k}
    e = case["rows"] * case["cols"]
    read = {"quantize_rows": 1, "swiglu_quantize": 2, "rmsnorm_quantize": 1 + case.get("residual", False)}[case["op"]]
    written = 1 + case.get("residual", False)       # the values, and the sum with the residual
    return {"bytes": e * b * (read + written) + 4 * case["rows"], "flops": e * {"quantize_rows": 3, "swiglu_quantize": 8, "rmsnorm_quantize": 7}[case["op"]]}


def exact(case, seed):
    """The definitions, a block of rows at a time, in 64 bits throughout: codes by comparison with the border between two of them."""
    s, op = _inputs(case, seed), case["op"]
    f64 = torch.float64
    if op == "gemm_int8":
        w = s["w"].to(f64).mul_(s["w_scale"].to(f64)[:, None]).t().contiguous()
        parts = []
        for r in range(0, case["m"], 2048):
            c = torch.mm(s["a"][r:r + 2048].to(f64).mul_(s["a_scale"][r:r + 2048].to(f64)[:, None]), w)
            parts.append(c if s["bias"] is None else c.add_(s["bias"].to(f64)))
        return torch.cat(parts)
    values, scales, sums = [], [], []
    for r in range(0, case["rows"], 2048):
        if op == "swiglu_quantize":
            g = s["gate"][r:r + 2048].to(f64)
            y = g * torch.sigmoid(g) * s["up"][r:r + 2048].to(f64)
        else:
            y = s["x"][r:r + 2048].to(f64)
        if op == "rmsnorm_quantize":
            if s["residual"] is not None:   # (the sum is rounded to the residual's type by the operator's definition)
                y = (y + s["residual"][r:r + 2048].to(f64)).to(_TYPES[case["type"]]).to(f64)
                sums.append(y)
            y = y * (torch.linalg.vector_norm(y, dim=1, keepdim=True).square() / case["cols"] + _EPS).rsqrt() * s["gain"].to(f64)
        step = torch.linalg.vector_norm(y, ord=float("inf"), dim=1, keepdim=True) / 127
        u = y / step
        low = torch.floor(u)
        up = (u - low > 0.5) | ((u - low == 0.5) & (low % 2 == 1))
        values.append((low + up) * step)
        scales.append(step[:, 0])
    out = {"values": torch.cat(values), "scale": torch.cat(scales)}
    return dict(out, h=torch.cat(sums)) if sums else out
