"""The 8-bit integer operators against their formulas in 64 bits: quantised rows (plain, RMSNorm with the residual's addition,
SwiGLU), the int8 product, a feed-forward made of them, their refusals and what they leave alone.

Tolerances, all derived: a scale is one fp32 rounding of the exact value (2^-24 relative; 2^-23 allows the double chain's own
errors next to a rounding border).  Codes equal the formula's.  The product: an exact integer
rounded to fp32, two products and a sum in fp32 (2^-24 each of the running value), then one rounding to the output's type."""
import pytest
import torch

import paper_2605_29233_amd as bb
from paper_2605_29233_amd import BBError

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
DEV = "cuda:0"


def gen(seed):
    return torch.Generator(device="cpu").manual_seed(seed)


def rnd(seed, rows, cols, dtype, scale=1.0):
    return (torch.randn(rows, cols, generator=gen(seed), dtype=torch.float32) * scale).to(TYPES[dtype])


def formula(y):
    """(codes, scale) of rows of doubles: codes as the correctly rounded quotient, ties to even."""
    top = y.abs().amax(1, keepdim=True)
    bad = ~torch.isfinite(y).all(1, keepdim=True)
    q = torch.where((top == 0) | bad, torch.zeros_like(y), torch.round(127 * y / top))
    q = torch.nan_to_num(q, nan=0.0).to(torch.int8)
    return q, torch.where(bad, torch.full_like(top, float("nan")), top / 127)[:, 0]


def norm_of(h, gain, eps):
    h = h.double()
    return h / torch.sqrt(h.square().mean(1, keepdim=True) + eps) * gain.double()


def same_scale(got, want):
    got, want = got.cpu().double(), want.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    ok = ~torch.isnan(want)
    assert ((got - want).abs()[ok] <= 2.0 ** -23 * want[ok] + 2.0 ** -150).all()


def check_codes(q, scale, y, same_codes=None):
    """same_codes: rows that differ from y's by a positive factor each (the norm's 1 / rms) and are exact, so that borders met
    exactly stay so."""
    codes, want = formula(y)
    same_scale(scale, want)
    assert torch.equal(q.cpu(), codes if same_codes is None else formula(same_codes)[0])


def check_norm(q, scale, h, gain, eps):
    y, p = norm_of(h, gain, eps), h.double() * gain.double()
    check_codes(q, scale, y, torch.where(torch.isfinite(y).all(1, keepdim=True), p, y))


def strided(t, extra, offset=0):
    """The same values as rows of a wider tensor, `offset` elements in; the gaps hold a recognisable value."""
    rows, cols = t.shape
    if t.dtype == torch.int8:
        base = torch.full((rows, cols + extra), 77, dtype=torch.int8)
    else:
        base = torch.full((rows, cols + extra), 1e4, dtype=t.dtype)
    base[:, offset:offset + cols] = t
    return base.to(DEV)[:, offset:offset + cols]


SHAPES = [(1, 1), (3, 7), (5, 8), (4, 64), (2, 511), (5, 512), (3, 513), (2, 2048), (3, 2049), (2, 4096), (2, 4097), (1, 8192), (3, 8200),
          (1, 18944), (2, 32768), (1, 32769), (2, 40001), (700, 33)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_quantize_rows_equals_the_formula(rows, cols, dtype):
    x = rnd(rows * 131 + cols, rows, cols, dtype)
    q, s = bb.quantize_rows(x.to(DEV))
    check_codes(q, s, x.double())
    # rows of a wider tensor, at an odd element offset, into rows of a wider tensor: the gaps stay as they were
    xs = strided(x, 5, 1)
    qbase = torch.full((rows + 2, cols + 3), 55, dtype=torch.int8, device=DEV)
    sbase = torch.full((rows + 2,), -1.0, device=DEV)
    bb.quantize_rows(xs, out=qbase[1:rows + 1, 2:cols + 2], scale=sbase[1:rows + 1])
    check_codes(qbase[1:rows + 1, 2:cols + 2], sbase[1:rows + 1], x.double())
    qbase[1:rows + 1, 2:cols + 2] = 55
    assert (qbase == 55).all() and sbase[0] == -1 and sbase[-1] == -1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("residual", [False, True])
def test_rmsnorm_quantize_equals_the_formula(rows, cols, dtype, residual):
    x, r, g = rnd(1 + cols, rows, cols, dtype), rnd(2 + cols, rows, cols, dtype, 3.0), rnd(3 + cols, 1, cols, dtype)[0]
    h = (x.float() + r.float()).to(x.dtype) if residual else x
    dx, dr, dg = x.to(DEV), r.to(DEV), g.to(DEV)
    if residual:
        out = torch.empty_like(dr)
        q, s = bb.rmsnorm_quantize(dx, dg, 1e-5, residual=dr, residual_out=out)
        assert torch.equal(out.cpu(), h) and torch.equal(dr.cpu(), r)
        check_norm(q, s, h, g, 1e-5)
        q, s = bb.rmsnorm_quantize(strided(x, 3, 1), dg, 1e-5, residual=dr)         # in place
        assert torch.equal(dr.cpu(), h)
        xs = strided(x, 3, 2)
        q2, s2 = bb.rmsnorm_quantize(xs, dg, 1e-5, residual=r.to(DEV), residual_out=xs)     # over x
        assert torch.equal(xs.cpu(), h) and torch.equal(q, q2) and torch.equal(s, s2)
    else:
        q, s = bb.rmsnorm_quantize(dx, dg, 1e-5)
        assert torch.equal(dx.cpu(), x)
    check_norm(q, s, h, g, 1e-5)


def check_swiglu(q, scale, gate, up):
    g = gate.double()
    check_codes(q, scale, g / (1 + torch.exp(-g)) * up.double())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES)
def test_swiglu_quantize_against_the_formula(rows, cols, dtype):
    gu = rnd(5 + cols, rows, 2 * cols, dtype, 2.0)
    d = gu.to(DEV)
    q, s = bb.swiglu_quantize(d[:, :cols], d[:, cols:])
    check_swiglu(q, s, gu[:, :cols], gu[:, cols:])
    q2, s2 = bb.swiglu_quantize(strided(gu[:, :cols], 7, 3), strided(gu[:, cols:], 2, 1))
    assert torch.equal(q, q2) and torch.equal(s, s2)


@pytest.mark.gpu
def test_ties_go_to_the_even_code():
    """Rows whose values meet a border exactly: half the maximum is 63.5 codes, (2 j + 1) / 254 of it j + 0.5."""
    top = 254.0
    x = torch.tensor([[top] + [float(2 * j + 1) for j in range(127)] + [-float(2 * j + 1) for j in range(126)]])
    for dtype in TYPES.values():
        for factor in (1.0, 2.0 ** -9, 2.0 ** 7):
            y = (x * factor).to(dtype)
            q, s = bb.quantize_rows(y.to(DEV))
            check_codes(q, s, y.double())
            assert q[0, 0] == 127 and q[0, 1] == 0 and q[0, 2] == 2 and q[0, 128] == 0
            q, _ = bb.rmsnorm_quantize(y.to(DEV), torch.full((254,), 3.0, dtype=dtype, device=DEV), 0.0)
            assert torch.equal(q.cpu(), formula(y.double())[0])


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [40, 4096, 40000])
def test_extreme_rows(cols):
    """Zeros, one value, the type's largest and smallest values, infinities and NaN: rows beside them are as ever."""
    for name, dtype in TYPES.items():
        big, tiny = torch.finfo(dtype).max, torch.finfo(dtype).tiny
        x = rnd(9, 8, cols, name)
        x[1] = 0
        x[2] = 0
        x[2, cols // 2] = -3
        x[3, 0], x[3, 1] = big, -big
        x[4] *= tiny
        x[5, cols - 1] = float("inf")
        x[6, 1] = float("nan")
        q, s = bb.quantize_rows(x.to(DEV))
        check_codes(q, s, x.double())
        assert s[1] == 0 and (q[1] == 0).all() and q[2, cols // 2] == -127 and torch.isnan(s[5]) and torch.isnan(s[6]) and (q[5] == 0).all()
        gain = torch.ones(cols, dtype=dtype)
        q, s = bb.rmsnorm_quantize(x.to(DEV), gain.to(DEV), 1e-6)
        check_norm(q, s, x, gain, 1e-6)
        gain[3] = float("nan")
        q, s = bb.rmsnorm_quantize(x.to(DEV), gain.to(DEV), 1e-6)
        assert torch.isnan(s).all() and (q == 0).all()
        gate = x.clone()
        gate[5, cols - 1], gate[6, 1] = float("-inf"), -200.0        # -inf / (1 + inf) is NaN; -200 / (1 + exp 200) is next to nothing
        gate[3] = 0
        up = rnd(10, 8, cols, name)
        q, s = bb.swiglu_quantize(gate.to(DEV), up.to(DEV))
        keep = [0, 1, 2, 3, 6, 7]
        check_swiglu(q[keep], s[keep], gate[keep], up[keep])
        assert torch.isnan(s[5]) and (q[5] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [6, 40, 700, 4096, 40000])
@pytest.mark.parametrize("dtype", TYPES)
def test_norm_of_rows_whose_products_leave_fp32(cols, dtype):
    """Gains by which h * gain overflows or underflows fp32 while the norm itself does not; with the sum over x or the residual, and rows
    of zeros between them."""
    t = TYPES[dtype]
    x, r = rnd(60 + cols, 5, cols, dtype), rnd(61 + cols, 5, cols, dtype)
    if dtype == "fp16":
        gain, by = rnd(62, 1, cols, dtype)[0] * 2.0 ** -12, 2.0 ** -10
    else:
        gain, by = (rnd(62, 1, cols, dtype)[0].float() * 1e-25).to(t), 1e-25
    x[1], r[1] = x[1] * by, r[1] * by
    x[2], r[2] = 0, 0
    for g, eps in ((gain, 0.0), (gain, 1e-5)) + (() if dtype == "fp16" else ((1 / gain.clamp(min=1e-27), 1e-5),)):
        if dtype != "fp16":
            x[3] = x[3] * 1e13 if g is not gain else x[3]
        h = (x.float() + r.float()).to(t)
        if eps == 0.0:
            keep = [0, 1, 3, 4]                 # (0 / 0 of the row of zeros is NaN in the formula too)
        else:
            keep = [0, 1, 2, 3, 4]
        over, into = x.to(DEV), r.to(DEV)
        q, s = bb.rmsnorm_quantize(over, g.to(DEV), eps, residual=into, residual_out=over)
        q2, s2 = bb.rmsnorm_quantize(x.to(DEV), g.to(DEV), eps, residual=into)
        assert torch.equal(over.cpu(), h) and torch.equal(into.cpu(), h) and torch.equal(q, q2) and torch.equal(s.view(torch.int32), s2.view(torch.int32))
        check_norm(q[keep], s[keep], h[keep], g, eps)


@pytest.mark.gpu
def test_more_rows_than_one_launch_holds():
    rows = (1 << 21) + 3
    x = (torch.arange(rows * 8, device=DEV) % 509 - 254).view(rows, 8).float()
    q, s = bb.quantize_rows(x)
    top = x.abs().amax(1).double()
    assert torch.equal(s, (top / 127).float())
    assert torch.equal(q, torch.round(127 * x.double() / top[:, None]).to(torch.int8))


def codes(seed, rows, cols):
    return torch.randint(-128, 128, (rows, cols), generator=gen(seed), dtype=torch.int16).to(torch.int8)


def check_gemm(out, a, sa, w, sw, bias):
    acc = a.double() @ w.double().t()           # (exact: integers below 2^53)
    scaled = acc * sa.double()[:, None] * sw.double()
    want = scaled if bias is None else scaled + bias.double()
    half = torch.finfo(out.dtype).eps / 2
    size = scaled.abs() + (0 if bias is None else bias.double().abs())
    tol = 4 * 2.0 ** -24 * size + (half if out.dtype != torch.float32 else 0) * want.abs() * (1 + 2.0 ** -20) + (2.0 ** -25 if out.dtype == torch.float16 else 2.0 ** -149)
    err = (out.cpu().double() - want).abs()
    assert (err <= tol).all(), f"worst {(err / tol).max().item()} of the tolerance"


GEMMS = [(1, 1, 1), (1, 64, 64), (1, 33, 17), (2, 5, 130), (7, 48, 1000), (16, 256, 688), (17, 100, 64), (31, 130, 4096), (33, 63, 257), (56, 768, 256),
         (64, 64, 63), (65, 129, 65), (120, 512, 1536), (128, 128, 128), (129, 260, 1040), (250, 96, 5000), (256, 512, 512), (257, 513, 520),
         (300, 1000, 333), (512, 768, 2048), (640, 1300, 704), (1, 4096, 18944), (3, 24576, 96), (2000, 40, 100), (1030, 1026, 1111)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", GEMMS)
def test_gemm_int8_against_the_exact_product(M, N, K, dtype):
    a, w = codes(M + K, M, K), codes(N + K, N, K)
    sa, sw, bias = torch.rand(M, generator=gen(1)) * 0.02, torch.rand(N, generator=gen(2)) * 0.001, torch.randn(N, generator=gen(3))
    if dtype == "fp16":
        sw = sw * min(1.0, 50.0 / K)            # (fp16 ends at 65504)
    t = TYPES[dtype]
    da, dw, dsa, dsw, db = (x.to(DEV) for x in (a, w, sa, sw, bias))
    check_gemm(bb.gemm_int8(da, dsa, dw, dsw, dtype=t), a, sa, w, sw, None)
    # strided operands at odd offsets, a bias, rows of a wider output whose gaps stay
    base = torch.full((M + 2, N + 3), 7.0, dtype=t, device=DEV)
    bb.gemm_int8(strided(a, 11, 3), dsa, strided(w, 5, 1), dsw, bias=db, out=base[1:M + 1, 2:N + 2])
    check_gemm(base[1:M + 1, 2:N + 2], a, sa, w, sw, bias)
    base[1:M + 1, 2:N + 2] = 7
    assert (base == 7).all()
    # rows at multiples of 16 bytes with something in the gaps
    pad = 16 - K % 16 if K % 16 else 16
    out = bb.gemm_int8(strided(a, pad), dsa, strided(w, pad), dsw, bias=db, dtype=t)
    check_gemm(out, a, sa, w, sw, bias)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,bias", [("bf16", True), ("fp32", False), ("fp16", True)])
@pytest.mark.parametrize("M,N,K", [
    (2047, 8190, 4100),                         # 256 x 256 tiles
    (511, 24570, 1030), (767, 3582, 18950),     # 256 x 192, k whole and in four
    (2999, 5001, 1200), (271, 8117, 19000),     # 128 x 128, and k in two; several tiles per workgroup
    (897, 4096, 12290), (199, 4610, 8200),      # 128 x 128 with the deeper ring, k whole and in three
    (549, 4094, 1100),
    (2600, 7700, 260), (119, 4090, 12300),      # 128 x 64, and k in four
    (255, 1023, 8193),                          # 64 x 64, k in four
    (15, 1022, 8200), (1, 24576, 1040),         # 32 x 32, k in eight and whole
])
def test_gemm_int8_every_tile_and_split(M, N, K, dtype, bias):
    """Large enough for each of the tiles, with ragged rows, columns and k; on the GPU in 64 bits (integers below 2^53: exact)."""
    g = torch.Generator(device=DEV).manual_seed(M + N + K)
    ld = (K + 15) // 16 * 16
    a, w = (torch.randint(-128, 128, (rows, ld), generator=g, device=DEV, dtype=torch.int8)[:, :K] for rows in (M, N))
    sa, sw = torch.rand(M, generator=g, device=DEV) * 0.02, torch.rand(N, generator=g, device=DEV) * (0.5 / K)
    b = torch.randn(N, generator=g, device=DEV) if bias else None
    base = torch.full((M + 1, N + 5), 7.0, dtype=TYPES[dtype], device=DEV)
    out = base[:M, 3:N + 3]
    bb.gemm_int8(a, sa, w, sw, bias=b, out=out)
    scaled = torch.mm(a.double(), w.double().t().contiguous()) * sa.double()[:, None] * sw.double()
    want, size = scaled, scaled.abs()
    if bias:
        want, size = want + b.double(), size + b.double().abs()
    half = 0.0 if dtype == "fp32" else torch.finfo(out.dtype).eps / 2 * (1 + 2.0 ** -20)
    assert ((out.double() - want).abs() <= 4 * 2.0 ** -24 * size + half * want.abs() + (2.0 ** -25 if dtype == "fp16" else 2.0 ** -149)).all()
    base[:M, 3:N + 3] = 7
    assert (base == 7).all()


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 40, 300])
def test_gemm_int8_longest_sum_and_bad_scales(M):
    """131071 products of -128 by -128 (just below 2^31) and by 127; a row whose scale is NaN stays a row of NaN, beside others."""
    K, N = 131071, 40
    a, w = torch.full((M, K), -128, dtype=torch.int8), torch.full((N, K), -128, dtype=torch.int8)
    w[1::2] = 127
    sa, sw = torch.rand(M, generator=gen(1)) * 1e-3, torch.rand(N, generator=gen(2)) * 1e-3
    check_gemm(bb.gemm_int8(a.to(DEV), sa.to(DEV), w.to(DEV), sw.to(DEV), dtype=torch.float32), a, sa, w, sw, None)
    sa[M // 2] = float("nan")
    out = bb.gemm_int8(a.to(DEV), sa.to(DEV), w.to(DEV), sw.to(DEV))
    assert torch.isnan(out[M // 2]).all() and torch.isnan(out).sum() == N


def ffn_weights(d, f, seed):
    return [rnd(seed + i, *shape, "bf16", 0.05) for i, shape in enumerate(((2 * f, d), (d, f)))]


@pytest.mark.gpu
@pytest.mark.parametrize("rows", [1, 56, 300])
@pytest.mark.parametrize("dtype", ["bf16", "fp32"])
def test_feed_forward_in_eight_bits(rows, dtype):
    """norm -> gate/up product -> SwiGLU -> down product -> next norm, each step's own input taken for its reference."""
    d, f, t = 256, 688, TYPES[dtype]
    w1, w2 = ffn_weights(d, f, 20)
    x, res, gain = rnd(30, rows, d, dtype), rnd(31, rows, d, dtype), rnd(32, 1, d, dtype)[0]
    q1, s1 = bb.quantize_rows(w1.to(DEV))
    q2, s2 = bb.quantize_rows(w2.to(DEV))
    check_codes(q1, s1, w1.double())
    h = res.to(DEV)
    q, s = bb.rmsnorm_quantize(x.to(DEV), gain.to(DEV), 1e-5, residual=h)
    check_norm(q, s, (x.float() + res.float()).to(t), gain, 1e-5)
    gu = bb.gemm_int8(q, s, q1, s1, dtype=t)
    check_gemm(gu, q.cpu(), s.cpu(), q1.cpu(), s1.cpu(), None)
    qa, sa = bb.swiglu_quantize(gu[:, :f], gu[:, f:])
    check_swiglu(qa, sa, gu.cpu()[:, :f], gu.cpu()[:, f:])
    y = bb.gemm_int8(qa, sa, q2, s2, dtype=t)
    check_gemm(y, qa.cpu(), sa.cpu(), q2.cpu(), s2.cpu(), None)
    before = h.cpu()
    q, s = bb.rmsnorm_quantize(y, gain.to(DEV), 1e-5, residual=h)
    check_norm(q, s, (y.cpu().float() + before.float()).to(t), gain, 1e-5)


@pytest.mark.gpu
def test_capture_replay_and_another_stream():
    """The feed-forward captured into a graph and replayed with new inputs between eager calls; then on a stream of its own."""
    d, f, rows = 256, 688, 40
    w1, w2 = (bb.quantize_rows(w.to(DEV)) for w in ffn_weights(d, f, 40))
    gain = rnd(41, 1, d, "bf16")[0].to(DEV)
    x, res = torch.zeros(rows, d, dtype=torch.bfloat16, device=DEV), torch.zeros(rows, d, dtype=torch.bfloat16, device=DEV)
    h = torch.empty_like(res)

    def ffn(stream=None):
        q, s = bb.rmsnorm_quantize(x, gain, 1e-5, residual=res, residual_out=h, stream=stream)
        gu = bb.gemm_int8(q, s, *w1, stream=stream)
        return bb.gemm_int8(*bb.swiglu_quantize(gu[:, :f], gu[:, f:], stream=stream), *w2, stream=stream)

    ffn()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        y = ffn()
    for seed in (50, 51, 52):
        x.copy_(rnd(seed, rows, d, "bf16"))
        res.copy_(rnd(seed + 10, rows, d, "bf16"))
        want, hw = ffn(), h.clone()
        torch.cuda.synchronize()
        h.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(h, hw)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = ffn(side)
    torch.cuda.current_stream().wait_stream(side)
    assert torch.equal(got, want)


@pytest.mark.gpu
def test_two_streams_at_once():
    """Products whose k is split, on two streams together: each has its own partial sums."""
    M, N, K = 120, 2048, 8192
    g = torch.Generator(device=DEV).manual_seed(9)
    sides = []
    for _ in range(2):
        a, w = (torch.randint(-128, 128, (n, K), generator=g, device=DEV, dtype=torch.int8) for n in (M, N))
        sides.append((a, torch.rand(M, generator=g, device=DEV), w, torch.rand(N, generator=g, device=DEV)))
    want = [bb.gemm_int8(*s, dtype=torch.float32) for s in sides]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    for st in streams:
        st.wait_stream(torch.cuda.current_stream())
    got = [[], []]
    for _ in range(20):
        for i, st in enumerate(streams):
            got[i].append(bb.gemm_int8(*sides[i], dtype=torch.float32, stream=st))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in range(2) for o in got[i])


def fake(*shape, dtype=torch.float32):
    return torch.zeros(*shape, dtype=dtype)


def test_cpu_tensors_are_refused():
    """There is no CPU fallback."""
    with pytest.raises(BBError):
        bb.quantize_rows(fake(2, 8))
    with pytest.raises(BBError):
        bb.rmsnorm_quantize(fake(2, 8), fake(8), 1e-5)
    with pytest.raises(BBError):
        bb.swiglu_quantize(fake(2, 8), fake(2, 8))
    with pytest.raises(BBError):
        bb.gemm_int8(fake(2, 8, dtype=torch.int8), fake(2), fake(4, 8, dtype=torch.int8), fake(4))


def test_the_library_refuses_malformed_arguments_on_the_host():
    import ctypes as C
    from paper_2605_29233_amd.binding import load_library
    lib = load_library()
    p = 4096                                    # never dereferenced: every call below is refused first, or has no rows
    bf16, bad = 1, 3
    ok = dict(x=p, ldx=64, q=p, ldq=64, scale=p, rows=2, cols=64, type=bf16)

    def rows(**kw):
        a = dict(ok, **kw)
        return lib.bb_quantize_rows(a["x"], a["ldx"], a["q"], a["ldq"], a["scale"], a["rows"], a["cols"], a["type"], None)

    def norm(res=None, ldr=64, h=None, ldh=64, gain=p, eps=1e-5, **kw):
        a = dict(ok, **kw)
        return lib.bb_rmsnorm_quantize(a["x"], a["ldx"], res, ldr, h, ldh, gain, eps, a["q"], a["ldq"], a["scale"], a["rows"], a["cols"], a["type"], None)

    def swiglu(up=p, ldu=64, **kw):
        a = dict(ok, **kw)
        return lib.bb_swiglu_quantize(a["x"], a["ldx"], up, ldu, a["q"], a["ldq"], a["scale"], a["rows"], a["cols"], a["type"], None)

    for f in (rows, norm, swiglu):
        for kw in (dict(x=None), dict(q=None), dict(scale=None), dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=-4), dict(type=bad), dict(type=-1),
                   dict(ldq=63), dict(ldx=-1), dict(x=p + 1), dict(scale=p + 2), dict(x=p + 2, type=0)):
            assert f(**kw) == -1, (f, kw)
        assert f(rows=0) == 0
    for kw in (dict(gain=None), dict(gain=p + 1), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(res=p), dict(h=p), dict(res=p, h=p, ldh=63),
               dict(res=p, h=p, ldr=-1), dict(res=p + 1, h=p), dict(res=p, h=p + 1)):
        assert norm(**kw) == -1, kw
    for kw in (dict(up=None), dict(up=p + 1), dict(ldu=-1)):
        assert swiglu(**kw) == -1, kw

    ok2 = dict(A=p, lda=64, sa=p, W=p, ldw=64, sw=p, bias=None, C=p, ldc=32, type=bf16, M=2, N=32, K=64, ws=None, nws=0)

    def gemm(**kw):
        return lib.bb_gemm_int8(*dict(ok2, **kw).values(), None)

    for kw in (dict(A=None), dict(sa=None), dict(W=None), dict(sw=None), dict(C=None), dict(M=-1), dict(N=-1), dict(K=0), dict(K=131072), dict(type=bad), dict(lda=-1),
               dict(ldw=-1), dict(ldc=31), dict(sa=p + 1), dict(sw=p + 2), dict(bias=p + 1), dict(C=p + 1), dict(C=p + 2, type=0)):
        assert gemm(**kw) == -1, kw
    assert gemm(M=0) == 0 and gemm(N=0, ldc=0) == 0
    # a workspace that is missing, too small or misaligned
    big = dict(M=120, N=4096, K=12288, lda=12288, ldw=12288, ldc=4096)
    need = lib.bb_gemm_int8_workspace_bytes(120, 4096, 12288, 1)
    assert need > 0 and gemm(**big) == -3 and gemm(**big, ws=p, nws=need - 1) == -3 and gemm(**big, ws=p + 8, nws=need) == -1
    odd = lib.bb_gemm_int8_workspace_bytes(120, 4096, 12288, 0)
    assert odd >= need + (120 + 4096) * 12288 and gemm(**dict(big, lda=12289), ws=p, nws=odd - 1) == -3
    for sizes in ((-1, 5, 5), (0, 0, 0), (0, 8, 8), (5, 5, 0), (5, 5, 131072), ((1 << 30) + 1, 5, 5)):
        assert lib.bb_gemm_int8_workspace_bytes(*sizes, 1) == 0 and lib.bb_gemm_int8_workspace_bytes(*sizes, 0) == 0


@pytest.mark.gpu
def test_the_binding_refuses_what_does_not_fit():
    x, q, s, gain = fake(4, 64).to(DEV), fake(4, 64, dtype=torch.int8).to(DEV), fake(4).to(DEV), fake(64).to(DEV)
    for call in (lambda: bb.quantize_rows(x[0]), lambda: bb.quantize_rows(x.double()), lambda: bb.quantize_rows(x.t()), lambda: bb.quantize_rows(x, out=q[:3]),
                 lambda: bb.quantize_rows(x, out=x), lambda: bb.quantize_rows(x, scale=s[:3]), lambda: bb.quantize_rows(x, scale=s.half()),
                 lambda: bb.quantize_rows(x, out=q[:1].expand(4, 64)), lambda: bb.quantize_rows(x, scale=s.cpu()),
                 lambda: bb.rmsnorm_quantize(x, gain.half(), 1e-5), lambda: bb.rmsnorm_quantize(x, gain[:8], 1e-5), lambda: bb.rmsnorm_quantize(x, gain, -1.0),
                 lambda: bb.rmsnorm_quantize(x, gain, 1e-5, residual=x.half()), lambda: bb.rmsnorm_quantize(x, gain, 1e-5, residual_out=x),
                 lambda: bb.rmsnorm_quantize(x, gain, 1e-5, residual=x[:2]), lambda: bb.swiglu_quantize(x, x[:2]), lambda: bb.swiglu_quantize(x, x.half()),
                 lambda: bb.gemm_int8(q, s, q[:, :32], s), lambda: bb.gemm_int8(x, s, q, s), lambda: bb.gemm_int8(q, s[:2], q, s), lambda: bb.gemm_int8(q, s, q, s[:2]),
                 lambda: bb.gemm_int8(q, s, q, s, bias=s.half()), lambda: bb.gemm_int8(q, s, q, s, out=x), lambda: bb.gemm_int8(q, s, q, s, dtype=torch.float64),
                 lambda: bb.gemm_int8(q, s, q, s, out=x[:, :4], dtype=torch.bfloat16), lambda: bb.gemm_int8(q.t(), s, q.t(), s)):
        with pytest.raises(BBError):
            call()
    # nothing to do: empty results, nothing launched
    assert bb.quantize_rows(x[:0])[0].shape == (0, 64) and bb.gemm_int8(q[:0], s[:0], q, s).shape == (0, 4) and bb.gemm_int8(q, s, q[:0], s[:0]).shape == (4, 0)
    # rows that overlap may be read: one row seen four times
    one = x[:1].expand(4, 64)
    assert torch.equal(bb.quantize_rows(one)[1], s)
