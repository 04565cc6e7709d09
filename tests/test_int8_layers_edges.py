"""The int8 layers at the edges: shapes whose sums would not be exact, codes that a captured forward has yet to make, attention's output on its way into the output
projection, and fewer live rows than a forward is sized for."""
import ctypes as C
import types

import numpy as np
import pytest
import torch

import paper_2605_29233_amd as pkg
from paper_2605_29233_amd import BB_INIT, BBError, BlockBatch, Limits
from paper_2605_29233_amd.binding import gemm_int8_plan, load_library
from test_int8_ops import check_codes, gen
from workload import gen_prompt, gen_weights
from workload.configs import TINY, DecodeParams, ModelShape

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d_ffn", [131056, 131072])
def test_sums_that_may_leave_int32_are_refused(d_ffn):
    """The product's own limit is 131071 terms; the down projection sums d_ffn of them.  (Nothing is run: the format is asked for only.)"""
    lib = load_library()
    bb = BlockBatch(ModelShape("longsum", 1, 64, 2, 2, 64, d_ffn, 256), DecodeParams(), Limits(1, 1, 48, 16, 16))
    n = lib.bb_int8_layers_bytes(bb._ctx)
    if d_ffn <= 131071:
        assert n > 3 * 64 * d_ffn
        bb.int8_layers()
        bb.int8_layers(False)
    else:
        assert n == 0
        mem = torch.empty(1 << 28, dtype=torch.uint8, device="cuda")
        assert lib.bb_int8_layers(bb._ctx, C.c_void_p((mem.data_ptr() + 255) // 256 * 256), (1 << 28) - 256) == -1
        assert b"BB_GEMM_INT8_MAX_K" in lib.bb_last_error(bb._ctx)
        with pytest.raises(BBError):
            bb.int8_layers()
    bb.close()


def test_a_captured_forward_does_not_count_as_having_made_the_codes():
    """A step captured right after the format is switched on, and an eager one before the graph runs; then replays between eager steps."""
    model, gen_len, blocks = TINY, 24, (4, 8)
    weights, prompt = dict(gen_weights(model, 11)), gen_prompt(model, 11, 0, 40)

    def make(stream=None):
        bb = BlockBatch(model, DecodeParams(), Limits(1, len(blocks), len(prompt) + gen_len, gen_len, sum(blocks)), stream=stream)
        bb.load_weights(weights.items())
        bb.keep_logits(True)
        rid = bb.request_open(prompt, gen_len, blocks)
        bb.refresh([rid], BB_INIT)
        bb.denoise_step([rid])                      # (the request's list is uploaded)
        bb.int8_layers()
        bb._i8.zero_()
        torch.cuda.synchronize()
        return bb, rid

    bb, rid = make()
    want = bb.denoise_step([rid]).logits()
    bb.close()
    bb, rid = make(torch.cuda.Stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=bb._stream):
        bb.denoise_step([rid], want_view=False)
    assert np.array_equal(bb.denoise_step([rid]).logits(), want)
    X, branches = bb.get_tokens(rid), list(bb.get_stats(rid).branch)[:len(blocks)]
    seen = [want]
    for k in range(3):                              # other tokens each time, seen by the graph first
        X[:, :len(prompt)] = gen_prompt(model, 12 + k, 0, len(prompt))
        X[:, len(prompt):len(prompt) + 2] = 5 + k
        bb.set_state(rid, X, branches)
        graph.replay()
        torch.cuda.synchronize()
        replayed = bb.latest_view().logits()
        assert np.array_equal(bb.denoise_step([rid]).logits(), replayed)
        assert not any(s.shape == replayed.shape and np.array_equal(s, replayed) for s in seen)
        seen.append(replayed)
    bb.close()


def two_terms(x):
    """fp32 as the sum of two bf16 terms, in doubles (exact)."""
    hi = x.to(torch.bfloat16).float()
    return hi.double() + (x - hi).to(torch.bfloat16).double()


@pytest.mark.parametrize("rows,cols", [(1, 128), (31, 256), (33, 128), (70, 768), (200, 4096), (1100, 1024), (1030, 3584), (2, 16400)])
def test_rows_of_a_panel_equal_the_formula(rows, cols):
    """Codes and scales of the two-term values, for rows of every kind: ordinary, with borders met exactly, large, small, zero, infinite, NaN; rows past the live ones are
    left alone."""
    lib = load_library()
    x = torch.randn(rows, cols, generator=gen(rows + cols))
    kinds = [lambda r: r, lambda r: torch.round(r * 40) * 2.0 ** -9, lambda r: r * 1e30, lambda r: r * 1e-33, lambda r: r * 0, lambda r: torch.where(r > 3, r / 0, r), lambda r: r * 1e-3]
    for k, kind in enumerate(kinds):
        x[k::len(kinds)] = kind(x[k::len(kinds)])
    if rows > 20:
        x[9, 3] = float("nan")
        x[11, cols // 2:] = 0
    dx = x.cuda()
    nbytes = (rows + 31) // 32 * 32 * ((cols + 63) // 64 * 64) * 4
    panel, live = torch.empty(nbytes, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    for n in (None, rows, rows // 2, 0):
        q, scale = torch.full((rows, cols), 55, dtype=torch.int8, device="cuda"), torch.full((rows,), -1.0, device="cuda")
        if n is not None:
            live.fill_(n)
        assert lib.bb_debug_panel_quantize(dx.data_ptr(), rows, cols, panel.data_ptr(), nbytes, q.data_ptr(), scale.data_ptr(), None if n is None else live.data_ptr(),
                                           torch.cuda.current_stream().cuda_stream) == 0
        n = rows if n is None else n
        check_codes(q[:n], scale[:n], two_terms(x)[:n])
        assert (q[n:] == 55).all() and (scale[n:] == -1).all()
    for bad in (dict(rows=0), dict(cols=0), dict(cols=cols + 8), dict(panel=panel.data_ptr() + 8), dict(x=None), dict(q=None), dict(scale=None)):
        a = dict(dict(x=dx.data_ptr(), rows=rows, cols=cols, panel=panel.data_ptr(), n=nbytes, q=q.data_ptr(), scale=scale.data_ptr()), **bad)
        assert lib.bb_debug_panel_quantize(*a.values(), None, None) == -1, bad
    assert lib.bb_debug_panel_quantize(dx.data_ptr(), rows, cols, panel.data_ptr(), nbytes - 1, q.data_ptr(), scale.data_ptr(), None, None) == -3


def test_attention_output_through_its_codes_into_the_output_projection():
    """One layer whose queries are zero (attention is then the mean of V, which the cache holds), whose feed-forward gives nothing and whose LM head is the identity: the logits are
    the norm of embedding + O(codes of attention's output), in the initial forward and in a block step.

    Tolerance.  Attention adds 2 L fp32 terms in an order of its own and splits the result into two bf16 terms: off by at most delta = (2 L + 40) 2^-23 mean |V| + 2^-16 |a|.  Only
    codes within that of a border may fall the other way, by one: those, and the scale's delta / max, are counted column by column through the exact product.  The norm
    divides by the rms of the same values; the LM head's two bf16 terms are off by 2^-15.  Three forwards that a looser bound would let pass are
    measured against it too: one that does not quantise there, one that keeps a single bf16 term, and a scale off by a hundredth."""
    d, prompt_len, gen_len, blocks, n_req = 256, 10, 8, (4, 8), 6
    model = ModelShape("opath", 1, d, 4, 2, 64, 64, 512)
    weights = dict(gen_weights(model, 21))
    weights["l0.wq"] = torch.zeros_like(weights["l0.wq"])
    weights["l0.w_down"] = torch.zeros_like(weights["l0.w_down"])
    weights["l0.wo"] = weights["l0.wo"] * 16
    weights["lm_head"] = torch.eye(model.vocab, d).to(torch.bfloat16)
    weights["final_norm"] = (1 + torch.rand(d, generator=gen(4))).to(torch.bfloat16)
    L = prompt_len + gen_len
    bb = BlockBatch(model, DecodeParams(), Limits(n_req, len(blocks), L, gen_len, n_req * sum(blocks)), poison_workspace=True)
    bb.load_weights(weights.items())
    bb.keep_logits(True)
    bb.int8_layers()
    ids = [bb.request_open(gen_prompt(model, 21, i, prompt_len), gen_len, blocks) for i in range(n_req)]
    qo, so = (t.cpu().double() for t in pkg.quantize_rows(weights["l0.wo"].cuda()))
    emb, gain = weights["tok_emb"][model.mask_id].double(), weights["final_norm"].double().reshape(-1)

    def expected(rid, branch):
        V = torch.from_numpy(bb.get_kv(rid, branch, 0)[1]).double()                     # [L][kv heads][64]
        a, size = (t.repeat_interleave(2, 0).reshape(-1) for t in (V.mean(0), V.abs().mean(0)))
        delta = (2 * L + 40) * 2.0 ** -23 * size + 2.0 ** -16 * a.abs()

        def o_of(x, by=1.0):
            top = x.abs().max()
            return (qo @ torch.round(127 * x / top)) * so * (top / 127 * by)

        def y_of(o):
            h = emb + o
            return h / torch.sqrt(h.square().mean() + model.rms_eps) * gain

        top, at = a.abs().max(), a.abs().argmax()
        t, scale_off = 127 * a.abs() / top, delta.max() / top
        near = (t - torch.floor(t) - 0.5).abs() <= 127 * (delta / top + a.abs() / top * scale_off) * 1.01
        near[at] = False                                                                # (127 whatever its value)
        o = o_of(a)
        tol_o = (qo.abs() @ near.double()) * so * top / 127 * (1 + scale_off) + o.abs() * (scale_off + 2.0 ** -20)
        h, tol_h = emb + o, tol_o + 2.0 ** -23 * (emb.abs() + o.abs())
        ms = h.square().mean() + model.rms_eps
        ms_off = (2 * h.abs() * tol_h + tol_h.square()).mean() / ms
        y = y_of(o)
        tol = (tol_h * gain / torch.sqrt(ms)) * (1 + ms_off) + y.abs() * (ms_off + 2.0 ** -15) + 2.0 ** -30
        other = [y_of(qx) for qx in ((qo * so[:, None]) @ a, o_of(a.to(torch.bfloat16).double()), o_of(a, 1.01))]
        return y, tol, [((x - y).abs() > 2 * tol).double().mean().item() for x in other]

    seen = []
    for rid in ids:
        bb.refresh([rid], BB_INIT)
        y, tol, others = expected(rid, 0)
        rows = torch.from_numpy(bb.latest_view().logits()).double()
        assert rows.shape == (gen_len, model.vocab) and ((rows[:, :d] - y).abs() <= tol).all(), ((rows[:, :d] - y).abs() / tol).max()
        seen.append(others)
    seen = np.mean(seen, axis=0)
    print("share of outputs by which other forwards would be seen:", seen, flush=True)
    assert (seen > 0.3).all()
    view = bb.denoise_step(ids)
    got = torch.from_numpy(view.logits()).double()
    branch = view.rows()[0][view.lm_rows()]
    assert len(got) == n_req * sum(blocks)
    for row, gbr in zip(got, branch):
        y, tol, _ = expected(ids[gbr // len(blocks)], int(gbr % len(blocks)))
        assert ((row[:d] - y).abs() <= tol).all(), ((row[:d] - y).abs() / tol).max()
    bb.close()


@pytest.mark.parametrize("d_ffn", [8192, 688])
def test_fewer_live_rows_give_the_rows_that_are_left_their_results(d_ffn):
    """A step sized for 288 rows of which some branches have finished: the rows of the others keep their logits bit for bit, although they lie elsewhere in the products, whose tiles
    and k splits (twelve of the down projection with d_ffn 8192) are those of 288 rows."""
    model = ModelShape("int8live", 2, 256, 4, 2, 64, d_ffn, 512)
    blocks, gen_len, prompt_len = (32, 96, 160), 160, 24
    if d_ffn == 8192:
        assert gemm_int8_plan(288, 256, 8192)["split"] > 1 and gemm_int8_plan(288, 256, 8192)["bm"] < 288
    bb = BlockBatch(model, DecodeParams(), Limits(1, 3, prompt_len + gen_len, gen_len, sum(blocks)), poison_workspace=True)
    bb.load_weights(gen_weights(model, 31))
    bb.keep_logits(True)
    bb.int8_layers()
    bb._i8.fill_(0x5A)
    torch.cuda.synchronize()
    rid = bb.request_open(gen_prompt(model, 31, 0, prompt_len), gen_len, blocks)
    bb.refresh([rid], BB_INIT)
    X = bb.get_tokens(rid)
    X[:, prompt_len::3] = np.arange(len(X[0, prompt_len::3])) % 500             # some rows of every window are decoded already
    every = None
    for done in ((), (0,), (1,), (2,), (0, 1), (1, 2), (0, 2), (0, 1, 2), ()):
        bb.set_state(rid, X, [types.SimpleNamespace(start=prompt_len, end=prompt_len + b, done=k in done, mean_conf=0.5) for k, b in enumerate(blocks)])
        print("finished:", done, flush=True)
        view = bb.denoise_step([rid])
        assert view.m_q == sum(b for k, b in enumerate(blocks) if k not in done)
        if view.m_lm == 0:
            assert len(done) == 3
            continue
        gbr, pos = view.rows()
        at = view.lm_rows()
        rows = {(int(gbr[m]), int(pos[m])): logits for m, logits in zip(at, view.logits())}
        every = every or rows
        assert len(rows) == sum(g not in done for g, _ in every)
        for key, logits in rows.items():
            assert np.array_equal(logits, every[key]), (done, key)
    bb.close()
