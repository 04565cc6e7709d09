"""The forward with its layers' products in 8-bit integers (bb_int8_layers): against the same operators called one by one, against the
oracle with every projection's operands quantised, switching it on, off and over, and what it refuses."""
import ctypes as C

import numpy as np
import pytest
import torch

import paper_2605_29233_amd as pkg
from paper_2605_29233_amd import BB_INIT, BB_PERIODIC, BBError, BlockBatch, Limits
from paper_2605_29233_amd.binding import load_library
from oracle.blockbatch import OracleRequest
from oracle.model import OracleModel
from workload import workload, gen_weights, gen_prompt
from workload.configs import DecodeParams, ModelShape, TINY, scaled

pytestmark = pytest.mark.gpu

GQA = ModelShape("int8_gqa", 2, 192, 4, 2, 64, 208, 512, qkv_bias=True, lm_std=0.5)      # d_ffn no multiple of 32 or 64


def make(model, weights, prompt, gen_len, blocks, decode=DecodeParams(), int8=True, poison=False, requests=1):
    bb = BlockBatch(model, decode, Limits(requests, len(blocks), len(prompt) + gen_len, gen_len, requests * sum(blocks)), poison_workspace=poison)
    bb.load_weights(weights.items())
    bb.keep_logits(True)
    if int8:
        bb.int8_layers()
    return bb, bb.request_open(prompt, gen_len, blocks)


def matrix(weights, names):
    return pkg.quantize_rows(torch.cat([weights[n] for n in names]).cuda().contiguous())


def layer0_qkv(weights, tokens, model):
    """(rows of the embedding stream, q|k|v of layer 0) by the operators."""
    emb = weights["tok_emb"].cuda()[torch.as_tensor(tokens, device="cuda").long()].float()
    q, s = pkg.rmsnorm_quantize(emb, weights["l0.attn_norm"].cuda().float().reshape(-1), model.rms_eps)
    bias = torch.cat([weights[f"l0.b{c}"].reshape(-1) for c in "qkv"]).cuda().float() if model.qkv_bias else None
    return emb, pkg.gemm_int8(q, s, *matrix(weights, ["l0.wq", "l0.wk", "l0.wv"]), bias=bias, dtype=torch.float32)


@pytest.mark.parametrize("model,prompt_len,gen_len,blocks", [(TINY, 64, 64, (8, 16, 32)), (GQA, 37, 27, (5, 13)), (scaled(TINY, n_layers=1), 900, 300, (32,))])
def test_first_layer_equals_the_operators(model, prompt_len, gen_len, blocks):
    """V of layer 0 after the initial forward: norm, product and bias as the operators give them, kept as two fp16 terms (2^-21 of
    the value, and 2^-24 where the second is subnormal)."""
    weights = dict(gen_weights(model, 3))
    prompt = gen_prompt(model, 3, 0, prompt_len)
    bb, rid = make(model, weights, prompt, gen_len, blocks)
    bb.refresh([rid], BB_INIT)
    _, V = bb.get_kv(rid, len(blocks) - 1, 0)
    tokens = np.concatenate([prompt, np.full(gen_len, model.mask_id)])
    _, qkv = layer0_qkv(weights, tokens, model)
    nkv = model.n_kv_heads * model.head_dim
    want = qkv[:, -nkv:].double().cpu().numpy()
    got = V.reshape(len(tokens), nkv).astype(np.float64)
    assert (np.abs(got - want) <= 2.0 ** -21 * np.abs(want) + 2.0 ** -24).all()
    bb.close()


def test_feed_forward_equals_the_operators():
    """With an output projection of zeros the residual stream after one layer is the embedding plus the feed-forward, which the operators
    give bit for bit; the logits then differ by the LM head's two bf16 terms (2^-17 of each product, summed) and fp32 sums."""
    model = scaled(TINY, n_layers=1)
    weights = dict(gen_weights(model, 5))
    weights["l0.wo"] = torch.zeros_like(weights["l0.wo"])
    prompt, gen_len = gen_prompt(model, 5, 0, 40), 24
    bb, rid = make(model, weights, prompt, gen_len, (8,))
    bb.refresh([rid], BB_INIT)
    got = bb.latest_view().logits().astype(np.float64)
    f = model.d_ffn
    h = weights["tok_emb"].cuda()[torch.full((gen_len,), model.mask_id).cuda()].float()
    q, s = pkg.rmsnorm_quantize(torch.zeros_like(h), weights["l0.ffn_norm"].cuda().float().reshape(-1), model.rms_eps, residual=h)
    gu = pkg.gemm_int8(q, s, *matrix(weights, ["l0.w_gate", "l0.w_up"]), dtype=torch.float32)
    qa, sa = pkg.swiglu_quantize(gu[:, :f], gu[:, f:])
    h = (h + pkg.gemm_int8(qa, sa, *matrix(weights, ["l0.w_down"]), dtype=torch.float32)).double().cpu()
    y = h / torch.sqrt(h.square().mean(1, keepdim=True) + model.rms_eps) * weights["final_norm"].double().reshape(-1)
    w = weights["lm_head"].double()
    want, size = (y @ w.t()).numpy(), (y.abs() @ w.abs().t()).numpy()
    assert (np.abs(got - want)[:, :-1] <= (2.0 ** -16 * size)[:, :-1]).all()
    bb.close()


def quantised(x):
    top = np.abs(x).max(-1, keepdims=True)
    q = np.rint(127 * x / np.where(top == 0, 1, top))
    return q * (top / 127).astype(np.float32).astype(np.float64)


class Int8Oracle(OracleModel):
    """The oracle with both operands of every projection of the layers quantised by rows."""

    def __init__(self, shape, weights):
        super().__init__(shape, weights)
        for k in self.w:
            if k[0] == "l" and k.rsplit(".", 1)[-1] in ("wq", "wk", "wv", "wo", "w_gate", "w_up", "w_down"):
                self.w[k] = quantised(self.w[k])

    def forward_rows(self, tokens, pos, cacheK, cacheV, seq_len, want_hidden=True):
        s, w, T = self.s, self.w, len(pos)
        h = w["tok_emb"][tokens].astype(self.dtype)
        for i in range(s.n_layers):
            p = f"l{i}."
            n1 = quantised(self.rmsnorm(h, w[p + "attn_norm"]))
            q, k, v = n1 @ w[p + "wq"].T, n1 @ w[p + "wk"].T, n1 @ w[p + "wv"].T
            if s.qkv_bias:
                q, k, v = q + w[p + "bq"], k + w[p + "bk"], v + w[p + "bv"]
            cacheK[i][pos] = self.rope(k.reshape(T, s.n_kv_heads, s.head_dim), pos)
            cacheV[i][pos] = v.reshape(T, s.n_kv_heads, s.head_dim)
            if i == s.n_layers - 1 and not want_hidden:
                return None
            a, _ = self.attention(self.rope(q.reshape(T, s.n_q_heads, s.head_dim), pos), cacheK[i][:seq_len], cacheV[i][:seq_len])
            h = h + quantised(a) @ w[p + "wo"].T
            n2 = quantised(self.rmsnorm(h, w[p + "ffn_norm"]))
            g, u = n2 @ w[p + "w_gate"].T, n2 @ w[p + "w_up"].T
            h = h + quantised((g / (1.0 + np.exp(-g))) * u) @ w[p + "w_down"].T
        return h


def rms(a, b=None):
    """Of a's logits, or of their difference to b's (the mask's column, which no token takes, aside)."""
    a = a[:, :-1] if b is None else a[:, :-1] - b[:, :-1]
    return float(np.sqrt(np.mean(np.square(a))))


@pytest.mark.parametrize("model,prompt_len,gen_len,blocks", [(TINY, 64, 64, (8, 16, 32)), (GQA, 37, 27, (5, 13))])
def test_logits_against_the_oracle_with_quantised_projections(model, prompt_len, gen_len, blocks):
    """Initial forward, then a block step from the same tokens and windows.  The rows that the GPU quantises differ from the oracle's by
    fp32 and fp16 roundings, so some codes fall the other way, and each such code moves the next rows.  At worst all roundings
    are independent: then the two sides differ by sqrt(2) of what quantisation moves the logits by (measured between the oracles; a tenth
    is added for the finite sample).  A wrong scale, order or operand moves them by their whole size."""
    weights = dict(gen_weights(model, 7))
    prompt = gen_prompt(model, 7, 0, prompt_len)
    bb, rid = make(model, weights, prompt, gen_len, blocks)
    om, op = (OracleRequest(M(model, weights), prompt, gen_len, blocks, DecodeParams()) for M in (Int8Oracle, OracleModel))
    f8, f = om.init_forward(), op.init_forward()
    bb.refresh([rid], BB_INIT)
    v = bb.latest_view()
    moved = rms(f8.logits, f.logits)
    assert 0 < rms(v.logits(), f8.logits) <= 1.1 * 2 ** 0.5 * moved
    assert moved < 0.2 * rms(f.logits)
    om.commit_merge()
    bb.merge_commit([rid])
    bb.set_state(rid, om.X, om.br)
    s8 = om.block_forward()
    op.X[:] = om.X
    for a, b in zip(op.br, om.br):
        a.start, a.end, a.done = b.start, b.end, b.done
    s = op.block_forward()
    v = bb.denoise_step([rid])
    assert v.m_lm == len(s8.pos) and s.logits.shape == s8.logits.shape
    assert rms(v.logits(), s8.logits) <= 1.1 * 2 ** 0.5 * rms(s8.logits, s.logits)
    bb.close()


def test_on_off_and_reloaded_weights():
    model = GQA
    a, b = dict(gen_weights(model, 1)), dict(gen_weights(model, 2))
    prompt, gen_len, blocks = gen_prompt(model, 1, 0, 50), 30, (8, 16)

    def logits(bb, rid):
        bb.refresh([rid], BB_PERIODIC)
        return bb.denoise_step([rid]).logits()

    def fresh(weights, int8, poison=False):
        bb, rid = make(model, weights, prompt, gen_len, blocks, int8=int8, poison=poison)
        bb.refresh([rid], BB_INIT)
        out = logits(bb, rid)
        bb.close()
        return out

    plain, int8, other = fresh(a, False), fresh(a, True), fresh(b, True)
    assert not np.array_equal(plain, int8) and not np.array_equal(int8, other)
    assert np.array_equal(int8, fresh(a, True, poison=True))        # nothing is taken from what the memory held
    bb, rid = make(model, a, prompt, gen_len, blocks, int8=False)
    bb.refresh([rid], BB_INIT)
    assert np.array_equal(logits(bb, rid), plain)
    bb.int8_layers()
    bb._i8.fill_(0xFF)
    torch.cuda.synchronize()
    assert np.array_equal(logits(bb, rid), int8)
    bb.int8_layers(False)
    assert np.array_equal(logits(bb, rid), plain)
    bb.int8_layers()
    bb.int8_layers()                            # other memory
    assert np.array_equal(logits(bb, rid), int8)
    bb.load_weights(b.items())                  # the codes follow the weights
    assert np.array_equal(logits(bb, rid), other)
    bb.close()


def test_a_decode_runs_to_its_end():
    w = workload("tiny")
    weights = dict(gen_weights(w.model, w.seed))
    prompts = [gen_prompt(w.model, w.seed, i, n) for i, n in enumerate((64, 33))]
    bb = BlockBatch(w.model, w.decode, Limits(2, len(w.block_sizes), 64 + w.gen_len, w.gen_len, 2 * sum(w.block_sizes)))
    bb.load_weights(weights.items())
    bb.int8_layers()
    runs = []
    for _ in range(2):
        ids = [bb.request_open(p, w.gen_len, w.block_sizes) for p in prompts]
        st = bb.generate(ids)
        assert all(s.finished for s in st)
        runs.append([bb.get_tokens(i)[s.winner] for i, s in zip(ids, st)])
        for i in ids:
            bb.request_close(i)
    for x, y, p in zip(*runs, prompts):
        assert np.array_equal(x, y) and np.array_equal(x[:len(p)], p) and (x != w.model.mask_id).all()
    bb.close()


def test_refusals():
    lib = load_library()
    assert lib.bb_int8_layers_bytes(None) == 0 and lib.bb_int8_layers(None, None, 0) == -1
    model = scaled(TINY, n_layers=1)
    weights = dict(gen_weights(model, 1))
    bb, rid = make(model, weights, gen_prompt(model, 1, 0, 20), 12, (4,), int8=False)
    n = lib.bb_int8_layers_bytes(bb._ctx)
    assert n > sum(weights[k].numel() for k in weights if k.startswith("l0.w"))
    mem = torch.empty(n + 512, dtype=torch.uint8, device="cuda")
    base = (mem.data_ptr() + 255) // 256 * 256
    assert lib.bb_int8_layers(bb._ctx, C.c_void_p(base + 16), n) == -1
    assert lib.bb_int8_layers(bb._ctx, C.c_void_p(base), n - 1) == -3
    assert b"bb_int8_layers_bytes" in lib.bb_last_error(bb._ctx)
    bb.refresh([rid], BB_INIT)                  # nothing was switched on
    before = bb.latest_view().logits()
    other, rid2 = make(model, weights, gen_prompt(model, 1, 0, 20), 12, (4,), int8=False)
    other.refresh([rid2], BB_INIT)
    assert np.array_equal(before, other.latest_view().logits())
    bb.close()
    other.close()
    with pytest.raises(BBError):
        BlockBatch.int8_layers(bb)              # closed
