"""The int8 layers at the edges: shapes whose sums would not be exact, and codes that a captured forward has yet to make."""
import ctypes as C

import numpy as np
import pytest
import torch

from paper_2605_29233_amd import BB_INIT, BBError, BlockBatch, Limits
from paper_2605_29233_amd.binding import load_library
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
