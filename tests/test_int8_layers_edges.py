"""The int8 layers at the edges: shapes whose sums would not be exact."""
import ctypes as C

import pytest
import torch

from paper_2605_29233_amd import BBError, BlockBatch, Limits
from paper_2605_29233_amd.binding import load_library
from workload.configs import DecodeParams, ModelShape

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
