"""Every body of the int8 product at every hand-over: workgroups that take several tiles (the next one's chunks and scales on their way while one is stored,
a ragged chunk followed by another tile, a tile of one chunk, a last round that not every XCD has work in), k splits and their join, and fewer live rows than the launch
is planned for; and which body the sizes of tests/test_int8_ops.py reach.

The reference is the integer product (exact in 64 bits), scaled: an exact integer rounded to fp32 and two products in fp32, 2^-24 of the value each."""
import pytest
import torch

from paper_2605_29233_amd.binding import gemm_int8_plan, load_library
from test_int8_ops import DEV

BODIES = [(256, 256, 1), (256, 192, 1), (128, 128, 2), (128, 128, 1), (128, 64, 2), (64, 64, 2), (32, 32, 3)]


def test_the_plans_of_the_sizes_that_stand_for_each_tile():
    """(256 x 192 by 2, and the others, as test_gemm_int8_every_tile_and_split says.)"""
    for M, N, K, body, split in (
            (2047, 8190, 4100, 0, 1), (511, 24570, 1030, 1, 1), (767, 3582, 18950, 1, 4), (2999, 5001, 1200, 2, 1), (271, 8117, 19000, 2, 2), (897, 4096, 12290, 3, 1),
            (199, 4610, 8200, 3, 3), (549, 4094, 1100, 3, 1), (2600, 7700, 260, 4, 1), (119, 4090, 12300, 4, 4), (255, 1023, 8193, 5, 4), (15, 1022, 8200, 6, 8),
            (1, 24576, 1040, 6, 1), (8192, 24576, 4096, 1, 1)):
        p = gemm_int8_plan(M, N, K)
        assert (p["body"], p["split"]) == (body, split) and (p["bm"], p["bn"], p["per_cu"]) == BODIES[body], (M, N, K, p)


def test_refusals():
    lib, p, M, N, K = load_library(), 4096, 300, 200, 1000
    ok = dict(A=p, sa=p, W=p, sw=p, ld=1008, C=p, M=M, N=N, K=K, body=2, split=2, live=None, ws=p, nws=1 << 30)
    for kw in (dict(A=None), dict(W=None), dict(sa=None), dict(sw=None), dict(C=None), dict(M=0), dict(N=0), dict(K=15), dict(ld=999), dict(ld=992), dict(body=-1), dict(body=len(BODIES)), dict(split=0),
               dict(split=9), dict(split=17, K=10000, ld=10000), dict(ws=None), dict(ws=p + 8), dict(A=p + 8)):
        assert lib.bb_debug_gemm_int8(*dict(ok, **kw).values(), None) == -1, kw
    assert lib.bb_debug_gemm_int8(*dict(ok, nws=3 * 2 * 2 * 128 * 128 * 4 - 1).values(), None) == -3
    for sizes in ((0, 5, 50), (5, 0, 50), (5, 5, 15), (5, 5, 131072)):
        with pytest.raises(ValueError):
            gemm_int8_plan(*sizes)


# rows, columns beyond one round of tiles (more than 256 times the workgroups per CU of them), and beyond two
SIZES = {0: (2500, 7100), 1: (2500, 5400), 2: (3000, 3300), 3: (2500, 2000), 4: (3000, 1500), 5: (1500, 1500), 6: (1100, 1000)}


@pytest.mark.gpu
@pytest.mark.parametrize("K,splits", [(16, (1,)), (100, (1,)), (128, (1,)), (200, (1, 2)), (1000, (1, 3)), (2176, (2, 16))])
@pytest.mark.parametrize("body", range(len(BODIES)))
def test_every_body_with_several_tiles_a_workgroup(body, K, splits):
    lib, (M, N), (bm, bn, per_cu) = load_library(), SIZES[body], BODIES[body]
    tiles = -(-M // bm) * -(-N // bn)
    assert tiles > 256 * per_cu
    g = torch.Generator(device=DEV).manual_seed(body * 10000 + K)
    ld = (K + 15) // 16 * 16 + 16 * (K % 3)
    a, w = (torch.randint(-128, 128, (rows, ld), generator=g, device=DEV, dtype=torch.int8) for rows in (M, N))
    sa, sw = torch.rand(M, generator=g, device=DEV) + 0.01, torch.rand(N, generator=g, device=DEV) * (1 / K)
    exact = torch.mm(a[:, :K].double(), w[:, :K].double().t().contiguous()) * sa.double()[:, None] * sw.double()
    live = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.empty(tiles * max(splits) * bm * bn * 4 if max(splits) > 1 else 16, dtype=torch.uint8, device=DEV)
    for split in splits:
        for rows in (None, M, M - 1, M // 2 + 1, bm + 1, bm, 1, 0):         # (live rows: whole tile rows, or all, fall away)
            out = torch.full((M, N), 7.0, device=DEV)
            if rows is not None:
                live.fill_(rows)
            print("body", body, "K", K, "split", split, "live", rows, flush=True)
            assert lib.bb_debug_gemm_int8(a.data_ptr(), sa.data_ptr(), w.data_ptr(), sw.data_ptr(), ld, out.data_ptr(), M, N, K, body, split, None if rows is None else live.data_ptr(),
                                          ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream) == 0
            n = M if rows is None else rows
            assert ((out[:n].double() - exact[:n]).abs() <= 4 * 2.0 ** -24 * exact[:n].abs() + 2.0 ** -149).all()
            assert (out[n:] == 7).all()
