"""Adapters at sizes, alignments and values where their parts meet: against the formulas in 64 bits."""
import pytest
import torch

import paper_2408_06995_b200 as fpq
import test_adapters as A

F32, BF, HF = torch.float32, torch.bfloat16, torch.float16
KIND = {F32: fpq.FP32, BF: fpq.BF16, HF: fpq.FP16}


def backward(t, u, **given):
    return fpq.fpq_adapter_backward(t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"], **given)


@pytest.mark.gpu
@pytest.mark.parametrize("xt,wt", A.TYPES)
@pytest.mark.parametrize("K", [32, 96, 160, 224, 288])
@pytest.mark.parametrize("M,R", [(9400, 64), (18900, 64), (18900, 24)])
def test_tiles_of_few_stages(M, R, K, xt, wt):
    """One to nine stages of a tile's reduction, in clusters of two blocks and alone: what the output reads takes the stages' place."""
    if xt != F32:
        K *= 2                                             # as many stages, of 64 columns each
    N = 1280
    assert fpq.fpq_adapter_route(M, N, K, 1, R, 1, KIND[xt], KIND[wt]) == fpq.ADAPTER_TILES
    t = A.make(M, K, N, R, [0, M - 5], [0], 1, xt, wt)
    first = A.run_forward(t)
    A.check_forward(t, *first)
    for _ in range(3):
        assert torch.equal(A.run_forward(t)[1], first[1])
    assert fpq.fpq_read_status() == fpq.OK


@pytest.mark.gpu
@pytest.mark.parametrize("xt", [BF, HF, F32])
@pytest.mark.parametrize("K,N,ldx,ldy", [(257, 96, 257, 96), (96, 257, 96, 257), (96, 130, 98, 131), (131, 96, 131, 98), (64, 64, 67, 72), (64, 64, 72, 67)])
def test_rows_and_base_of_different_alignment(K, N, ldx, ldy, xt):
    """Rows of x, or of dy, that start between words while those of base allow wider copies, and the other way round."""
    t = A.make(210, K, N, 16, [1, 12, 101, 103, 207], [1, 0, 1, 0], 2, xt, xt, ldx=ldx, ldy=ldy)
    A.check_forward(t, *A.run_forward(t, ldy=ldy))
    u, dx = torch.randn(210, 16, device="cuda"), torch.full((210, ldx), -7.0, dtype=xt, device="cuda")[:, :K]
    before = dx.clone()
    A.check_backward(t, u, *backward(t, u, base=t["dbase"], dx=dx), before)
