"""Adapters at sizes, alignments and values where their parts meet: against the formulas in 64 bits."""
import os
import re

import pytest
import torch

import paper_2408_06995_b200 as fpq
import test_adapters as A
from paper_2408_06995_b200 import build as fpq_build

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


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("xt,M", [(F32, 60), (F32, 3000), (BF, 60), (BF, 3000)])
def test_an_adapter_without_rows_has_zeros_whatever_its_scale(xt, M, value):
    t = A.make(M, 64, 96, 8, [0, M // 3, M // 3, M], [0, 1, 2], 4, xt, xt)
    t["scale"][1] = t["scale"][3] = value                  # an empty segment's adapter, and one that no segment names
    u = torch.randn(M, 8, device="cuda")
    _, da, db = backward(t, u)
    for g in (1, 3):
        assert not bool(da[g].any()) and not bool(db[g].any())
    t["scale"][2] = value                                  # with rows: zeros of u times it are NaN, as the formula has it
    u[:, 5] = 0
    _, da, db = backward(t, u)
    assert bool(torch.isnan(db[2][:, 5]).all()) and not bool(torch.isfinite(db[2]).any()) and bool(torch.isfinite(db[0]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("sizes", [{"M": 0}, {"S": 0}])
def test_without_rows_only_the_gradients_are_touched(sizes):
    """The other arguments may be anything: a scale between words is no error, and is not read."""
    da, db, scale = torch.ones(2, 4, 16, device="cuda"), torch.ones(2, 8, 4, device="cuda"), torch.ones(4, device="cuda")
    call = A.Call(ld_base=16, da=da.data_ptr(), db=db.data_ptr(), scale=scale.data_ptr() + 2, workspace=None, x=None, dy=None, u=None, a=None, b=None,
                  offsets=None, ids=None, base=None, dx=None, stream=torch.cuda.current_stream().cuda_stream, **sizes)
    assert call.run("backward") == fpq.OK
    assert not bool(da.any()) and not bool(db.any())


class Layers:
    """Stands in for the extension: remembers the call, computes nothing."""

    def adapter_forward(self, *args):
        self.args = args
        return 0

    adapter_backward = adapter_forward


@pytest.mark.parametrize("with_base", [True, False])
def test_outputs_made_by_the_call_have_no_history(monkeypatch, with_base):
    """The kernels' results are no function of `base` alone: an autograd graph that says so would lose every other gradient without a word."""
    layers = Layers()
    monkeypatch.setattr(fpq, "_layers", layers)
    x, a, b = torch.randn(6, 8, requires_grad=True), torch.randn(1, 2, 8, requires_grad=True), torch.randn(1, 4, 2, requires_grad=True)
    offsets, ids = torch.tensor([0, 6], dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    base = torch.randn(6, 4, requires_grad=True) if with_base else None
    y = fpq.fpq_adapter_forward(x, a, b, offsets, ids, base=base)
    assert not y.requires_grad and y.grad_fn is None and layers.args[7] is y
    assert torch.equal(y, base if with_base else torch.zeros(6, 4)) and (not with_base or y.data_ptr() != base.data_ptr())
    dbase = torch.randn(6, 8, requires_grad=True) if with_base else None
    for g in fpq.fpq_adapter_backward(torch.randn(6, 4), x, torch.randn(6, 2), a, b, offsets, ids, base=dbase):
        assert not g.requires_grad and g.grad_fn is None


# tall requests whose backward pass goes by tiles, on padded weights, while the forward pass may not: M, K, N, R, cuts, ids, G
TALL_ODD_RANKS = [
    (8192, 1280, 640, 36, [0, 8192], [0], 1),
    (9000, 640, 1288, 20, [0, 1, 4400, 8999], [1, 0, 1], 2),
    (18900, 1288, 648, 18, [3, 9000, 18899], [1, 0], 2),
    (28001, 648, 1288, 12, [0, 14000, 28001], [0, 1], 2),
    (28000, 1288, 648, 28, [1, 20000, 27999], [1, 0], 2),
    (20000, 648, 1288, 63, [0, 19990], [2], 3),
    (20000, 648, 1288, 33, [0, 10000, 20000], [1, 0], 2),
    (20000, 648, 1288, 17, [0, 20000], [0], 1),
    (30000, 640, 640, 5, [9, 15000, 30000], [0, 1], 2),
]


def backward_by_tiles(shape, xt, wt, dx=True, base=True):
    M, K, N, R, cuts, _, G = shape
    return fpq.fpq_adapter_backward_route(M, N, K, G, R, len(cuts) - 1, KIND[xt], KIND[wt], dx, base) == fpq.ADAPTER_TILES


def test_the_backward_route_is_that_of_padded_weights():
    for xt, wt in A.TYPES:
        for K, N in ((1280, 640), (648, 1288)):
            for R in (12, 18, 20, 28, 36, 60):
                for dx, base in ((True, True), (True, False), (False, False)):
                    shape = (32768, K, N, R, [0, 32768], [0], 1)
                    padded = shape[:3] + (-(-R // 8) * 8,) + shape[4:]
                    assert backward_by_tiles(shape, xt, wt, dx, base) == backward_by_tiles(padded, xt, wt, dx, base)
                assert backward_by_tiles(padded, xt, wt) == (fpq.fpq_adapter_route(32768, K, N, 1, padded[3], 1, KIND[xt], KIND[wt]) == fpq.ADAPTER_TILES)
    for xt, wt in A.TYPES:                                 # every type and padded rank is among the cases below
        ranks = {max(16, 1 << (s[3] - 1).bit_length()) for s in TALL_ODD_RANKS if backward_by_tiles(s, xt, wt)}
        assert ranks >= ({32, 64} if xt == F32 else {16, 32, 64})
    with pytest.raises(fpq.FpqError, match="shape"):
        fpq.fpq_adapter_backward_route(1, 1, 1, 1, 200, 1, fpq.FP32, fpq.FP32)
    with pytest.raises(fpq.FpqError, match="unsupported"):
        fpq.fpq_adapter_backward_route(1, 1, 1, 1, 2, 1, fpq.BF16, fpq.FP32)


@pytest.mark.gpu
@pytest.mark.parametrize("xt,wt", A.TYPES)
@pytest.mark.parametrize("shape", TALL_ODD_RANKS, ids=lambda s: "x".join(map(str, s[:4])))
def test_tall_backward_of_ranks_that_are_padded(shape, xt, wt):
    t = A.make(*shape, xt=xt, wt=wt)
    M, K, R = t["x"].shape[0], t["x"].shape[1], t["a"].shape[1]
    u = torch.randn(M, R, device="cuda")
    dx = torch.full((M, K), -7.0, dtype=xt, device="cuda")
    before = dx.clone()
    A.check_backward(t, u, *backward(t, u, base=t["dbase"], dx=dx), before)
    _, da, db = backward(t, u, need_dx=False)
    A.check_backward(t, u, None, da, db, None, have_dx=False)
    A.check_forward(t, *A.run_forward(t))
    assert fpq.fpq_read_status() == fpq.OK


# ---- the documented bounds --------------------------------------------------------------------------------------------

def documented():
    """FPQ_ADAPTER_ERROR as the header has it."""
    text = open(os.path.join(fpq_build.ROOT, "include", "fpq.h")).read()
    add, unit = re.search(r"#define FPQ_ADAPTER_ERROR\(n\) \(\(([\d.]+) \+ \(n\)\) / ([\d.]+)\)", text).groups()
    return lambda n: (float(add) + n) / float(unit)


def test_the_documented_bounds_hold_what_the_terms_add_up_to():
    """Units of 2^-23.  Operands: 2^-20 three times, 24.  t: up to 24 sums cut off inside the tensor cores (64 FP32 columns: eight MMAs of
    three products), then K / 64 FP32 additions and up to 20 of warps and blocks.  y: 3 R / 8 sums inside, and 2^-18 of t beside BF16
    weights.  Gradients: a sum of 8 rows at a time and warp, two warps at least, each addition rounded by half a unit."""
    bound = documented()
    for D in (1, 64, 1280, 1 << 24):
        assert bound(D / 64) >= A.product_error(D, 24) >= 2.0 ** -24
        assert bound(D / 32) >= 3 * 2.0 ** -20 + (24 + 20 + D / 16 / 2) * 2.0 ** -23
    for R in (1, 128):
        assert 2.0 ** -16 >= A.product_error(R, 3 * R / 8) + 2.0 ** -23 + 2.0 ** -18


def full(shape, dtype, g):
    """Positive numbers in [0.5, 4) whose every mantissa bit but a few is set: the longest remainders of every split, and sums that are cut off
    towards one side throughout."""
    bits = {F32: 23, BF: 7, HF: 10}[dtype]
    m = (1 << bits) - 1 - (torch.randint(0, 8, shape, generator=g, device="cuda") << torch.randint(0, bits - 2, shape, generator=g, device="cuda")) % (1 << bits)
    return ((1 + m.double() / (1 << bits)) * 2.0 ** torch.randint(-1, 2, shape, generator=g, device="cuda").double()).to(dtype)


BOUNDED = [(1, 1280, 640, 16), (300, 1280, 320, 128), (257, 96, 2560, 128), (3000, 320, 96, 24), (9000, 640, 1288, 64), (20000, 640, 1288, 32),
           (30000, 328, 648, 60), (70000, 64, 32, 128), (12000, 2560, 64, 64)]


@pytest.mark.gpu
@pytest.mark.parametrize("xt,wt", A.TYPES)
@pytest.mark.parametrize("M,K,N,R", BOUNDED)
def test_the_documented_bounds(M, K, N, R, xt, wt):
    g = torch.Generator(device="cuda").manual_seed(M)
    bound = documented()
    x, dy, a, b, u0 = full((M, K), xt, g), full((M, N), xt, g), full((1, R, K), wt, g), full((1, N, R), wt, g), full((M, R), F32, g)
    if xt == HF:                                           # (sums that its range holds)
        a, b = a * 2.0 ** -8, b * 2.0 ** -10
    s = 1.2345678806304932
    scale, offsets, ids = torch.tensor([s], device="cuda"), torch.tensor([0, M], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    u = torch.empty(M, R, device="cuda")
    y = fpq.fpq_adapter_forward(x, a, b, offsets, ids, scale, None, None, u)
    dx, da, db = fpq.fpq_adapter_backward(dy, x, u0, a, b, offsets, ids, scale)
    x, dy, a, b, u0 = x.double(), dy.double(), a[0].double(), b[0].double(), u0.double()
    ue, te = x @ a.T, s * (dy @ b)                         # (everything is positive: each sum is that of its absolute terms)
    second = 2.0 ** -16
    for name, got, want, error in (("u", u, ue, bound(K / 64)), ("y", y, s * (ue @ b.T), bound(K / 64) + second), ("dx", dx, te @ a, bound(N / 64) + second),
                                   ("da", da[0], te.T @ x, bound(M / 32) + bound(N / 64)), ("db", db[0], s * (dy.T @ u0), bound(M / 32))):
        assert bool(torch.isfinite(got).all())
        off = (got.double() - want).abs()
        allowed = error * want + A.half_step(got.dtype, want * (1 + error)) + 2.0 ** -24 * want
        worst = float((off / allowed).max())
        assert worst <= 1, (name, worst)


@pytest.mark.gpu
@pytest.mark.parametrize("xt,wt", [(F32, F32), (F32, BF), (BF, BF)])
@pytest.mark.parametrize("M,K,N,R", [(64, 128, 96, 16), (20000, 640, 1280, 32)])
@pytest.mark.parametrize("x_exp,a_exp,b_exp,dy_exp,u_exp", [(-112, 10, 10, 0, 0), (-130, 20, 10, -118, 5), (-145, 30, 30, -130, 20), (10, -130, 20, 10, -125), (0, 20, -130, 5, -140), (-70, -75, 0, -40, -40),
                                                          (-100, -40, 10, -140, 30)])
def test_operands_near_the_smallest_numbers(M, K, N, R, x_exp, a_exp, b_exp, dy_exp, u_exp, xt, wt):
    """What is lost of an FP32 operand lies below 2^-133, and sums end at FP32's 2^-149 (each cut-off addition, up to three for 8 terms)."""
    bound, lost, least = documented(), 2.0 ** -133, 2.0 ** -149
    g = torch.Generator(device="cuda").manual_seed(M)

    def numbers(shape, exponent, dtype):
        return ((1 + torch.rand(shape, generator=g, device="cuda", dtype=torch.float64)) * 2.0 ** exponent).to(F32).to(dtype)

    x, a, b, dy, u0 = numbers((M, K), x_exp, xt), numbers((1, R, K), a_exp, wt), numbers((1, N, R), b_exp, wt), numbers((M, N), dy_exp, xt), numbers((M, R), u_exp, F32)
    offsets, ids = torch.tensor([0, M], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    u = torch.empty(M, R, device="cuda")
    y = fpq.fpq_adapter_forward(x, a, b, offsets, ids, None, None, None, u)
    dx, da, db = fpq.fpq_adapter_backward(dy, x, u0, a, b, offsets, ids)
    x, a, b, dy, u0 = x.double(), a[0].double(), b[0].double(), dy.double(), u0.double()

    def product(p, q, p_off, q_off, error):
        """p q^T, and how far it may be off when p and q are."""
        D = p.shape[1]
        return p @ q.T, (error * p + p_off) @ q.T + (p + p_off).sum(1, keepdim=True) * q_off + D * least

    x_off, w_off = lost if xt == F32 else 0.0, lost if wt == F32 else 0.0
    ue, u_off = product(x, a, x_off, w_off, bound(K / 64))
    ye, y_off = product(ue, b, u_off + lost, w_off, 2.0 ** -16)
    te, t_off = product(dy, b.T, x_off, w_off, bound(N / 64))
    xe, dx_off = product(te, a.T, t_off + lost, w_off, 2.0 ** -16)
    ae, da_off = product(te.T, x.T, (t_off + lost).T, x_off, bound(M / 32))
    be, db_off = product(dy.T, u0.T, torch.full_like(dy.T, x_off), lost, bound(M / 32))
    for name, got, want, off in (("u", u, ue, u_off), ("y", y, ye, y_off), ("dx", dx, xe, dx_off), ("da", da[0], ae, da_off), ("db", db[0], be, db_off)):
        allowed = off + A.half_step(got.dtype, want + off) + 2.0 ** -24 * want
        assert bool(((got.double() - want).abs() <= allowed).all()), (name, float(((got.double() - want).abs() / allowed).max()))


@pytest.mark.gpu
@pytest.mark.parametrize("xt,R", [(BF, 64), (BF, 32), (F32, 64), (HF, 24)])
def test_tiles_on_two_streams_and_replayed(xt, R):
    """Tall calls of two streams share the SMs and their tensor memory; a captured one serves other segments."""
    M, K, N, G = 20000, 648, 1288, 2
    assert fpq.fpq_adapter_route(M, N, K, G, R, 3, KIND[xt], KIND[xt]) == fpq.ADAPTER_TILES
    t = A.make(M, K, N, R, [0, 7000, 12000, 20000], [0, -1, 1], G, xt, xt)
    u0 = torch.randn(M, R, device="cuda")

    def both():
        u = torch.zeros(M, R, device="cuda")
        y = fpq.fpq_adapter_forward(t["x"], t["a"], t["b"], t["offsets"], t["ids"], t["scale"], t["base"], None, u)
        return (y, u) + backward(t, u0, base=t["dbase"])

    want = both()
    torch.cuda.synchronize()
    got, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(both())
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = both()
    t["offsets"].copy_(torch.tensor([5, 6, 15000, 19000], dtype=torch.int32))
    t["ids"].copy_(torch.tensor([1, 0, 1], dtype=torch.int32))
    for _ in range(2):
        graph.replay()
    want = both()
    assert all(torch.equal(a, b) for a, b in zip(out, want))
    assert fpq.fpq_read_status() == fpq.OK


@pytest.mark.gpu
@pytest.mark.parametrize("M,K,N,R", [(24000, 640, 640, 64), (24000, 640, 1280, 32), (12000, 64, 640, 64), (20000, 1280, 320, 24), (300, 640, 640, 128), (900, 64, 320, 100),
                                     (64, 1280, 1280, 16)])
def test_fp32_outputs_on_average(M, K, N, R):
    """Root mean square errors of FP32 outputs, in units of 2^-23.  A sum that is cut off loses a third of a unit on average, of a running sum
    that is some 0.7 of the last one: 16 for 64 columns of t (the tails of the first half cost nothing) 4, 8 for 64 ranks 2, and twice
    0.9 for the product of two tails: 8 in all."""
    g = torch.Generator(device="cuda").manual_seed(R)
    x, dy = torch.randn(M, K, generator=g, device="cuda"), torch.randn(M, N, generator=g, device="cuda")
    a, b = torch.randn(1, R, K, generator=g, device="cuda") / K ** 0.5, torch.randn(1, N, R, generator=g, device="cuda")
    offsets, ids = torch.tensor([0, M], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    u = torch.empty(M, R, device="cuda")
    y = fpq.fpq_adapter_forward(x, a, b, offsets, ids, None, None, None, u)
    dx, da, db = fpq.fpq_adapter_backward(dy, x, u, a, b, offsets, ids)
    x, dy, a, b = x.double(), dy.double(), a[0].double(), b[0].double()
    for name, got, want in (("u", u, x @ a.T), ("y", y, x @ a.T @ b.T), ("dx", dx, dy @ b @ a), ("da", da[0], (dy @ b).T @ x), ("db", db[0], dy.T @ (x @ a.T))):
        off = float((got.double() - want).norm() / want.norm())
        assert off <= 8 * 2.0 ** -23, (name, off)
