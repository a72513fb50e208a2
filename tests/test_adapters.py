"""Low-rank adapters of many requests: forward and backward against the formulas in 64 bits."""
import ctypes

import pytest
import torch

import paper_2408_06995_b200 as fpq
from paper_2408_06995_b200 import build as fpq_build

fpq_build.build()
F32, BF, HF = torch.float32, torch.bfloat16, torch.float16


WS = 10 * 4 * 4 + 2 * 4 * (16 + 8) * 4          # t [M][R], A and B transposed


# ---- refusals, without a GPU ------------------------------------------------------------------------------------------

class Call:
    """fpq_adapter_forward / _backward with arguments that pass, but for those that a test changes; nothing is ever launched."""
    forward = ["x", "ldx", "x_type", "a", "b", "w_type", "scale", "G", "R", "offsets", "ids", "S", "base", "ld_base", "y", "ldy", "u", "M", "N",
               "K", "stream"]
    backward = ["dy", "ld_dy", "x", "ldx", "x_type", "u", "a", "b", "w_type", "scale", "G", "R", "offsets", "ids", "S", "base", "ld_base", "dx",
                "ld_dx", "da", "db", "M", "N", "K", "workspace", "ws_bytes", "stream"]

    def __init__(self, **given):
        pointers = {k: 4096 for k in ("x", "a", "b", "scale", "offsets", "ids", "base", "y", "u", "dy", "dx", "da", "db", "workspace")}
        self.v = {**pointers, "x_type": fpq.FP32, "w_type": fpq.FP32, "G": 2, "R": 4, "S": 3, "M": 10, "N": 8, "K": 16, "ldx": 16, "ldy": 8,
                  "ld_base": 8, "ld_dy": 8, "ld_dx": 16, "ws_bytes": WS, "stream": None, **given}

    def run(self, name):
        return getattr(fpq.lib(), "fpq_adapter_" + name)(*[self.v[k] for k in getattr(self, name)])


BAD = [({"x_type": 3}, "ERR_UNSUPPORTED"), ({"x_type": -1}, "ERR_UNSUPPORTED"), ({"w_type": 3}, "ERR_UNSUPPORTED"),
       ({"x_type": fpq.BF16}, "ERR_UNSUPPORTED"), ({"x_type": fpq.FP16, "w_type": fpq.BF16}, "ERR_UNSUPPORTED"),
       ({"M": -1}, "ERR_SHAPE"), ({"M": 1 << 31}, "ERR_SHAPE"), ({"N": 0}, "ERR_SHAPE"), ({"K": 0}, "ERR_SHAPE"), ({"K": (1 << 24) + 1}, "ERR_SHAPE"),
       ({"G": 0}, "ERR_SHAPE"), ({"G": 65536}, "ERR_SHAPE"), ({"R": 0}, "ERR_SHAPE"), ({"R": 129}, "ERR_SHAPE"), ({"S": -1}, "ERR_SHAPE"),
       ({"S": (1 << 24) + 1}, "ERR_SHAPE"), ({"ldx": 15}, "ERR_SHAPE"), ({"G": 65535, "R": 128, "N": 1 << 18}, "ERR_SHAPE"), ({"G": 32768, "R": 1, "N": 1 << 18}, "ERR_SHAPE"),
       ({"a": None}, "ERR_NULL"), ({"b": None}, "ERR_NULL"), ({"offsets": None}, "ERR_NULL"), ({"ids": None}, "ERR_NULL"), ({"x": None}, "ERR_NULL"),
       ({"x": 4098}, "ERR_ALIGN"), ({"a": 4098}, "ERR_ALIGN"), ({"b": 4097}, "ERR_ALIGN"), ({"scale": 4098}, "ERR_ALIGN"),
       ({"offsets": 4098}, "ERR_ALIGN"), ({"ids": 4097}, "ERR_ALIGN"), ({"base": 4098}, "ERR_ALIGN"), ({"u": 4098}, "ERR_ALIGN")]


@pytest.mark.parametrize("given,error", BAD + [({"y": None}, "ERR_NULL"), ({"y": 4097}, "ERR_ALIGN"), ({"ldy": 7}, "ERR_SHAPE"),
                                               ({"ld_base": 7}, "ERR_SHAPE")])
def test_forward_refuses(given, error):
    assert Call(**given).run("forward") == getattr(fpq, error)


@pytest.mark.parametrize("given,error", BAD + [({"u": None}, "ERR_NULL"), ({"dy": None}, "ERR_NULL"), ({"da": None}, "ERR_NULL"),
                                               ({"db": None}, "ERR_NULL"), ({"dy": 4098}, "ERR_ALIGN"), ({"da": 4098}, "ERR_ALIGN"),
                                               ({"dx": 4098}, "ERR_ALIGN"), ({"workspace": 4100}, "ERR_ALIGN"), ({"ld_dy": 7}, "ERR_SHAPE"),
                                               ({"ld_dx": 15}, "ERR_SHAPE"), ({"ld_base": 15}, "ERR_SHAPE"), ({"workspace": None}, "ERR_WORKSPACE"),
                                               ({"ws_bytes": WS - 1}, "ERR_WORKSPACE")])
def test_backward_refuses(given, error):
    assert Call(**{"ld_base": 16, "N": 8, **({"ld_dy": given["N"]} if "N" in given and given["N"] > 8 else {}), **given}).run("backward") == getattr(fpq, error)


def test_nothing_to_do_is_no_error():
    assert Call(M=0, x=None, y=None).run("forward") == fpq.OK
    assert Call(S=0, ids=None).run("forward") == fpq.OK


def test_workspace_size():
    assert fpq.fpq_adapter_backward_workspace_size(10, 8, 16, 2, 4, fpq.FP32) == WS
    assert fpq.fpq_adapter_backward_workspace_size(-1, 8, 16, 2, 4, fpq.FP32) == 0
    assert fpq.fpq_adapter_backward_workspace_size(10, 8, 16, 2, 129, fpq.FP32) == 0
    assert fpq.fpq_adapter_backward_workspace_size(10, 8, 16, 2, 4, 3) == 0


def test_binding_takes_no_cpu_tensors():
    x, a, b = torch.zeros(4, 8), torch.zeros(1, 2, 8), torch.zeros(1, 8, 2)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(AssertionError, match="current device"):
        fpq.fpq_adapter_forward(x, a, b, i, i[:1])
    with pytest.raises(TypeError):
        fpq._load_layers().adapter_forward(x)


# ---- on the GPU -------------------------------------------------------------------------------------------------------

def make(M, K, N, R, cuts, ids, G, xt=F32, wt=F32, seed=0, ldx=None, ldy=None, scale=True):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    ldx, ldy = ldx or K, ldy or N
    return {"x": normal(M, ldx).to(xt)[:, :K], "a": (normal(G, R, K) / K ** 0.5).to(wt), "b": (normal(G, N, R) * 0.3).to(wt),
            "scale": torch.rand(G, generator=g, device="cuda") + 0.5 if scale else None,
            "offsets": torch.tensor(cuts, dtype=torch.int32, device="cuda"), "ids": torch.tensor(ids, dtype=torch.int32, device="cuda"),
            "base": normal(M, ldy).to(xt)[:, :N], "dy": normal(M, ldy).to(xt)[:, :N], "dbase": normal(M, ldx).to(xt)[:, :K]}


def segments(t):
    cuts, ids, G = t["offsets"].tolist(), t["ids"].tolist(), t["a"].shape[0]
    return [(lo, hi, i if 0 <= i < G else -1) for lo, hi, i in zip(cuts, cuts[1:], ids) if hi > lo]


def product_error(D, terms):
    """Error of a sum of D products relative to the sum of their magnitudes: two TF32 terms each (where the first term is the number cut off,
    the second is below 2^-10 of it: their product, 2^-20, is left out, and of each second term 2^-10 of it is cut off, 2^-20 twice), at
    most `terms` cut-off additions of the tensor cores, each 2^-23 at most, and the FP32 additions behind them."""
    return 3 * 2.0 ** -20 + (terms + 20 + D / 64) * 2.0 ** -23


def half_step(t, v):
    tiny = {F32: 2.0 ** -149, BF: 2.0 ** -133, HF: 2.0 ** -24}[t]
    return torch.finfo(t).eps / 2 * v.abs() + tiny / 2


def rows_exact(x, w1, w2, base, s, R, xt=F32):
    """t, y and their error bounds for the rows of one adapter: t = x w1^T, y = base + s t w2^T.  With BF16 operands t is multiplied as two
    BF16 terms: the first is off by 2^-9 of t at most, the second by 2^-9 of that."""
    D1 = x.shape[1]
    t = x @ w1.T
    dt = product_error(D1, 24) * (x.abs() @ w1.abs().T)
    y = s * (t @ w2.T)
    split = 2.0 ** -18 if xt == BF else 0.0
    dy = s * (dt @ w2.abs().T + (product_error(R, 3 * R / 8) + 2.0 ** -23 + split) * (t.abs() @ w2.abs().T))
    if base is not None:
        y = y + base
    return t, dt, y, dy + 2.0 ** -23 * y.abs()


def check_rows(got, y, dy, what):
    err = (got.double() - y).abs()
    tol = dy + half_step(got.dtype, y.abs() + dy)
    worst = (err - tol).argmax()
    assert bool((err <= tol).all()), (what, float(err.flatten()[worst]), float(tol.flatten()[worst]))


def run_forward(t, base=True, in_place=False, ldy=None):
    M, N, R = t["x"].shape[0], t["b"].shape[1], t["a"].shape[1]
    y = torch.full((M, ldy or N), -7.0, dtype=t["x"].dtype, device="cuda")[:, :N]
    u = torch.full((M, R), -7.0, device="cuda")
    if in_place:
        y.copy_(t["base"])
    before = y.clone()
    fpq.fpq_adapter_forward(t["x"], t["a"], t["b"], t["offsets"], t["ids"], t["scale"], y if in_place else t["base"] if base else None, y, u)
    return before, y, u


def check_forward(t, before, y, u, base=True):
    inside = torch.zeros(y.shape[0], dtype=torch.bool, device="cuda")
    for lo, hi, i in segments(t):
        inside[lo:hi] = True
        b0 = t["base"][lo:hi].double() if base else None
        if i < 0:
            assert torch.equal(y[lo:hi], t["base"][lo:hi] if base else torch.zeros_like(y[lo:hi])) and not bool(u[lo:hi].any())
            continue
        s = float(t["scale"][i]) if t["scale"] is not None else 1.0
        te, dt, ye, dy = rows_exact(t["x"][lo:hi].double(), t["a"][i].double(), t["b"][i].double(), b0, s, u.shape[1], y.dtype)
        check_rows(u[lo:hi], te, dt, "u")
        check_rows(y[lo:hi], ye, dy, "y")
    assert torch.equal(y[~inside], before[~inside]) and bool((u[~inside] == -7).all())


SHAPES = [  # M, K, N, R, cuts, ids, G
    (1, 1280, 1280, 16, [0, 1], [0], 1),
    (1, 1, 1, 1, [0, 1], [0], 1),
    (5, 320, 320, 8, [0, 1, 2, 3, 4, 5], [4, 0, -1, 2, 0], 5),
    (64, 640, 320, 16, list(range(65)), [i % 7 for i in range(64)], 7),
    (77, 768, 320, 4, [0, 77], [0], 1),
    (130, 35, 33, 3, [0, 17, 17, 64, 130], [1, 0, 2, 1], 3),
    (200, 802, 70, 24, [3, 40, 171], [1, 0], 2),
    (333, 96, 257, 17, [0, 100, 300], [9, 0], 1),
    (256, 320, 640, 32, [0, 33, 256], [0, 1], 2),
    (150, 200, 132, 64, [0, 64, 150], [1, 0], 2),
    (100, 136, 72, 128, [0, 31, 100], [0, 1], 2),
    (90, 64, 40, 100, [0, 90], [0], 1),
    (4100, 320, 96, 16, [0, 4096, 4099], [0, 0], 1),
    (40, 4100, 36, 40, [0, 40], [0], 1),
]
TYPES = [(F32, F32), (F32, BF), (F32, HF), (BF, BF), (HF, HF)]


@pytest.mark.gpu
@pytest.mark.parametrize("xt,wt", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:4])))
def test_forward(shape, xt, wt):
    t = make(*shape, xt=xt, wt=wt)
    check_forward(t, *run_forward(t))


# requests of many rows: tiles of 128 rows on tcgen05 MMAs, in clusters of two blocks or alone, forward or (N and K exchanged) backward
TALL = [
    (8192, 640, 1280, 64, [0, 8192], [0], 1),
    (8000, 648, 1288, 56, [7, 3000, 3000, 7990], [1, 0, 0], 2),
    (9000, 1288, 640, 32, [0, 1, 4400, 8999], [1, 0, 1], 2),
    (9400, 648, 1288, 24, [0, 4600, 9400], [0, -1], 1),
    (18900, 1288, 648, 16, [3, 18899], [1], 2),
    (18931, 640, 1280, 32, [0, 18931], [0], 1),
    (21000, 328, 648, 64, [0, 9000, 9000, 20990], [1, 0, 0], 2),
    (28001, 648, 1288, 16, [0, 14000, 28001], [0, 1], 2),
    (28000, 1288, 648, 24, [1, 20000, 27999], [1, 0], 2),
    (12000, 64, 1032, 40, [5, 6000, 11990], [0, 1], 2),
]


def by_tiles(shape, xt, wt):
    M, K, N, R, cuts, _, G = shape
    kind = {F32: fpq.FP32, BF: fpq.BF16, HF: fpq.FP16}
    return [fpq.fpq_adapter_route(M, n, k, G, R, len(cuts) - 1, kind[xt], kind[wt], base) == fpq.ADAPTER_TILES
            for n, k, base in ((N, K, True), (N, K, False), (K, N, True))]


TALL_CASES = [(s, x, w) for s in TALL for x, w in TYPES if any(by_tiles(s, x, w))]


def test_tall_requests_reach_their_kernel():
    """Every type and padded rank that the kernel is built for is among the cases, forward and backward."""
    seen = {(x, w, max(16, 1 << (s[3] - 1).bit_length()), s[0] > 148 * 128, way)
            for s, x, w in TALL_CASES for way, yes in enumerate(by_tiles(s, x, w)) if yes}
    for x, w in TYPES:
        for rp in (32, 64) if x == F32 else (16, 32, 64):
            for more_than_sms in (False, True):            # up to a tile for every SM, and more
                assert {way for *k, way in seen if k == [x, w, rp, more_than_sms]} >= {0, 2}, (x, w, rp, more_than_sms)
    assert not any(by_tiles((8192, 640, 640, 128, [0, 8192], [0], 1), F32, F32))
    with pytest.raises(fpq.FpqError, match="shape"):
        fpq.fpq_adapter_route(1, 1, 1, 1, 200, 1, fpq.FP32, fpq.FP32)


@pytest.mark.gpu
@pytest.mark.parametrize("shape,xt,wt", TALL_CASES, ids=lambda s: "x".join(map(str, s[:4])) if isinstance(s, tuple) else str(s)[6:])
def test_tall_requests(shape, xt, wt):
    t = make(*shape, xt=xt, wt=wt)
    check_forward(t, *run_forward(t))
    check_forward(t, *run_forward(t, base=False), base=False)
    M, K, R = t["x"].shape[0], t["x"].shape[1], t["a"].shape[1]
    u = torch.randn(M, R, device="cuda")
    dx = t["dbase"].clone()
    before = dx.clone()
    _, da, db = fpq.fpq_adapter_backward(t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"], dx, dx)
    check_backward(t, u, dx, da, db, before)
    assert fpq.fpq_read_status() == fpq.OK


@pytest.mark.gpu
@pytest.mark.parametrize("xt", [F32, BF])
def test_tall_requests_in_slices_and_with_odd_values(xt):
    shape = (9300, 320, 1032, 64, [0, 9290], [0], 1)
    assert all(by_tiles(shape, xt, xt)[:2])
    t = make(*shape, xt, xt, ldx=704, ldy=1160)
    check_forward(t, *run_forward(t, ldy=1160))
    clean = run_forward(t)[1].clone()
    t["x"][3, 17], t["x"][200, 0], t["x"][9289, 5] = float("inf"), float("nan"), 3e38
    t["x"][9290:] = float("nan")
    before, y, u = run_forward(t)
    keep = torch.ones(9300, dtype=torch.bool, device="cuda")
    keep[[3, 200, 9289]] = False
    assert torch.equal(y[keep], clean[keep]) and bool(torch.isnan(y[200]).all())
    for r in (3, 9289):
        want = t["x"][r].float().cpu() @ t["a"][0].float().cpu().T
        assert torch.equal(torch.isnan(u[r].cpu()), torch.isnan(want)) and torch.equal(torch.isinf(u[r].cpu()), torch.isinf(want))
    assert fpq.fpq_read_status() == fpq.OK


@pytest.mark.gpu
@pytest.mark.parametrize("xt,wt", TYPES)
@pytest.mark.parametrize("ldx,ldy", [(700, 1000), (643, 963)])
def test_forward_in_slices_of_wider_tensors(xt, wt, ldx, ldy):
    t = make(100, 640, 960, 16, [0, 60, 100], [1, 0], 2, xt, wt, ldx=ldx, ldy=ldy)
    check_forward(t, *run_forward(t, ldy=ldy))


@pytest.mark.gpu
@pytest.mark.parametrize("xt", [F32, BF])
def test_forward_base_absent_or_in_place(xt):
    t = make(300, 320, 96, 16, [0, 100, 120, 290], [1, -1, 0], 2, xt, xt, scale=False)
    check_forward(t, *run_forward(t, base=False), base=False)
    before, y, u = run_forward(t, in_place=True)
    check_forward(t, before, y, u)
    assert torch.equal(y, fpq.fpq_adapter_forward(t["x"], t["a"], t["b"], t["offsets"], t["ids"], None, t["base"]))


@pytest.mark.gpu
def test_rows_of_no_segment_are_not_read():
    t = make(64, 320, 64, 16, [8, 20, 50], [0, 1], 2)
    clean = run_forward(t)[1].clone()
    t["x"][:8], t["x"][50:], t["base"][50:] = float("nan"), float("inf"), float("nan")
    y = run_forward(t)[1]
    assert torch.equal(y, clean)
    t["dy"][:8] = float("nan")
    u = torch.randn(64, 16, device="cuda")
    u[:8], u[50:] = float("nan"), float("inf")
    for g in fpq.fpq_adapter_backward(t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"])[1:]:
        assert bool(torch.isfinite(g).all())


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("inf"), float("-inf"), float("nan"), 3.4e38])
def test_forward_values_without_a_split(value):
    """One operand that is not finite (or rounds up to infinity as TF32): what multiply-adds give, and no other row changes."""
    t = make(40, 256, 48, 8, [0, 40], [0], 1)
    clean, cu = (v.clone() for v in run_forward(t)[1:])
    t["x"][5, 77] = value
    _, y, u = run_forward(t)
    others = torch.arange(40, device="cuda") != 5
    assert torch.equal(y[others], clean[others]) and torch.equal(u[others], cu[others])
    want = t["x"][5].float().cpu() @ t["a"][0].cpu().T
    got = u[5].cpu()
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(torch.isinf(got), torch.isinf(want))
    fine = torch.isfinite(want)
    assert torch.equal(got[~fine & ~torch.isnan(want)], want[~fine & ~torch.isnan(want)])
    bound = product_error(256, 24) * (t["x"][5].cpu().double().abs() @ t["a"][0].cpu().double().abs().T)
    assert bool(((got.double() - t["x"][5].cpu().double() @ t["a"][0].cpu().double().T).abs()[fine] <= bound[fine]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("S,G,M", [(40, 40, 700), (1500, 300, 2600), (2500, 7, 900)])
def test_many_segments(S, G, M):
    """More segments than a warp looks through at a time, empty ones among them, and many adapters."""
    g = torch.Generator().manual_seed(S)
    cuts = [0] + torch.randint(0, M + 1, (S - 1,), generator=g).sort().values.tolist() + [M - 3]
    cuts = [min(c, M - 3) for c in cuts]
    ids = torch.randint(-1, G, (S,), generator=g).tolist()
    t = make(M, 64, 72, 4, cuts, ids, G)
    check_forward(t, *run_forward(t))
    u = torch.randn(M, 4, device="cuda")
    dx = torch.full((M, 64), -7.0, device="cuda")
    before = dx.clone()
    _, da, db = fpq.fpq_adapter_backward(t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"], t["dbase"], dx)
    check_backward(t, u, dx, da, db, before)


@pytest.mark.gpu
@pytest.mark.parametrize("R", [4, 64])
def test_offsets_beyond_32_bits(R):
    """An output of more than 2^32 bytes and 2^31 elements: the last rows, by both kernels."""
    M, K, N = 140000, 64, 16384
    x = torch.randn(M, K, device="cuda").bfloat16()
    a, b = (torch.randn(1, R, K, device="cuda") / 8).bfloat16(), (torch.randn(1, N, R, device="cuda") / 8).bfloat16()
    offsets, ids = torch.tensor([5, M - 1], dtype=torch.int32, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
    y = torch.zeros(M, N, dtype=BF, device="cuda")
    fpq.fpq_adapter_forward(x, a, b, offsets, ids, None, None, y)
    for lo, hi in ((5, 40), (131060, 131090), (M - 40, M - 1)):
        _, _, want, dy = rows_exact(x[lo:hi].double(), a[0].double(), b[0].double(), None, 1.0, R, BF)
        check_rows(y[lo:hi], want, dy, "y")
    assert not bool(y[:5].any()) and not bool(y[M - 1].any())
    dy, u = y[:, :], torch.randn(M, R, device="cuda")
    _, da, db = fpq.fpq_adapter_backward(dy, x, u, a, b, offsets, ids, need_dx=False)
    ea, ta = torch.zeros(R, K, dtype=torch.float64, device="cuda"), torch.zeros(R, K, dtype=torch.float64, device="cuda")
    for lo in range(5, M - 1, 10000):
        rows = slice(lo, min(lo + 10000, M - 1))
        te, dt, _, _ = rows_exact(dy[rows].double(), b[0].double().T, a[0].double().T, None, 1.0, R, BF)
        ea += te.T @ x[rows].double()
        ta += dt.T @ x[rows].double().abs() + product_error(M, 24) * (te.abs().T @ x[rows].double().abs())
    check_rows(da[0], ea, ta, "da")
    cols = torch.tensor([0, 1, 8191, N - 1], device="cuda")
    d = dy[5:M - 1, cols].double()
    uu = u[5:M - 1].double()
    check_rows(db[0, cols], d.T @ uu, (product_error(M, 24) + 2.0 ** -23) * (d.abs().T @ uu.abs()), "db")


@pytest.mark.gpu
def test_wrong_lists_stay_in_bounds():
    """Offsets out of range are clamped and ids out of range mean no adapter: every row keeps base or gets some adapter's result."""
    t = make(50, 64, 32, 8, [-100, 20, 1000], [0, 5], 2)
    _, y, _ = run_forward(t)
    assert torch.equal(y[20:], t["base"][20:])
    _, _, want, dy = rows_exact(t["x"][:20].double(), t["a"][0].double(), t["b"][0].double(), t["base"][:20].double(), float(t["scale"][0]), 8)
    check_rows(y[:20], want, dy, "y")
    t["offsets"] = torch.tensor([40, 10, 45], dtype=torch.int32, device="cuda")
    run_forward(t)
    torch.cuda.synchronize()


@pytest.mark.gpu
def test_replayed_with_other_segments():
    t = make(120, 320, 64, 16, [0, 50, 120], [0, 1], 3)
    y, u = torch.zeros(120, 64, device="cuda"), torch.zeros(120, 16, device="cuda")
    da, db, dx = torch.zeros_like(t["a"]), torch.zeros_like(t["b"]), torch.zeros(120, 320, device="cuda")
    ws = torch.empty(fpq.fpq_adapter_backward_workspace_size(120, 64, 320, 3, 16, fpq.FP32), dtype=torch.uint8, device="cuda")

    def both():
        fpq.fpq_adapter_forward(t["x"], t["a"], t["b"], t["offsets"], t["ids"], t["scale"], t["base"], y, u)
        fpq.fpq_adapter_backward(t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"], None, dx, da, db, ws)

    both()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        both()
    t["offsets"].copy_(torch.tensor([0, 9, 113], dtype=torch.int32))
    t["ids"].copy_(torch.tensor([2, 0], dtype=torch.int32))
    for v in (y, u, dx, da, db):
        v.fill_(-7.0)
    graph.replay()
    got = [v.clone() for v in (y, u, dx, da, db)]
    for v in (y, u, dx, da, db):
        v.fill_(-7.0)
    both()
    for v, w in zip(got, (y, u, dx, da, db)):
        assert torch.equal(v, w)
    check_forward(t, torch.full_like(y, -7.0), y, u)


def check_backward(t, u, dx, da, db, before, base=True, have_dx=True):
    R, G = u.shape[1], t["a"].shape[0]
    ea, eb = torch.zeros_like(t["a"], dtype=torch.float64), torch.zeros_like(t["b"], dtype=torch.float64)
    ta, tb = torch.zeros_like(ea), torch.zeros_like(eb)
    inside = torch.zeros(u.shape[0], dtype=torch.bool, device="cuda")
    M = u.shape[0]
    for lo, hi, i in segments(t):
        inside[lo:hi] = True
        b0 = t["dbase"][lo:hi].double() if base else None
        if i < 0:
            if have_dx:
                assert torch.equal(dx[lo:hi], t["dbase"][lo:hi] if base else torch.zeros_like(dx[lo:hi]))
            continue
        s = float(t["scale"][i]) if t["scale"] is not None else 1.0
        dy, x, uu = t["dy"][lo:hi].double(), t["x"][lo:hi].double(), u[lo:hi].double()
        te, dt, xe, dxe = rows_exact(dy, t["b"][i].double().T, t["a"][i].double().T, b0, s, R, t["x"].dtype)
        if have_dx:
            check_rows(dx[lo:hi], xe, dxe, "dx")
        te, dt = s * te, s * dt + 2.0 ** -23 * s * te.abs()
        ea[i] += te.T @ x
        ta[i] += dt.T @ x.abs() + product_error(M, 24) * (te.abs().T @ x.abs())
        eb[i] += s * (dy.T @ uu)
        tb[i] += s * (product_error(M, 24) + 2.0 ** -23) * (dy.abs().T @ uu.abs())
    check_rows(da, ea, ta, "da")
    check_rows(db, eb, tb, "db")
    if have_dx:
        assert torch.equal(dx[~inside], before[~inside])


@pytest.mark.gpu
@pytest.mark.parametrize("xt,wt", TYPES)
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s[:4])))
def test_backward(shape, xt, wt):
    t = make(*shape, xt=xt, wt=wt)
    M, K, R = t["x"].shape[0], t["x"].shape[1], t["a"].shape[1]
    u = torch.randn(M, R, device="cuda")
    dx = torch.full((M, K), -7.0, dtype=xt, device="cuda")
    before = dx.clone()
    _, da, db = fpq.fpq_adapter_backward(t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"], t["dbase"], dx)
    check_backward(t, u, dx, da, db, before)


@pytest.mark.gpu
@pytest.mark.parametrize("xt", [F32, HF])
def test_backward_strides_in_place_and_without_dx(xt):
    t = make(210, 640, 320, 16, [0, 90, 100, 205], [1, -1, 0], 3, xt, xt, ldx=643, ldy=328)
    u = torch.randn(210, 16, device="cuda")
    args = (t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"])
    none, da, db = fpq.fpq_adapter_backward(*args, need_dx=False)
    assert none is None
    check_backward(t, u, None, da, db, None, have_dx=False)
    dx = t["dbase"].clone()
    before = dx.clone()
    _, da2, db2 = fpq.fpq_adapter_backward(*args, base=dx, dx=dx)
    check_backward(t, u, dx, da2, db2, before)
    assert torch.equal(da, da2) and torch.equal(db, db2)
    assert not bool(da2[2].any()) and not bool(db2[2].any())          # an adapter without rows


@pytest.mark.gpu
@pytest.mark.parametrize("xt", [F32, BF])
def test_tensors_at_any_element(xt):
    """Every tensor one element behind an aligned address."""
    def behind(v):
        flat = torch.empty(v.numel() + 1, dtype=v.dtype, device="cuda")[1:]
        return flat.view(v.shape).copy_(v)

    M, K, N, R, G = 150, 96, 64, 16, 2
    t = {k: behind(v) for k, v in make(M, K, N, R, [0, 60, 148], [1, 0], G, xt, xt).items()}
    y, u = behind(torch.full((M, N), -7.0, device="cuda").to(xt)), behind(torch.full((M, R), -7.0, device="cuda"))
    before = y.clone()
    fpq.fpq_adapter_forward(t["x"], t["a"], t["b"], t["offsets"], t["ids"], t["scale"], t["base"], y, u)
    check_forward(t, before, y, u)
    dx, da, db = behind(torch.full((M, K), -7.0, device="cuda").to(xt)), behind(torch.empty_like(t["a"], dtype=F32)), behind(torch.empty_like(t["b"], dtype=F32))
    before = dx.clone()
    fpq.fpq_adapter_backward(t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"], t["dbase"], dx, da, db)
    check_backward(t, u, dx, da, db, before)


@pytest.mark.gpu
def test_backward_without_rows_gives_zeros():
    for M, cuts, ids in ((0, [0, 0], [0]), (4, [0], [])):
        t = make(M, 40, 24, 4, cuts, ids, 2)
        _, da, db = fpq.fpq_adapter_backward(t["dy"], t["x"], torch.zeros(M, 4, device="cuda"), t["a"], t["b"], t["offsets"], t["ids"])
        assert not bool(da.any()) and not bool(db.any())


@pytest.mark.gpu
def test_gradients_against_differences():
    """y is linear in each of x, A and B alone: <dy, y(A + d) - y(A)> is <dA, d> but for rounding (64-bit sums of FP32 results)."""
    t = make(150, 96, 80, 8, [0, 70, 150], [1, 0], 2)

    def forward(**changed):
        c = {**t, **changed}
        y, u = torch.zeros(150, 80, device="cuda"), torch.zeros(150, 8, device="cuda")
        fpq.fpq_adapter_forward(c["x"], c["a"], c["b"], c["offsets"], c["ids"], c["scale"], None, y, u)
        return y.double(), u

    y0, u = forward()
    dy = t["dy"].double()
    dx, da, db = fpq.fpq_adapter_backward(t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"])
    for name, grad in (("x", dx), ("a", da), ("b", db)):
        d = torch.randn_like(t[name])
        moved = (t[name] + d)                                          # (rounded: the step that was made is moved - t[name])
        y1, _ = forward(**{name: moved})
        lhs = float((dy * (y1 - y0)).sum())
        rhs = float((grad.double() * (moved.double() - t[name].double())).sum())
        # each y is off by less than 2^-16 of its magnitude (product_error of 96 and 8 terms, twice the sum of magnitudes)
        size = float((dy.abs() * (y1.abs() + y0.abs())).sum()) + float((grad.double().abs() * d.double().abs()).sum())
        assert abs(lhs - rhs) <= 2.0 ** -15 * size, (name, lhs, rhs)


@pytest.mark.gpu
def test_equal_calls_give_equal_bits_on_two_streams():
    t = make(2000, 640, 320, 16, [0, 700, 2000], [1, 0], 2)
    u = torch.randn(2000, 16, device="cuda")
    args = (t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"])
    want = fpq.fpq_adapter_backward(*args)
    torch.cuda.synchronize()
    got, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(4):
        for s in streams:
            with torch.cuda.stream(s):
                got.append(fpq.fpq_adapter_backward(*args))
    torch.cuda.synchronize()
    for g in got:
        assert all(torch.equal(a, b) for a, b in zip(g, want))


GRAD_TILES = [  # M, K, N, R, cuts, ids, G: BF16 rows whose gradients come from tcgen05 tiles of 128 columns and runs of 64 rows
    (2048, 128, 64, 16, [0, 2048], [0], 1),
    (2100, 8, 16, 4, [0, 63, 127, 128, 2100], [0, 1, 0, 0], 2),
    (2777, 200, 328, 32, [3, 70, 70, 1000, 2769], [1, 0, 2, 4], 5),
    (4099, 320, 136, 12, list(range(0, 4100, 41)), [i % 3 for i in range(99)], 3),
    (3001, 648, 264, 20, [0, 1, 2, 66, 3001], [0, 1, 1, 0], 2),
    (5000, 136, 520, 64, [0, 2500, 4990], [1, 0], 2),
    (2050, 1288, 72, 40, [0, 1025, 2050], [-1, 0], 1),
    (30000, 64, 64, 8, [0, 29000, 30000], [0, 1], 2),
    (6000, 128, 64, 8, [0] + list(range(40, 4041, 50)) + [6000], [i % 41 for i in range(81)] + [7], 41),
    (9000, 64, 128, 24, [0, 8800] + list(range(8801, 8900)), [i % 32 for i in range(100)], 32),
    (1030, 72, 72, 4, [0, 300, 1029], [1, 0], 2),
    (1500, 136, 200, 128, [0, 600, 1499], [1, 0], 2),
    (5000, 320, 72, 100, [0, 4000, 4500, 5000], [0, 0, 1], 3),
]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", GRAD_TILES, ids=lambda s: "x".join(map(str, s[:4])))
def test_gradients_by_tiles(shape):
    M, K, N, R, cuts, ids, G = shape
    t = make(M, K, N, R, cuts, ids, G, BF, BF)
    outside = torch.ones(M, dtype=torch.bool, device="cuda")
    for lo, hi, i in segments(t):
        outside[lo:hi] = i < 0
    u = torch.randn(M, R, device="cuda")
    for v in (t["x"], t["dy"], u):                         # rows of no adapter hold what they like
        v[outside] = float("nan")
    t["dbase"][outside] = 0
    dx = torch.zeros_like(t["x"])
    got = fpq.fpq_adapter_backward(t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"], None, dx)
    check_backward(t, u, *got, torch.zeros_like(dx), base=False)
    again = fpq.fpq_adapter_backward(t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"], need_dx=False)
    assert torch.equal(got[1], again[1]) and torch.equal(got[2], again[2])


@pytest.mark.gpu
@pytest.mark.parametrize("K,N,ldx,ldy", [(1, 3, 8, 8), (5, 130, 16, 136), (200, 64, 1000, 2000)])
def test_gradients_by_tiles_in_slices(K, N, ldx, ldy):
    M, R = 1700, 8
    t = make(M, K, N, R, [0, 900, 1690], [1, 0], 2, BF, BF, ldx=ldx, ldy=ldy)
    u, dx = torch.randn(M, R, device="cuda"), torch.zeros(M, K, dtype=BF, device="cuda")
    got = fpq.fpq_adapter_backward(t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"], None, dx)
    check_backward(t, u, *got, torch.zeros_like(dx), base=False)


@pytest.mark.gpu
@pytest.mark.parametrize("xt", [F32, HF])
@pytest.mark.parametrize("G", [32, 33])
def test_gradients_of_many_adapters_that_share_blocks(G, xt):
    cuts = [0, 5000] + [5000 + 13 * i for i in range(1, 60)] + [6400]
    t = make(6400, 64, 48, 8, cuts, [i * 7 % (G + 1) for i in range(61)], G, xt, xt)
    u, dx = torch.randn(6400, 8, device="cuda"), torch.zeros_like(t["x"])
    got = fpq.fpq_adapter_backward(t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"], None, dx)
    check_backward(t, u, *got, torch.zeros_like(dx), base=False)


@pytest.mark.gpu
@pytest.mark.parametrize("value", [float("inf"), float("nan"), 3.3e38])
def test_gradients_by_tiles_of_values_that_are_not_finite(value):
    t = make(2200, 136, 72, 16, [0, 1000, 2200], [0, 1], 2, BF, BF)
    u = torch.randn(2200, 16, device="cuda")
    t["x"][500, 3] = value
    t["x"][600, 3] = -1.0
    t["dy"][1500, 5] = value
    u[700, 2] = value
    _, da, db = fpq.fpq_adapter_backward(t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"], need_dx=False)
    for i, (lo, hi) in enumerate(((0, 1000), (1000, 2200))):
        dy, x, s = t["dy"][lo:hi].float(), t["x"][lo:hi].float(), float(t["scale"][i])
        ea, eb = (s * (dy.double() @ t["b"][i].double())).T @ x.double(), s * (dy.double().T @ u[lo:hi].double())
        for got, want in ((da[i], ea), (db[i], eb)):
            fits = want.abs() < 3.0e38                     # (NaN and infinities are not; in between, FP32 sums may run over)
            assert bool(torch.isfinite(got[fits & (want.abs() < 1e37)]).all())
            assert not bool(torch.isfinite(got[~(want.abs() <= 3.5e38)]).any())


@pytest.mark.gpu
def test_workspaces_hold_nothing_between_calls():
    # many blocks share each sum: whatever the workspace holds, and after a call of other sizes in it, the bits are the same
    t, other = make(4000, 640, 320, 24, [0, 1500, 4000], [1, 0], 2), make(900, 96, 200, 8, [0, 900], [0], 1)
    u, v = torch.randn(4000, 24, device="cuda"), torch.randn(900, 8, device="cuda")
    work = torch.empty(fpq.fpq_adapter_backward_workspace_size(4000, 320, 640, 2, 24, fpq.FP32), dtype=torch.uint8, device="cuda")
    want = None
    for fill in (0, 255, 1):
        work.fill_(fill)
        for _ in range(2):
            got = fpq.fpq_adapter_backward(t["dy"], t["x"], u, t["a"], t["b"], t["offsets"], t["ids"], t["scale"], workspace=work)
            want = want or got
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            fpq.fpq_adapter_backward(other["dy"], other["x"], v, other["a"], other["b"], other["offsets"], other["ids"], workspace=work)


@pytest.mark.gpu
@pytest.mark.parametrize("xt", [F32, BF])
def test_another_adapters_values_change_no_bit(xt):
    # the last 64 columns of adapter 0 reach into adapter 1's rows of B, its last ranks into those of A: infinite ones may not change how
    # its own rows are worked out
    t = make(21000, 648, 328, 40, [0, 20000, 21000], [0, 1], 2, xt, xt)
    assert fpq.fpq_adapter_route(21000, 328, 648, 2, 40, 2, fpq._REAL[xt], fpq._REAL[xt]) == fpq.ADAPTER_TILES
    _, y, u = run_forward(t)
    t["b"][1] = float("inf")
    t["a"][1] = float("nan")
    _, z, v = run_forward(t)
    assert torch.equal(y[:20000], z[:20000]) and torch.equal(u[:20000], v[:20000])
    assert not bool(torch.isfinite(z[20000:]).any())


@pytest.mark.gpu
def test_binding_refuses():
    t = make(10, 32, 16, 4, [0, 10], [0], 1)
    ok = [t["x"], t["a"], t["b"], t["offsets"], t["ids"], t["scale"], t["base"], torch.zeros(10, 16, device="cuda"), None]
    for at, bad in ((0, t["x"].double()), (0, t["x"].T), (0, t["x"][:, :31]), (0, t["x"][:1].expand(10, 32)), (1, t["a"].half()), (1, t["a"][0]),
                    (2, t["b"][:, :15]), (3, t["offsets"].long()), (3, t["offsets"][:1]), (4, t["ids"].cpu()), (5, t["scale"].half()),
                    (6, t["base"][:9]), (6, t["base"].bfloat16()), (7, torch.zeros(9, 16, device="cuda")), (8, torch.zeros(10, 5, device="cuda"))):
        with pytest.raises(AssertionError):
            fpq.fpq_adapter_forward(*(bad if i == at else v for i, v in enumerate(ok)))
    big = torch.zeros(1, 129, 32, device="cuda"), torch.zeros(1, 16, 129, device="cuda")
    with pytest.raises(fpq.FpqError, match="shape"):
        fpq.fpq_adapter_forward(t["x"], *big, *ok[3:])
    with pytest.raises(fpq.FpqError, match="unsupported"):
        fpq.fpq_adapter_forward(t["x"].half(), t["a"], t["b"], t["offsets"], t["ids"])


def test_ctypes_signature_matches_the_header():
    assert ctypes.sizeof(fpq._CAdamwTensor) == 64
