"""The AdamW step over many tensors: FP32 moments against the formulas in 64 bits, 8-bit moments bit for bit."""
import ctypes
import math

import numpy as np
import pytest
import torch

import paper_2408_06995_b200 as fpq
from paper_2408_06995_b200 import build as fpq_build

fpq_build.build()
F32, BF, HF = torch.float32, torch.bfloat16, torch.float16


# ---- refusals, without a GPU ------------------------------------------------------------------------------------------

class Options(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("lr", "beta1", "beta2", "eps", "weight_decay")] + [("seed", ctypes.c_uint32), ("reserved", ctypes.c_uint32)]


def call(count=1, g_type=fpq.FP32, copy_type=fpq.BF16, state_type=fpq.FP32, step=4096, factors=None, tensors=True, options=True, tensor=None, **opt):
    o = Options(**{"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01, **opt})
    t = (fpq._CAdamwTensor * max(1, count))()
    for e in t:
        for k, v in {**dict.fromkeys(("p", "g", "m", "v", "m_scale", "v_scale", "copy"), 4096), "n": 10, **(tensor or {})}.items():
            setattr(e, k, v)
    return fpq.lib().fpq_adamw_step(t if tensors else None, count, g_type, copy_type, state_type, ctypes.byref(o) if options else None, factors,
                                    step, None)


@pytest.mark.parametrize("given,error", [
    ({"g_type": 3}, "ERR_UNSUPPORTED"), ({"copy_type": fpq.FP32}, "ERR_UNSUPPORTED"), ({"state_type": fpq.BF16}, "ERR_UNSUPPORTED"),
    ({"count": -1}, "ERR_SHAPE"), ({"lr": math.inf}, "ERR_SHAPE"), ({"beta1": 1.0}, "ERR_SHAPE"), ({"beta1": -0.1}, "ERR_SHAPE"),
    ({"beta2": math.nan}, "ERR_SHAPE"), ({"eps": -1e-8}, "ERR_SHAPE"), ({"eps": math.nan}, "ERR_SHAPE"), ({"eps": 1e-39}, "ERR_SHAPE"), ({"weight_decay": math.inf}, "ERR_SHAPE"),
    ({"tensor": {"n": -1}}, "ERR_SHAPE"), ({"tensor": {"n": 1 << 40}}, "ERR_SHAPE"), ({"count": 2, "tensor": {"n": 1 << 39}}, "ERR_SHAPE"),
    ({"step": None}, "ERR_NULL"), ({"tensors": False}, "ERR_NULL"), ({"options": False}, "ERR_NULL"), ({"tensor": {"p": None}}, "ERR_NULL"),
    ({"tensor": {"g": None}}, "ERR_NULL"), ({"tensor": {"v": None}}, "ERR_NULL"),
    ({"state_type": fpq.E4M3_BLOCK32, "tensor": {"m_scale": None}}, "ERR_NULL"), ({"state_type": fpq.E4M3_BLOCK32, "tensor": {"v_scale": None}}, "ERR_NULL"),
    ({"step": 4100}, "ERR_ALIGN"), ({"factors": 4098}, "ERR_ALIGN"), ({"tensor": {"p": 4098}}, "ERR_ALIGN"), ({"tensor": {"g": 4098}}, "ERR_ALIGN"),
    ({"g_type": fpq.BF16, "tensor": {"g": 4097}}, "ERR_ALIGN"), ({"tensor": {"m": 4097}}, "ERR_ALIGN"), ({"tensor": {"copy": 4097}}, "ERR_ALIGN")])
def test_refuses(given, error):
    assert call(**given) == getattr(fpq, error)


def test_the_table_refuses_cpu_tensors():
    z = torch.zeros(4)
    with pytest.raises(AssertionError):
        fpq.fpq_adamw_table([z], [z.clone()], [z.clone()], [z.clone()])


# ---- the step, written out --------------------------------------------------------------------------------------------

def mix(z):
    z = np.uint32(z) * np.uint32(0x9E3779B1)
    z = z ^ (z >> np.uint32(15))
    z = z * np.uint32(0x243F6A89)
    return z ^ (z >> np.uint32(16))


def noise(first, n, t, seed):
    number = np.arange(first, first + n, dtype=np.uint64)
    with np.errstate(over="ignore"):
        high = (number >> np.uint64(32)).astype(np.uint32) * np.uint32(0x243F6A89)
        key = mix(np.uint32(t & 0xFFFFFFFF) * np.uint32(0x9E3779B1) + np.uint32(seed) + np.uint32(1) + high)
        z = mix((number & np.uint64(0xFFFFFFFF)).astype(np.uint32) ^ key)
    return (z >> np.uint32(16)).astype(np.int64), (z & np.uint32(0xFFFF)).astype(np.int64)


GRID = np.array([(c & 7) * 2.0 ** -9 if c < 8 else (1 + (c & 7) / 8) * 2.0 ** ((c >> 3) - 7) for c in range(127)])     # E4M3 magnitudes


def decode(codes, scale):
    mag = np.append(GRID, np.nan)[codes & 127] * np.where(codes & 128, -1.0, 1.0)
    return (mag.reshape(-1, 32) * np.ldexp(1.0, scale.astype(int) - 127)[:, None]).reshape(-1)


def encode(value, bits, least):
    """Codes by the definition: the FP32 value on the grid of its block, up by chance of the remainder, and the noise that decides."""
    v = value.reshape(-1, 32).astype(np.float64)
    finite = np.isfinite(v)
    top = np.where(finite, np.abs(v), 0).max(1)
    _, e = np.frexp(top)
    power = np.where(top > 0, np.maximum(e - 1 - 7, -126), -126)
    with np.errstate(invalid="ignore"):
        q = np.abs(np.ldexp(v, -power[:, None]))
    # (scaling by a power of two is exact in FP32 but for what falls below its smallest numbers)
    q32 = np.where(finite, q, 0).astype(np.float32).astype(np.float64)
    below = np.clip(np.searchsorted(GRID, q32.reshape(-1), "right") - 1, 0, 125).reshape(q32.shape)
    step = GRID[below + 1] - GRID[below]
    # the remainder as a fraction of the step, in 20 bits: below 2^-6 what FP32 keeps of it next to 2^-6
    fine = np.where(q32 < 2.0 ** -6, (q32.astype(np.float32) + np.float32(2.0 ** -6)).astype(np.float64) - 2.0 ** -6, q32)
    below = np.where((q32 < 2.0 ** -6), np.floor(fine / 2.0 ** -9).astype(int), below)
    rest = np.floor((fine - GRID[np.minimum(below, 126)]) / step * 2 ** 20).astype(np.int64)
    code = below + ((rest + bits.reshape(rest.shape) * 16) >= 2 ** 20)
    code = np.where((q32 > 0) & (code < least), least, code)
    code = np.where((code > 0) & (v < 0), code | 128, code)
    return np.where(finite, code, 127).reshape(-1).astype(np.uint8), (power + 127).astype(np.uint8)


def moments(g, m, v, o, factor=None):
    """m and v (FP32, each product and sum rounded on its own) as the header defines them."""
    f = np.float32
    g = g.astype(f)
    if factor is not None:
        g = g * f(factor)
    m = m * f(o["beta1"]) + g * f(1 - o["beta1"])
    v = v * f(o["beta2"]) + (g * g) * f(1 - o["beta2"])
    return m.astype(f), v.astype(f)


def pad(a):
    return np.concatenate([a, np.zeros(-len(a) % 32, a.dtype)])


O = {"lr": 2e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.02}


def check_p(got, p, m, v, t, o, rate=None, ulps=8):
    """p' from the new FP32 moments: eight FP32 operations and an approximate division (2 units in the last place) on the update."""
    rate = o["lr"] if rate is None else rate
    m, v, p = m.astype(np.float64), v.astype(np.float64), p.astype(np.float64)
    update = rate / (1 - o["beta1"] ** t) * m / (np.sqrt(v) / math.sqrt(1 - o["beta2"] ** t) + o["eps"])
    want = p * (1 - rate * o["weight_decay"]) - update
    tol = 2.0 ** -24 * (3 * np.abs(p) + 2 * ulps * np.abs(update) + np.abs(want)) + 1e-44
    assert np.all(np.abs(got.astype(np.float64) - want) <= tol), float((np.abs(got - want) / tol).max())


def make(sizes, g_type, codes, copy, seed=0, off=0):
    """Tensors of the given sizes; off: elements by which each lies behind an aligned address."""
    g = torch.Generator(device="cuda").manual_seed(seed)

    def tensors(f, dtype=F32, unit=1):
        out = []
        for n in sizes:
            n = -(-n // unit)
            out.append(f(n + off).to(dtype)[off:])
        return out

    def normal(n):
        return torch.randn(n, generator=g, device="cuda")

    t = {"params": tensors(lambda n: normal(n)), "grads": tensors(lambda n: normal(n) * 10.0 ** (torch.rand(n, generator=g, device="cuda") * 4 - 5), g_type)}
    if codes:
        t["m"] = [c.view(torch.uint8) for c in tensors(lambda n: (normal(n) * 60).clamp(-250, 250), torch.float8_e4m3fn)]
        t["v"] = [c.view(torch.uint8) for c in tensors(lambda n: (normal(n).abs() * 60).clamp(0, 250), torch.float8_e4m3fn)]
        t["m_scale"] = tensors(lambda n: torch.randint(104, 112, (n,), generator=g, device="cuda"), torch.uint8, 32)
        t["v_scale"] = tensors(lambda n: torch.randint(104, 112, (n,), generator=g, device="cuda"), torch.uint8, 32)
    else:
        t["m"], t["v"] = tensors(lambda n: normal(n) * 1e-3), tensors(lambda n: normal(n) ** 2 * 1e-6)
    t["copies"] = tensors(lambda n: normal(n), copy) if copy else None
    return t


def host(ts):
    return [[x.detach().float().cpu().numpy() if x.dtype in (F32, BF, HF) else x.cpu().numpy() for x in t] if t is not None else None for t in ts]


def counter(t):
    return torch.tensor([t, 0], dtype=torch.int64, device="cuda")


def check_step(t, before, sizes, made, codes, seed=0, o=O, factors=None):
    keys = ["params", "grads", "m", "v"] + (["m_scale", "v_scale"] if codes else [])
    now = dict(zip(keys, host([t[k] for k in keys])))
    rate = o["lr"] * (factors[0] if factors else 1.0)
    first = 0
    for i, n in enumerate(sizes):
        b = {k: before[k][i] for k in keys}
        if codes:
            m = decode(pad(b["m"]), b["m_scale"])[:n].astype(np.float32)
            r = decode(pad(b["v"]), b["v_scale"])[:n].astype(np.float32)
            v = r * r
        else:
            m, v = b["m"], b["v"]
        m, v = moments(b["grads"], m, v, o, factors[1] if factors else None)
        check_p(now["params"][i], b["params"], m, v, made + 1, o, rate)
        if t["copies"] is not None and t["copies"][i] is not None:
            assert torch.equal(t["copies"][i], t["params"][i].to(t["copies"][i].dtype))
        if codes:
            for k, value, which, least in (("m", m, 0, 0), ("v", np.sqrt(v), 1, 1)):
                c, s = encode(pad(value), noise(first, -(-n // 32) * 32, made + 1, seed)[which], least)
                assert np.array_equal(now[k + "_scale"][i], s), (k, i)
                assert np.array_equal(now[k][i], c[:n]), (k, i, np.nonzero(now[k][i] != c[:n])[0][:5])
        else:
            assert np.array_equal(now["m"][i], m) and np.array_equal(now["v"][i], v)
        first += -(-n // 32) * 32


def snapshot(t, codes):
    keys = ["params", "grads", "m", "v"] + (["m_scale", "v_scale"] if codes else [])
    return dict(zip(keys, host([t[k] for k in keys])))


def table(t):
    return fpq.fpq_adamw_table(t["params"], t["grads"], t["m"], t["v"], t.get("m_scale"), t.get("v_scale"), t["copies"])


SIZES = {"one": [1], "few": [5, 32, 33, 1000], "sixteen": [100 + 7 * i for i in range(16)], "seventeen": [31 + i for i in range(17)],
         "runs": [1024, 1025, 4096, 4097, 12288], "many": [17 + i % 90 for i in range(805)], "empty_ones": [0, 64, 0, 3, 0],
         "large": [3000001, 2500000, 77]}


@pytest.mark.gpu
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("g_type,copy", [(F32, None), (BF, BF), (HF, HF)])
@pytest.mark.parametrize("name", SIZES)
def test_step(name, g_type, copy, codes):
    sizes = SIZES[name]
    t = make(sizes, g_type, codes, copy)
    before = snapshot(t, codes)
    step = counter(41)
    fpq.fpq_adamw_step(table(t), step, seed=77, **O)
    check_step(t, before, sizes, 41, codes, 77)
    assert step.tolist() == [42, 0]


@pytest.mark.gpu
@pytest.mark.parametrize("codes", [False, True])
@pytest.mark.parametrize("off", [1, 2, 3])
def test_unaligned_tensors(codes, off):
    sizes = [100, 4097, 31]
    t = make(sizes, BF, codes, HF, off=off)
    before = snapshot(t, codes)
    fpq.fpq_adamw_step(table(t), counter(0), seed=5, **O)
    check_step(t, before, sizes, 0, codes, 5)


@pytest.mark.gpu
@pytest.mark.parametrize("codes", [False, True])
def test_neighbours_stay_as_they_are(codes):
    """Parameters and states that are slices of one storage: what lies between them is not written."""
    flat = {k: torch.full((400,), 3, dtype=d, device="cuda") for k, d in
            (("params", F32), ("grads", F32), ("m", torch.uint8 if codes else F32), ("v", torch.uint8 if codes else F32))}
    t = {k: [f[1:98], f[131:300]] for k, f in flat.items()}
    t["copies"] = None
    if codes:
        scales = {k: torch.full((20,), 120, dtype=torch.uint8, device="cuda") for k in ("m_scale", "v_scale")}
        t.update({k: [s[1:5], s[9:15]] for k, s in scales.items()})
    keep = torch.ones(400, dtype=torch.bool, device="cuda")
    keep[1:98] = keep[131:300] = False
    fpq.fpq_adamw_step(table(t), counter(0), **O)
    for f in flat.values():
        assert bool((f[keep] == 3).all())
    if codes:
        for s in scales.values():
            assert bool((s[5:9] == 120).all()) and bool((s[15:] == 120).all()) and int(s[0]) == 120


@pytest.mark.gpu
@pytest.mark.parametrize("codes", [False, True])
def test_the_first_steps_from_zeros(codes):
    sizes = [2000, 333]
    t = make(sizes, F32, codes, None)
    for k in ("m", "v") + (("m_scale", "v_scale") if codes else ()):
        for x in t[k]:
            x.zero_()
    t["grads"][0][::3] = 0.0                       # never a gradient: the parameter only decays
    tab, step = table(t), counter(0)
    p0 = t["params"][0][::3].clone()
    for made in range(3):
        before = snapshot(t, codes)
        fpq.fpq_adamw_step(tab, step, seed=9, **O)
        check_step(t, before, sizes, made, codes, 9)
    # three products, and the constant itself, rounded
    want = p0.double() * (1 - O["lr"] * O["weight_decay"]) ** 3
    assert bool(((t["params"][0][::3].double() - want).abs() <= 6 * 2.0 ** -24 * want.abs()).all())


@pytest.mark.gpu
@pytest.mark.parametrize("codes", [False, True])
def test_captured_steps_count_on(codes):
    sizes = [700, 64]
    t, f = make(sizes, F32, codes, BF), torch.tensor([0.5, 2.0], device="cuda")
    twin = {k: [x.clone() for x in v] for k, v in t.items()}
    tab, step, step2 = table(t), counter(0), counter(0)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        fpq.fpq_adamw_step(tab, step, seed=3, factors=f, **O)
    tab2 = table(twin)
    for made in range(4):
        f.copy_(torch.tensor([0.5 + made, 2.0 - made / 4]))
        for a, b in zip(t["grads"], twin["grads"]):
            a.normal_()
            b.copy_(a)
        graph.replay()
        before = snapshot(twin, codes)
        fpq.fpq_adamw_step(tab2, step2, seed=3, factors=f, **O)
        check_step(twin, before, sizes, made, codes, 3, factors=f.tolist())
    assert step.tolist() == step2.tolist() == [4, 0]
    for k in t:
        assert all(torch.equal(a, b) for a, b in zip(t[k], twin[k])), k


@pytest.mark.gpu
def test_stochastic_rounding_keeps_the_mean():
    """A moment that moves by far less than a code's step follows its recursion on the average: 4096 elements, 300 steps of
    v = 0.999 v + 0.001 from 0.25 towards 1; rounded to nearest it would stay at 0.25."""
    n, steps = 4096, 300
    t = {"params": [torch.zeros(n, device="cuda")], "grads": [torch.ones(n, device="cuda")], "copies": None,
         "m": [torch.zeros(n, dtype=torch.uint8, device="cuda")], "v": [torch.full((n,), 0.5, device="cuda").to(torch.float8_e4m3fn)],
         "m_scale": [torch.zeros(n // 32, dtype=torch.uint8, device="cuda")], "v_scale": [torch.full((n // 32,), 127, dtype=torch.uint8, device="cuda")]}
    tab, step = table(t), counter(0)
    for _ in range(steps):
        fpq.fpq_adamw_step(tab, step, lr=0.0)
    r = decode(t["v"][0].view(torch.uint8).cpu().numpy(), t["v_scale"][0].cpu().numpy())
    path = math.sqrt(1 - 0.75 * 0.999 ** steps)
    # f(r) = sqrt(0.999 r^2 + 0.001) increases and is convex, and each rounding leaves the mean of f(r) as it is: the mean is never below
    # the path (Jensen), and exceeds it by f'' <= 0.001 / r^3 times half the variance a step (which only grows from the common start)
    sigma = r.std() / math.sqrt(n)
    assert r.mean() >= path - 6 * sigma
    assert r.mean() <= path + steps * 0.5 * 0.001 * (r ** -3.0).max() * r.var() + 6 * sigma
    assert path > 0.65 and r.mean() < 0.8


@pytest.mark.gpu
def test_values_that_are_not_finite():
    t = make([96], F32, True, None)
    t["grads"][0][3], t["grads"][0][40], t["grads"][0][70] = float("inf"), float("nan"), 3e38
    before = snapshot(t, True)
    with np.errstate(over="ignore", invalid="ignore"):
        fpq.fpq_adamw_step(table(t), counter(10), seed=1, **O)
        m = t["m"][0].cpu()
        assert int(m[3]) & 127 == 127 and int(m[40]) & 127 == 127          # 3e38 squared is infinite: the square root's code is NaN
        assert int(t["v"][0][3]) == int(t["v"][0][40]) == int(t["v"][0][70]) == 127
        mm = decode(before["m"][0], before["m_scale"][0]).astype(np.float32)
        rr = decode(before["v"][0], before["v_scale"][0]).astype(np.float32)
        new_m, new_v = moments(before["grads"][0], mm, rr * rr, O)
        for k, value, which, least in (("m", new_m, 0, 0), ("v", np.sqrt(new_v), 1, 1)):
            c, s = encode(value, noise(0, 96, 11, 1)[which], least)
            assert np.array_equal(t[k][0].cpu().numpy() & (127 + 128 * (c != 127)), c) and np.array_equal(t[k + "_scale"][0].cpu().numpy(), s)
    others = torch.ones(96, dtype=torch.bool)
    others[[3, 40, 70]] = False
    assert bool(torch.isfinite(t["params"][0].cpu()[others]).all())


@pytest.mark.gpu
def test_tiny_and_huge_moments():
    """Blocks whose largest magnitude is zero, below FP32's normal numbers, or near its largest."""
    g = torch.zeros(128, device="cuda")
    g[32:64] = 1e-39
    g[64:96] = 1e-22
    g[96:] = 1.5e19
    t = {"params": [torch.ones(128, device="cuda")], "grads": [g], "m": [torch.zeros(128, dtype=torch.uint8, device="cuda")],
         "v": [torch.zeros(128, dtype=torch.uint8, device="cuda")], "copies": None,
         "m_scale": [torch.zeros(4, dtype=torch.uint8, device="cuda")], "v_scale": [torch.zeros(4, dtype=torch.uint8, device="cuda")]}
    before = snapshot(t, True)
    fpq.fpq_adamw_step(table(t), counter(0), seed=2, **O)
    check_step(t, before, [128], 0, True, 2)


@pytest.mark.gpu
def test_a_tensor_of_more_than_2_to_31_elements():
    n, tail, o = (1 << 31) + 4131, 1000, {**O, "lr": 0.5}
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=BF, device="cuda")
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    scales = [torch.zeros(-(-n // 32), dtype=torch.uint8, device="cuda") for _ in range(2)]
    first = n - tail - (n - tail) % 32                    # a block's first element
    g[first:] = torch.randn(n - first, device="cuda").bfloat16()
    step = counter(0)
    fpq.fpq_adamw_step(fpq.fpq_adamw_table([p], [g], [m], [v], [scales[0]], [scales[1]]), step, seed=1, **o)
    gg = g[first:].float().cpu().numpy()
    new_m, new_v = moments(gg, np.zeros_like(gg), np.zeros_like(gg), o)
    check_p(p[first:].cpu().numpy(), np.zeros_like(gg), new_m, new_v, 1, o)
    for k, s, value, which, least in ((m, scales[0], new_m, 0, 0), (v, scales[1], np.sqrt(new_v), 1, 1)):
        c, e = encode(pad(value), noise(first, -(-len(gg) // 32) * 32, 1, 1)[which], least)
        assert np.array_equal(k[first:].cpu().numpy(), c[:len(gg)]) and np.array_equal(s[first // 32:].cpu().numpy(), e)
    assert not bool(p[:first].any())


@pytest.mark.gpu
def test_no_tensors_still_count():
    step = counter(7)
    fpq.fpq_adamw_step(fpq.fpq_adamw_table([], [], [], []), step, lr=1e-3)
    assert step.tolist() == [8, 0]


@pytest.mark.gpu
def test_binding_refuses():
    t = make([64, 64], F32, False, None)
    tab = table(t)
    for bad in (torch.zeros(1, dtype=torch.int64, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int64)):
        with pytest.raises(AssertionError):
            fpq.fpq_adamw_step(tab, bad, lr=1e-3)
    with pytest.raises(AssertionError):
        fpq.fpq_adamw_step(tab, counter(0), lr=1e-3, factors=torch.zeros(1, device="cuda"))
    with pytest.raises(ValueError):
        fpq.fpq_adamw_step(tab, counter(0), lr=1e-3, seed=-1)
    with pytest.raises(fpq.FpqError):
        fpq.fpq_adamw_step(tab, counter(0), lr=1e-3, beta1=1.0)
    p, g, m, v = t["params"], t["grads"], t["m"], t["v"]
    for args in (([p[0], p[0]], g, m, v), (p, g, m, m), (p, g[:1], m, v), (p, [g[0], g[1].bfloat16()], m, v), ([p[0], p[1].double()], g, m, v),
                 ([p[0], p[1][::2]], g, m, v), (p, g, [m[0], m[1][:63]], v)):
        with pytest.raises(AssertionError):
            fpq.fpq_adamw_table(*args)
    codes = make([64], F32, True, None)
    with pytest.raises(AssertionError):
        fpq.fpq_adamw_table(codes["params"], codes["grads"], codes["m"], codes["v"])
