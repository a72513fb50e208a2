"""What the speed of training and serving low-rank adapters beside quantized layers is measured on.

Three operators, each in its plain form (elementary torch operations in 32 bits) and as the call of this library:

  forward   y_i = base_i + s_a B_a (A_a x_i) for the rows i of every request, a the request's adapter: rows of many requests
            at once, the base usually the output of the shared quantized projection;
  backward  its gradients: dx_i = base_i + A_a^T (s_a B_a^T dy_i), dA_a = sum_i (s_a B_a^T dy_i) x_i^T,
            dB_a = sum_i s_a dy_i (A_a x_i)^T over the rows of adapter a;
  adamw     one AdamW step over many tensors at once, moments in 32 bits or in 8 (E4M3 codes with a power-of-two scale per 32
            elements; the second moment as its square root; stochastic rounding by a hash of seed, step and element number).

Layer widths are those of the Stable-Diffusion-v1-style U-Net (320, 640, 1280; contexts of 768), row counts those of its
latents and of single tokens.
"""
import math

import torch

own = False

TYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
BYTES = {"fp32": 4, "bf16": 2, "fp16": 2}
C1, C2, M32 = 0x9E3779B1, 0x243F6A89, 0xFFFFFFFF


def listed():
    return [
        # serving, the smallest call: one row (a time embedding's projection, or one token) through one adapter
        {"name": "forward_one_row", "op": "forward", "M": 1, "K": 1280, "N": 1280, "R": 16, "G": 4, "S": 1, "x": "fp32", "w": "bf16",
         "base": True, "save": False, "tail": 0},
        # serving single tokens of 64 requests, an adapter of its own for each
        {"name": "forward_64_tokens", "op": "forward", "M": 64, "K": 1280, "N": 1280, "R": 16, "G": 64, "S": 64, "x": "bf16", "w": "bf16",
         "base": True, "save": False, "tail": 0},
        # a batch of images of odd sizes, each request with its own adapter or none, padded behind the last: QKV projection
        {"name": "forward_ragged_qkv", "op": "forward", "M": 9001, "K": 320, "N": 960, "R": 24, "G": 5, "S": 7, "x": "fp32", "w": "fp16",
         "base": True, "save": False, "tail": 55},
        # training one adapter on a 64 x 64 latent, batch 2: the forward pass that keeps A x for the backward one
        {"name": "forward_train_ffn", "op": "forward", "M": 8192, "K": 1280, "N": 320, "R": 16, "G": 1, "S": 1, "x": "fp32", "w": "fp32",
         "base": True, "save": True, "tail": 0},
        # throughput serving: the feed-forward input of a batch of 8, 4 adapters of rank 64
        {"name": "forward_geglu_batch8", "op": "forward", "M": 32768, "K": 320, "N": 2560, "R": 64, "G": 4, "S": 8, "x": "bf16", "w": "bf16",
         "base": True, "save": False, "tail": 0},
        # training on a text context of 77 rows (cross-attention keys)
        {"name": "backward_context_77", "op": "backward", "M": 77, "K": 768, "N": 320, "R": 4, "G": 1, "S": 1, "x": "fp32", "w": "fp32",
         "base": True, "tail": 0},
        # training the output projection of a 64 x 64 latent, batch 2, one adapter
        {"name": "backward_attn_out", "op": "backward", "M": 8192, "K": 640, "N": 640, "R": 16, "G": 1, "S": 1, "x": "fp32", "w": "fp32",
         "base": True, "tail": 0},
        # several adapters trained at once on a larger batch, 16-bit activations, odd lengths
        {"name": "backward_multi_bf16", "op": "backward", "M": 30011, "K": 1280, "N": 640, "R": 32, "G": 3, "S": 6, "x": "bf16", "w": "bf16",
         "base": False, "tail": 11},
        # the step of one layer's adapter
        {"name": "adamw_one_layer", "op": "adamw", "tensors": 2, "elements": 20480, "bits": 32, "grad": "fp32", "copy": None},
        # the step of the adapters of a whole U-Net, 16-bit copies for the forward pass written along
        {"name": "adamw_unet_adapters", "op": "adamw", "tensors": 256, "elements": 6200000, "bits": 32, "grad": "fp32", "copy": "bf16"},
        # the same with moments in 8 bits and 16-bit gradients
        {"name": "adamw_unet_adapters_8bit", "op": "adamw", "tensors": 256, "elements": 6200000, "bits": 8, "grad": "bf16", "copy": "bf16"},
        # rounding parameters of a level's 3 x 3 convolutions (five of 1280 x 1280 x 9), moments in 8 bits
        {"name": "adamw_rounding_8bit", "op": "adamw", "tensors": 5, "elements": 73728000, "bits": 8, "grad": "fp32", "copy": None},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    # most widths are multiples of 32; some are not even multiples of 4
    c = _log(rng, lo, hi)
    return c if rng.random() < 0.25 else max(32, c // 32 * 32)


def draw(rng):
    """One more call of the ranges above."""
    while True:
        op = rng.choice(["forward", "forward", "backward", "adamw"])
        if op == "adamw":
            t = _log(rng, 1, 300)
            c = {"op": op, "tensors": t, "elements": max(t, _log(rng, 1000, 60000000)), "bits": rng.choice([8, 32]),
                 "grad": rng.choice(["fp32", "bf16", "fp16"]), "copy": rng.choice([None, "bf16", "fp16"])}
        else:
            x = rng.choice(["fp32", "fp32", "bf16", "fp16"])
            S = _log(rng, 1, 64)
            M = S if rng.random() < 0.25 else _log(rng, S, 32768)
            c = {"op": op, "M": M, "K": _width(rng, 32, 2560), "N": _width(rng, 32, 2560), "R": rng.choice([1, 3, 4, 8, 16, 16, 24, 32, 64, 128]),
                 "G": rng.randint(1, max(1, min(S, 16))), "S": S, "x": x, "w": rng.choice(["fp32", "bf16", "fp16"]) if x == "fp32" else x,
                 "base": rng.random() < 0.7, "tail": min(M - 1, rng.choice([0, 0, 5, 130]))}
            if op == "forward":
                c["save"] = rng.random() < 0.3
            # the plain form multiplies every row by every adapter: bounded
            if c["M"] * c["G"] * c["R"] * (c["K"] + c["N"]) > 2e12:
                continue
        if work(c)["bytes"] <= work(listed()[-1])["bytes"]:
            return c


def work(c):
    if c["op"] == "adamw":
        n = c["elements"]
        state = 8 * 2 if c["bits"] == 32 else 2 * (2 + 2 / 32)
        return {"bytes": n * (8 + BYTES[c["grad"]] + state + (2 if c["copy"] else 0)), "flops": 15 * n}
    M, K, N, R = c["M"] - c["tail"], c["K"], c["N"], c["R"]
    xs, weights = BYTES[c["x"]], min(c["G"], c["S"]) * (K + N) * R * BYTES[c["w"]]
    if c["op"] == "forward":
        return {"bytes": M * K * xs + M * N * xs * (2 if c["base"] else 1) + weights + (4 * M * R if c["save"] else 0),
                "flops": 2 * M * R * (K + N)}
    return {"bytes": M * (K + N) * xs + M * K * xs * (2 if c["base"] else 1) + weights + 4 * M * R + 4 * c["G"] * (K + N) * R,
            "flops": 4 * M * R * (K + N)}


def _sizes(c):
    """Elements of each tensor: powers of two apart, odd ones among them, `elements` in all."""
    t, left = c["tensors"], c["elements"]
    weights = [1 + (7 * i) % 13 for i in range(t)] if t > 8 else [1] * t
    sizes = [max(1, c["elements"] * w // sum(weights)) for w in weights]
    sizes[-1] = max(1, left - sum(sizes[:-1]))
    return sizes


def _adamw_options(c):
    return {"lr": 1e-3, "beta1": 0.9, "beta2": 0.999, "eps": 1e-8, "weight_decay": 0.01, "seed": 1234}


def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape):
        return torch.randn(*shape, generator=g, device="cuda")

    if c["op"] == "adamw":
        sizes = _sizes(c)
        first, total = [], 0                              # every tensor starts at a multiple of 32 elements of flat storage
        for n in sizes:
            first.append(total)
            total += -(-n // 32) * 32
        st = {"case": c, "p": normal(total) * 0.05, "g": (normal(total) * 1e-3).to(TYPES[c["grad"]]),
              "step": torch.tensor([99, 0], dtype=torch.int64, device="cuda")}
        if c["bits"] == 32:
            st["m"], st["v"] = normal(total) * 1e-3, normal(total).square() * 1e-6
        else:
            st["m"] = (normal(total) * 50).clamp(-250, 250).to(torch.float8_e4m3fn)
            st["v"] = (normal(total).abs() * 50 + 0.01).clamp(0, 250).to(torch.float8_e4m3fn)
            for name in ("m_scale", "v_scale"):
                st[name] = torch.randint(110, 114, (total // 32,), generator=g, device="cuda", dtype=torch.uint8).view(torch.float8_e8m0fnu)
        if c["copy"]:
            st["copy"] = torch.zeros(total, dtype=TYPES[c["copy"]], device="cuda")
        for f, n in zip(first, sizes):                    # what pads a tensor holds zeros
            for name in ("p", "g", "m", "v"):
                st[name][f + n:f + -(-n // 32) * 32] = 0
        if own:
            # the table that a program keeps beside its tensors
            import paper_2408_06995_b200 as fpq

            def parts(name, unit=1):
                return [st[name][f // unit:f // unit + -(-n // unit)] for f, n in zip(first, sizes)] if name in st else None

            st["table"] = fpq.fpq_adamw_table(parts("p"), parts("g"), parts("m"), parts("v"), parts("m_scale", 32), parts("v_scale", 32),
                                              parts("copy"))
        return st
    M, K, N, R, G, S, xt, wt = c["M"], c["K"], c["N"], c["R"], c["G"], c["S"], TYPES[c["x"]], TYPES[c["w"]]
    used = M - c["tail"]
    if S >= used:
        cuts = list(range(used)) + [used] * (S + 1 - used)
    else:
        cuts = torch.randperm(used - 1, generator=torch.Generator().manual_seed(seed))[:S - 1].add(1).sort().values.tolist()
        cuts = [0] + cuts + [used]
    ids = torch.randperm(max(G, S), generator=torch.Generator().manual_seed(seed + 1))[:S] % G
    if S > 3:
        ids[S // 2] = -1                                   # a request without an adapter
    x = normal(M, K)
    x[:, ::97] *= 4.0                                      # channels that stand out
    st = {"case": c, "a": ((torch.rand(G, R, K, generator=g, device="cuda") * 2 - 1) / math.sqrt(K)).to(wt), "b": (normal(G, N, R) * 0.02).to(wt),
          "scale": 2.0 ** torch.randint(-1, 2, (G,), generator=g, device="cuda").float(),
          "offsets": torch.tensor(cuts, dtype=torch.int32, device="cuda"), "ids": ids.to(torch.int32).cuda(), "x": x.to(xt)}
    if c["op"] == "forward":
        st["base"] = normal(M, N).to(xt) if c["base"] else None
        st["y"] = torch.zeros(M, N, dtype=xt, device="cuda")
        st["u"] = torch.zeros(M, R, device="cuda") if c["save"] else None
    else:
        st["dy"] = (normal(M, N) * 0.1).to(xt)
        st["u"] = normal(M, R)                             # what the forward pass kept
        st["base"] = (normal(M, K) * 0.1).to(xt) if c["base"] else None
        st["dx"] = torch.zeros(M, K, dtype=xt, device="cuda")
        st["da"], st["db"] = torch.empty(G, R, K, device="cuda"), torch.empty(G, N, R, device="cuda")
    return st


# ---- the plain forms ------------------------------------------------------------------------------------------------

def _rows(st, M, G):
    """For every row whether it is some request's, and [M][G] whether adapter g is its own."""
    rows = torch.arange(M, device="cuda", dtype=torch.int32)
    segment = torch.searchsorted(st["offsets"][1:], rows, right=True)
    inside = segment < st["ids"].numel()
    mine = st["ids"][segment.clamp(max=st["ids"].numel() - 1)]
    return inside, (torch.arange(G, device="cuda") == mine[:, None]) & inside[:, None]


def _forward(st):
    c = st["case"]
    M, K, N, R, G = c["M"], c["K"], c["N"], c["R"], c["G"]
    inside, mine = _rows(st, M, G)
    h = (st["x"].float() @ st["a"].float().reshape(G * R, K).T).reshape(M, G, R)
    h = torch.where(mine[:, :, None], h, 0.0)
    y = (h * st["scale"][:, None]).reshape(M, G * R) @ st["b"].float().permute(0, 2, 1).reshape(G * R, N)
    if c["base"]:
        y = y + st["base"].float()
    st["y"].copy_(torch.where(inside[:, None], y.to(st["y"].dtype), st["y"]))
    if not c["save"]:
        return {"y": st["y"]}
    st["u"].copy_(torch.where(inside[:, None], h.sum(1), st["u"]))
    return {"y": st["y"], "u": st["u"]}


def _backward(st):
    c = st["case"]
    M, K, N, R, G = c["M"], c["K"], c["N"], c["R"], c["G"]
    inside, mine = _rows(st, M, G)
    dy = st["dy"].float()
    du = (dy @ st["b"].float().permute(1, 0, 2).reshape(N, G * R)).reshape(M, G, R)
    du = torch.where(mine[:, :, None], du * st["scale"][:, None], 0.0).reshape(M, G * R)
    dx = du @ st["a"].float().reshape(G * R, K)
    if c["base"]:
        dx = dx + st["base"].float()
    st["dx"].copy_(torch.where(inside[:, None], dx.to(st["dx"].dtype), st["dx"]))
    st["da"].copy_((du.T @ st["x"].float()).reshape(G, R, K))
    u = torch.where(mine[:, :, None], st["u"][:, None, :] * st["scale"][:, None], 0.0).reshape(M, G * R)
    st["db"].copy_((dy.T @ u).reshape(N, G, R).permute(1, 0, 2))
    return {"dx": st["dx"], "da": st["da"], "db": st["db"]}


def _mix(z):
    z = (z * C1) & M32
    z = z ^ (z >> 15)
    z = (z * C2) & M32
    return z ^ (z >> 16)


def _decode(codes, scale):
    return codes.float().reshape(-1, 32) * scale.float()[:, None]


def _encode(value, bits16, least):
    """E4M3 codes of value [blocks][32] and the blocks' scale exponents: the scale brings the largest magnitude into [128, 256); the
    remainder below a code's step plus 16 random bits decides its rounding; nonzero values get the code `least` at least."""
    exponent = (value.abs().amax(1).view(torch.int32) >> 23) - 7
    exponent = exponent.clamp(min=1)
    q = value * ((254 - exponent) << 23).view(torch.float32)[:, None]
    a = q.abs()
    low = a < 2.0 ** -6
    word = torch.where(low, a + 2.0 ** -6, a).view(torch.int32)
    code = ((word + (bits16 << 4)) >> 20) - torch.where(low, 968, 960)
    code = torch.where(a > 0, code.clamp(min=least), code) | ((q.view(torch.int32) >> 24) & 128)
    return code.to(torch.uint8).reshape(-1), exponent.to(torch.uint8)


def _adamw(st):
    c = st["case"]
    o = _adamw_options(c)
    st["step"][0] += 1
    t = st["step"][0]
    bias1, bias2 = 1 - o["beta1"] ** t.double(), 1 - o["beta2"] ** t.double()
    g = st["g"].float()
    if c["bits"] == 32:
        m, v = st["m"], st["v"]
    else:
        m = _decode(st["m"], st["m_scale"])
        r = _decode(st["v"], st["v_scale"])
        v, g = r * r, g.reshape(-1, 32)
    m = m * o["beta1"] + g * (1 - o["beta1"])
    v = v * o["beta2"] + (g * g) * (1 - o["beta2"])
    r = torch.sqrt(v)
    update = m / (r * (1 / torch.sqrt(bias2)).float() + o["eps"]) * (o["lr"] / bias1).float()
    st["p"].mul_(1 - o["lr"] * o["weight_decay"]).sub_(update.reshape(-1))
    if c["copy"]:
        st["copy"].copy_(st["p"])
    if c["bits"] == 32:
        st["m"].copy_(m)
        st["v"].copy_(v)
    else:
        number = torch.arange(st["p"].numel(), device="cuda").reshape(-1, 32)
        z = _mix((number & M32) ^ _mix(((t & M32) * C1 + o["seed"] + 1 + (number >> 32) * C2) & M32)).to(torch.int64)
        for name, value, bits, least in (("m", m, z >> 16, 0), ("v", r, z & 0xFFFF, 1)):
            codes, exponent = _encode(value, bits.to(torch.int32), least)
            st[name].view(torch.uint8).copy_(codes)
            st[name + "_scale"].view(torch.uint8).copy_(exponent)
    return {k: st[k] for k in ("p", "m", "v", "m_scale", "v_scale", "copy", "step") if k in st}


def run(st):
    c = st["case"]
    if not own:
        return {"forward": _forward, "backward": _backward, "adamw": _adamw}[c["op"]](st)
    import paper_2408_06995_b200 as fpq
    if c["op"] == "forward":
        fpq.fpq_adapter_forward(st["x"], st["a"], st["b"], st["offsets"], st["ids"], st["scale"], st["base"], st["y"], st["u"])
        return {"y": st["y"], "u": st["u"]} if c["save"] else {"y": st["y"]}
    if c["op"] == "backward":
        fpq.fpq_adapter_backward(st["dy"], st["x"], st["u"], st["a"], st["b"], st["offsets"], st["ids"], st["scale"], st["base"], st["dx"],
                                 st["da"], st["db"])
        return {"dx": st["dx"], "da": st["da"], "db": st["db"]}
    fpq.fpq_adamw_step(st["table"], st["step"], **_adamw_options(c))
    return {k: st[k] for k in ("p", "m", "v", "m_scale", "v_scale", "copy", "step") if k in st}


# ---- from the definitions, in 64 bits ---------------------------------------------------------------------------------

def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "adamw":
        return _exact_adamw(c, s)
    cuts, ids, a, b = s["offsets"].tolist(), s["ids"].tolist(), s["a"].double(), s["b"].double()
    if c["op"] == "forward":
        y, u = s["y"].double(), torch.zeros(c["M"], c["R"], dtype=torch.float64, device="cuda")
        for lo, hi, i in zip(cuts, cuts[1:], ids):
            y[lo:hi] = s["base"][lo:hi].double() if c["base"] else 0.0
            if i >= 0:
                u[lo:hi] = torch.einsum("mk,rk->mr", s["x"][lo:hi].double(), a[i])
                y[lo:hi] += torch.einsum("mr,nr->mn", u[lo:hi], b[i]) * s["scale"][i].double()
        return {"y": y, "u": u} if c["save"] else {"y": y}
    dx, da, db = s["dx"].double(), torch.zeros_like(a), torch.zeros_like(b)
    for lo, hi, i in zip(cuts, cuts[1:], ids):
        dx[lo:hi] = s["base"][lo:hi].double() if c["base"] else 0.0
        if i >= 0:
            dy, f = s["dy"][lo:hi].double(), s["scale"][i].double()
            du = torch.einsum("mn,nr->mr", dy, b[i]) * f
            dx[lo:hi] += torch.einsum("mr,rk->mk", du, a[i])
            da[i] += torch.einsum("mr,mk->rk", du, s["x"][lo:hi].double())
            db[i] += torch.einsum("mn,mr->nr", dy, s["u"][lo:hi].double()) * f
    return {"dx": dx, "da": da, "db": db}


def _exact_codes(value, noise, least):
    """Values of the codes and of the scales, by the definition: the grid below and above, and how far the value lies between."""
    value = value.reshape(-1, 32)
    top = torch.frexp(value.abs().amax(1))[1] - 1                     # floor(log2)
    power = (top - 7).clamp(min=-126)
    q = torch.ldexp(value, -power[:, None])
    step = torch.ldexp(torch.ones_like(q), (torch.frexp(q.abs())[1] - 1).clamp(min=-6) - 3)
    code = torch.floor(q.abs() / step + noise.reshape(-1, 32) / 65536.0) * step
    code = torch.where((q != 0) & (code < least * 2.0 ** -9), torch.full_like(code, least * 2.0 ** -9), code)
    return (code * torch.sign(q)).reshape(-1), torch.ldexp(torch.ones_like(power, dtype=torch.float64), power)


def _exact_adamw(c, s):
    beta1, beta2, lr, eps, decay, seed = 0.9, 0.999, 1e-3, 1e-8, 0.01, 1234
    t = int(s["step"][0]) + 1
    g = s["g"].double()
    m, v = s["m"].double(), s["v"].double()
    if c["bits"] == 8:
        m = (m.reshape(-1, 32) * s["m_scale"].double()[:, None]).reshape(-1)
        v = (v.reshape(-1, 32) * s["v_scale"].double()[:, None]).reshape(-1).square()
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = s["p"].double() * (1 - lr * decay) - lr * (m / (1 - beta1 ** t)) / (torch.sqrt(v / (1 - beta2 ** t)) + eps)
    out = {"p": p, "m": m, "v": v}
    if c["bits"] == 8:
        def scramble(z):
            z = z * C1 % 2 ** 32
            z = z ^ z // 2 ** 15
            z = z * C2 % 2 ** 32
            return z ^ z // 2 ** 16

        z = scramble(torch.arange(p.numel(), device="cuda") ^ scramble((t * C1 + seed + 1) % 2 ** 32))
        out["m"], out["m_scale"] = _exact_codes(m, (z // 65536).double(), 0)
        out["v"], out["v_scale"] = _exact_codes(torch.sqrt(v), (z % 65536).double(), 1)
    if c["copy"]:
        out["copy"] = p
    out["step"] = torch.tensor([t, 0])
    return out
