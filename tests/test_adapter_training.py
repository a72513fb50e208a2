"""The quantized layer, its adapters and the AdamW step as a program runs them together: fine-tuning beside a W4A8 projection, and the
learned rounding with AdamW in the place of plain descent."""
import math

import pytest
import torch

import paper_2408_06995_b200 as fpq
from paper_2408_06995_b200 import build as fpq_build

fpq_build.build()
pytestmark = pytest.mark.gpu
LR, B1, B2, EPS, WD = 1e-2, 0.9, 0.99, 1e-8, 0.01


class Layer:
    """A quantized linear layer with adapters for two requests, 16-bit adapters copied from FP32 masters by the step."""

    def __init__(self, M=192, K=320, N=640, R=8, G=2, bits=32):
        g = torch.Generator(device="cuda").manual_seed(7)
        self.N = N
        self.x = torch.randn(M, K, generator=g, device="cuda")
        w = torch.randn(N, K, generator=g, device="cuda") * 0.02
        self.w_scale = (w.abs().amax(1) / fpq.fpq_format_max(fpq.E2M1)).contiguous()
        self.prepared = fpq.fpq_prepare_weight(fpq.fpq_quantize_weight(w, self.w_scale, fpq.E2M1), fpq.E2M1, fpq.LINEAR, N, K)
        self.x_scale = fpq.fpq_scale_from_max(float(self.x.abs().max()), fpq.E4M3)
        self.target = self.x @ w.T
        self.master = [torch.randn(G, R, K, generator=g, device="cuda") / math.sqrt(K), torch.randn(G, N, R, generator=g, device="cuda") * 0.01]
        self.copy = [p.bfloat16() for p in self.master]
        self.grad = [torch.empty_like(p) for p in self.master]
        codes, state = bits == 8, torch.uint8 if bits == 8 else torch.float32
        self.m, self.v = ([torch.zeros(p.shape, dtype=state, device="cuda") for p in self.master] for _ in range(2))
        self.m_scale, self.v_scale = ([torch.zeros(-(-p.numel() // 32), dtype=torch.uint8, device="cuda") for p in self.master] if codes else None
                                      for _ in range(2))
        self.table = fpq.fpq_adamw_table(self.master, self.grad, self.m, self.v, self.m_scale, self.v_scale, self.copy)
        self.step = torch.zeros(2, dtype=torch.int64, device="cuda")
        self.offsets = torch.tensor([0, 77, M], dtype=torch.int32, device="cuda")
        self.ids = torch.tensor([1, 0], dtype=torch.int32, device="cuda")
        self.scale = torch.tensor([2.0, 0.5], device="cuda")
        self.y, self.dy, self.u = torch.empty(M, N, device="cuda"), torch.empty(M, N, device="cuda"), torch.empty(M, R, device="cuda")
        self.work = torch.empty(fpq.fpq_linear_workspace_size(M, N, K, fpq.E4M3, fpq.E2M1), dtype=torch.uint8, device="cuda")
        self.work2 = torch.empty(fpq.fpq_adapter_backward_workspace_size(M, N, K, G, R, fpq.BF16), dtype=torch.uint8, device="cuda")

    def forward(self):
        fpq.fpq_linear(self.x, self.prepared, self.w_scale, self.x_scale, fpq.E4M3, fpq.E2M1, None, self.N, self.y, self.work)
        fpq.fpq_adapter_forward(self.x, *self.copy, self.offsets, self.ids, self.scale, self.y, self.y, self.u)

    def backward(self):
        torch.sub(self.y, self.target, out=self.dy)
        self.dy.mul_(2.0 / self.dy.numel())
        fpq.fpq_adapter_backward(self.dy, self.x, self.u, *self.copy, self.offsets, self.ids, self.scale, None, None, *self.grad, self.work2,
                                 need_dx=False)

    def train(self):
        self.forward()
        self.backward()
        fpq.fpq_adamw_step(self.table, self.step, LR, B1, B2, EPS, WD, seed=3)

    def state(self):
        return [self.y, self.u, *self.grad, *self.master, *self.copy, *self.m, *self.v, *(self.m_scale or []), *(self.v_scale or []), self.step]


def test_one_training_step_is_the_chain_rule_and_adamw():
    s = Layer()
    a, b = (p.double() for p in s.copy)
    masters = [p.double() for p in s.master]
    y0 = fpq.fpq_linear(s.x, s.prepared, s.w_scale, s.x_scale, fpq.E4M3, fpq.E2M1, None, s.N).double()
    s.train()
    assert fpq.fpq_read_status() == fpq.OK
    a.requires_grad_(), b.requires_grad_()
    rows = [(0, 77, 1), (77, 192, 0)]
    y = torch.cat([y0[lo:hi] + s.scale[i].double() * (s.x[lo:hi].double() @ a[i].T @ b[i].T) for lo, hi, i in rows])
    loss = (y - s.target.double()).square().mean()
    loss.backward()
    # FP32 sums of at most 640 terms (2^-17 of the sum of magnitudes and less); what cancels in them is bounded by the largest gradient
    assert float((s.y.double() - y).abs().max()) <= 2.0 ** -16 * float(y.abs().max())
    for got, want in zip(s.grad, (a.grad, b.grad)):
        assert float((got.double() - want).abs().max()) <= 2.0 ** -12 * float(want.abs().max())
    # the first step: the moments' bias cancels, the update is lr g / (|g| + eps)
    for p, c, before, g in zip(s.master, s.copy, masters, s.grad):
        want = before * (1 - LR * WD) - LR * g.double() / (g.double().abs() + EPS)
        assert float((p.double() - want).abs().max()) <= 2.0 ** -20
        assert torch.equal(c, p.bfloat16())
    assert s.step.tolist() == [1, 0]


@pytest.mark.parametrize("bits", [32, 8])
def test_captured_training_steps_equal_eager_ones(bits):
    eager, captured = Layer(bits=bits), Layer(bits=bits)
    for _ in range(4):
        eager.train()
    captured.forward()                                 # (the first layer call on a device is made outside a capture)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.train()
    for _ in range(4):
        graph.replay()
    torch.cuda.synchronize()
    assert fpq.fpq_read_status() == fpq.OK
    for got, want in zip(captured.state(), eager.state()):
        assert torch.equal(got, want)


def test_rounding_learned_with_adamw():
    """The gradient of fpq_round_learn_step, with lr = 0, for two layers, and one AdamW step over both alphas; the bits are alpha's signs."""
    g = torch.Generator(device="cuda").manual_seed(1)
    layers, table = [], [[], [], [], [], [], []]
    for N, K in ((96, 64), (40, 128)):
        w = torch.randn(N, K, generator=g, device="cuda") * 0.05
        scale = (w.abs().amax(1) / fpq.fpq_format_max(fpq.E2M1)).contiguous()
        alpha, a = torch.randn(N, K, generator=g, device="cuda"), torch.randn(256, K, generator=g, device="cuda")
        grad = torch.empty_like(w)
        layers.append((w, scale, alpha, a, grad))
        blocks = -(-w.numel() // 32)
        for t, v in zip(table, (alpha, grad, torch.zeros(N, K, dtype=torch.uint8, device="cuda"), torch.zeros(N, K, dtype=torch.uint8, device="cuda"),
                                torch.zeros(blocks, dtype=torch.uint8, device="cuda"), torch.zeros(blocks, dtype=torch.uint8, device="cuda"))):
            t.append(v)
    tab, step = fpq.fpq_adamw_table(*table), torch.zeros(2, dtype=torch.int64, device="cuda")
    before = [layer[2].double().clone() for layer in layers]
    for w, scale, alpha, a, grad in layers:
        fpq.fpq_round_learn_step(w, scale, fpq.E2M1, alpha, a, reg=1e-3, lr=0.0, grad=grad)
    fpq.fpq_adamw_step(tab, step, LR, eps=1e-8, seed=5)
    for (w, scale, alpha, a, grad), b in zip(layers, before):
        want = b - LR * grad.double() / (grad.double().abs() + 1e-8)
        assert float((alpha.double() - want).abs().max()) <= 2.0 ** -20      # |alpha| below 8: four roundings of 2^-22 and the update's
        bits = fpq.fpq_round_learn_harden(alpha)
        assert torch.equal((bits[:, 0] & 1).bool(), alpha[:, 0] >= 0)
    assert fpq.fpq_read_status() == fpq.OK
