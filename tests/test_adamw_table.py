"""The AdamW step's table and roots, apart from the step itself."""
import pytest
import torch

import paper_2408_06995_b200 as fpq

F32, BF = torch.float32, torch.bfloat16


class Memory:
    """Stands in for a tensor on the GPU: the table looks at a tensor's place and type alone."""
    is_cuda = True

    def __init__(self, at, n, dtype=F32):
        self.at, self.n, self.dtype = at, n, dtype

    def data_ptr(self):
        return self.at

    def numel(self):
        return self.n

    def get_device(self):
        return 0

    def is_contiguous(self):
        return True


def memory_table(codes=False, **changed):
    """Two tensors of 64 and 40 elements, every buffer directly behind another; {name: tensor 0's or 1's} are put elsewhere."""
    at, given = 1 << 20, {}
    state = torch.uint8 if codes else F32
    for name, dtype, unit in (("params", F32, 1), ("grads", BF, 1), ("m", state, 1), ("v", state, 1), ("m_scale", torch.uint8, 32), ("v_scale", torch.uint8, 32),
                              ("copies", BF, 1)):
        given[name] = []
        for n in (64, 40):
            given[name].append(Memory(at, -(-n // unit), dtype))
            at += given[name][-1].numel() * dtype.itemsize
    for name, (i, place) in changed.items():
        given[name][i] = Memory(place(given), given[name][i].n, given[name][i].dtype)
    if not codes:
        given["m_scale"] = given["v_scale"] = None
    return fpq.fpq_adamw_table(**given)


@pytest.mark.parametrize("codes", [False, True])
def test_the_table_takes_buffers_side_by_side(codes):
    memory_table(codes)
    memory_table(codes, grads=(1, lambda t: t["grads"][0].at))         # gradients are only read: two may be one
    memory_table(codes, grads=(1, lambda t: t["grads"][0].at + 2))


@pytest.mark.parametrize("codes,changed", [
    (False, {"grads": (0, lambda t: t["copies"][0].at)}), (False, {"grads": (1, lambda t: t["copies"][0].at + 100)}), (True, {"grads": (0, lambda t: t["copies"][1].at - 126)}),
    (False, {"grads": (0, lambda t: t["params"][0].at)}), (True, {"grads": (1, lambda t: t["params"][1].at + 158)}), (False, {"grads": (1, lambda t: t["v"][0].at + 16)}),
    (True, {"grads": (1, lambda t: t["v_scale"][0].at)}), (False, {"params": (1, lambda t: t["params"][0].at + 252)}), (False, {"m": (0, lambda t: t["m"][1].at - 252)}),
    (False, {"copies": (1, lambda t: t["params"][0].at + 4)}), (True, {"m": (0, lambda t: t["v"][0].at + 8)}), (True, {"m_scale": (0, lambda t: t["v_scale"][0].at + 1)}),
    (True, {"m_scale": (1, lambda t: t["m"][0].at + 63)}), (False, {"params": (1, lambda t: t["params"][0].at)})])
def test_the_table_refuses_memory_in_two_roles(codes, changed):
    with pytest.raises(AssertionError, match="overlap|twice"):
        memory_table(codes, **changed)
