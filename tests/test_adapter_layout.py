"""Shared memory of the adapters' tile kernel, without a GPU: no two things lie in one place, in any form of the kernel."""
import os
import subprocess

import pytest

from paper_2408_06995_b200 import build as fpq_build

# bytes of x and of the weights, BF16, padded rank, two blocks on an SM: what fpq_adapter_tile.cu builds
FORMS = [(4, wb, 0, rp, two) for wb in (4, 2) for rp in (32, 64) for two in (0, 1) if rp == 32 or not two]
FORMS += [(2, 2, bf, rp, two) for bf in (0, 1) for rp in (16, 32, 64) for two in (0, 1) if rp <= 32 or bf or not two]
NAMES = ["FP32", "STAGES", "STAGE", "W2_SETS", "GROUPS", "WORK_WARPS", "SLOTS", "SLOT_BASE", "END", "SMEM", "W2_BASE", "W2_SET", "KEPT_BASE", "T_KEPT",
         "T_BYTES", "FULL", "EMPTY", "READY", "T_FULL", "T_FREE", "T_READY", "T_DONE", "W_FULL", "W_EMPTY", "W_READY", "Y_FULL", "SLOT_FULL", "TMEM_WORD",
         "BARRIERS"]


@pytest.fixture(scope="module")
def sizes(tmp_path_factory):
    """{form: {name: value}}, and where the barriers lie for each gap in front of the stages, as the kernel's header has them."""
    folder = tmp_path_factory.mktemp("layout")
    rows = "".join("    { using T = fpq::TileSizes<%d, %d, %s, %d, %s>;\n      %s\n      for (int gap = 0; gap < 1024; gap += 16) put(T::barriers_at(gap));\n"
                   "      std::puts(\"\"); }\n" % (x, w, "true" if b else "false", r, "true" if t else "false", " ".join(f"put(T::{n});" for n in NAMES))
                   for x, w, b, r, t in FORMS)
    source = folder / "sizes.cpp"
    source.write_text('#include <cstdio>\n#include "fpq_adapter_layout.h"\nstatic void put(long v) { std::printf("%ld ", v); }\n'
                      "int main()\n{\n" + rows + "}\n")
    subprocess.run(["g++", "-std=c++17", "-I", fpq_build.CSRC, str(source), "-o", str(folder / "sizes")], check=True)
    lines = subprocess.run([str(folder / "sizes")], check=True, capture_output=True, text=True).stdout.splitlines()
    out = {}
    for form, line in zip(FORMS, lines):
        v = [int(w) for w in line.split()]
        out[form] = dict(zip(NAMES, v)), v[len(NAMES):]
    assert len(out) == len(FORMS)
    return out


def apart(ranges):
    ranges = sorted(ranges)
    return all(end <= start for (_, end), (start, _) in zip(ranges, ranges[1:]))


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(map(str, f)))
def test_barriers_and_the_tensor_memory_word_lie_apart(sizes, form):
    t, places = sizes[form]
    counts = {"FULL": t["STAGES"], "EMPTY": t["STAGES"], "READY": t["STAGES"] if t["FP32"] else 0, "T_FULL": 2, "T_FREE": 2, "T_READY": 1, "T_DONE": 1,
              "W_FULL": t["W2_SETS"], "W_EMPTY": t["W2_SETS"], "W_READY": t["GROUPS"], "Y_FULL": t["GROUPS"],
              "SLOT_FULL": t["WORK_WARPS"] * t["SLOTS"]}
    barriers = [(t[n] + 8 * i, t[n] + 8 * i + 8) for n, k in counts.items() for i in range(k)]
    assert all(b % 8 == 0 for b, _ in barriers) and t["TMEM_WORD"] % 4 == 0
    inside = barriers + [(t["TMEM_WORD"], t["TMEM_WORD"] + 4)]
    assert apart(inside) and min(inside)[0] >= 0 and max(e for _, e in inside) <= t["BARRIERS"]
    for i, at in enumerate(places):                        # the gap in front of the stages is 16 i bytes of SMEM in all
        gap = 16 * i
        assert at % 16 == 0 and at >= -gap and gap + at + t["BARRIERS"] <= t["SMEM"]
        assert apart([(at, at + t["BARRIERS"]), (0, t["END"])]) and gap + t["END"] <= t["SMEM"]


@pytest.mark.parametrize("form", FORMS, ids=lambda f: "-".join(map(str, f)))
def test_stages_operands_and_slots_lie_apart(sizes, form):
    t, _ = sizes[form]
    slots = (t["SLOT_BASE"], t["SLOT_BASE"] + t["WORK_WARPS"] * t["SLOTS"] * 32 * 128)
    assert apart([(0, t["STAGES"] * t["STAGE"]), slots]) and slots[1] <= t["END"]
    assert apart([(0, 2 * t["T_BYTES"]), (t["W2_BASE"], t["W2_BASE"] + t["W2_SETS"] * t["W2_SET"]), (t["KEPT_BASE"], t["KEPT_BASE"] + t["T_KEPT"]), slots])
    assert t["SMEM"] <= 227 * 1024 and (not form[4] or 2 * (t["SMEM"] + 1024) <= 228 * 1024)
