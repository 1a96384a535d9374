"""Records of the gate, the experts and the adapters as the binding and the C compiler lay them out, and the registers of their kernels.
No GPU needed."""
import ctypes as C
import os
import subprocess

import pytest

from paper_2605_22428_amd import binding as B
from test_kernel_resources import _device_elf, _kernels
from paper_2605_22428_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_records_match_the_header(tmp_path):
    recs = [("mw_gate", B.MwGate), ("mw_experts", B.MwExperts), ("mw_adapters", B.MwAdapters)]
    lines = []
    for name, cls in recs:
        lines.append('printf("%%zu", sizeof(%s));' % name)
        lines += ['printf(" %%zu", offsetof(%s, %s));' % (name, f) for f, _ in cls._fields_]
        lines.append('printf("\\n");')
    (tmp_path / "t.c").write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"mw.h\"\nint main(void) {\n%s\nreturn 0; }\n" % "\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(tmp_path / "t.c"), "-o", str(tmp_path / "t")], check=True)
    out = subprocess.run([str(tmp_path / "t")], check=True, capture_output=True, text=True).stdout.splitlines()
    for line, (name, cls) in zip(out, recs):
        assert [int(v) for v in line.split()] == [C.sizeof(cls)] + [getattr(cls, f).offset for f, _ in cls._fields_], name
    assert [C.sizeof(cls) for _, cls in recs] == [16, 40, 40]


def test_constants_match_the_header():
    text = open(os.path.join(ROOT, "include", "mw.h")).read()
    for name in ("MW_GATE_SOFTMAX", "MW_GATE_SOFTMAX_TOPK", "MW_GATE_SIGMOID_TOPK", "MW_LOGITS_F32", "MW_LOGITS_BF16", "MW_GATE_MAX_EXPERTS", "MW_GATE_MAX_GROUPS",
                 "MW_LAYER_MAX_TOKENS", "MW_ADAPT_MAX_ADAPTERS", "MW_ADAPT_MAX_RANK", "MW_ADAPT_MAX_ROWS", "MW_FLAG_BAD_ADAPTER"):
        line = [l.split() for l in text.splitlines() if l.startswith("#define " + name + " ")]
        assert len(line) == 1 and int(line[0][2].rstrip("u"), 0) == getattr(B, name), name


def test_workspaces_grow_with_the_batch_and_hold_the_limits():
    a = B.MwAdapters(16, 16, 0, 8, 32, 4096, 4096)
    need, sizes = C.c_int64(0), []
    for rows in (0, 1, 255, 256, 257, 4096, 65536):
        for backward in (0, 1):
            assert B.load().mw_adapt_workspace_bytes(C.byref(a), C.c_int32(rows), C.c_int32(backward), C.byref(need)) == B.MW_OK
            sizes.append(need.value)
    assert sizes[::2] == sorted(sizes[::2]) and sizes[1::2] == sorted(sizes[1::2]) and all(f <= b for f, b in zip(sizes[::2], sizes[1::2]))
    assert B.load().mw_adapt_workspace_bytes(C.byref(a), C.c_int32(65537), C.c_int32(0), C.byref(need)) == B.MW_ERR_CAPACITY
    assert B.load().mw_adapt_workspace_bytes(None, C.c_int32(1), C.c_int32(0), C.byref(need)) == B.MW_ERR_INVALID_ARG


@pytest.mark.parametrize("kernel", ["k_route", "k_layer_up", "k_layer_down", "k_layer_sum", "k_adapt_order", "k_adapt_prepare", "k_adapt_down", "k_adapt_up",
                                    "k_adapt_grads"])
def test_nothing_is_spilled(kernel):
    """A stream whose registers go through memory waits for its own spills."""
    path = build.LIB if os.path.exists(build.LIB) else build.build()
    found = [k for elf in _device_elf(path) for k in _kernels(elf) if kernel in k[".name"]]
    assert found
    for k in found:
        assert k[".private_segment_fixed_size"] == 0, (k[".name"], k[".private_segment_fixed_size"])
