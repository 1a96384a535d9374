"""What mw_quantize_rows and mw_matmul_int8 refuse, by status and before anything is launched, and the record of matrices.  No GPU needed."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2605_22428_amd import binding as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
I, CAP, UN = B.MW_ERR_INVALID_ARG, B.MW_ERR_CAPACITY, B.MW_ERR_UNSUPPORTED


@pytest.fixture
def memory():
    t = torch.zeros(4096 + 64, dtype=torch.uint8)
    return t[(-t.data_ptr()) % 64:]


def test_quantize(memory):
    call, good = B._native().mw_quantize_rows, [memory, 64, 0, 64, memory, 64, memory, 0]
    assert call(*good) == B.MW_OK                                    # (no rows: nothing to do)
    good[2] = 4
    for at, bad, status in ((0, None, I), (0, memory[8:], I), (1, 56, I), (1, 68, I), (1, (1 << 21) + 8, UN), (2, -1, I), (2, (1 << 24) + 1, CAP), (3, 0, I), (3, 24, I), (3, 65552, UN), (4, None, I),
                            (4, memory[8:], I), (5, 48, I), (5, 72, I), (5, 1 << 22, UN), (6, None, I), (6, memory[2:], I)):
        assert call(*(good[:at] + [bad] + good[at + 1:])) == status, (at, bad)


def test_matmul(memory):
    rec = B.MwMatricesInt8(memory.data_ptr(), memory.data_ptr(), 2, 64, 32, 0)
    call, good = B._native().mw_matmul_int8, [C.addressof(rec), memory, 64, memory, memory, 0, memory, B.MW_LOGITS_BF16, 32, 0]
    assert call(*good) == B.MW_OK
    good[5] = 4
    for at, bad, status in ((0, 0, I), (1, None, I), (1, memory[8:], I), (2, 48, I), (2, 72, I), (2, 1 << 22, UN), (3, None, I), (3, memory[2:], I), (4, None, I), (4, memory[4:], I), (5, -1, I),
                            (5, (1 << 24) + 1, CAP), (6, None, I), (6, memory[8:], I), (7, 2, I), (8, 24, I), (8, 36, I), (8, 1 << 22, UN)):
        assert call(*(good[:at] + [bad] + good[at + 1:])) == status, (at, bad)
    for change, status in ((dict(n_matrices=0), I), (dict(n_in=0), I), (dict(n_in=72), I), (dict(n_out=40), I), (dict(n_in=65552), UN), (dict(n_out=(1 << 20) + 16), UN), (dict(codes_dev=0), I), (dict(scale_dev=0), I),
                           (dict(codes_dev=memory.data_ptr() + 8), I), (dict(scale_dev=memory.data_ptr() + 2), I)):
        bad = B.MwMatricesInt8(*[change.get(f, getattr(rec, f)) for f, _ in B.MwMatricesInt8._fields_])
        assert call(*([C.addressof(bad)] + good[1:])) == status, change


class Calls:
    def __getattr__(self, name):
        def call(*args):
            raise AssertionError("%s was called" % name)
        return call


def test_tensors_of_another_kind_or_device(monkeypatch):
    monkeypatch.setattr(B, "_native", Calls)
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 0)
    w, scale = torch.zeros((2, 32, 64), dtype=torch.int8), torch.zeros((2, 32))
    codes, scales, out, offsets = torch.zeros((3, 64), dtype=torch.int8), torch.zeros(3), torch.zeros((3, 32)), torch.zeros(3, dtype=torch.int64)
    m = B.MatricesInt8(w, scale)
    for args in ((codes.float(), scales, offsets, out), (codes, scales[:2], offsets, out), (codes, scales, offsets.int(), out), (codes, scales, offsets[:2], out), (codes, scales, offsets, out.half()),
                 (codes, scales, offsets, out[:2]), (codes[:, :32], scales, offsets, out), (codes, scales, offsets, out[:, ::2])):
        with pytest.raises(ValueError):
            m.mw_matmul_int8(*args)
    x = torch.zeros((3, 64), dtype=torch.bfloat16)
    for args in ((x.float(), codes, scales), (x, codes[:, :32], scales), (x, codes.float(), scales), (x, codes, scales[:2])):
        with pytest.raises(ValueError):
            B.mw_quantize_rows(*args)
    for bad in (lambda: B.MatricesInt8(w.float(), scale), lambda: B.MatricesInt8(w, scale[:1]), lambda: B.Experts(torch.zeros((1, 2, 16, 32), dtype=torch.int8), torch.zeros((1, 32, 16), dtype=torch.int8)),
                lambda: B.Experts(torch.zeros((1, 2, 16, 32), dtype=torch.int8), torch.zeros((1, 32, 16), dtype=torch.int8), torch.zeros((1, 2, 1, 1)), torch.zeros((1, 32)))):
        with pytest.raises(ValueError):
            bad()
    for device in (torch.device("cpu"), torch.device("cuda", 1)):
        m.device = device
        with pytest.raises(B.MwError, match="arrays on"):
            m.mw_matmul_int8(codes, scales, offsets, out)


def test_experts_of_another_device(monkeypatch):
    monkeypatch.setattr(B, "_native", Calls)
    ctx = B.Context.__new__(B.Context)
    ctx._h, ctx.n_local, ctx.hidden = None, 1, 16
    ctx.workspace = torch.empty(0, device="meta")
    experts = B.Experts(torch.zeros((1, 2, 8, 16), dtype=torch.bfloat16), torch.zeros((1, 16, 8), dtype=torch.bfloat16))
    x, offsets, ws, kept = torch.zeros((3, 16), dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int64), torch.zeros(1024, dtype=torch.uint8), torch.zeros((3, 2, 8), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="weights on cpu"):
        ctx.mw_ffn(experts, x, offsets, torch.empty_like(x), ws)
    with pytest.raises(ValueError, match="weights on cpu"):
        ctx.mw_ffn_backward(experts, x, offsets, kept, x, None, None, None, ws)


class Elsewhere(torch.Tensor):
    """An array that says that it is on another device."""

    def get_device(self):
        return 1


def test_arrays_of_another_device(monkeypatch):
    """Each array of each call, alone on another device than the weights (or rows), is refused before anything is launched."""
    monkeypatch.setattr(B, "_native", Calls)
    monkeypatch.setattr(B, "_stream_on", lambda device, where: 0)
    monkeypatch.setattr(B, "_stream_handle", lambda: 0)
    ctx = B.Context.__new__(B.Context)
    ctx._h, ctx.n_local, ctx.hidden, ctx.workspace = None, 1, 16, torch.empty(0)
    bf, f = dict(dtype=torch.bfloat16), torch.zeros(3)
    experts = B.Experts(torch.zeros((1, 2, 8, 16), **bf), torch.zeros((1, 16, 8), **bf))
    m = B.MatricesInt8(torch.zeros((1, 32, 16), dtype=torch.int8), torch.zeros((1, 32)))
    x, codes, offsets, ws, kept = torch.zeros((3, 16), **bf), torch.zeros((3, 16), dtype=torch.int8), torch.zeros(2, dtype=torch.int64), torch.zeros(1024, dtype=torch.uint8), torch.zeros((3, 2, 8), **bf)
    calls = ((lambda *a: ctx.mw_ffn(experts, *a), (x, offsets, x.clone(), ws, f, kept)),
             (lambda *a: ctx.mw_ffn_backward(experts, *a), (x, offsets, kept, x.clone(), x.clone(), torch.zeros((1, 2, 8, 16), **bf), torch.zeros((1, 16, 8), **bf), ws, f, f.clone())),
             (m.mw_matmul_int8, (codes, f, offsets, torch.zeros((3, 32)))), (B.mw_quantize_rows, (x, codes, f)))
    for call, args in calls:
        for at, t in enumerate(args):
            with pytest.raises(ValueError, match="expected device"):
                call(*(args[:at] + (t.as_subclass(Elsewhere),) + args[at + 1:]))


def test_record_and_constants_match_the_header(tmp_path):
    lines = ['printf("%zu", sizeof(mw_matrices_int8));'] + ['printf(" %%zu", offsetof(mw_matrices_int8, %s));' % f for f, _ in B.MwMatricesInt8._fields_]
    lines += ['printf(" %%lld", (long long)%s);' % n for n in ("MW_WEIGHT_INT8_CHANNEL", "MW_FFN_MAX_ROWS", "MW_MAX_STRIDE", "MW_INT8_MAX_IN")]
    (tmp_path / "t.c").write_text("#include <stdio.h>\n#include <stddef.h>\n#include \"mw.h\"\nint main(void) {\n%s\nreturn 0; }\n" % "\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-I", os.path.join(ROOT, "include"), str(tmp_path / "t.c"), "-o", str(tmp_path / "t")], check=True)
    out = subprocess.run([str(tmp_path / "t")], check=True, capture_output=True, text=True).stdout
    assert [int(v) for v in out.split()] == ([C.sizeof(B.MwMatricesInt8)] + [getattr(B.MwMatricesInt8, f).offset for f, _ in B.MwMatricesInt8._fields_]
                                             + [B.MW_WEIGHT_INT8_CHANNEL, B.MW_FFN_MAX_ROWS, B.MW_MAX_STRIDE, B.MW_INT8_MAX_IN])
