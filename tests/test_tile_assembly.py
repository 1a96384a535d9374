"""The compiled kernels of the tiles, by their own assembly: the register that holds a load's place in LDS is written for those loads and used by nothing else (the
compiler does not know that they write it), nothing goes through scratch memory, and no wait for all loads stands inside the loops but those that are written there.
No GPU needed."""
import os
import re
import subprocess

import pytest

from paper_2605_22428_amd import build
from test_kernel_resources import _device_elf, _kernels

OBJDUMP = "/opt/rocm/llvm/bin/llvm-objdump"
KERNELS = ("k_tilesINS_5up_op", "k_tilesINS_7rows_op", "k_tilesINS_6act_op", "k_ffn_grads", "k_tilesINS_7int8_op")


@pytest.fixture(scope="module")
def listings(tmp_path_factory):
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    path = build.LIB if os.path.exists(build.LIB) else build.build()
    found = {}
    for i, elf in enumerate(_device_elf(path)):
        names = [k[".name"] for k in _kernels(elf) if any(n in k[".name"] for n in KERNELS)]
        if names:
            at = tmp_path_factory.mktemp("elf") / ("%d.elf" % i)
            at.write_bytes(elf)
            text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--disassemble-symbols=" + ",".join(names), str(at)], check=True, capture_output=True, text=True).stdout
            for part in re.split(r"\n(?=[0-9a-f]+ <)", text):
                m = re.match(r"[0-9a-f]+ <([^>]+)>:\n(.*)", part, re.S)
                if m and m.group(1) in names:
                    found[m.group(1)] = [line.split("//")[0].strip() for line in m.group(2).splitlines() if line.strip()]
    return found


def test_the_place_register_is_written_for_loads_alone(listings):
    assert all(any(k in name for name in listings) for k in KERNELS)
    for name, lines in listings.items():
        loads = [i for i, l in enumerate(lines) if re.match(r"buffer_load_dwordx4 .* lds$", l)]
        assert loads, name
        uses = [i for i, l in enumerate(lines) if re.search(r"\bm0\b", l)]
        assert uses == [i - 2 for i in loads], name
        for i in uses:
            assert re.match(r"s_mov_b32 m0, s\d+$", lines[i]) and lines[i + 1] == "s_nop 0", (name, lines[i:i + 3])


def test_no_scratch(listings):
    for name, lines in listings.items():
        assert not [l for l in lines if l.startswith("scratch_")], name


@pytest.fixture(scope="module")
def loops(tmp_path_factory):
    """Every kernel's loop over the steps: the shortest piece of code that a branch goes back over and that loads into LDS."""
    if not os.path.exists(OBJDUMP):
        pytest.skip("no llvm-objdump")
    path = build.LIB if os.path.exists(build.LIB) else build.build()
    found = {}
    for i, elf in enumerate(_device_elf(path)):
        names = [k[".name"] for k in _kernels(elf) if any(n in k[".name"] for n in KERNELS)]
        if not names:
            continue
        at = tmp_path_factory.mktemp("elf") / ("%d.elf" % i)
        at.write_bytes(elf)
        text = subprocess.run([OBJDUMP, "-d", "--no-show-raw-insn", "--disassemble-symbols=" + ",".join(names), str(at)], check=True, capture_output=True, text=True).stdout
        for part in re.split(r"\n(?=[0-9a-f]+ <)", text):
            m = re.match(r"([0-9a-f]+) <([^>]+)>:\n(.*)", part, re.S)
            if not m or m.group(2) not in names:
                continue
            lines = [(int(a, 16), what.strip(), after) for what, a, after in re.findall(r"^(.*?)// ([0-9A-F]+):(.*)$", m.group(3), re.M)]
            places = {a: n for n, (a, _, _) in enumerate(lines)}
            bodies = []
            for n, (a, what, after) in enumerate(lines):
                target = re.search(r"\+0x([0-9a-f]+)>", after) if re.match(r"s_c?branch", what) else None
                back = places[int(m.group(1), 16) + int(target.group(1), 16)] if target else n + 1
                body = [l for _, l, _ in lines[back:n + 1]]
                if any(re.match(r"buffer_load_dwordx4 .* lds$", l) for l in body):
                    bodies.append(body)
            found[m.group(2)] = min(bodies, key=len)
    return found


def test_loops_wait_for_the_loads_that_they_need_and_no_others(loops):
    """One wait for loads in a step: until those of the steps ahead alone are on the way (a step's loads for each stage but one), for none where there is room for one step.  No spilled
    register, scalar load or load of another kind stands among them, whose waits would count the loads into LDS too."""
    assert all(any(k in name for name in loops) for k in KERNELS)
    for name, body in loops.items():
        loads = sum(bool(re.match(r"buffer_load_dwordx4 .* lds$", l)) for l in body)
        columns, rows = (int(v) for v in re.search(r"ILi(\d+)ELi(\d+)E", name).groups())
        assert loads == (columns + rows) // 32, name
        stages = 1 if (columns, rows) == (128, 128) else 3 if (columns, rows) == (128, 64) else 2
        waits = [l for l in body if "vmcnt" in l]
        assert len(waits) == 1 and re.match(r"s_waitcnt vmcnt\(%d\)" % ((stages - 1) * loads), waits[0]), (name, waits)
        assert sum("mfma" in l for l in body) == columns * rows // 1024, name
        assert not [l for l in body if re.match(r"(buffer|global|flat|scratch|s)_(load|store)", l) and not l.endswith("lds")], name
