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
