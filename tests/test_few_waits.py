"""The counted waits of the kernel for products on few rows, from the built library: a wave that waits for its turn's weights and rows leaves the next turn's in flight, so
many copies and so many loads.  Both must be there, in the block of instructions in front of the wait: with fewer, some of the turn's own would be among those left."""
import os
import re
import subprocess

import pytest

from paper_2006_11735_amd import binding, build

LLVM = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")


def kernels(tmp_path):
    """{kernel: its instructions, labels as lines that end in ':'}, of the code object that holds them"""
    assert binding.icnn_version() >= 100               # (there is a library)
    os.symlink(build.LIB, tmp_path / "lib.so")
    run = lambda *a: subprocess.run([os.path.join(LLVM, a[0]), *a[1:]], check=True, capture_output=True, text=True, cwd=tmp_path).stdout  # noqa: E731
    run("llvm-objdump", "--offloading", "lib.so")
    out, name = {}, None
    for f in sorted(os.listdir(tmp_path)):
        if not f.endswith("gfx950") or "linear_few_kernel" not in run("llvm-readelf", "--symbols", "--wide", f):
            continue
        text = run("llvm-objdump", "-d", "--no-show-raw-insn", "--symbolize-operands", f)
        for line in text.splitlines():
            m = re.match(r"(?:[0-9a-f]+ )?<(_Z\w+)>:", line)
            if m:
                name = m[1]
                out[name] = []
            elif name:
                s = re.sub(r"\s*//.*", "", line).strip()
                out[name].append(s if not s.startswith("<") else "label:")
    return out


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    return kernels(tmp_path_factory.mktemp("few"))


@pytest.mark.parametrize("rows", [1, 2, 4])
@pytest.mark.parametrize("gated", [0, 1])
def test_what_a_turn_s_wait_leaves_in_flight(code, rows, gated):
    names = [n for n in code if re.search(r"linear_few_kernelILi%dELb%dELb1E" % (rows, gated), n)]
    assert len(names) == 1
    lines = code[names[0]]
    copies, loads = 4 * (1 + gated), 4 * rows
    found = 0
    for at, s in enumerate(lines):
        m = re.match(r"s_waitcnt vmcnt\((\d+)\)$", s)
        ahead = next((q for q in lines[at + 1:at + 12] if q.startswith(("ds_read", "buffer_", "global_", "s_waitcnt vmcnt"))), "")
        if not m or int(m[1]) != copies + loads or not ahead.startswith("ds_read"):
            continue
        seen = {"copies": 0, "loads": 0}
        for q in reversed(lines[:at]):
            if q.endswith(":") or q.startswith(("s_cbranch", "s_branch")):
                break
            seen["copies"] += q.startswith("buffer_load_dwordx4") and q.endswith("lds")
            seen["loads"] += q.startswith("global_load_dwordx4")
        assert seen == {"copies": copies, "loads": loads}, (names[0], at, seen)
        found += 1
    assert found == 2                                  # a pair of turns is the loop's body
