"""The counted waits of the tiled kernels for products with 4-bit weights, from the built library: in front of a step's barrier a wave leaves so many copies in flight; the
steps behind it must have issued as many, or some of the step's own would be among those left."""
import os
import re
import subprocess

import pytest

from paper_2006_11735_amd import binding, build

LLVM = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")
# (TN, TM, WN, WM, WK): stages by the size of a group
TILES = [(2, 2, 4, 2, 1), (2, 2, 2, 2, 2), (2, 1, 1, 2, 4), (1, 1, 1, 2, 4), (1, 1, 1, 1, 8)]


def sizes(tn, tm, wn, wm, wk, group):
    """(stages, copies of a wave: weights, rows), as S4Tile has them"""
    bn, bm, waves = 32 * tn * wn, 32 * tm * wm, wn * wm * wk
    stage, steps = bm * 128 * wk + bn * 64 * wk, (2 if group == 32 else 4) if wk == 1 else 1
    rest = 2 * (128 * wk * steps // group) * bn * 4 + bm * 4
    return (4 if 4 * stage + rest <= 163840 else 3), bn * 64 * wk // 1024 // waves, bm * 128 * wk // 1024 // waves


@pytest.fixture(scope="module")
def code(tmp_path_factory):
    path = tmp_path_factory.mktemp("s4")
    assert binding.icnn_version() >= 100               # (there is a library)
    os.symlink(build.LIB, path / "lib.so")
    run = lambda *a: subprocess.run([os.path.join(LLVM, a[0]), *a[1:]], check=True, capture_output=True, text=True, cwd=path).stdout  # noqa: E731
    run("llvm-objdump", "--offloading", "lib.so")
    out, name = {}, None
    for f in sorted(os.listdir(path)):
        if not f.endswith("gfx950") or "s4_tiled_kernel" not in run("llvm-readelf", "--symbols", "--wide", f):
            continue
        for line in run("llvm-objdump", "-d", "--no-show-raw-insn", "--symbolize-operands", f).splitlines():
            m = re.match(r"(?:[0-9a-f]+ )?<(_Z\w+)>:", line)
            if m:
                name = m[1]
                out[name] = []
            elif name:
                s = re.sub(r"\s*//.*", "", line).strip()
                out[name].append(s if not s.startswith("<") else "label:" + s)
    return out


@pytest.mark.parametrize("group", [32, 64, 128, 256])
@pytest.mark.parametrize("tile", TILES)
@pytest.mark.parametrize("direct", [0, 1])
def test_what_a_step_s_wait_leaves_in_flight(code, group, tile, direct):
    stages, of_weights, of_rows = sizes(*tile, group)
    copies = of_weights + (of_rows if direct else 0)
    left = (stages - 3 if stages == 4 else stages - 2) * copies
    names = [n for n in code if re.search("s4_tiled_kernelI%sLi%dELb[01]ELb%dELb[01]E" % ("".join("Li%dE" % t for t in tile), group, direct), n)]
    assert len(names) == (4 if tile[:2] == (2, 2) else 2)          # gated and not, scales of two bytes and four
    for n in names:
        lines = code[n]
        steps = 0
        for at, s in enumerate(lines):
            if s != "s_barrier" or not any(re.match(r"s_waitcnt vmcnt\(%d\)" % left, q) for q in lines[at - 6:at]):
                continue
            # from this barrier on, up to the loop's end: the next wait for copies' barrier, or the epilogue's
            body = lines[at + 1:next(i for i in range(at + 1, len(lines)) if lines[i] == "s_barrier")]
            issued = sum(q.startswith("buffer_load_dwordx4") and q.endswith("lds") for q in body)
            if not any("mfma" in q for q in body):
                continue                               # (the prologue's)
            assert issued == copies, (n, issued, copies)
            steps += 1
        assert steps == 1, n
