"""The instructions of the built library's kernels, for tests that count waits."""
import os
import re
import subprocess

from paper_2006_11735_amd import binding, build

LLVM = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin")


def kernels(path, wanted):
    """{kernel: its instructions, labels as lines 'label:L<number>'} of the code objects that hold one whose name has `wanted` in it"""
    assert binding.icnn_version() >= 100               # (there is a library)
    os.symlink(build.LIB, path / "lib.so")
    run = lambda *a: subprocess.run([os.path.join(LLVM, a[0]), *a[1:]], check=True, capture_output=True, text=True, cwd=path).stdout  # noqa: E731
    run("llvm-objdump", "--offloading", "lib.so")
    out, name = {}, None
    for f in sorted(os.listdir(path)):
        if not f.endswith("gfx950") or wanted not in run("llvm-readelf", "--symbols", "--wide", f):
            continue
        for line in run("llvm-objdump", "-d", "--no-show-raw-insn", "--symbolize-operands", f).splitlines():
            m = re.match(r"(?:[0-9a-f]+ )?<(_Z\w+)>:", line)
            if m:
                name = m[1] if wanted in m[1] else None
                if name:
                    out[name] = []
            elif name:
                s = re.sub(r"\s*//.*", "", line).strip()
                label = re.match(r"(?:[0-9a-f]+ )?<(L\d+)>:", s)
                out[name].append("label:" + label[1] if label else s)
    return out


def loops(lines):
    """Bodies of the loops that hold no other loop"""
    at = {s[6:]: i for i, s in enumerate(lines) if s.startswith("label:")}
    ends = [(at[m[1]], i) for i, s in enumerate(lines) for m in [re.match(r"s_c?branch\w* (L\d+)$", s)] if m and at.get(m[1], i) < i]
    return [lines[a:b + 1] for a, b in ends if not any(a <= c and d <= b and (a, b) != (c, d) for c, d in ends)]
