"""Lanes of a wave that hand each other values through LDS: between the writes and the reads stands an order that the
compiler has to keep (a barrier of the wave or of the workgroup), on every way through the kernels that do so.  Read
from the compiler's own intermediate form of the sources; no GPU needed."""
import os
import re
import subprocess

import pytest

from paper_2407_09577_amd import build

BARRIER = re.compile(r"call void @llvm\.amdgcn\.(wave\.barrier|s\.barrier)\b")
READ = re.compile(r" = load [^,]*, ptr addrspace\(3\)")
WRITE = re.compile(r"^\s*store [^,]*, ptr addrspace\(3\)")


def kernels(source, tmp_path):
    """{mangled name: lines} of the device code of csrc/<source>, as optimised."""
    if not os.path.exists(build.HIPCC):
        pytest.skip("hipcc not installed")
    out = str(tmp_path / "device.ll")
    r = subprocess.run([build.HIPCC, *build.CFLAGS, "--offload-device-only", "-S", "-emit-llvm",
                        os.path.join(build.CSRC, source), "-o", out], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    found, name = {}, None
    for line in open(out):
        m = re.match(r"define .*amdgpu_kernel void @(\w+)\(", line)
        if m:
            name, found[m.group(1)] = m.group(1), []
        elif line.startswith("}"):
            name = None
        elif name:
            found[name].append(line)
    return found


def successors(lines):
    """The blocks of a function and, of each, its lines and those that may follow it."""
    blocks, at = {"entry": []}, "entry"
    for line in lines:
        m = re.match(r"([\w.]+):", line)
        if m:
            at = m.group(1)
            blocks[at] = []
        else:
            blocks[at].append(line)
    first = next(iter(lines), "")
    if re.match(r"([\w.]+):", first):
        blocks.pop("entry")
    return {b: (ls, re.findall(r"label %([\w.]+)", "".join(ls))) for b, ls in blocks.items()}


def unordered(lines):
    """Reads of LDS that some way reaches from a write with no barrier between."""
    blocks = successors(lines)
    entry = next(iter(blocks))
    bad, seen, todo = set(), set(), [(entry, False)]
    while todo:
        b, written = todo.pop()
        if (b, written) in seen:
            continue
        seen.add((b, written))
        for line in blocks[b][0]:
            if BARRIER.search(line):
                written = False
            elif WRITE.search(line):
                written = True
            elif READ.search(line) and written:
                bad.add(line.strip())
        todo += [(s, written) for s in blocks[b][1]]
    return bad


@pytest.mark.parametrize("source,exchanges", [("w4_few_row.hip", r"w4_few_kernel.*ELb1EEE"), ("w4_few_glu.hip", r"w4_few_kernel.*ELb1EEE"),
                                              ("w4_fold.hip", r"w4_fold_kernelI.*ELb1EEE")])
def test_writes_and_reads_of_a_wave_are_in_order(source, exchanges, tmp_path):
    found = kernels(source, tmp_path)
    through = [n for n in found if re.search(exchanges, n)]
    assert len(through) >= 6 and all(any(READ.search(x) for x in found[n]) for n in through)
    assert {n: bad for n, lines in found.items() if (bad := unordered(lines))} == {}


def test_the_check_sees_what_is_missing():
    """The check itself, on a loop that writes, reads and goes round."""
    write, read, wave = ("  store <4 x i32> %a, ptr addrspace(3) %p, align 16", "  %b = load <4 x i32>, ptr addrspace(3) %q, align 16",
                         "  call void @llvm.amdgcn.wave.barrier()")
    loop = lambda *body: ["  br label %1", "1:", *body, "  br i1 %c, label %1, label %2", "2:", "  ret void"]
    assert not unordered(loop(wave, write, wave, read))
    assert not unordered(loop(write, wave, read))
    assert len(unordered(loop(wave, write, read))) == 1
    assert len(unordered(loop(read, write))) == 1  # the next time round
