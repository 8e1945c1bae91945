"""Build-time guard for matrix instructions written as assembly: the compiler does not know how long their results take, so nothing may read or
move them before that, on any path through a kernel.  The listings are made by cross-compiling the sources (no GPU needed)."""
import os
import re
import subprocess
import tempfile
from concurrent.futures import ThreadPoolExecutor

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2101_05615_amd", "csrc")

MATRIX = re.compile(r"v_mfma_\S*?_(\d+x\d+x\d+)\S*\s+([av])\[(\d+):(\d+)\]")
REGISTERS = re.compile(r"\b([av])(?:\[(\d+):(\d+)\]|(\d+)\b)")
# wait states until another instruction may read the result: of 4, 8 and 16 passes
STATES = {"16x16x32": 7, "16x16x128": 11, "32x32x16": 11, "32x32x64": 19}
PASSES = {"16x16x32": 4, "16x16x128": 8, "32x32x16": 8, "32x32x64": 16}


def kernels(text):
    for m in re.finditer(r"^(_Z\S+):\s*; @", text, re.M):
        yield m.group(1), text[m.end():text.index(".Lfunc_end", m.end())]


def registers(operands):
    found = set()
    for kind, first, last, one in REGISTERS.findall(operands):
        found |= {(kind, i) for i in (range(int(first), int(last) + 1) if first else (int(one),))}
    return found


def too_early(body):
    """Instructions that may read a result before it is there.  Forward over the blocks: register -> wait states that are left, at most."""
    blocks, index = [[]], {}
    for line in body.split("\n"):
        line = line.split(";")[0].strip()
        label = re.match(r"(\.LBB\S+):", line)
        if label:
            index[label.group(1)] = len(blocks)
            blocks.append([])
        elif line and not line.startswith("."):
            blocks[-1].append(line)
    at_start, work, found = [None] * len(blocks), [0], set()
    at_start[0] = {}

    def reaches(block, left):
        known = at_start[block]
        if known is None:
            at_start[block] = dict(left)
        else:
            later = {r: n for r, n in left.items() if known.get(r, 0) < n}
            if not later:
                return
            known.update(later)
        work.append(block)

    while work:
        block = work.pop()
        left, through = dict(at_start[block]), True
        for line in blocks[block]:
            name = line.split()[0]
            matrix = MATRIX.match(line)
            if matrix:                          # (it goes out when the ones before it have left the matrix unit)
                step = PASSES[matrix.group(1)]
                left = {r: n - step for r, n in left.items() if n > step}
                left.update({(matrix.group(2), i): STATES[matrix.group(1)] for i in range(int(matrix.group(3)), int(matrix.group(4)) + 1)})
                continue
            if not name.startswith("s_"):
                found |= {line for r in registers(line[len(name):]) if r in left}
            branch = re.match(r"s_c?branch\S*\s+(\.LBB\S+)", line)
            if branch:
                reaches(index[branch.group(1)], left)
            if name in ("s_branch", "s_endpgm"):
                through = False
                break
            step = int(line.split()[1]) + 1 if name == "s_nop" else 1
            left = {r: n - step for r, n in left.items() if n > step}
        if through and block + 1 < len(blocks):
            reaches(block + 1, left)
    return found


def listing(source):
    from paper_2101_05615_amd import build
    with tempfile.TemporaryDirectory() as folder:
        out = os.path.join(folder, "out.s")
        subprocess.run(["hipcc"] + [f for f in build.FLAGS if f != "-shared"] + ["--cuda-device-only", "-S", os.path.join(CSRC, source), "-o", out],
                       check=True, stderr=subprocess.DEVNULL)
        with open(out) as f:
            return f.read()


def test_the_reader_finds_a_move():
    """On listings written here: a move right behind the product, on one path only; the same with a wait; another register."""
    loop = "\n.LBB0_1:\n v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]\n s_cbranch_scc1 .LBB0_1\n%s v_accvgpr_mov_b32 a9, a%d\n s_endpgm\n"
    assert too_early(loop % ("", 3)) and not too_early(loop % (" s_nop 7\n", 3)) and not too_early(loop % ("", 4))


@pytest.mark.timeout(600)
def test_results_are_waited_for():
    with ThreadPoolExecutor(3) as pool:
        texts = list(pool.map(listing, ["fp8_tile.hip", "fp8_stream.hip", "fp8_gradient.hip"]))
    seen = 0
    for text in texts:
        for name, body in kernels(text):
            if "v_mfma" in body:
                seen += 1
                assert not too_early(body), f"{name}: {sorted(too_early(body))[:5]}"
    assert seen >= 40, seen
