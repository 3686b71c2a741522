"""The product kernels' matrix instructions and direct copies are written as inline assembly, around
which the compiler adds no wait states.  What they need of the instructions beside them is read
off the built library:

 - a vector instruction writes no operand of a matrix instruction in the two states before it;
 - a matrix instruction's sums are not touched in the next 18 states (the longest wait of a 16 x 16
   one is 11), but by matrix instructions, and by those not in the next eight;
 - a copy to LDS finds m0 as its own s_mov_b32 left it, one state or more before, in a straight line.
"""

import glob
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2601_17654_amd", "libkareus_mi355x.so")
OBJDUMP = os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "llvm", "bin", "llvm-objdump")
RANGE = re.compile(r"\b([va])(?:(\d+)\b|\[(\d+):(\d+)\])")


def registers(text):
    got = set()
    for kind, one, lo, hi in RANGE.findall(text):
        got.update((kind, r) for r in range(int(one or lo), int(one or hi) + 1))
    return got


class Instruction:
    def __init__(self, text, labels):
        self.text, self.labels = text, labels
        self.op, _, rest = text.partition(" ")
        parts = rest.split(",")
        self.mfma = self.op.startswith("v_mfma")
        self.first, self.rest = registers(parts[0]), registers(",".join(parts[1:]))
        self.touched = self.first | self.rest
        vector = self.op.startswith("v_") and not self.mfma
        self.written = self.first if vector else set()
        self.states = 1 + (int(rest) if self.op == "s_nop" else 0)
        self.target = rest.strip() if self.op.startswith(("s_branch", "s_cbranch")) else None


def functions(listing):
    """{name: instructions} of a disassembly with symbolic branch targets."""
    got, name, labels = {}, None, []
    for line in listing.splitlines():
        head = re.match(r"^[0-9a-f]+ <(_Z\S+)>:", line)
        label = re.match(r"^<(L\d+)>:|^[0-9a-f]+ <(L\d+)>:", line)
        if head:
            name, labels = head.group(1), []
            got[name] = []
        elif label:
            labels.append(label.group(1) or label.group(2))
        elif name and line.startswith("\t"):
            got[name].append(Instruction(line.split("//")[0].strip(), labels))
            labels = []
    return got


def before(code, sources, at, states):
    """Instructions with fewer than `states` states between them and instruction `at`, on any way."""
    seen, todo = {}, [(at, 0)]
    while todo:
        i, gone = todo.pop()
        ways = [b for label in code[i].labels for b in sources.get(label, ())]
        if i > 0 and not code[i - 1].op.startswith(("s_branch", "s_endpgm", "s_setpc")):
            ways.append(i - 1)
        for j in ways:
            if gone < states and seen.get(j, states) > gone:
                seen[j] = gone
                yield code[j]
                todo.append((j, gone + code[j].states))


def faults(code):
    sources = {}
    for i, x in enumerate(code):
        if x.target:
            sources.setdefault(x.target, []).append(i)
    sums = set().union(*(x.first for x in code if x.mfma))
    for i, x in enumerate(code):
        if x.mfma:
            for y in before(code, sources, i, 2):
                if y.written & x.touched:
                    yield "%s: operand written by %s" % (x.text, y.text)
            for y in before(code, sources, i, 8):
                if y.mfma and y.first & x.touched:
                    yield "%s: too close to %s" % (x.text, y.text)
        elif x.touched & sums:
            for y in before(code, sources, i, 18):
                if y.mfma and y.first & x.touched:
                    yield "%s: sums of %s" % (x.text, y.text)
        if x.op.startswith("buffer_load") and x.text.endswith(" lds"):
            j, between = i - 1, 0
            while j > 0 and "m0" not in code[j].text and not code[j + 1].labels:
                if code[j].text.endswith(" lds"):
                    break
                between += code[j].states
                j -= 1
            if not code[j].text.startswith("s_mov_b32 m0,") or between < 1:
                yield "%s: m0 from %s" % (x.text, code[j].text)
        elif "m0" in x.text and not x.text.startswith("s_mov_b32 m0,"):
            yield "%s: a use of m0" % x.text


@pytest.fixture(scope="module")
def kernels(tmp_path_factory):
    assert os.path.exists(LIB), "the library is not built"
    at = str(tmp_path_factory.mktemp("code"))
    shutil.copy(LIB, os.path.join(at, "lib.so"))
    subprocess.check_call([OBJDUMP, "--offloading", "lib.so"], cwd=at, stdout=subprocess.DEVNULL)
    got = {}
    for path in glob.glob(os.path.join(at, "*gfx950")):
        with open(path, "rb") as f:
            if b"mma_kernel" not in f.read():
                continue
        got.update(functions(subprocess.check_output(
            [OBJDUMP, "-d", "--no-show-raw-insn", "--symbolize-operands", path], text=True)))
    return {k: v for k, v in got.items() if "10mma_kernel" in k}


def test_product_kernels(kernels):
    # 16-bit: forward, its gradients' three products, of two types; bytes of three; two tile sizes
    assert len(kernels) == 2 * (2 * 4 + 3)
    for name, code in kernels.items():
        assert sum(x.mfma for x in code) in (2 * 16, 2 * 64), name
        assert sum(x.text.endswith(" lds") for x in code) in (3 * 8, 3 * 16), name
        found = list(faults(code))
        assert not found, "%s: %s" % (name, found[:5])


GOOD = """0000 <_Zgood>:
	v_mov_b32_e32 v1, 0
	s_nop 1
	s_mov_b32 m0, s4
	v_mfma_f32_16x16x32_bf16 a[0:3], v[0:3], v[4:7], a[0:3]
	buffer_load_dwordx4 v9, s[4:7], 0 offen lds
	s_nop 15
	s_nop 15
	ds_write_b128 v8, a[0:3]
	s_endpgm
"""


@pytest.mark.parametrize("old,new", [
    ("\ts_nop 1\n", ""), ("v_mov_b32_e32 v1, 0", "v_mov_b32_e32 v3, 0\n\ts_cbranch_scc0 L1\n\ts_nop 0\n<L1>:"),
    ("\ts_nop 15\n\ts_nop 15\n", "\ts_nop 15\n"), ("ds_write_b128 v8, a[0:3]", "s_nop 0\n\ts_branch L0"),
    ("\tbuffer", "\ts_mov_b32 m0, s5\n\tbuffer"), ("\tbuffer", "<L7>:\n\tbuffer"),
    ("\tv_mfma", "\ts_add_i32 m0, m0, 4\n\tv_mfma")])
def test_faults_are_found(old, new):
    assert not list(faults(functions(GOOD)["_Zgood"]))
    bad = GOOD.replace(old, new)
    assert bad != GOOD
    if "L0" in new:  # a loop whose head is too close to its end
        bad = bad.replace("\ts_nop 15\n\ts_nop 15\n", "").replace("\tv_mov", "<L0>:\n\tv_mov", 1)
        bad = bad.replace("v_mov_b32_e32 v1, 0", "v_accvgpr_read_b32 v30, a1")
    elif "m0" not in new and "L7" not in new and "s_nop 15" not in old:
        bad = bad.replace("\ts_nop 1\n", "").replace("\ts_mov_b32 m0, s4\n", "", 1).replace(
            "\tbuffer_load_dwordx4 v9, s[4:7], 0 offen lds\n", "")
    assert list(faults(functions(bad)["_Zgood"]))
