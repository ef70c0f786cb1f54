"""CPU check of the compiled kernels: a matrix product's result is not touched before it is there.

The hardware does not hold back an instruction that reads a product's registers too early; the compiler has to put enough others, or s_nop, between them.  Where two paths meet before the first
read it has counted along the longer one only (a maximum then read sums without the last product's part), so every kernel's assembly is searched here for the shortest path from each product to the
first instruction that touches its result.  What is enough is what the compiler puts in straight code: 8 states behind a 16x16x32 product, 12 behind a 32x32x16 one (4 more than its passes).
"""
import heapq
import os
import re
import subprocess
from concurrent.futures import ThreadPoolExecutor

import pytest

from paper_2506_07900_amd import build

STATES = {"16x16x32": 8, "32x32x16": 12}


def registers(operand):
    """v3, -v3, |v3|, v[4:7], a[0:15] -> {("v", 3)}, .."""
    found = set()
    for kind, first, last, one in re.findall(r"(?<![\w.])([va])(?:\[(\d+):(\d+)\]|(\d+))(?!\w)", operand):
        found |= {(kind, i) for i in (range(int(first), int(last) + 1) if first else [int(one)])}
    return found


def operands(text):
    return [registers(x) for x in re.split(r",(?![^\[]*\])", text)]


def kernels(assembly):
    """name -> (instructions [(mnemonic, operands' text)], label -> index)"""
    found, code, labels = {}, None, None
    for line in assembly.splitlines():
        line = line.split(";")[0].strip()
        label = re.match(r"^([\w.$]+):", line)
        if label and not label[1].startswith("."):
            code, labels = [], {}
            found[label[1]] = (code, labels)
        elif code is None or not line:
            continue
        elif label:
            labels[label[1]] = len(code)
        elif line.startswith((".section", ".end_amdhsa_kernel")):
            code = None
        elif not line.startswith("."):
            code.append(tuple((line.split(None, 1) + [""])[:2]))
    return {name: x for name, x in found.items() if x[0]}


def following(code, labels, i):
    """[(next instruction, whether the branch says that no lane is active)]"""
    name, text = code[i]
    if name == "s_endpgm":
        return []
    if name == "s_branch":
        return [(labels[text], False)]
    if name.startswith("s_cbranch"):
        return [(i + 1, name == "s_cbranch_execnz"), (labels[text], name == "s_cbranch_execz")]
    return [(i + 1, False)] if i + 1 < len(code) else []


def early_reads(code, labels):
    """[(states, product, the instruction that touches its result)] of those that come too early"""
    touched = [operands(text) for _, text in code]
    early = []
    for i, (name, text) in enumerate(code):
        if not name.startswith("v_mfma"):
            continue
        need, result = STATES[re.search(r"\d+x\d+x\d+", name)[0]], touched[i][0]
        heap, seen = [(0, j, dead) for j, dead in following(code, labels, i)], set()
        while heap:
            states, j, dead = heapq.heappop(heap)
            if states >= need:
                break
            if (j, dead) in seen:
                continue
            seen.add((j, dead))
            other, rest = code[j]
            if other.startswith("v_mfma") and result & set().union(*touched[j]):
                if not result & (touched[j][1] | touched[j][2]):
                    continue                                     # adds to the result: the hardware waits, and what follows waits for that product
            if result & set().union(*touched[j]) and not (dead and not other.startswith(("v_readlane", "v_readfirstlane"))):
                early.append((states, text, "%s %s" % code[j]))
                break
            dead = dead and not re.match(r"exec\b", rest) and "saveexec" not in other
            cost = int(rest, 0) + 1 if other == "s_nop" else 1
            for k, none in following(code, labels, j):
                heapq.heappush(heap, (states + cost, k, dead or none))
    return early


DIAMOND = """
f:
  v_mfma_f32_32x32x16_bf16 v[0:15], v[16:19], v[20:23], v[0:15]
  s_cbranch_vccnz .LBB0_2
  s_nop %d
.LBB0_2:
  s_nop %d
  v_max_f32_e32 v30, v3, v30
  s_endpgm
"""


@pytest.mark.parametrize("long,after,states", [(15, 0, 2), (0, 9, 11), (0, 10, None), (15, 15, None)])
def test_the_search_takes_the_shortest_path(long, after, states):
    (code, labels), = kernels(DIAMOND % (long, after)).values()
    assert [x[0] for x in early_reads(code, labels)] == ([] if states is None else [states])


def test_the_search_knows_what_touches():
    assert registers("-|v3|") == {("v", 3)} and registers("a[2:3]") == {("a", 2), ("a", 3)} and registers("vcc") == set() and registers("v_x") == set()
    for middle, want in (("v_mfma_f32_32x32x16_bf16 v[0:15], v[16:19], v[20:23], v[0:15]\n s_nop 11", []),         # the second product's wait counts
                         ("v_mfma_f32_32x32x16_bf16 v[32:47], v[0:3], v[20:23], v[32:47]\n s_nop 15", [0]),
                         ("buffer_load_dwordx4 v[12:15], v40, s[0:3], 0 offen", [0]),
                         ("s_cbranch_execnz .LBB0_9\n v_mov_b32_e32 v50, v1\n.LBB0_9:\n s_nop 11", []),          # (no lane reads it)
                         ("s_cbranch_execnz .LBB0_9\n s_mov_b64 exec, s[0:1]\n v_mov_b32_e32 v50, v1\n.LBB0_9:\n s_nop 11", [2])):
        text = "f:\n v_mfma_f32_32x32x16_bf16 v[0:15], v[16:19], v[20:23], v[0:15]\n %s\n ds_write_b32 v40, v0\n s_endpgm" % middle
        (code, labels), = kernels(text).values()
        assert [x[0] for x in early_reads(code, labels)] == want, middle


@pytest.fixture(scope="module")
def assembly(tmp_path_factory):
    """source -> assembly, with the flags that the library is built with"""
    folder, hipcc = tmp_path_factory.mktemp("assembly"), os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")

    def compiled(source):
        to = os.path.join(str(folder), source + ".s")
        done = subprocess.run([hipcc] + build.FLAGS + ["-S", "--cuda-device-only", os.path.join(build.CSRC, source), "-o", to], stdout=subprocess.PIPE, stderr=subprocess.STDOUT, text=True)
        assert done.returncode == 0, done.stdout
        with open(to) as f:
            return source, f.read()
    with ThreadPoolExecutor(max_workers=min(8, os.cpu_count() or 1)) as pool:
        return dict(pool.map(compiled, build.SOURCES))


@pytest.mark.parametrize("source", build.SOURCES)
def test_no_kernel_reads_a_product_too_early(assembly, source):
    early = {name: early_reads(*x) for name, x in kernels(assembly[source]).items()}
    assert {name: x for name, x in early.items() if x} == {}


def test_products_are_found(assembly):
    count = sum(name.startswith("v_mfma") for text in assembly.values() for code, _ in kernels(text).values() for name, _ in code)
    assert count > 1000
