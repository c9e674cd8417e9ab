"""Products pass their results through the LDS from lane to lane of one wavefront, part by part of a tile: the order of those writes and
reads, and of the reads and the next part's writes, is told to the compiler.  Checked in the library's own LLVM IR, because a build
that happens to keep the order gives the right results without it."""
import importlib.util
import os
import re
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def ir(tmp_path_factory):
    spec = importlib.util.spec_from_file_location("lib_build", os.path.join(ROOT, "paper_2205_00119_amd", "build.py"))
    lib_build = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(lib_build)
    if not os.path.exists(lib_build.HIPCC):
        pytest.skip("no hipcc")
    out = str(tmp_path_factory.mktemp("ir") / "linear.ll")
    flags = [f for f in lib_build.FLAGS if f not in ("-shared", "-fPIC")]
    subprocess.run([lib_build.HIPCC, *flags, "--offload-device-only", "-S", "-emit-llvm", "-o", out,
                    os.path.join(ROOT, "paper_2205_00119_amd", "csrc", "linear.hip")], check=True, capture_output=True)
    return open(out).read().splitlines()


@pytest.fixture(scope="module")
def kernels(ir):
    """name -> accesses to the LDS: W stores of floats, w other stores, r loads, | fences."""
    found, accesses = {}, None
    for line in ir:
        start = re.match(r"define .*@(\S+?)\(", line)
        if start:
            accesses = found.setdefault(start.group(1), [])
        elif re.match(r'\s+fence syncscope\("(wavefront|workgroup)"\) (release|acquire)', line):
            accesses.append("|")
        elif re.match(r"\s+store .*ptr addrspace\(3\)", line):
            accesses.append("W" if "float" in line.split("ptr addrspace")[0] else "w")
        elif re.match(r"\s+%\S+ = load .*ptr addrspace\(3\)", line):
            accesses.append("r")
    return {name: re.sub(r"\|+", "|", "".join(a)) for name, a in found.items()}


def test_results_pass_through_the_lds_in_an_order_that_the_compiler_knows(kernels):
    tiles = {name: a for name, a in kernels.items() if "product_kernel" in name}
    few = {name: a for name, a in kernels.items() if "few_rows_kernel" in name}
    assert len(tiles) >= 30 and len(few) >= 12
    parts = set()
    for name, a in {**tiles, **few}.items():
        assert "W" in a, name
        # operands are no floats; the results begin behind a barrier
        before, order = a[:a.index("W")], a[a.index("W"):]
        assert not before or before.endswith("|"), (name, a)
        assert re.fullmatch(r"(W+\|r+\|)+", order), (name, order)
        parts.add(len(re.findall("W+", order)))
    assert parts == {1, 2}                                       # tiles of 256 rows come in two parts


def test_assembly_that_sets_m0_says_so(ir):
    """A value that the compiler holds in m0, as it does for some LDS and message instructions, is then not taken to be there still."""
    sets = [line for line in ir if re.search(r'asm sideeffect "[^"]*\bm0\b', line)]
    assert sets and all("~{m0}" in line for line in sets)
