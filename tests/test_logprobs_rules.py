"""The launch rules of the log probabilities (csrc/logprobs_rules.h), built with plain g++ and asked for their answers: what the
kernels rely on, and that the sizes of the tests on the GPU reach every kernel.  No GPU involved."""
import ctypes
import os
import random
import subprocess

import pytest

from logprobs_shapes import GRADIENTS, SHAPES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
WIDTH = {"bf16": 2, "f16": 2, "f32": 4}


@pytest.fixture(scope="module")
def rules(tmp_path_factory):
    lib = tmp_path_factory.mktemp("rules") / "rules.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC",
                    f"-I{os.path.join(ROOT, 'paper_2205_00119_amd', 'csrc')}", "-o", str(lib),
                    os.path.join(ROOT, "tests", "host", "logprobs_rules_c.cpp")], check=True)
    lib = ctypes.CDLL(str(lib))
    to = ctypes.POINTER(ctypes.c_longlong)
    lib.rules_splits.argtypes = [ctypes.c_size_t, ctypes.c_size_t, ctypes.c_int]
    lib.rules_logprobs.argtypes = [ctypes.c_size_t, ctypes.c_size_t, ctypes.c_int, ctypes.c_size_t, to]
    lib.rules_gradient.argtypes = [ctypes.c_size_t, ctypes.c_size_t, ctypes.c_size_t, to]
    return lib


def logprobs(rules, rows, vocab, top, width):
    got = (ctypes.c_longlong * 5)()
    rules.rules_logprobs(rows, vocab, top, width, got)
    return list(got)


def gradient(rules, rows, vocab, width):
    got = (ctypes.c_longlong * 3)()
    rules.rules_gradient(rows, vocab, width, got)
    return list(got)


def test_parts_of_a_row_cover_it(rules):
    """No part is empty or has fewer logits than there are alternatives; the join can rank all keys and has a lane for every part."""
    rng = random.Random(3)
    ends = [(r, v, t) for r in (1, 2, 255, 256, 257) for v in (1, 7, 8, 16383, 16384, 32767, 32768, 2 ** 24) for t in (0, 1, 64) if t <= v]
    for rows, vocab, top in ends + [(int(2 ** rng.uniform(0, 12)), max(64, int(2 ** rng.uniform(6, 24))), rng.randrange(65)) for _ in range(20000)]:
        splits, chunk, lanes, flight, uncached = logprobs(rules, rows, vocab, top, 2)
        vecs = -(-vocab // 8)
        assert splits == rules.rules_splits(rows, vocab, top) and 1 <= splits <= 64 and splits * max(top, 1) <= max(rules.rules_candidates(), top)
        assert (splits - 1) * chunk < vecs <= splits * chunk, (rows, vocab, top)
        assert vocab - (splits - 1) * chunk * 8 >= top
        assert (lanes, flight) in ((1024, 4), (256, 4), (256, 2)) and (not uncached or (lanes, flight) == (256, 4))
    assert rules.rules_splits(0, 10 ** 6, 0) == 1


def test_sizes_of_the_tests_run_what_they_are_meant_to(rules):
    seen = set()
    for rows, vocab, _, _, fmt, top, want in SHAPES:
        splits, _, lanes, flight, uncached = logprobs(rules, rows, vocab, top, WIDTH[fmt])
        assert (lanes, flight, bool(uncached), splits) == want, (rows, vocab, fmt, top)
        seen.add((fmt, lanes, flight, bool(uncached), top > 0))
        seen.add(("join", fmt, top > 0) if splits > 1 else None)
    for fmt in WIDTH:
        for top in (False, True):
            for lanes, flight, uncached in ((1024, 4, False), (256, 4, False), (256, 4, True)):
                assert (fmt, lanes, flight, uncached, top) in seen
            assert ("join", fmt, top) in seen
    assert all((fmt, 256, 2, False, True) in seen for fmt in WIDTH)
    of = set()
    for rows, vocab, _, _, fmt, unkept in GRADIENTS:
        chunk, chunks, past = gradient(rules, rows, vocab, WIDTH[fmt])
        assert bool(past) == unkept and (chunks - 1) * chunk < -(-vocab // 8) <= chunks * chunk
        of.add((fmt, unkept, "tiny" if vocab < 8 else vocab % 8 > 0))
    assert all((fmt, True, part) in of for fmt in WIDTH for part in (False, True))
