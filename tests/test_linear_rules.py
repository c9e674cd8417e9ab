"""How products are cut: the rules of linear_rules.h on the CPU, and that the sizes of the GPU tests reach every kernel."""
import ctypes
import os
import random
import subprocess

import pytest

from linear_shapes import SHAPES

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
FIELDS = ("few", "bm", "bn", "whole", "shared", "splits", "depth", "a_copy", "b_copy", "workspace", "most")
WIDTH = {"bf16": 2, "f16": 2, "f32": 4}


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    so = tmp_path_factory.mktemp("rules") / "rules.so"
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wextra", "-Werror", "-fPIC", "-shared",
                    f"-I{os.path.join(ROOT, 'paper_2205_00119_amd', 'csrc')}", "-o", str(so),
                    os.path.join(ROOT, "tests", "host", "linear_rules_c.cpp")], check=True)
    f = ctypes.CDLL(str(so)).plan_of_product

    def of(m, n, k, width, a_turned, b_turned, a16=True, b16=True, chunks=True, blocks=False):
        out = (ctypes.c_size_t * 11)()
        f((ctypes.c_size_t * 4)(m, n, k, width), (ctypes.c_int * 6)(a_turned, b_turned, a16, b16, chunks, blocks), out)
        return dict(zip(FIELDS, out))
    return of


def ceil(a, b):
    return -(-a // b)


def test_every_tile_and_every_k_is_taken_once(plan):
    rng = random.Random(3)
    size = lambda: int(2 ** rng.uniform(0, 14.5))                                      # noqa: E731
    for _ in range(3000):
        m, n, k, width = size(), size(), rng.choice([0, size(), size(), size()]), rng.choice([2, 4])
        turned = rng.choice([(False, False), (False, True), (True, True)])
        a16, b16, chunks, blocks = (rng.random() < p for p in (0.5, 0.5, 0.9, 0.2))
        p = plan(m, n, k, width, *turned, a16, b16, chunks, blocks)
        tiles = ceil(m, p["bm"]) * ceil(n, p["bn"])
        depths = ceil(k, 128 // width)
        what = (m, n, k, width, turned, a16, b16, chunks, blocks, p)
        assert p["whole"] + p["shared"] == tiles and (p["splits"] == 1) == (p["shared"] == 0), what
        if p["splits"] > 1:
            # no part is empty, all of k is there
            assert p["depth"] * p["splits"] >= depths and p["depth"] * (p["splits"] - 1) < depths, what
        assert p["workspace"] <= p["most"] <= 1 << 26, what
        if p["few"]:
            assert m <= p["bm"] <= 32 and not turned[0] and chunks and k > 0 and p["bm"] % 16 == 0, what
            assert turned[1] or b16, what
            assert not blocks or turned[1] or p["bn"] == 64, what
        else:
            tile = p["bm"], p["bn"]
            assert tile == (128, 128) or chunks, what
            assert tile in [(128, 128)] + ([(256, 256)] if width == 2 else [(64, 64), (32, 128)]), what
            assert tile != (32, 128) or not turned[0], what
        copied = [p["a_copy"], p["b_copy"]]
        assert (not copied[0] or not a16) and (not copied[1] or not b16) and (chunks or copied == [0, 0]), what
        if any(copied):                                                                # all that is off 16 bytes
            kp = k if a16 or b16 else depths * 128 // width
            rows = [(kp, m) if turned[0] else (m, kp), (kp, n) if turned[1] else (n, kp)]
            for bytes_, on, (r, c) in zip(copied, (a16, b16), rows):
                assert bytes_ == (0 if on else r * ceil(c * width, 16) * 16), what


def test_sizes_of_the_gpu_tests_reach_every_kernel(plan):
    seen = set()
    for rows, cin, cout, pad, skew, fmt in SHAPES:
        w = WIDTH[fmt]
        for op, m, n, k, turned in (("linear", rows, cout, cin, (False, False)), ("input", rows, cin, cout, (False, True)),
                                    ("weight", cout, cin, rows, (True, True))):
            def operand(high, wide, is_turned):
                on = (64 + skew) * w % 16 == 0 and (wide + pad) * w % 16 == 0 and (not is_turned or wide * w % 16 == 0)
                return on, wide * w >= 16
            a16, ac = operand(*((k, m) if turned[0] else (m, k)), turned[0])
            b16, bc = operand(*((k, n) if turned[1] else (n, k)), turned[1])
            for blocks in ((False, True) if op == "linear" else (False,)):
                p = plan(m, n, k, w, *turned, a16, b16, ac and bc, blocks)
                how = "few" if p["few"] else "guarded" if not (ac and bc) else \
                    "direct" if (a16 or p["a_copy"]) and (b16 or p["b_copy"]) else "through"
                seen.add((op, w, how, p["bm"], p["bn"] if p["few"] else 0))
                if p["a_copy"] + p["b_copy"]:
                    seen.add((op, w, "copy"))
                if p["splits"] > 1:
                    seen.add((op, w, how, p["bm"], "parts", p["whole"] > 0))
    wanted = []
    for op in ("linear", "input", "weight"):
        wanted += [(op, w, how, 128, 0) for w in (2, 4) for how in ("guarded", "direct", "through")]
        wanted += [(op, 4, how, 64, 0) for how in ("direct", "through")]
        wanted += [x for how in ("direct", "through") for x in ((op, 4, how, 32, 0), (op, 4, how, 32, "parts", False)) if op != "weight"]
        wanted += [(op, 2, how, 256, 0) for how in ("direct", "through") if (op, how) != ("weight", "through")]
        wanted += [(op, w, how, bm, "parts", False) for w, bm in ((2, 128), (4, 64)) for how in ("direct", "through")]
        wanted += [(op, 2, "copy")]
    wanted += [("input", w, "few", bm, 256 // w) for w in (2, 4) for bm in (16, 32)]
    wanted += [(op, w, "few", bm, "parts", False) for op in ("linear", "input") for w in (2, 4) for bm in (16, 32)]
    wanted += [("linear", w, "few", bm, bn) for w in (2, 4) for bm in (16, 32) for bn in (16, 64)]
    # whole tiles and shared ones in one launch
    wanted += [("linear", 2, "direct", bm, "parts", True) for bm in (128, 256)]
    assert not [x for x in wanted if x not in seen]
