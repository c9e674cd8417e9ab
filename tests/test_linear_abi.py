"""The linear layer and activations without a GPU: every argument error is reported by the host-side checks before any HIP call,
workspaces are what the header says, and the binding hands over what ctypes does."""
import ctypes
import types

import numpy as np
import pytest
import torch

mics = pytest.importorskip("paper_2205_00119_amd")

A = 0x7F0000000000          # a pretend device address
BUF = 1 << 30
P = [A + BUF * i for i in range(16)]
INVALID, ALIGN, UNSUPPORTED = mics.MICS_ERR_INVALID_ARG, mics.MICS_ERR_ALIGNMENT, mics.MICS_ERR_UNSUPPORTED

# name -> (arguments by name in order, keywords, columns of the matrices in the order of their strides, results, what may be NULL,
# inputs that no result may replace)
WORK = dict(workspace=P[15], workspace_bytes=1 << 26)
CALLS = {
    "activation": (dict(y=P[0], codes=P[1], scales=P[2], x=P[3], bias=P[4], rows=8, cols=64), dict(act=2, dtype=0, param_dtype=0),
                   dict(y="cols", codes="cols", x="cols"), ["y", "codes", "scales"], ["y", "bias"], []),
    "checkpoint_read": (dict(y=P[0], codes=P[1], scales=P[2], rows=8, cols=64), dict(act=2, dtype=0), dict(y="cols", codes="cols"), ["y"],
                        [], ["codes"]),
    "activation_backward": (dict(dx=P[0], dbias=P[1], dy=P[2], z=None, codes=P[4], scales=P[5], rows=8, cols=64),
                            dict(act=2, dtype=0, grad_dtype=0, **WORK), dict(dx="cols", dy="cols", z="cols", codes="cols"), ["dx", "dbias"],
                            ["dx", "dbias"], ["codes"]),
    "linear": (dict(out=P[0], pre=P[1], codes=P[2], scales=P[3], x=P[4], weight=P[5], bias=P[6], residual=P[7], rows=8, in_features=128,
                    out_features=64), dict(act=2, dtype=0, param_dtype=0, **WORK),
               dict(out="out_features", pre="out_features", codes="out_features", x="in_features", weight="in_features",
                    residual="out_features"), ["out", "pre", "codes", "scales"], ["pre", "bias", "residual"], ["x", "weight"]),
    "linear_backward_input": (dict(dx=P[0], dz=P[1], weight=P[2], dsum=P[3], rows=8, in_features=128, out_features=64),
                              dict(dtype=0, **WORK), dict(dx="in_features", dz="out_features", weight="in_features", dsum="in_features"),
                              ["dx"], ["dsum"], ["dz", "weight"]),
    "linear_backward_weight": (dict(dweight=P[0], dz=P[1], x=P[2], rows=8, in_features=128, out_features=64),
                               dict(dtype=0, grad_dtype=0, **WORK), dict(dweight="in_features", dz="out_features", x="in_features"),
                               ["dweight"], [], ["dz", "x"]),
}
NAMES = list(CALLS)


def call(name, **changes):
    args, kwargs = CALLS[name][:2]
    kwargs = {**kwargs, **{k: v for k, v in changes.items() if k not in args}}
    return lambda: getattr(mics, "mics_" + name)(*[changes.get(k, v) for k, v in args.items()], stream=0, **kwargs)


def expect(code, fragment, call):
    with pytest.raises(mics.MicsError) as e:
        call()
    assert e.value.code == code and fragment in str(e.value), str(e.value)
    assert fragment in mics.mics_last_error()


def sizes(name):
    return [k for k in CALLS[name][0] if k in ("cols", "in_features", "out_features")]


@pytest.mark.parametrize("name", NAMES)
def test_sizes(name):
    for n in sizes(name):
        expect(INVALID, f"{n} = 0", call(name, **{n: 0}))
        expect(UNSUPPORTED, f"{n} = {2 ** 24 + 1} exceeds", call(name, **{n: 2 ** 24 + 1}))
    expect(INVALID, "overflows", call(name, rows=2 ** 60))
    expect(INVALID, "overflows", call(name, rows=-1))


@pytest.mark.parametrize("name", NAMES)
def test_types_and_activations(name):
    for key in CALLS[name][1]:
        if key.endswith("dtype"):
            for bad in (3, -1, 99):
                expect(UNSUPPORTED, f"{key} = {bad}", call(name, **{key: bad}))
        if key == "act":
            for bad in (5, -1):
                expect(UNSUPPORTED, f"act = {bad}", call(name, act=bad))


@pytest.mark.parametrize("name", NAMES)
def test_missing_buffers(name):
    args, kwargs, _, _, optional, _ = CALLS[name]
    for key, value in args.items():
        if value in P and key not in optional:
            expect(INVALID, f"mics_{name}: {key} is NULL", call(name, **{key: None}))
    if name == "activation_backward":
        expect(INVALID, "workspace is NULL", call(name, workspace=None))
        need = mics.mics_column_workspace_bytes(8, 64)
        expect(INVALID, f"workspace_bytes = {need - 1}, needs {need}", call(name, workspace_bytes=need - 1))
        expect(ALIGN, "workspace", call(name, workspace=P[15] + 4))
        expect(INVALID, "z and codes are NULL", call(name, codes=None, scales=None))
        expect(INVALID, "are NULL", call(name, dx=None, dbias=None))
        expect(INVALID, "z or codes has to be NULL", call(name, z=P[3]))
    if name == "activation":
        expect(INVALID, "y and codes are NULL", call(name, y=None, codes=None, scales=None))


def test_missing_workspace_of_products():
    """Products of few tiles take one, and say how much."""
    for name, shape in (("linear", (8, 20000, 130)), ("linear_backward_input", (40, 130, 20000)), ("linear_backward_weight", (20000, 130, 128))):
        n = dict(zip(("rows", "in_features", "out_features"), shape))
        if name == "linear":
            n["rows"] = 40
        expect(INVALID, "workspace_bytes = 0, needs", call(name, workspace_bytes=0, **n))
        expect(INVALID, "workspace is NULL", call(name, workspace=None, **n))
        expect(ALIGN, "workspace", call(name, workspace=P[15] + 4, **n))


@pytest.mark.parametrize("name", NAMES)
def test_alignment(name):
    for key, value in CALLS[name][0].items():
        if value in P and key != "codes":
            expect(ALIGN, key, call(name, **{key: value + 1}))


@pytest.mark.parametrize("name", NAMES)
def test_overlaps(name):
    args, kwargs, matrices, outs, _, whole = CALLS[name]
    for out in outs:
        for other, value in args.items():
            if value not in P or other == out:
                continue
            expect(INVALID, "overlaps", call(name, **{out: value + (16 if other in matrices and out in matrices else 0)}))
        for other in whole:                                         # not even in the same place
            strides = tuple(256 for _ in matrices)
            expect(INVALID, f"{out} overlaps {other}", call(name, **{out: args[other], "strides": strides}))


@pytest.mark.parametrize("name", NAMES)
def test_strides(name):
    args, _, matrices, _, _, _ = CALLS[name]
    good = [128 + 8 * i for i in range(len(matrices))]
    for i, (m, cols) in enumerate(matrices.items()):
        if args[m] is None:
            continue
        expect(INVALID, f"the row stride of {m}", call(name, strides=tuple(args[cols] - 1 if k == i else s for k, s in enumerate(good))))
        expect(INVALID, "overflows", call(name, strides=tuple(2 ** 61 if k == i else s for k, s in enumerate(good))))
    for wrong in (good[:-1], good + [64], []):
        with pytest.raises(ValueError, match="row strides"):
            call(name, strides=tuple(wrong))()


def test_codes_in_the_place_of_wider_rows():
    """Rows of the same distance in bytes, but not of the same length: no place to be replaced."""
    expect(INVALID, "dx overlaps codes", call("activation_backward", dx=P[4], strides=(128, 64, 64, 256)))


def test_workspaces():
    w = mics.mics_linear_workspace_bytes
    assert w(10, 0, 5) == 0 and w(10, 5, 2 ** 24 + 1) == 0 and w(2 ** 60, 64, 64) == 0
    for shape in ((1, 64, 64), (100, 4096, 4096), (2047, 5121, 2561), (4095, 8193, 4095), (8192, 512, 512), (64, 16384, 16384), (0, 5, 7),
                  (10 ** 9, 1, 1), (513, 100003, 257), (4096, 8192, 32768)):
        assert 0 <= w(*shape) <= 1 << 26, shape
    s = mics.mics_checkpoint_scales
    assert s(3, 64) == 3 and s(3, 65) == 6 and s(5, 1) == 5 and s(0, 64) == 0 and s(3, 0) == 0


# ---- the binding -------------------------------------------------------------------------------

T = torch.zeros(64, 128)
LIKE = {"as it is": lambda x: x, "numpy's integers": lambda x: np.int64(x) if type(x) is int and x < 2 ** 40 else x,
        "lists": lambda x: list(x) if type(x) is tuple else x, "a parameter": lambda x: torch.nn.Parameter(x) if x is T else x,
        "packed": lambda x: None if type(x) is tuple else x, "rows apart": lambda x: T[:, :40] if x is T else x,
        "transposed": lambda x: T[:, :40].t() if x is T else x, "text": lambda x: "7" if type(x) is int else x,
        "too few": lambda x: x[1:] if type(x) is tuple else x}


@pytest.mark.parametrize("like", list(LIKE))
@pytest.mark.parametrize("name", NAMES)
def test_whole_calls_hand_over_what_ctypes_does(monkeypatch, name, like):
    """Both ways with the library's entry point replaced by one that records its arguments."""
    args, kwargs, matrices, _, _, _ = CALLS[name]
    at = list(args).index("rows") + len([k for k in args if k in ("rows", "cols", "in_features", "out_features")])
    first = next(iter(matrices))
    args = {k: (T if k == first else v) for k, v in args.items()}
    kwargs = {**kwargs, "strides": tuple(128 + 2 * i for i in range(len(matrices)))}
    args, kwargs = [LIKE[like](x) for x in args.values()], {k: LIKE[like](x) for k, x in kwargs.items()}
    real, seen = getattr(mics.lib, "mics_" + name), []

    def record(*got):
        got = list(got)
        if got[at]:
            got[at] = list((ctypes.c_size_t * len(matrices)).from_address(got[at]))
        seen.append(got)
        return 0

    stub = ctypes.CFUNCTYPE(ctypes.c_int, *real.argtypes)(record)
    addresses = [ctypes.cast(getattr(mics.lib, "mics_" + n), ctypes.c_void_p).value for n in mics._LINEAR_CALLS]
    fake = [ctypes.cast(stub, ctypes.c_void_p).value if n == name else a for n, a in zip(mics._LINEAR_CALLS, addresses)]

    def outcome():
        try:
            return getattr(mics, "mics_" + name)(*args, stream=64, **kwargs), seen.pop()
        except Exception as e:                                      # noqa: BLE001
            return type(e), str(e)

    mics._marshal.bind_linear(tuple(fake))
    monkeypatch.setattr(mics, "lib", types.SimpleNamespace(**{"mics_" + name: stub}))
    asked = []
    fast = getattr(mics._marshal, name)
    monkeypatch.setattr(mics, "_marshal", types.SimpleNamespace(**{**vars(mics._marshal), name: lambda *a: asked.append(fast(*a)) or asked[-1]}))
    try:
        got = outcome()
        monkeypatch.setattr(mics, "_marshal", types.SimpleNamespace(**{**vars(mics._marshal), name: lambda *a: None}))
        assert got == outcome()
        if like in ("as it is", "lists", "packed", "rows apart"):
            assert asked == [0]                                     # this one does go past ctypes
    finally:
        monkeypatch.undo()
        mics._marshal.bind_linear(tuple(addresses))


def test_bind_linear_refuses_what_is_no_table():
    for bad in ([], (1,), tuple(range(9)), ("x",) * 6):
        with pytest.raises((TypeError, ValueError)):
            mics._marshal.bind_linear(bad)
