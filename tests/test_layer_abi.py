"""Layer norm, dropout and log probabilities without a GPU: every argument error is reported by the host-side checks before
any HIP call, workspaces and counters are what the header says, and the binding hands over what ctypes does."""
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


def expect(code, fragment, call):
    with pytest.raises(mics.MicsError) as e:
        call()
    assert e.value.code == code and fragment in str(e.value), str(e.value)
    assert fragment in mics.mics_last_error()


# name -> (function, its arguments by name in order, keywords, matrices in the order of their strides, vectors of parameters,
# float32 vectors)
TYPES = dict(dtype=0, param_dtype=0)
KEY = dict(drop=0.1, seed=1, offset=2)
WORK = dict(grad_dtype=0, workspace=P[15], workspace_bytes=1 << 28)
CALLS = {
    "bias_dropout_add": (dict(out=P[0], x=P[1], bias=P[2], residual=P[3], rows=8, cols=64), {**KEY, **TYPES},
                         ["out", "x", "residual"], ["out"], ["bias", "residual"]),
    "bias_dropout_add_backward": (dict(dx=P[0], dbias=P[1], dout=P[2], rows=8, cols=64), {**KEY, **WORK, "dtype": 0},
                                  ["dx", "dout"], ["dx", "dbias"], ["dbias"]),
    "layer_norm": (dict(y=P[0], mean=P[1], rstd=P[2], x=P[3], weight=P[4], bias=P[5], rows=8, cols=64), {"eps": 1e-5, **TYPES},
                   ["y", "x"], ["y", "mean", "rstd"], ["mean", "rstd", "weight", "bias"]),
    "layer_norm_backward": (dict(dx=P[0], dweight=P[1], dbias=P[2], dy=P[3], x=P[4], mean=P[5], rstd=P[6], weight=P[7], rows=8, cols=64),
                            {**TYPES, **WORK}, ["dx", "dy", "x"], ["dx", "dweight", "dbias"], ["dweight", "dbias", "weight"]),
    "dropout_add_layer_norm": (dict(y=P[0], sum=P[1], mean=P[2], rstd=P[3], x=P[4], bias=P[5], residual=P[6], weight=P[7], norm_bias=P[8],
                                    rows=8, cols=64), {**KEY, "eps": 1e-5, **TYPES}, ["y", "sum", "x", "residual"],
                               ["y", "sum", "mean", "rstd"], ["sum", "mean", "rstd", "bias", "residual", "weight", "norm_bias"]),
    "dropout_add_layer_norm_backward": (
        dict(dx=P[0], dresidual=P[1], dbias=P[2], dweight=P[3], dnorm_bias=P[4], dy=P[5], dsum=P[6], sum=P[7], mean=P[8], rstd=P[9],
             weight=P[10], rows=8, cols=64), {**KEY, **TYPES, **WORK}, ["dx", "dresidual", "dy", "dsum", "sum"],
        ["dx", "dresidual", "dbias", "dweight", "dnorm_bias"], ["dresidual", "dbias", "dweight", "dnorm_bias", "dsum", "weight"]),
    "token_logprobs": (dict(logprob=P[0], entropy=P[1], lse=P[2], top_ids=P[3], top_logprobs=P[4], logits=P[5], targets=P[6], rows=8,
                            vocab=64), dict(dtype=0, top_k=3), ["logits"], ["logprob", "entropy", "lse", "top_ids", "top_logprobs"],
                       ["entropy", "lse"]),
    "token_logprobs_backward": (dict(dlogits=P[0], logits=P[1], targets=P[2], lse=P[3], entropy=P[4], dlogprob=P[5], dentropy=P[6], rows=8,
                                     vocab=64), dict(dtype=0), ["dlogits", "logits"], ["dlogits"], ["dentropy"]),
}
NAMES = list(CALLS)


def call(name, **changes):
    args, kwargs = CALLS[name][:2]
    kwargs = {**kwargs, **{k: v for k, v in changes.items() if k not in args}}
    return lambda: getattr(mics, "mics_" + name)(*[changes.get(k, v) for k, v in args.items()], stream=0, **kwargs)


def size_names(name):
    return "vocab" if name.startswith("token") else "cols"


@pytest.mark.parametrize("name", NAMES)
def test_sizes(name):
    n = size_names(name)
    expect(INVALID, f"{n} = 0", call(name, **{n: 0}))
    expect(UNSUPPORTED, "exceeds", call(name, **{n: 2 ** 24 + 1}))
    expect(INVALID, "overflows", call(name, rows=2 ** 60))
    expect(INVALID, "overflows", call(name, rows=-1))


@pytest.mark.parametrize("name", NAMES)
def test_types(name):
    for key in CALLS[name][1]:
        if key.endswith("dtype"):
            for bad in (3, -1, 99):
                expect(UNSUPPORTED, f"{key} = {bad}", call(name, **{key: bad}))


@pytest.mark.parametrize("name", NAMES)
def test_missing_buffers(name):
    args, kwargs, _, _, optional = CALLS[name]
    for key, value in args.items():
        if value in P and key not in optional:
            changes = {key: None}
            expect(INVALID, f"mics_{name}: {key} is NULL", call(name, **changes))
    if "workspace" in kwargs:
        expect(INVALID, "workspace is NULL", call(name, workspace=None))
        need = mics.mics_column_workspace_bytes(8, 64)
        expect(INVALID, f"workspace_bytes = {need - 1}, needs {need}", call(name, workspace_bytes=need - 1))
        expect(ALIGN, "workspace", call(name, workspace=P[15] + 4))


@pytest.mark.parametrize("name", NAMES)
def test_alignment(name):
    args = CALLS[name][0]
    for key, value in args.items():
        if value in P:
            expect(ALIGN, key, call(name, **{key: value + 1}))


@pytest.mark.parametrize("name", NAMES)
def test_overlaps(name):
    args, kwargs, matrices, outs, _ = CALLS[name]
    for out in outs:
        for other, value in args.items():
            if value not in P or other == out:
                continue
            shifted = value + 16 if other in matrices and out in matrices else value
            expect(INVALID, "overlaps", call(name, **{out: shifted}))
        if "workspace" in kwargs:
            expect(INVALID, "overlaps", call(name, **{out: kwargs["workspace"]}))


@pytest.mark.parametrize("name", [n for n in NAMES if n != "token_logprobs"])
def test_strides(name):
    args, _, matrices, _, _ = CALLS[name]
    good = [64 + 8 * i for i in range(len(matrices))]
    for i, m in enumerate(matrices):
        expect(INVALID, f"the row stride of {m}", call(name, strides=tuple(63 if k == i else s for k, s in enumerate(good))))
        expect(INVALID, "overflows", call(name, strides=tuple(2 ** 61 if k == i else s for k, s in enumerate(good))))
    for wrong in (good[:-1], good + [64], []):
        with pytest.raises(ValueError, match="row strides"):
            call(name, strides=tuple(wrong))()


def test_rows_between_each_other():
    """Halves of one wide buffer are no overlap; a column more is one."""
    name = "layer_norm"
    expect(INVALID, "y overlaps x", call(name, y=A, x=A + 2 * 63, strides=(128, 128)))
    expect(INVALID, "y overlaps x", call(name, y=A + 2 * 65, x=A, strides=(128, 128)))
    expect(INVALID, "y overlaps x", call(name, y=A, x=A + 2 * 64, strides=(128, 136)))
    expect(INVALID, "eps", call(name, y=A, x=A + 2 * 64, strides=(128, 128), eps=-1.0))
    # what is left of the check: the next argument error is another
    expect(ALIGN, "weight", call(name, y=A, x=A + 2 * 64, strides=(128, 128), weight=P[9] + 1))


@pytest.mark.parametrize("name", [n for n in NAMES if "dropout" in n])
def test_share_that_is_dropped(name):
    for bad in (1.0, -0.1, float("nan"), 2.0, float("inf")):
        expect(INVALID, "must lie in [0, 1)", call(name, drop=bad))


def test_eps():
    for name in ("layer_norm", "dropout_add_layer_norm"):
        for bad in (-1e-5, float("nan")):
            expect(INVALID, "eps", call(name, eps=bad))


def test_log_probabilities():
    f = "token_logprobs"
    for bad in (-1, 65, 1000):
        expect(INVALID, f"top_k = {bad}", call(f, top_k=bad, vocab=5000, stride=5000))
    expect(INVALID, "top_k = 9", call(f, vocab=8, stride=8, top_k=9))
    expect(INVALID, "row stride of logits", call(f, stride=63))
    need = mics.mics_token_logprobs_workspace_bytes(2, 100000, 3)
    assert need > 0
    expect(INVALID, "workspace_bytes = 0", call(f, rows=2, vocab=100000, stride=100000))
    expect(INVALID, "workspace is NULL", call(f, rows=2, vocab=100000, stride=100000, workspace_bytes=need))
    expect(INVALID, "top_ids is NULL", call(f, top_ids=None))
    expect(INVALID, "entropy is NULL", call("token_logprobs_backward", entropy=None))


def test_workspaces_and_counters():
    assert mics.mics_dropout_counters(3, 17) == 9 and mics.mics_dropout_counters(5, 16) == 10 and mics.mics_dropout_counters(0, 8) == 0
    w = mics.mics_column_workspace_bytes
    assert w(0, 64) == 0 and w(10, 0) == 0 and w(10, 2 ** 24 + 1) == 0
    assert w(1, 64) <= w(512, 64) == w(10 ** 6, 64)
    l = mics.mics_token_logprobs_workspace_bytes
    assert l(8192, 65536, 64) == 0 and l(0, 65536, 5) == 0 and l(4, 131072, -1) == 0 and l(4, 131072, 65) == 0
    assert l(4, 131072, 8) >= l(4, 131072, 0) > 0


# ---- the binding -------------------------------------------------------------------------------

T = torch.zeros(64, 64)
LIKE = {"as it is": lambda x: x, "numpy's integers": lambda x: np.int64(x) if type(x) is int and x < 2 ** 40 else x,
        "lists": lambda x: list(x) if type(x) is tuple else x, "a parameter": lambda x: torch.nn.Parameter(x) if x is T else x,
        "packed": lambda x: None if type(x) is tuple else x, "rows apart": lambda x: T[:, :40] if x is T else x,
        "transposed": lambda x: T[:, :40].t() if x is T else x, "text": lambda x: "7" if type(x) is int else x,
        "too few": lambda x: x[1:] if type(x) is tuple else x}


@pytest.mark.parametrize("like", list(LIKE))
@pytest.mark.parametrize("name", NAMES)
def test_whole_calls_hand_over_what_ctypes_does(monkeypatch, name, like):
    """Both ways with the library's entry point replaced by one that records its arguments."""
    args, kwargs, matrices, _, _ = CALLS[name]
    args = {k: (T if k in matrices[:1] else v) for k, v in args.items()}
    if name == "token_logprobs":
        kwargs = {**kwargs, "stride": 64}
    else:
        kwargs = {**kwargs, "strides": tuple(64 + 2 * i for i in range(len(matrices)))}
    args, kwargs = [LIKE[like](x) for x in args.values()], {k: LIKE[like](x) for k, x in kwargs.items()}
    real, seen = getattr(mics.lib, "mics_" + name), []
    at = {"bias_dropout_add": 6, "bias_dropout_add_backward": 5, "layer_norm": 8, "layer_norm_backward": 10,
          "dropout_add_layer_norm": 11, "dropout_add_layer_norm_backward": 13, "token_logprobs": None, "token_logprobs_backward": 9}[name]

    def record(*got):
        got = list(got)
        if at is not None and got[at]:
            got[at] = list((ctypes.c_size_t * len(matrices)).from_address(got[at]))
        seen.append(got)
        return 0

    stub = ctypes.CFUNCTYPE(ctypes.c_int, *real.argtypes)(record)
    addresses = [ctypes.cast(getattr(mics.lib, "mics_" + n), ctypes.c_void_p).value for n in mics._LAYER_CALLS]
    fake = [ctypes.cast(stub, ctypes.c_void_p).value if n == name else a for n, a in zip(mics._LAYER_CALLS, addresses)]

    def outcome():
        try:
            return getattr(mics, "mics_" + name)(*args, stream=64, **kwargs), seen.pop()
        except Exception as e:                                      # noqa: BLE001
            return type(e), str(e)

    mics._marshal.bind_layer(tuple(fake))
    monkeypatch.setattr(mics, "lib", types.SimpleNamespace(**{"mics_" + name: stub}))
    asked = []
    fast = getattr(mics._marshal, name)
    monkeypatch.setattr(mics, "_marshal", types.SimpleNamespace(**{**vars(mics._marshal), name: lambda *a: asked.append(fast(*a)) or asked[-1]}))
    try:
        first = outcome()
        monkeypatch.setattr(mics, "_marshal", types.SimpleNamespace(**{**vars(mics._marshal), name: lambda *a: None}))
        assert first == outcome()
        if like in ("as it is", "lists", "packed", "rows apart"):
            assert asked == [0]                                     # this one does go past ctypes
    finally:
        monkeypatch.undo()
        mics._marshal.bind_layer(tuple(addresses))


def test_bind_layer_refuses_what_is_no_table():
    for bad in ([], (1,), tuple(range(9)), ("x",) * 8):
        with pytest.raises((TypeError, ValueError)):
            mics._marshal.bind_layer(bad)
