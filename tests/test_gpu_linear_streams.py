"""The linear layer, its gradients, activations and checkpoints on streams and in replayed graphs: every result is overwritten first,
so that only what a call or a replay writes itself can be right."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

mics = pytest.importorskip("paper_2205_00119_amd")

DEV = "cuda:0"
GELU = mics.MICS_ACT_GELU


class Step:
    """Inputs, results and scratch of a run of the calls as a sublayer makes them.  Sizes: few rows, which have a kernel of their own;
    products whose last tiles are shared; operands off 16 bytes that are copied first."""

    def __init__(self, rows, cin, cout):
        r = np.random.default_rng(21)
        half = lambda *s: torch.from_numpy(r.normal(size=s)).to(torch.bfloat16).to(DEV)      # noqa: E731
        self.sizes = rows, cin, cout
        self.x, self.w, self.b, self.res, self.dy = half(rows, cin), half(cout, cin), half(cout), half(rows, cout), half(rows, cout)
        self.inputs = [self.x, self.w, self.res, self.dy]
        o = lambda *s, t=torch.bfloat16: torch.empty(*s, dtype=t, device=DEV)                 # noqa: E731
        n = mics.mics_checkpoint_scales(rows, cout)
        self.out = {"y": o(rows, cout), "pre": o(rows, cout), "codes": o(rows, cout, t=torch.int8), "scales": o(n, t=torch.float32),
                    "g": o(rows, cout), "codes2": o(rows, cout, t=torch.int8), "scales2": o(n, t=torch.float32), "again": o(rows, cout),
                    "dz": o(rows, cout), "db": o(cout, t=torch.float32), "dx": o(rows, cin), "dw": o(cout, cin, t=torch.float32)}
        self.n = max(mics.mics_linear_workspace_bytes(rows, cin, cout), mics.mics_column_workspace_bytes(rows, cout))
        self.ws = o(self.n, t=torch.uint8)

    def __call__(self, stream=None):
        (n, i, c), o = self.sizes, self.out
        work = dict(workspace=self.ws, workspace_bytes=self.n, stream=stream)
        t = dict(dtype=0, param_dtype=0)
        mics.mics_linear(o["y"], o["pre"], o["codes"], o["scales"], self.x, self.w, self.b, self.res, n, i, c, act=GELU, **t, **work)
        mics.mics_activation(o["g"], o["codes2"], o["scales2"], o["pre"], self.b, n, c, act=GELU, stream=stream, **t)
        mics.mics_checkpoint_read(o["again"], o["codes2"], o["scales2"], n, c, act=GELU, dtype=0, stream=stream)
        mics.mics_activation_backward(o["dz"], o["db"], self.dy, None, o["codes"], o["scales"], n, c, act=GELU, dtype=0, grad_dtype=2, **work)
        mics.mics_linear_backward_input(o["dx"], o["dz"], self.w, None, n, i, c, dtype=0, **work)
        mics.mics_linear_backward_weight(o["dw"], o["dz"], self.x, n, i, c, dtype=0, grad_dtype=2, **work)

    def spoil(self):
        for x in self.out.values():
            x.fill_(float("nan") if x.is_floating_point() else -128)        # a code that no call writes
        self.ws.fill_(0xFF)
        torch.cuda.synchronize()

    def results(self):
        torch.cuda.synchronize()
        return {n: x.clone() for n, x in self.out.items()}


SIZES = [(7, 1024, 700), (300, 1100, 650), (301, 2047, 1003)]


def differing(got, want):
    return [n for n in want if not torch.equal(got[n], want[n])]


@pytest.mark.parametrize("sizes", SIZES)
def test_replays_write_every_result_anew(sizes):
    s = Step(*sizes)
    s()
    before = s.results()
    s.spoil()
    assert differing(s.results(), before) == list(before)        # what the comparisons rest on
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s()
    for k in range(1, 5):
        for x in s.inputs:
            x.copy_(x.roll(k, 0) * (1.0 + 0.125 * k))
        s.spoil()
        s()
        want = s.results()
        assert differing(before, want) == list(want)
        s.spoil()
        graph.replay()
        assert not differing(s.results(), want), k
        before = want


@pytest.mark.parametrize("sizes", SIZES[:2])
@pytest.mark.parametrize("explicit", [True, False])
def test_calls_run_where_they_are_told_to(sizes, explicit):
    """Inputs are right on the side stream only, and only after a long piece of work there.  What is launched anywhere else reads
    zeros, or writes before results are spoilt."""
    s, side, other = Step(*sizes), torch.cuda.Stream(), torch.cuda.Stream()
    s()
    want = s.results()
    held = [x.clone() for x in s.inputs]
    big = torch.zeros(1 << 29, device=DEV)
    s.spoil()
    with torch.cuda.stream(side):
        for x in s.inputs:
            x.zero_()
        side.synchronize()                                       # zeros are there before anything else starts
        for _ in range(32):
            big.add_(1.0)                                        # 2 GB each way: some 25 ms, the calls take one to queue
        for x, h in zip(s.inputs, held):
            x.copy_(h)
        if not explicit:
            s()                                                  # torch's current stream
    if explicit:
        with torch.cuda.stream(other):
            s(stream=side)
    side.synchronize()
    assert not differing(s.results(), want)


def test_two_streams_at_once_with_scratch_of_their_own():
    steps = [Step(*SIZES[1]) for _ in range(2)]
    steps[1].x.mul_(2.0)
    want = []
    for s in steps:
        s()
        want.append(s.results())
        s.spoil()
    streams = [torch.cuda.Stream() for _ in steps]
    for _ in range(20):
        for s, st in zip(steps, streams):
            s(stream=st)
    for s, w in zip(steps, want):
        assert not differing(s.results(), w)


def test_places_beyond_32_bits():
    """Rows whose places pass 2^31 elements: the last ones are right."""
    rows, cols = 70000, 40000                                    # 2.8e9 elements
    x = torch.empty(rows, cols, dtype=torch.bfloat16, device=DEV)
    y = torch.empty_like(x)
    for r in range(0, rows, 7000):
        x[r:r + 7000].normal_()
    codes, scales = torch.empty(rows, cols, dtype=torch.int8, device=DEV), torch.empty(mics.mics_checkpoint_scales(rows, cols), device=DEV)
    mics.mics_activation(y, codes, scales, x, None, rows, cols, act=mics.MICS_ACT_RELU, dtype=0, param_dtype=0)
    top = x[-3:].float().view(3, cols // 64, 64).abs().amax(2)
    assert torch.equal(y[-3:], x[-3:].clamp(min=0)) and torch.equal(scales.view(rows, -1)[-3:], top / torch.full_like(top, 127.0))
    mics.mics_checkpoint_read(y, codes, scales, rows, cols, act=mics.MICS_ACT_NONE, dtype=0)
    want = codes[-3:].float() * scales.view(rows, -1)[-3:].repeat_interleave(64, dim=1)
    assert torch.equal(y[-3:], want.to(torch.bfloat16))
    n = mics.mics_column_workspace_bytes(rows, cols)
    ws, db = torch.empty(n, dtype=torch.uint8, device=DEV), torch.empty(cols, device=DEV)
    mics.mics_activation_backward(y, db, x, None, codes, scales, rows, cols, act=mics.MICS_ACT_RELU, dtype=0, grad_dtype=2, workspace=ws,
                                  workspace_bytes=n)
    assert torch.equal(y[-3:], torch.where(codes[-3:] > 0, x[-3:], torch.zeros_like(x[-3:])))
    del y, codes
    # the product: x beyond 2^31 elements, its last rows against the same rows alone
    w = torch.randn(64, cols, device=DEV).to(torch.bfloat16)
    need = mics.mics_linear_workspace_bytes(rows, cols, 64)
    ws = torch.empty(max(need, mics.mics_linear_workspace_bytes(200, cols, 64)), dtype=torch.uint8, device=DEV)
    out = torch.empty(rows, 64, dtype=torch.bfloat16, device=DEV)
    mics.mics_linear(out, None, None, None, x, w, None, None, rows, cols, 64, act=0, dtype=0, param_dtype=0, workspace=ws, workspace_bytes=ws.numel())
    want = x[-200:].double() @ w.double().t()
    assert float((out[-200:].double() - want).norm() / want.norm()) < 2.0 ** -8
    dw = torch.empty(64, cols, device=DEV)
    dz = torch.zeros(rows, 64, dtype=torch.bfloat16, device=DEV)
    dz[-200:].normal_()                                          # all but the last rows are zeros
    mics.mics_linear_backward_weight(dw, dz, x, rows, cols, 64, dtype=0, grad_dtype=2, workspace=ws, workspace_bytes=ws.numel())
    want = dz[-200:].double().t() @ x[-200:].double()
    assert float((dw.double() - want).norm() / want.norm()) < 1e-5
