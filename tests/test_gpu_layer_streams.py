"""All eight layer operators on streams and in replayed graphs: every result is overwritten first, so that only what a call or a
replay writes itself can be right."""
import numpy as np
import pytest
import torch

from test_gpu_layer_ops import scratch

pytestmark = pytest.mark.gpu

mics = pytest.importorskip("paper_2205_00119_amd")

DEV = "cuda:0"


class Step:
    """Inputs, results and scratch of one call of each operator.  The sizes decide the launches: a second one for the columns'
    sums with many rows, one that joins the parts of few long rows of logits."""

    def __init__(self, rows=200, cols=1027, vocab=40000):
        r = np.random.default_rng(21)
        half = lambda *s: torch.from_numpy(r.normal(size=s)).to(torch.bfloat16).to(DEV)      # noqa: E731
        f = lambda *s: torch.zeros(*s, device=DEV)                                            # noqa: E731
        self.sizes = rows, cols, vocab
        self.x, self.res, self.dy, self.w, self.nb, self.bias = half(rows, cols), half(rows, cols), half(rows, cols), half(cols), half(cols), half(cols)
        few = 7                                                                               # rows of logits: several workgroups each
        self.few, self.logits, self.t = few, half(few, vocab), torch.from_numpy(r.integers(0, vocab, few)).to(DEV)
        like = lambda *names: {n: torch.empty_like(self.x) for n in names}                    # noqa: E731
        self.out = {**like("y", "dx", "o", "do", "by", "bs", "bdx", "bdr"), "dl": torch.empty_like(self.logits),
                    **{n: f(rows) for n in ("mean", "rstd", "bmean", "brstd")}, **{n: f(cols) for n in ("dw", "db", "dob", "bdb", "bdw", "bdn")},
                    **{n: f(few) for n in ("lp", "ent", "lse")}, "ids": torch.zeros(few, 5, dtype=torch.int64, device=DEV), "best": f(few, 5)}
        self.dlp, self.dent = f(few) - 1, f(few) + 0.5
        self.ws, self.n = scratch(rows, cols)
        self.ln = mics.mics_token_logprobs_workspace_bytes(few, vocab, 5)
        assert self.ln > 0
        self.lw = torch.zeros(self.ln, dtype=torch.uint8, device=DEV)

    def __call__(self, stream=None):
        (n, c, v), o, k = self.sizes, self.out, self.few
        t, key = dict(dtype=0, param_dtype=0, stream=stream), dict(drop=0.1, seed=5, offset=6)
        back = dict(grad_dtype=2, workspace=self.ws, workspace_bytes=self.n)
        mics.mics_layer_norm(o["y"], o["mean"], o["rstd"], self.x, self.w, self.nb, n, c, eps=1e-5, **t)
        mics.mics_layer_norm_backward(o["dx"], o["dw"], o["db"], self.dy, self.x, o["mean"], o["rstd"], self.w, n, c, **t, **back)
        mics.mics_bias_dropout_add(o["o"], self.x, self.bias, self.res, n, c, **key, **t)
        mics.mics_bias_dropout_add_backward(o["do"], o["dob"], self.dy, n, c, dtype=0, stream=stream, **key, **back)
        mics.mics_dropout_add_layer_norm(o["by"], o["bs"], o["bmean"], o["brstd"], self.x, self.bias, self.res, self.w, self.nb, n, c,
                                         eps=1e-5, **key, **t)
        mics.mics_dropout_add_layer_norm_backward(o["bdx"], o["bdr"], o["bdb"], o["bdw"], o["bdn"], self.dy, self.res, o["bs"], o["bmean"],
                                                  o["brstd"], self.w, n, c, **key, **t, **back)
        mics.mics_token_logprobs(o["lp"], o["ent"], o["lse"], o["ids"], o["best"], self.logits, self.t, k, v, dtype=0, top_k=5,
                                 workspace=self.lw, workspace_bytes=self.ln, stream=stream)
        mics.mics_token_logprobs_backward(o["dl"], self.logits, self.t, o["lse"], o["ent"], self.dlp, self.dent, k, v, dtype=0, stream=stream)

    def spoil(self):
        for x in self.out.values():
            x.fill_(float("nan") if x.is_floating_point() else -7)
        self.ws.fill_(0xFF)
        self.lw.fill_(0xFF)
        torch.cuda.synchronize()

    def results(self):
        torch.cuda.synchronize()
        return {n: x.clone() for n, x in self.out.items()}


def differing(got, want):
    return [n for n in want if not torch.equal(got[n], want[n])]


def test_spoilt_results_are_told_apart():
    """What the comparisons below rest on: no result holds what spoil() leaves."""
    s = Step()
    s()
    first = s.results()
    s.spoil()
    assert differing(s.results(), first) == list(first)
    assert all(bool(torch.isfinite(x).all()) for x in first.values())


def change(s, k):
    """Other inputs in the same places."""
    for x in (s.x, s.res, s.dy, s.logits):
        x.copy_(x.roll(k, 0) * (1.0 + 0.125 * k))
    s.t.add_(k).remainder_(s.sizes[2])


def test_replays_write_every_result_anew():
    s = Step()
    s()
    before = s.results()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s()
    for k in range(1, 5):
        change(s, k)
        s.spoil()
        s()
        want = s.results()
        assert differing(before, want) == list(want)             # the inputs did change, and every result with them
        s.spoil()
        graph.replay()
        assert not differing(s.results(), want), k
        before = want


@pytest.mark.parametrize("explicit", [True, False])
def test_calls_run_where_they_are_told_to(explicit):
    """Inputs are right on the side stream only, and only after a long piece of work there.  What is launched anywhere else reads
    zeros, or writes before results are spoilt."""
    s, side, other = Step(), torch.cuda.Stream(), torch.cuda.Stream()
    s()
    want = s.results()
    held = [x.clone() for x in (s.x, s.res, s.dy, s.logits)]
    big = torch.zeros(1 << 29, device=DEV)
    s.spoil()
    with torch.cuda.stream(side):
        for x in (s.x, s.res, s.dy, s.logits):
            x.zero_()
        side.synchronize()                                       # zeros are there before anything else starts
        for _ in range(32):
            big.add_(1.0)                                        # 2 GB each way: some 25 ms, the calls take one to queue
        for x, h in zip((s.x, s.res, s.dy, s.logits), held):
            x.copy_(h)
        if not explicit:
            s()                                                  # torch's current stream
    if explicit:
        with torch.cuda.stream(other):
            s(stream=side)
    side.synchronize()
    assert not differing(s.results(), want)
