"""What the order of a product's sums depends on: sizes, element type, strides and alignment, and up to 32 rows whether a checkpoint is
written.  On the CPU by the rule that cuts products; on the GPU by results that stay the same bit by bit while all else changes."""
import random

import numpy as np
import pytest
import torch

from test_linear_rules import plan      # noqa: F401

mics = pytest.importorskip("paper_2205_00119_amd")

DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
CODE = {"bf16": mics.MICS_DTYPE_BF16, "f32": mics.MICS_DTYPE_F32}


def test_a_checkpoint_changes_the_cut_of_few_rows_alone(plan):             # noqa: F811
    rng = random.Random(9)
    size = lambda: int(2 ** rng.uniform(0, 14.5))                                      # noqa: E731
    few = 0
    for _ in range(4000):
        m, n, k, width = size(), size(), size(), rng.choice([2, 4])
        a16, b16, chunks = (rng.random() < p for p in (0.6, 0.6, 0.9))
        with_codes, without = (plan(m, n, k, width, False, False, a16, b16, chunks, b) for b in (True, False))
        assert m <= 32 or with_codes == without, (m, n, k, width)
        few += with_codes != without
    assert few                                                   # which is why the header says so


def rows_of(data, fmt, shift):
    """On 16 bytes, `shift` of them behind the allocation's start."""
    t = torch.from_numpy(data).to(TORCH[fmt])
    whole = torch.empty(t.numel() + 64, dtype=t.dtype, device=DEV)
    at = shift * 16 // t.element_size()
    m = whole[at:at + t.numel()].view(t.shape)
    m.copy_(t)
    return m


@pytest.mark.gpu
@pytest.mark.parametrize("rows,cin,cout,fmt", [(1, 8192, 640, "bf16"), (20, 2048, 96, "f32"), (300, 1100, 650, "bf16"), (64, 4096, 512, "bf16"),
                                               (700, 2049, 1030, "bf16"), (200, 1030, 320, "f32")])
def test_nothing_else_changes_a_sum(rows, cin, cout, fmt):
    r = np.random.default_rng(cin)
    xd, wd, zd = r.normal(0, 1, (rows, cin)), r.normal(0, 1, (cout, cin)), r.normal(0, 1, (rows, cout))
    n = mics.mics_linear_workspace_bytes(rows, cin, cout)
    seen = {"pre": [], "dx": [], "dw": []}
    for i in range(3):                                           # addresses, workspaces, what is in them, the epilogue
        x, w, dz = (rows_of(d, fmt, i) for d in (xd, wd, zd))
        ws = torch.full((n + 64 * i + 8,), 255 - i, dtype=torch.uint8, device=DEV)
        work = dict(workspace=ws, workspace_bytes=ws.numel())
        out, pre = (torch.empty(rows, cout, dtype=TORCH[fmt], device=DEV) for _ in range(2))
        bias = torch.zeros(cout, dtype=TORCH["f32" if i == 1 else fmt], device=DEV) if i else None
        residual = torch.ones_like(out) if i == 2 else None
        keep = (None, None)
        if i == 2 and rows > 32:
            keep = (torch.empty(rows, cout, dtype=torch.int8, device=DEV), torch.empty(mics.mics_checkpoint_scales(rows, cout), device=DEV))
        mics.mics_linear(out, pre, *keep, x, w, bias, residual, rows, cin, cout, act=i, dtype=CODE[fmt],
                         param_dtype=CODE["f32" if i == 1 else fmt], **work)
        dx, dw = torch.empty_like(x), torch.empty(cout, cin, dtype=TORCH["f32" if i else fmt], device=DEV)
        mics.mics_linear_backward_input(dx, dz, w, torch.zeros_like(dx) if i else None, rows, cin, cout, dtype=CODE[fmt], **work)
        mics.mics_linear_backward_weight(dw, dz, x, rows, cin, cout, dtype=CODE[fmt], grad_dtype=CODE["f32" if i else fmt], **work)
        for name, t in (("pre", pre), ("dx", dx), ("dw", dw.to(TORCH[fmt]))):
            seen[name].append(t.clone())
    for name, (a, b, c) in seen.items():
        assert torch.equal(a, b) and torch.equal(a, c), name
