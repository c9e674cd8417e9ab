"""The sizes of the GPU test of products that write a checkpoint reach every kernel that does, as the rules cut them."""
from linear_shapes import WITH_CODES
from test_linear_rules import WIDTH, plan      # noqa: F401


def reached(plan, rows, cin, cout, pad, skew, fmt):             # noqa: F811
    w = WIDTH[fmt]
    on, chunks = (64 + skew) * w % 16 == 0 and (cin + pad) * w % 16 == 0, cin * w >= 16
    p = plan(rows, cout, cin, w, False, False, on, on, chunks, True)
    how = "few" if p["few"] else "guarded" if not chunks else "copy" if p["a_copy"] else "direct" if on else "through"
    return w, how, p["bm"], "whole" if p["splits"] == 1 else "mixed" if p["whole"] else "parts"


def test_sizes_with_codes_reach_every_kernel(plan):             # noqa: F811
    seen = {reached(plan, *s) for s in WITH_CODES}
    wanted = [(w, "few", bm, cut) for w in (2, 4) for bm in (16, 32) for cut in ("whole", "parts")]
    wanted += [(w, "guarded", 128, "whole") for w in (2, 4)]
    wanted += [(2, "direct", bm, cut) for bm in (128, 256) for cut in ("whole", "mixed")] + [(2, "direct", bm, "parts") for bm in (128, 256)]
    wanted += [(2, "through", bm, cut) for bm in (128, 256) for cut in ("whole", "parts")] + [(2, "copy", bm, "whole") for bm in (128, 256)]
    wanted += [(4, how, bm, cut) for how in ("direct", "through") for bm in (32, 64, 128) for cut in ("whole", "parts")]
    wanted += [(4, how, 64, "mixed") for how in ("direct", "through")] + [(4, "copy", 128, "whole")]
    assert not [x for x in wanted if x not in seen]
