"""Performance cases of a transformer layer's matrix products and of what is kept of them for the backward pass: the linear
layer with bias, activation and residual in its epilogue, the gradients of its input and of its weight, the activation that
leaves an 8-bit checkpoint of what it was applied to, and its gradient from that checkpoint.

A case is one pass as a training or scoring program makes it.  Hidden sizes are the repository's own (h = 2560, 4096, 5120,
8192, inner sizes 4h) and odd ones, tokens are micro-batches of 8 or 16 sequences of 512 and fewer, down to a single token.
`draw` spreads all of them over the whole range.
"""
import math

import torch

own = False

DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
WIDTH = {"bf16": 2, "f16": 2, "f32": 4}
ACTS = ("none", "relu", "gelu", "gelu_tanh", "silu")
BLOCK = 64                              # columns of a row that share a scale in a checkpoint
SMALLEST = 2.0 ** -100                  # a scale is not made from less than this
# scratch that a training program keeps for the calls: parts of a product that is split over its sum, and sums of columns
# over groups of rows
LINEAR_SCRATCH, COLUMN_PARTS, COLUMN_SUMS = 1 << 26, 256, 3


def listed():
    return [
        # scoring one token: the first product of the h = 2560 feed-forward, weights are read once
        dict(name="linear_1x2560x10240", op="linear", rows=1, cin=2560, cout=10240, pad=0, dtype="bf16", param="bf16",
             act="gelu", bias=True, residual=False, keep="no"),
        # 8 sequences of 512 through the h = 8192 feed-forward's first product; z is kept in 8 bits for the backward pass
        dict(name="linear_4096x8192x32768_keep8", op="linear", rows=4096, cin=8192, cout=32768, pad=0, dtype="bf16",
             param="bf16", act="gelu", bias=True, residual=False, keep="8"),
        # an output projection with its residual; binary16, odd sizes, rows that are slices of a wider buffer
        dict(name="linear_2047x5121x2561_f16", op="linear", rows=2047, cin=5121, cout=2561, pad=3, dtype="f16", param="f16",
             act="none", bias=True, residual=True, keep="no"),
        # the input's gradient of the h = 5120 feed-forward's second product, 8 sequences of 512
        dict(name="linear_input_4096x20480x5120", op="linear_input", rows=4096, cin=20480, cout=5120, pad=0, dtype="bf16",
             dsum=False),
        # a short micro-batch in plain float32, with a gradient that reaches the input as well
        dict(name="linear_input_37x4096x1000_f32", op="linear_input", rows=37, cin=4096, cout=1000, pad=0, dtype="f32",
             dsum=True),
        # the weight's gradient of the h = 4096 feed-forward's first product, 16 sequences of 512
        dict(name="linear_weight_8192x4096x16384", op="linear_weight", rows=8192, cin=4096, cout=16384, pad=0, dtype="bf16",
             grad="bf16"),
        # the same with odd sizes and gradients in 32 bits
        dict(name="linear_weight_1003x2563x1285", op="linear_weight", rows=1003, cin=2563, cout=1285, pad=0, dtype="bf16",
             grad="f32"),
        # a short micro-batch's activation and its checkpoint, read back as the next product's operand: latency counts
        dict(name="activation_8x10240", op="activation", rows=8, cols=10240, pad=0, dtype="bf16", param="bf16", act="gelu",
             bias=True, again="gelu"),
        # the h = 8192 feed-forward's, 8 sequences of 512
        dict(name="activation_4096x32768", op="activation", rows=4096, cols=32768, pad=0, dtype="bf16", param="bf16",
             act="gelu_tanh", bias=True, again="gelu_tanh"),
        # its gradient from the checkpoint, with the bias's
        dict(name="activation_backward_4096x32768", op="activation_backward", rows=4096, cols=32768, pad=0, dtype="bf16",
             grad="bf16", act="gelu_tanh", bias=True, keep="8"),
        # plain float32 training, odd sizes, padded rows
        dict(name="activation_backward_1003x5125_f32", op="activation_backward", rows=1003, cols=5125, pad=3, dtype="f32",
             grad="f32", act="gelu", bias=True, keep="8"),
    ]


MOST_FLOPS = 2 * 4096 * 8192 * 32768    # of a drawn case's pass, the largest listed one's
MOST_FLOPS_F32 = MOST_FLOPS // 8
MOST_ELEMENTS = 1 << 27                 # of a drawn matrix


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        case = _draw(rng)
        if case["op"].startswith("activation"):
            return case
        m, k, n = case["rows"], case["cin"], case["cout"]
        if max(m * k, m * n, n * k) <= MOST_ELEMENTS and \
           2 * m * k * n <= (MOST_FLOPS_F32 if case["dtype"] == "f32" else MOST_FLOPS):
            return case


def _draw(rng):
    op = rng.choice(["linear", "linear", "linear_input", "linear_weight", "activation", "activation_backward"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    pad = rng.choice([0, 0, 0, 8, 3])
    if op.startswith("activation"):
        cols = rng.choice([10240, 16384, 20480, 32768, _between(rng, 64, 32768), _between(rng, 64, 32768)])
        rows = _between(rng, 1, min(32768, MOST_ELEMENTS // cols))
        case = dict(op=op, rows=rows, cols=cols, pad=pad, dtype=dtype, act=rng.choice(ACTS), bias=rng.random() < 0.7)
        if op == "activation":
            case.update(param=rng.choice([dtype, dtype, "f32"]), again=rng.choice(["none", case["act"]]))
        else:
            case.update(grad=rng.choice([dtype, dtype, "f32"]), keep=rng.choice(["8", "8", "full"]))
        return case
    size = lambda: rng.choice([2560, 4096, 5120, 8192, 10240, 16384, _between(rng, 64, 16384), _between(rng, 64, 16384)])  # noqa: E731
    case = dict(op=op, rows=_between(rng, 1, 8192), cin=size(), cout=size(), pad=pad, dtype=dtype)
    if op == "linear":
        case.update(param=rng.choice([dtype, dtype, "f32"]), act=rng.choice(ACTS), bias=rng.random() < 0.75,
                    residual=rng.random() < 0.4, keep=rng.choice(["no", "no", "8", "full"]))
    elif op == "linear_input":
        case["dsum"] = rng.random() < 0.4
    else:
        case["grad"] = rng.choice([dtype, dtype, "f32"])
    return case


# ---- inputs ------------------------------------------------------------------------------------

def _rows(rows, cols, pad, dtype):
    """An uninitialised matrix, `pad` elements between its rows."""
    return torch.empty(rows, cols + pad, dtype=dtype, device=DEV)[:, :cols]


def _normal(gen, rows, cols, case, sigma, mean=0.0):
    m = _rows(rows, cols, case["pad"], TORCH[case["dtype"]])
    step = max(1, (1 << 26) // cols)
    for r in range(0, rows, step):
        part = m[r:r + step]
        part.copy_(torch.empty(part.shape, dtype=torch.float32, device=DEV).normal_(mean, sigma, generator=gen))
    return m


def _vector(gen, n, sigma, kind):
    return torch.empty(n, dtype=torch.float32, device=DEV).normal_(0.0, sigma, generator=gen).to(TORCH[kind])


def _blocks(cols):
    return -(-cols // BLOCK)


def _coded(z):
    """The checkpoint of a matrix in 32 bits: codes, scales."""
    rows, cols = z.shape
    n = _blocks(cols)
    wide = torch.nn.functional.pad(z, (0, n * BLOCK - cols)).view(rows, n, BLOCK)
    top = wide.abs().amax(2).clamp(min=SMALLEST)
    codes = torch.round(wide * (127.0 / top)[:, :, None]).to(torch.int8).view(rows, n * BLOCK)[:, :cols]
    return codes, top / 127.0


def _restored(codes, scales):
    rows, cols = codes.shape
    n = scales.shape[1]
    wide = torch.nn.functional.pad(codes, (0, n * BLOCK - cols)).view(rows, n, BLOCK)
    return (wide.float() * scales[:, :, None]).view(rows, n * BLOCK)[:, :cols]


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    op, rows, pad, t = case["op"], case["rows"], case["pad"], TORCH[case["dtype"]]
    st = {"case": case}
    if op.startswith("linear"):
        cin, cout = case["cin"], case["cout"]
        st["scratch"] = torch.empty(LINEAR_SCRATCH, dtype=torch.uint8, device=DEV)
        if op != "linear_weight":
            st["weight"] = _normal(gen, cout, cin, case, cin ** -0.5)
        if op == "linear":
            st["x"] = _normal(gen, rows, cin, case, 1.0)
            st["bias"] = _vector(gen, cout, 0.5, case["param"]) if case["bias"] else None
            st["residual"] = _normal(gen, rows, cout, case, 1.5) if case["residual"] else None
            st["out"] = _rows(rows, cout, pad, t)
            full, eight = case["keep"] == "full", case["keep"] == "8"
            st["pre"] = _rows(rows, cout, pad, t) if full else None
            st["codes"] = _rows(rows, cout, pad, torch.int8) if eight else None
            st["scales"] = torch.empty(rows, _blocks(cout), dtype=torch.float32, device=DEV) if eight else None
            st["z"] = _rows(rows, cout, pad, t) if eight else None
        else:
            st["dz"] = _normal(gen, rows, cout, case, 0.1)
            if op == "linear_input":
                st["dsum"] = _normal(gen, rows, cin, case, 0.1) if case["dsum"] else None
                st["dx"] = _rows(rows, cin, pad, t)
            else:
                st["x"] = _normal(gen, rows, cin, case, 1.0)
                st["dweight"] = _rows(cout, cin, pad, TORCH[case["grad"]])
        return st
    cols = case["cols"]
    # activations have a few columns that are far larger than the others
    x = _normal(gen, rows, cols, case, 1.0)
    x *= torch.where(torch.rand(cols, generator=gen, device=DEV) < 0.01, 12.0, 1.0).to(t)
    if op == "activation":
        st.update(x=x, bias=_vector(gen, cols, 0.5, case["param"]) if case["bias"] else None, y=_rows(rows, cols, pad, t),
                  codes=_rows(rows, cols, pad, torch.int8), again=_rows(rows, cols, pad, t),
                  scales=torch.empty(rows, _blocks(cols), dtype=torch.float32, device=DEV))
        return st
    st.update(dy=_normal(gen, rows, cols, case, 0.1), dx=_rows(rows, cols, pad, t), z=None, codes=None, scales=None,
              dbias=torch.empty(cols, dtype=TORCH[case["grad"]], device=DEV) if case["bias"] else None,
              scratch=torch.empty(4 * COLUMN_PARTS * COLUMN_SUMS * cols + 8 * rows, dtype=torch.uint8, device=DEV))
    if case["keep"] == "8":                 # what the forward pass left
        codes, st["scales"] = _coded(x.float())
        st["codes"] = _rows(rows, cols, pad, torch.int8).copy_(codes)
    else:
        st["z"] = x
    return st


# ---- one pass ----------------------------------------------------------------------------------

def run(st):
    return (_own if own else _plain)(st, st["case"])


def _own(st, case):
    import paper_2205_00119_amd as mics
    code = {"bf16": mics.MICS_DTYPE_BF16, "f16": mics.MICS_DTYPE_F16, "f32": mics.MICS_DTYPE_F32}
    acts = {"none": mics.MICS_ACT_NONE, "relu": mics.MICS_ACT_RELU, "gelu": mics.MICS_ACT_GELU,
            "gelu_tanh": mics.MICS_ACT_GELU_TANH, "silu": mics.MICS_ACT_SILU}
    op, rows, pad, dtype = case["op"], case["rows"], case["pad"], code[case["dtype"]]
    if op.startswith("linear"):
        i, o = case["cin"], case["cout"]
        si, so = i + pad, o + pad
        scratch = dict(workspace=st["scratch"], workspace_bytes=LINEAR_SCRATCH)
        if op == "linear_input":
            mics.mics_linear_backward_input(st["dx"], st["dz"], st["weight"], st["dsum"], rows, i, o, dtype=dtype,
                                            strides=(si, so, si, si), **scratch)
            return [st["dx"]]
        if op == "linear_weight":
            mics.mics_linear_backward_weight(st["dweight"], st["dz"], st["x"], rows, i, o, dtype=dtype,
                                             grad_dtype=code[case["grad"]], strides=(si, so, si), **scratch)
            return [st["dweight"]]
        mics.mics_linear(st["out"], st["pre"], st["codes"], st["scales"], st["x"], st["weight"], st["bias"], st["residual"],
                         rows, i, o, act=acts[case["act"]], dtype=dtype, param_dtype=code[case["param"]],
                         strides=(so, so, so, si, si, so), **scratch)
        if case["keep"] == "8":
            mics.mics_checkpoint_read(st["z"], st["codes"], st["scales"], rows, o, act=mics.MICS_ACT_NONE, dtype=dtype,
                                      strides=(so, so))
        return [st["out"], {"no": None, "8": st["z"], "full": st["pre"]}[case["keep"]]]
    cols = case["cols"]
    s = cols + pad
    if op == "activation":
        mics.mics_activation(st["y"], st["codes"], st["scales"], st["x"], st["bias"], rows, cols, act=acts[case["act"]],
                             dtype=dtype, param_dtype=code[case["param"]], strides=(s, s, s))
        mics.mics_checkpoint_read(st["again"], st["codes"], st["scales"], rows, cols, act=acts[case["again"]], dtype=dtype,
                                  strides=(s, s))
        return [st["y"], st["again"]]
    mics.mics_activation_backward(st["dx"], st["dbias"], st["dy"], st["z"], st["codes"], st["scales"], rows, cols,
                                  act=acts[case["act"]], dtype=dtype, grad_dtype=code[case["grad"]], strides=(s, s, s, s),
                                  workspace=st["scratch"], workspace_bytes=st["scratch"].numel())
    return [st["dx"], st["dbias"]]


def _tanh_part(z):
    return math.sqrt(2.0 / math.pi) * (z + 0.044715 * z * z * z)


def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1.0 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return z / (1.0 + torch.exp(-2.0 * _tanh_part(z)))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "gelu_tanh":
        s = 1.0 / (1.0 + torch.exp(-2.0 * _tanh_part(z)))
        return s + z * s * (1.0 - s) * (2.0 * math.sqrt(2.0 / math.pi)) * (1.0 + 3 * 0.044715 * z * z)
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return s * (1.0 + z * (1.0 - s))
    return torch.ones_like(z)


def _plain(st, case):
    op, t = case["op"], TORCH[case["dtype"]]
    if op == "linear_input":
        dx = st["dz"].float() @ st["weight"].float()
        return [(dx + st["dsum"].float() if case["dsum"] else dx).to(t)]
    if op == "linear_weight":
        return [(st["dz"].float().t() @ st["x"].float()).to(TORCH[case["grad"]])]
    if op == "linear":
        z = st["x"].float() @ st["weight"].float().t()
        if case["bias"]:
            z = z + st["bias"].float()
        y = _act(z, case["act"])
        if case["residual"]:
            y = st["residual"].float() + y
        kept = None
        if case["keep"] == "8":
            kept = _restored(*_coded(z)).to(t)
        elif case["keep"] == "full":
            kept = z.to(t)
        return [y.to(t), kept]
    if op == "activation":
        z = st["x"].float()
        if case["bias"]:
            z = z + st["bias"].float()
        return [_act(z, case["act"]).to(t), _act(_restored(*_coded(z)), case["again"]).to(t)]
    z = _restored(st["codes"], st["scales"]) if case["keep"] == "8" else st["z"].float()
    dx = st["dy"].float() * _slope(z, case["act"])
    return [dx.to(t), dx.sum(0).to(TORCH[case["grad"]]) if case["bias"] else None]


# ---- what a pass cannot do without ---------------------------------------------------------------

def work(case):
    op, m, e = case["op"], case["rows"], WIDTH[case["dtype"]]
    if op.startswith("linear"):
        i, o = case["cin"], case["cout"]
        if op == "linear_weight":
            nbytes = e * (m * i + m * o) + WIDTH[case["grad"]] * i * o
        elif op == "linear_input":
            nbytes = e * (m * i * (1 + case["dsum"]) + m * o + i * o)
        else:
            nbytes = e * (m * i + i * o + m * o * (1 + case["residual"])) + (WIDTH[case["param"]] * o if case["bias"] else 0)
            if case["keep"] == "full":
                nbytes += e * m * o
            elif case["keep"] == "8":       # written, read, and what it stands for written
                nbytes += m * (2 * (o + 4 * _blocks(o)) + e * o)
        return {"bytes": nbytes, "flops": 2 * m * i * o}
    n = case["cols"]
    kept = n + 4 * _blocks(n)
    if op == "activation":
        return {"bytes": m * (3 * e * n + 2 * kept) + (WIDTH[case["param"]] * n if case["bias"] else 0), "flops": 30 * m * n}
    nbytes = m * (2 * e * n + (kept if case["keep"] == "8" else e * n)) + (WIDTH[case["grad"]] * n if case["bias"] else 0)
    return {"bytes": nbytes, "flops": 20 * m * n}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _normal_cdf(z):
    return torch.special.ndtr(z)


def _act64(z, act):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0), "gelu": lambda: z * _normal_cdf(z),
            "gelu_tanh": lambda: z * torch.sigmoid(2 * (2 / math.pi) ** 0.5 * (z + 0.044715 * z ** 3)),
            "silu": lambda: z * torch.sigmoid(z)}[act]()


def _slope64(z, act):
    if act == "gelu":
        return _normal_cdf(z) + z * torch.exp(-z * z / 2) / (2 * math.pi) ** 0.5
    if act == "gelu_tanh":
        c = (2 / math.pi) ** 0.5
        th = torch.tanh(c * (z + 0.044715 * z ** 3))
        return (1 + th) / 2 + z / 2 * (1 - th * th) * c * (1 + 0.134145 * z * z)
    if act == "silu":
        s = torch.sigmoid(z)
        return s + z * s * torch.sigmoid(-z)
    return (z > 0).double() if act == "relu" else torch.ones_like(z)


def _kept64(z, case):
    """What a checkpoint of z stands for: the nearest of 255 equally spaced values up to its block's largest."""
    rows, cols = z.shape
    n = (cols + 63) // 64
    full = z.new_zeros(rows, n * 64)
    full[:, :cols] = z
    full = full.reshape(rows * n, 64)
    step = full.abs().max(dim=1, keepdim=True).values.clamp(min=SMALLEST) / 127
    return (torch.round(full / step) * step).reshape(rows, n * 64)[:, :cols]


def exact(case, seed):
    st = prepare(case, seed)
    op = case["op"]
    if op == "linear_input":
        d = torch.mm(st["dz"].double(), st["weight"].double())
        return [d + st["dsum"].double() if case["dsum"] else d]
    if op == "linear_weight":
        return [torch.mm(st["dz"].double().t(), st["x"].double())]
    if op == "linear":
        z = torch.mm(st["x"].double(), st["weight"].double().t())
        if case["bias"]:
            z += st["bias"].double()
        y = _act64(z, case["act"])
        if case["residual"]:
            y = y + st["residual"].double()
        return [y, {"no": lambda: None, "8": lambda: _kept64(z, case), "full": lambda: z}[case["keep"]]()]
    if op == "activation":
        z = st["x"].double()
        if case["bias"]:
            z = z + st["bias"].double()
        return [_act64(z, case["act"]), _act64(_kept64(z, case), case["again"])]
    if case["keep"] == "8":
        z = st["codes"].double() * st["scales"].double().repeat_interleave(64, dim=1)[:, :case["cols"]]
    else:
        z = st["z"].double()
    d = st["dy"].double() * _slope64(z, case["act"])
    return [d, d.sum(dim=0) if case["bias"] else None]
