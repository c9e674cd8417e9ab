"""Performance cases of the operators that a transformer layer's training step runs between the
parameter gather and the gradient reduction: layer norm, dropout with bias and residual, both in one
pass, and the log probabilities of given tokens; each forward and backward.

A case is one call as a training or scoring program makes it.  Hidden sizes are the repository's own
(h = 2560, 4096, 5120, 8192) and odd ones, tokens are micro-batches of 8 or 16 sequences of 512 and
fewer, vocabularies are generic.  `draw` spreads all of them over the whole range.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
TORCH = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
WIDTH = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-5
# scratch that a training program keeps for the calls: sums of three gradients over up to 512 groups
# of rows, and the parts of rows that are scored by several workgroups
COLUMN_PARTS, COLUMN_SUMS = 512, 3
ROW_PARTS_BYTES = 1 << 20


def listed():
    return [
        # a short micro-batch's norm, forward only: latency counts
        dict(name="norm_8x2560", op="norm", rows=8, cols=2560, pad=0, dtype="bf16", param="bf16"),
        # 16 sequences of 512 through the norm of the h = 8192 layer
        dict(name="norm_8192x8192", op="norm", rows=8192, cols=8192, pad=0, dtype="bf16", param="bf16"),
        # its backward pass on 8 sequences of 512 of the h = 4096 layer
        dict(name="norm_backward_4096x4096", op="norm_backward", rows=4096, cols=4096, pad=0, dtype="bf16",
             param="bf16", grad="bf16"),
        # plain float32 training, odd sizes, rows that are slices of a wider buffer
        dict(name="norm_backward_1003x5125_f32", op="norm_backward", rows=1003, cols=5125, pad=3, dtype="f32",
             param="f32", grad="f32"),
        # an attention output's bias, dropout and residual, 8 sequences of 512, h = 8192
        dict(name="dropout_4096x8192", op="dropout", rows=4096, cols=8192, pad=0, dtype="bf16", param="bf16",
             drop=0.1, bias=True, residual=True),
        # its backward pass with the bias's gradient; binary16 training, odd width
        dict(name="dropout_backward_2047x5121_f16", op="dropout_backward", rows=2047, cols=5121, pad=0, dtype="f16",
             param="f16", grad="f16", drop=0.1, bias=True),
        # the whole epilogue of a sublayer in one pass, 8 sequences of 512, h = 5120
        dict(name="block_4096x5120", op="block", rows=4096, cols=5120, pad=0, dtype="bf16", param="bf16", drop=0.1),
        # its backward pass, h = 8192, with a gradient that reaches the sum as well
        dict(name="block_backward_4096x8192", op="block_backward", rows=4096, cols=8192, pad=0, dtype="bf16",
             param="bf16", grad="bf16", drop=0.1, dsum=True),
        # scoring one new token of four sequences with the eight best alternatives
        dict(name="logprobs_4x131072_top8", op="logprobs", rows=4, cols=131072, pad=0, dtype="bf16", top=8,
             given=1.0, masked=0.3),
        # the loss of 8 sequences of 512, with entropy
        dict(name="logprobs_4096x65536", op="logprobs", rows=4096, cols=65536, pad=0, dtype="bf16", top=0,
             given=1.0, masked=0.0),
        # evaluation with alternatives, float32 logits, an odd vocabulary
        dict(name="logprobs_500x50001_f32_top5", op="logprobs", rows=500, cols=50001, pad=0, dtype="f32", top=5,
             given=1.0, masked=0.0),
        # the loss's gradient of 8 sequences of 512, some of whose tokens are padding
        dict(name="logprobs_backward_4096x65536", op="logprobs_backward", rows=4096, cols=65536, pad=0, dtype="bf16",
             given=0.9, entropy=True),
    ]


MOST_HIDDEN = 1 << 26                   # elements of a drawn activation
MOST_LOGITS = 1 << 28                   # of drawn logits
MOST_BYTES = 1.07e9                     # of a drawn case's pass, the largest listed one's


def _between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        case = _draw(rng)
        if work(case)["bytes"] <= MOST_BYTES:
            return case


def _draw(rng):
    op = rng.choice(["norm", "norm_backward", "dropout", "dropout_backward", "block", "block_backward", "logprobs",
                     "logprobs_backward"])
    dtype = rng.choice(["bf16", "bf16", "f16", "f32"])
    if op.startswith("logprobs"):
        cols = _between(rng, 1000, 200000)
        rows = _between(rng, 1, max(1, min(8192, MOST_LOGITS // cols)))
        case = dict(op=op, rows=rows, cols=cols, pad=rng.choice([0, 0, 0, 7]), dtype=dtype,
                    given=rng.choice([1.0, 0.9, 0.15]))
        if op == "logprobs":
            case.update(top=rng.choice([0, 0, 1, 5, 20, 50]), masked=rng.choice([0.0, 0.0, 0.5, 0.999]))
        else:
            case["entropy"] = rng.random() < 0.5
        return case
    cols = rng.choice([2560, 4096, 5120, 8192, _between(rng, 64, 16384), _between(rng, 64, 16384)])
    rows = _between(rng, 1, max(1, min(32768, MOST_HIDDEN // cols)))
    case = dict(op=op, rows=rows, cols=cols, pad=rng.choice([0, 0, 0, 8, 3]), dtype=dtype,
                param=rng.choice([dtype, dtype, "f32"]))
    if op.endswith("backward"):
        case["grad"] = rng.choice([dtype, dtype, "f32"])
    if "norm" not in op:
        case["drop"] = rng.choice([0.1, 0.1, 0.0, round(rng.uniform(0.0, 0.9), 3)])
    if op.startswith("dropout"):
        case["bias"] = rng.random() < 0.75
    if op == "dropout":
        case["residual"] = rng.random() < 0.75
    if op == "block_backward":
        case["dsum"] = rng.random() < 0.5
    return case


# ---- inputs ------------------------------------------------------------------------------------

def _rows(case):
    """An uninitialised matrix of the case, `pad` elements between its rows."""
    buf = torch.empty(case["rows"], case["cols"] + case["pad"], dtype=TORCH[case["dtype"]], device=DEV)
    return buf[:, :case["cols"]]


def _normal(gen, case, sigma, mean=0.0):
    m = _rows(case)
    return m.copy_(torch.empty(m.shape, dtype=torch.float32, device=DEV).normal_(mean, sigma, generator=gen))


def _vector(gen, case, sigma, mean=0.0):
    v = torch.empty(case["cols"], dtype=torch.float32, device=DEV).normal_(mean, sigma, generator=gen)
    return v.to(TORCH[case["param"]])


def _out(case, names, of):
    return {n: torch.empty(of, dtype=TORCH[case["grad"]], device=DEV) for n in names}


def _stats(x):
    """Mean and reciprocal deviation of every row, which the forward pass left behind."""
    x = x.double()
    mean = x.mean(1)
    return mean.float(), (1.0 / torch.sqrt((x - mean[:, None]).square().mean(1) + EPS)).float()


def prepare(case, seed):
    gen = torch.Generator(device=DEV).manual_seed(seed)
    op, rows, cols = case["op"], case["rows"], case["cols"]
    st = {"case": case}
    f32 = dict(dtype=torch.float32, device=DEV)
    if op.startswith("logprobs"):
        st["logits"] = x = _normal(gen, case, 3.0)
        if case.get("masked"):          # tokens that a grammar or a sampler has ruled out
            x.masked_fill_(torch.rand(x.shape, generator=gen, **f32) < case["masked"], float("-inf"))
        t = torch.randint(0, cols, (rows,), generator=gen, device=DEV)
        if case.get("masked"):          # the given token is always allowed
            x.scatter_(1, t[:, None], torch.zeros((), dtype=x.dtype, device=DEV).expand(rows, 1))
        st["targets"] = torch.where(torch.rand(rows, generator=gen, **f32) < case["given"], t, torch.full_like(t, -1))
        if op == "logprobs":
            for n in ("logprob", "entropy", "lse"):
                st[n] = torch.empty(rows, **f32)
            st["top_ids"] = torch.empty(rows, case["top"], dtype=torch.int64, device=DEV)
            st["top_logprobs"] = torch.empty(rows, case["top"], **f32)
            st["scratch"] = torch.empty(ROW_PARTS_BYTES, dtype=torch.uint8, device=DEV)
        else:
            wide = x.double()
            lse = torch.logsumexp(wide, 1)
            logp = wide - lse[:, None]
            st["lse"], st["entropy"] = lse.float(), -(logp.exp() * logp).sum(1).float()
            del wide, logp
            given = (st["targets"] >= 0).float()
            st["dlogprob"] = -given / given.sum().clamp(min=1.0)
            st["dentropy"] = -0.01 * given / given.sum().clamp(min=1.0) if case["entropy"] else None
            st["dlogits"] = _rows(case)
        return st
    if op.endswith("backward"):
        st["scratch"] = torch.empty(COLUMN_PARTS * COLUMN_SUMS * cols * 4, dtype=torch.uint8, device=DEV)
    st["seed"], st["offset"] = 0x9E3779B97F4A7C15 ^ seed, 1 << 33
    if op == "norm":
        st.update(x=_normal(gen, case, 1.5, 0.25), weight=_vector(gen, case, 0.1, 1.0), bias=_vector(gen, case, 0.1),
                  y=_rows(case), mean=torch.empty(rows, **f32), rstd=torch.empty(rows, **f32))
    elif op == "norm_backward":
        st.update(dy=_normal(gen, case, 0.1), x=_normal(gen, case, 1.5, 0.25), weight=_vector(gen, case, 0.1, 1.0),
                  dx=_rows(case), **_out(case, ("dweight", "dbias"), cols))
        st["mean"], st["rstd"] = _stats(st["x"])
    elif op == "dropout":
        st.update(x=_normal(gen, case, 1.0), bias=_vector(gen, case, 0.1) if case["bias"] else None,
                  residual=_normal(gen, case, 1.5) if case["residual"] else None, out=_rows(case))
    elif op == "dropout_backward":
        st.update(dout=_normal(gen, case, 0.1), dx=_rows(case))
        st["dbias"] = _out(case, ("dbias",), cols)["dbias"] if case["bias"] else None
    elif op == "block":
        st.update(x=_normal(gen, case, 1.0), bias=_vector(gen, case, 0.1), residual=_normal(gen, case, 1.5),
                  weight=_vector(gen, case, 0.1, 1.0), norm_bias=_vector(gen, case, 0.1), y=_rows(case), sum=_rows(case),
                  mean=torch.empty(rows, **f32), rstd=torch.empty(rows, **f32))
    else:
        st.update(dy=_normal(gen, case, 0.1), dsum=_normal(gen, case, 0.1) if case["dsum"] else None,
                  sum=_normal(gen, case, 1.5, 0.25), weight=_vector(gen, case, 0.1, 1.0), dx=_rows(case),
                  dresidual=_rows(case), **_out(case, ("dbias", "dweight", "dnorm_bias"), cols))
        st["mean"], st["rstd"] = _stats(st["sum"])
    return st


# ---- one pass ----------------------------------------------------------------------------------

def run(st):
    return (_own if own else _plain)(st, st["case"])


def _own(st, case):
    import paper_2205_00119_amd as mics
    code = {"bf16": mics.MICS_DTYPE_BF16, "f16": mics.MICS_DTYPE_F16, "f32": mics.MICS_DTYPE_F32}
    op, rows, cols, dtype = case["op"], case["rows"], case["cols"], code[case["dtype"]]
    stride = cols + case["pad"]
    if op == "logprobs":
        mics.mics_token_logprobs(st["logprob"], st["entropy"], st["lse"], st["top_ids"], st["top_logprobs"], st["logits"],
                                 st["targets"], rows, cols, top_k=case["top"], dtype=dtype, stride=stride,
                                 workspace=st["scratch"], workspace_bytes=ROW_PARTS_BYTES)
        return [st[n] for n in ("logprob", "entropy", "lse", "top_ids", "top_logprobs")]
    if op == "logprobs_backward":
        mics.mics_token_logprobs_backward(st["dlogits"], st["logits"], st["targets"], st["lse"], st["entropy"],
                                          st["dlogprob"], st["dentropy"], rows, cols, dtype=dtype, strides=(stride, stride))
        return [st["dlogits"]]
    param = code[case["param"]]
    if op == "norm":
        mics.mics_layer_norm(st["y"], st["mean"], st["rstd"], st["x"], st["weight"], st["bias"], rows, cols, eps=EPS,
                             dtype=dtype, param_dtype=param, strides=(stride,) * 2)
        return [st["y"], st["mean"], st["rstd"]]
    if op == "dropout":
        mics.mics_bias_dropout_add(st["out"], st["x"], st["bias"], st["residual"], rows, cols, drop=case["drop"],
                                   seed=st["seed"], offset=st["offset"], dtype=dtype, param_dtype=param,
                                   strides=(stride,) * 3)
        return [st["out"]]
    if op == "block":
        mics.mics_dropout_add_layer_norm(st["y"], st["sum"], st["mean"], st["rstd"], st["x"], st["bias"], st["residual"],
                                         st["weight"], st["norm_bias"], rows, cols, drop=case["drop"], seed=st["seed"],
                                         offset=st["offset"], eps=EPS, dtype=dtype, param_dtype=param,
                                         strides=(stride,) * 4)
        return [st["y"], st["sum"], st["mean"], st["rstd"]]
    grad, scratch = code[case["grad"]], dict(workspace=st["scratch"], workspace_bytes=st["scratch"].numel())
    if op == "norm_backward":
        mics.mics_layer_norm_backward(st["dx"], st["dweight"], st["dbias"], st["dy"], st["x"], st["mean"], st["rstd"],
                                      st["weight"], rows, cols, dtype=dtype, param_dtype=param, grad_dtype=grad,
                                      strides=(stride,) * 3, **scratch)
        return [st["dx"], st["dweight"], st["dbias"]]
    if op == "dropout_backward":
        mics.mics_bias_dropout_add_backward(st["dx"], st["dbias"], st["dout"], rows, cols, drop=case["drop"],
                                            seed=st["seed"], offset=st["offset"], dtype=dtype, grad_dtype=grad,
                                            strides=(stride,) * 2, **scratch)
        return [st["dx"], st["dbias"]]
    mics.mics_dropout_add_layer_norm_backward(
        st["dx"], st["dresidual"], st["dbias"], st["dweight"], st["dnorm_bias"], st["dy"], st["dsum"], st["sum"],
        st["mean"], st["rstd"], st["weight"], rows, cols, drop=case["drop"], seed=st["seed"], offset=st["offset"],
        dtype=dtype, param_dtype=param, grad_dtype=grad, strides=(stride,) * 5, **scratch)
    return [st[n] for n in ("dx", "dresidual", "dbias", "dweight", "dnorm_bias")]


def _mul_wide(a, m):
    """High and low 32 bits of the product of 32-bit numbers, in 64-bit integers without their sign."""
    low, high = a * (m & 0xFFFF), a * (m >> 16)
    mid = (low >> 16) + (high & 0xFFFF)
    return (high >> 16) + (mid >> 16), ((mid & 0xFFFF) << 16) | (low & 0xFFFF)


def _round(c, k0, k1):
    """One round of Philox4x32 (Salmon, Moraes, Dror, Shaw 2011)."""
    h0, l0 = _mul_wide(c[0], 0xD2511F53)
    h1, l1 = _mul_wide(c[2], 0xCD9E8D57)
    return h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0


def _kept(case, seed, offset):
    """Which elements dropout keeps: column c of row r takes the 16-bit number c mod 8 of the generator's block
    offset + r * ceil(cols / 8) + c div 8 and stays where that is at least rint(65536 drop)."""
    groups = -(-case["cols"] // 8)
    n = torch.arange(case["rows"] * groups, dtype=torch.int64, device=DEV) + offset
    c = (n & 0xFFFFFFFF, (n >> 32) & 0xFFFFFFFF, torch.zeros_like(n), torch.zeros_like(n))
    k0, k1 = seed & 0xFFFFFFFF, seed >> 32
    for _ in range(10):
        c = _round(c, k0, k1)
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    words = torch.stack(c, 1)
    halves = torch.stack((words & 0xFFFF, words >> 16), 2).reshape(case["rows"], groups * 8)[:, :case["cols"]]
    return halves >= _threshold(case["drop"])


def _threshold(drop):
    return min(65535, round(65536 * drop))


def _dropped(v, case, st):
    t = _threshold(case["drop"])
    if t == 0:
        return v
    return torch.where(_kept(case, st["seed"], st["offset"]), v * (65536.0 / (65536.0 - t)), torch.zeros_like(v))


def _norm(x):
    """Normalised rows, mean, reciprocal deviation."""
    n = x.shape[1]
    mean = x.sum(1) / n
    d = x - mean[:, None]
    rstd = 1.0 / torch.sqrt((d * d).sum(1) / n + EPS)
    return d * rstd[:, None], mean, rstd


def _norm_gradient(dy, x, st):
    """Gradients of the rows, of the weight and of the bias."""
    n, rstd = x.shape[1], st["rstd"][:, None]
    hat = (x - st["mean"][:, None]) * rstd
    d = dy * st["weight"].float()
    dx = rstd * (d - d.sum(1, keepdim=True) / n - hat * ((d * hat).sum(1, keepdim=True) / n))
    return dx, (dy * hat).sum(0), dy.sum(0)


def _best(x, k):
    """The k largest of every row, the lowest index first among equals."""
    x, ids = x.clone(), []
    rest = torch.ones_like(x, dtype=torch.bool)
    at = torch.arange(x.shape[1], device=x.device)
    for _ in range(k):
        most = torch.where(rest, x, float("-inf")).amax(1, keepdim=True)
        i = torch.where(rest & (x == most), at, x.shape[1]).amin(1, keepdim=True)
        rest.scatter_(1, i, False)
        ids.append(i)
    return torch.cat(ids, 1)


def _plain(st, case):
    op, t = case["op"], TORCH[case["dtype"]]
    if op == "logprobs":
        x = st["logits"].float()
        most = x.amax(1, keepdim=True)
        d = x - most
        e = torch.exp(d)
        total = e.sum(1)
        lse = most[:, 0] + torch.log(total)
        entropy = torch.log(total) - torch.where(e > 0, d * e, torch.zeros_like(e)).sum(1) / total
        given = st["targets"] >= 0
        of = x.gather(1, st["targets"].clamp(min=0)[:, None])[:, 0] - lse
        out = [torch.where(given, of, torch.zeros_like(of)), entropy, lse]
        if not case["top"]:
            return out + [st["top_ids"], st["top_logprobs"]]
        ids = _best(x, case["top"])
        return out + [ids, x.gather(1, ids) - lse[:, None]]
    if op == "logprobs_backward":
        logp = st["logits"].float() - st["lse"][:, None]
        p = torch.exp(logp)
        d = -st["dlogprob"][:, None] * p
        if st["dentropy"] is not None:
            d = d - st["dentropy"][:, None] * p * (logp + st["entropy"][:, None])
        given = st["targets"] >= 0
        d.scatter_add_(1, st["targets"].clamp(min=0)[:, None], torch.where(given, st["dlogprob"], 0.0)[:, None])
        return [d.to(t)]
    if op == "norm":
        hat, mean, rstd = _norm(st["x"].float())
        return [(hat * st["weight"].float() + st["bias"].float()).to(t), mean, rstd]
    if op == "dropout":
        v = st["x"].float()
        if case["bias"]:
            v = v + st["bias"].float()
        v = _dropped(v, case, st)
        return [(v + st["residual"].float() if case["residual"] else v).to(t)]
    if op == "block":
        s = st["residual"].float() + _dropped(st["x"].float() + st["bias"].float(), case, st)
        hat, mean, rstd = _norm(s)
        return [(hat * st["weight"].float() + st["norm_bias"].float()).to(t), s.to(t), mean, rstd]
    g = TORCH[case["grad"]]
    if op == "norm_backward":
        dx, dw, db = _norm_gradient(st["dy"].float(), st["x"].float(), st)
        return [dx.to(t), dw.to(g), db.to(g)]
    if op == "dropout_backward":
        d = _dropped(st["dout"].float(), case, st)
        return [d.to(t), d.sum(0).to(g) if case["bias"] else None]
    ds, dw, db = _norm_gradient(st["dy"].float(), st["sum"].float(), st)
    if case["dsum"]:
        ds = ds + st["dsum"].float()
    d = _dropped(ds, case, st)
    return [d.to(t), ds.to(t), d.sum(0).to(g), dw.to(g), db.to(g)]


# ---- what a pass cannot do without ---------------------------------------------------------------

# matrices read and written, and operations on an element, by operator
TRAFFIC = {"norm": (2, 8), "norm_backward": (3, 14), "dropout": (2, 4), "dropout_backward": (2, 3), "block": (4, 12),
           "block_backward": (4, 18), "logprobs": (1, 6), "logprobs_backward": (2, 6)}


def work(case):
    op, rows, cols = case["op"], case["rows"], case["cols"]
    n, ops = TRAFFIC[op]
    n += bool(case.get("residual")) + bool(case.get("dsum"))
    nbytes = n * rows * cols * WIDTH[case["dtype"]]
    if op == "logprobs":
        nbytes += rows * (8 + 12 + 12 * case["top"])
    elif op == "logprobs_backward":
        nbytes += rows * (8 + 16 + 4 * case["entropy"])
    else:
        vectors = {"norm": 2, "norm_backward": 1, "dropout": int(case.get("bias", False)), "dropout_backward": 0, "block": 3,
                   "block_backward": 1}[op]
        grads = {"norm_backward": 2, "dropout_backward": int(case.get("bias", False)), "block_backward": 3}.get(op, 0)
        nbytes += cols * (vectors * WIDTH[case["param"]] + (grads * WIDTH[case["grad"]] if grads else 0))
        nbytes += 0 if op.startswith("dropout") else 8 * rows
    return {"bytes": nbytes, "flops": ops * rows * cols}


# ---- the definitions in 64 bits ------------------------------------------------------------------

def _mask64(case, seed, offset):
    """1 where an element is kept, from the generator's definition on unsigned 64-bit integers."""
    groups = (case["cols"] + 7) // 8
    block = np.arange(case["rows"] * groups, dtype=np.uint64) + np.uint64(offset)
    low, s32 = np.uint64(0xFFFFFFFF), np.uint64(32)
    x0, x1 = block & low, block >> s32
    x2, x3 = np.zeros_like(x0), np.zeros_like(x0)
    keys = (seed & 0xFFFFFFFF, seed >> 32)
    for i in range(10):
        a, b = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
        ka, kb = ((keys[0] + i * 0x9E3779B9) & 0xFFFFFFFF, (keys[1] + i * 0xBB67AE85) & 0xFFFFFFFF)
        x0, x1, x2, x3 = (b >> s32) ^ x1 ^ np.uint64(ka), b & low, (a >> s32) ^ x3 ^ np.uint64(kb), a & low
    u = np.empty((case["rows"] * groups, 8), dtype=np.int32)
    for w, word in enumerate((x0, x1, x2, x3)):
        u[:, 2 * w] = word & np.uint64(0xFFFF)
        u[:, 2 * w + 1] = word >> np.uint64(16)
    u = torch.from_numpy(u.reshape(case["rows"], groups * 8)).to(DEV)
    return (u[:, :case["cols"]] >= _threshold(case["drop"])).double()


def exact(case, seed):
    st = prepare(case, seed)
    f = {k: v.double() for k, v in st.items() if isinstance(v, torch.Tensor) and v.is_floating_point()}
    op, n = case["op"], case["cols"]
    scale = 1.0
    if case.get("drop"):
        t = _threshold(case["drop"])
        scale = _mask64(case, st["seed"], st["offset"]) * (65536 / (65536 - t)) if t else 1.0
    if op == "logprobs":
        x = f["logits"]
        lse = torch.logsumexp(x, dim=1)
        logp = x - lse.unsqueeze(1)
        p = torch.exp(logp)
        entropy = -torch.where(p == 0, 0.0, p * logp).sum(dim=1)
        rows = torch.arange(case["rows"], device=DEV)
        of = torch.where(st["targets"] < 0, 0.0, logp[rows, st["targets"].clamp(min=0)])
        if not case["top"]:
            return [of, entropy, lse, None, None]
        best, ids = torch.sort(x, dim=1, descending=True, stable=True)
        return [of, entropy, lse, ids[:, :case["top"]], best[:, :case["top"]] - lse.unsqueeze(1)]
    if op == "logprobs_backward":
        # the forward pass's results are inputs here, as they were rounded
        logp = f["logits"] - f["lse"].unsqueeze(1)
        p = torch.exp(logp)
        hit = torch.arange(n, device=DEV).unsqueeze(0) == st["targets"].unsqueeze(1)
        d = f["dlogprob"].unsqueeze(1) * (hit.double() - p)
        if case["entropy"]:
            d -= f["dentropy"].unsqueeze(1) * p * (logp + f["entropy"].unsqueeze(1))
        return [d]
    if op == "dropout":
        v = (f["x"] + f["bias"] if case["bias"] else f["x"]) * scale
        return [v + f["residual"] if case["residual"] else v]
    if op == "dropout_backward":
        d = f["dout"] * scale
        return [d, d.sum(dim=0) if case["bias"] else None]
    if op in ("norm", "block"):
        s = f["x"] if op == "norm" else f["residual"] + (f["x"] + f["bias"]) * scale
        mean = s.mean(dim=1)
        rstd = (s.var(dim=1, unbiased=False) + EPS) ** -0.5
        y = (s - mean.unsqueeze(1)) * rstd.unsqueeze(1) * f["weight"] + f["bias" if op == "norm" else "norm_bias"]
        return [y, mean, rstd] if op == "norm" else [y, s, mean, rstd]
    x = f["x" if op == "norm_backward" else "sum"]
    hat = (x - f["mean"].unsqueeze(1)) * f["rstd"].unsqueeze(1)
    g = f["dy"] * f["weight"]
    ds = (g - g.mean(dim=1, keepdim=True) - hat * (g * hat).mean(dim=1, keepdim=True)) * f["rstd"].unsqueeze(1)
    sums = [(f["dy"] * hat).sum(dim=0), f["dy"].sum(dim=0)]
    if op == "norm_backward":
        return [ds] + sums
    if case["dsum"]:
        ds = ds + f["dsum"]
    d = ds * scale
    return [d, ds, d.sum(dim=0)] + sums
