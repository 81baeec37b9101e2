"""Cases of the operators around the drafter layer: the norm in front of its projections, the log
probabilities of drafted tokens with their gradient, and the optimizer step, each in its plain form
(elementary torch operations) and through ``paper_2602_01469_b200.binding``.

A case's ``"op"`` says which call it is:

  norm_fwd       ``peagle_norm_fwd``: layer norm or RMS norm of rows
  norm_bwd       ``peagle_norm_bwd``: gradient of the rows, and of weight and bias added to fp32 sums
  logprobs_fwd   ``peagle_token_logprobs_fwd``: log probability of a token per row, log-sum-exp, entropy, top
                 alternatives
  logprobs_bwd   ``peagle_token_logprobs_bwd``: gradient of the logits
  adamw          ``peagle_adamw_step``: one step over many tensors, in place

``own`` chooses between the two forms.  Widths are those of the benchmark's layer (2,880 hidden, 64 and 128
per head) and of generic ones; row counts run from one token to the expanded tokens of the headline
sequence (4,096 x 8); vocabularies from a few hundred entries to 200,000.
"""
from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
BETA1, BETA2, ADAM_EPS, LR, DECAY, STEP, SEED = 0.9, 0.999, 1e-8, 1e-4, 0.1, 10, 1234
BLOCK = 256            # elements that share a scale where states are held in 8 bits
GOLDEN = 0x9E3779B9    # 2^32 / golden ratio: spreads the element numbers over 32 bits

DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
SIZE = {"bf16": 2, "f32": 4}


# ------------------------------------------------------------------ cases
def _norm(op, kind, rows, cols, dtype="bf16", wdtype="bf16", bias=False, pad=0, name=None):
    """``pad``: elements between the rows' ends and the next row (a view of a wider buffer)."""
    c = {"op": op, "kind": kind, "rows": rows, "cols": cols, "dtype": dtype, "wdtype": wdtype, "bias": bias, "pad": pad}
    return c if name is None else {"name": name, **c}


def _logprobs(op, rows, vocab, dtype="bf16", k=0, entropy=True, masked=0, pad=0, scale=1.0, name=None):
    """``masked``: vocabulary entries of every row that carry -inf (tokens that may not be drafted)."""
    c = {"op": op, "rows": rows, "vocab": vocab, "dtype": dtype, "k": k, "entropy": entropy, "masked": masked,
         "pad": pad, "scale": scale}
    return c if name is None else {"name": name, **c}


def _adamw(shape, width, layers, bits, dtype="bf16", gdtype="bf16", master=True, name=None):
    """``shape``: "layers" (weight matrices of ``layers`` decoder layers of hidden size ``width``, with
    their norms) or "vectors" (``layers`` small odd-sized tensors, ``width`` elements on average)."""
    c = {"op": "adamw", "shape": shape, "width": width, "layers": layers, "bits": bits, "dtype": dtype,
         "gdtype": gdtype, "master": master}
    return c if name is None else {"name": name, **c}


def listed():
    return [
        # one drafted token on its way into the layer: the time is the launch
        _norm("norm_fwd", "rms", 1, 2880, name="norm_fwd_one_token"),
        # the headline sequence's expanded tokens (4,096 x 8) at the layer's hidden size
        _norm("norm_fwd", "rms", 32768, 2880, name="norm_fwd_rms_hidden"),
        # its backward, once per segment
        _norm("norm_bwd", "rms", 32768, 2880, name="norm_bwd_rms_hidden"),
        # the norm of every query head of half the median trace (2,048 x 8 tokens, 32 heads of 128)
        _norm("norm_bwd", "layer", 524288, 128, bias=True, name="norm_bwd_layer_heads"),
        # fp32 rows of an odd width in a wider buffer, at the median trace length
        _norm("norm_bwd", "layer", 3891, 1001, dtype="f32", wdtype="f32", bias=True, pad=6, name="norm_bwd_layer_odd_f32"),
        # serving: the next token of one request with its twenty alternatives
        _logprobs("logprobs_fwd", 1, 128000, k=20, name="logprobs_fwd_one_token"),
        # scoring the median trace: entropy and a few alternatives for every position
        _logprobs("logprobs_fwd", 4096, 128000, k=8, name="logprobs_fwd_trace"),
        # fp32 logits of an odd vocabulary, some of them not allowed, at another temperature
        _logprobs("logprobs_fwd", 391, 50001, dtype="f32", k=5, masked=300, scale=0.7, name="logprobs_fwd_odd_f32"),
        # the loss's gradient over the median trace
        _logprobs("logprobs_bwd", 4096, 128000, entropy=False, name="logprobs_bwd_trace"),
        # many small tensors (norm weights, biases): the time is the launch and its table
        _adamw("vectors", 1500, 160, 32, dtype="f32", gdtype="f32", master=False, name="adamw_small_tensors"),
        # two decoder layers at the benchmark's hidden size, bf16 weights with fp32 masters
        _adamw("layers", 2880, 2, 32, name="adamw_layers"),
        # the same with states in 8 bits and without masters
        _adamw("layers", 2880, 2, 8, master=False, name="adamw_layers_8bit"),
    ]


def _spread(rng, lo, hi):
    """A whole number from [lo, hi], even over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        op = rng.choice(("norm_fwd", "norm_bwd", "logprobs_fwd", "logprobs_bwd", "adamw"))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        if op.startswith("norm"):
            cols = rng.choice((64, 128, 2880, 5120, _spread(rng, 1, 16384), 8 * _spread(rng, 8, 2048)))
            c = _norm(op, rng.choice(("rms", "layer")), _spread(rng, 1, 65536), cols, dtype=dtype,
                      wdtype=rng.choice((dtype, "f32")), bias=rng.random() < 0.5,
                      pad=rng.choice((0, 0, 8, rng.randint(1, 40))))
        elif op.startswith("logprobs"):
            vocab = rng.choice((32000, 128000, _spread(rng, 100, 200000), 8 * _spread(rng, 64, 25000)))
            forward = op == "logprobs_fwd"
            c = _logprobs(op, _spread(rng, 1, 16384), vocab, dtype=dtype, k=rng.choice((0, 1, 5, 20, 64)) if forward else 0,
                          entropy=rng.random() < 0.6, masked=rng.choice((0, 0, vocab // 3)),
                          pad=rng.choice((0, 0, rng.randint(1, 40))), scale=rng.choice((1.0, 1.0, 0.7, 1.3)))
        else:
            master = dtype == "bf16" and rng.random() < 0.5
            shape = rng.choice(("layers", "vectors"))
            c = _adamw(shape, 8 * _spread(rng, 16, 360) if shape == "layers" else _spread(rng, 10, 20000),
                       rng.randint(1, 2) if shape == "layers" else _spread(rng, 1, 600), rng.choice((8, 32)), dtype=dtype,
                       gdtype=rng.choice((dtype, "f32")), master=master)
        if _cost(c) <= most:
            return c


def _cost(case):
    return work(case)["bytes"]


def work(case):
    """Bytes: every input read once, every output written once.  Flops: counted roughly, no case is near
    the card's rate of them."""
    op = case["op"]
    if op.startswith("norm"):
        rows, cols, e = case["rows"], case["cols"], SIZE[case["dtype"]]
        vectors = (1 + case["bias"]) * cols
        stats = rows * (8 if case["kind"] == "layer" else 4)
        if op == "norm_fwd":
            return {"bytes": 2 * rows * cols * e + vectors * SIZE[case["wdtype"]] + stats, "flops": 6 * rows * cols}
        return {"bytes": 3 * rows * cols * e + cols * SIZE[case["wdtype"]] + 8 * vectors + stats, "flops": 12 * rows * cols}
    if op.startswith("logprobs"):
        rows, vocab, e = case["rows"], case["vocab"], SIZE[case["dtype"]]
        if op == "logprobs_fwd":
            return {"bytes": rows * (vocab * e + 4 + 8 + 4 * case["entropy"] + 8 * case["k"]), "flops": 6 * rows * vocab}
        return {"bytes": rows * (2 * vocab * e + 4 + 4 + 4 + 8 * case["entropy"]), "flops": 6 * rows * vocab}
    n = sum(_sizes(case))
    p = 2 * SIZE[case["dtype"]] if not case["master"] else 8 + SIZE[case["dtype"]]
    state = 16 if case["bits"] == 32 else 4 + 16 / BLOCK
    return {"bytes": n * (p + SIZE[case["gdtype"]] + state), "flops": 15 * n}


def _sizes(case):
    """Elements of the tensors, those with weight decay (matrices) first."""
    w = case["width"]
    if case["shape"] == "layers":
        # query | key | value projection, output projection, gate and up, down; the two norms
        matrices = [w * (w + w // 2), w * w, 2 * w * w, w * w]
        return matrices * case["layers"] + [w, w] * case["layers"]
    return [1 + (i * 7919 + 13) % (2 * w) for i in range(case["layers"])]


def _decayed(case):
    return 4 * case["layers"] if case["shape"] == "layers" else case["layers"] // 2


# ------------------------------------------------------------------ what a program holds
def _lib():
    from paper_2602_01469_b200 import binding as b
    return b


_contexts = {}


def _context():
    """A training program keeps one context for its whole run."""
    dev = torch.cuda.current_device()
    if dev not in _contexts:
        _contexts[dev] = _lib().Context(dev)
    return _contexts[dev]


def _rows(gen, rows, cols, pad, dtype, std=1.0):
    """Normal rows inside a buffer whose rows are ``pad`` elements longer."""
    t = torch.randn(rows, cols + pad, generator=gen, dtype=dtype, device="cuda")
    return (t * std if std != 1.0 else t)[:, :cols]


def _empty_rows(rows, cols, pad, dtype):
    return torch.zeros(rows, cols + pad, dtype=dtype, device="cuda")[:, :cols]


def _f32(*shape):
    return torch.zeros(*shape, dtype=torch.float32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = {"case": case}
    if case["op"].startswith("norm"):
        rows, cols, pad, dt = case["rows"], case["cols"], case["pad"], DTYPE[case["dtype"]]
        s["x"] = _rows(gen, rows, cols, pad, dt, 2.0)
        s["x"] += torch.randn(1, cols, generator=gen, dtype=dt, device="cuda")  # hidden units have means of their own
        s["w"] = (1.0 + 0.2 * torch.randn(cols, generator=gen, device="cuda")).to(DTYPE[case["wdtype"]])
        s["b"] = (0.1 * torch.randn(cols, generator=gen, device="cuda")).to(DTYPE[case["wdtype"]]) if case["bias"] else None
        layer = case["kind"] == "layer"
        if case["op"] == "norm_fwd":
            s["y"], s["rstd"] = _empty_rows(rows, cols, pad, dt), _f32(rows)
            s["mean"] = _f32(rows) if layer else None
        else:
            s["dy"] = _rows(gen, rows, cols, pad, dt)
            x = s["x"].float()
            s["mean"] = x.mean(1) if layer else None
            x = x - s["mean"][:, None] if layer else x
            s["rstd"] = (x.square().mean(1) + EPS).rsqrt()
            s["dx"], s["dw"] = _empty_rows(rows, cols, pad, dt), _f32(cols)
            s["db"] = _f32(cols) if case["bias"] else None
        return s
    if case["op"].startswith("logprobs"):
        rows, vocab, pad, dt, k = case["rows"], case["vocab"], case["pad"], DTYPE[case["dtype"]], case["k"]
        s["logits"] = _rows(gen, rows, vocab, pad, dt, 2.5)
        # the model is rather sure of one token per row, and that is the given one in most rows
        peak = torch.randint(vocab, (rows,), generator=gen, device="cuda")
        s["logits"][torch.arange(rows, device="cuda"), peak] += 12.0
        other = torch.randint(vocab, (rows,), generator=gen, device="cuda")
        tokens = torch.where(torch.rand(rows, generator=gen, device="cuda") < 0.7, peak, other)
        if rows > 8:
            tokens[torch.rand(rows, generator=gen, device="cuda") < 0.05] = -1  # padding: no token given
        if case["masked"]:
            s["logits"][:, torch.randperm(vocab, generator=gen, device="cuda")[:case["masked"]]] = -math.inf
        s["tokens"] = tokens.to(torch.int32)
        s["lse"], s["entropy"] = _f32(rows), _f32(rows) if case["entropy"] else None
        if case["op"] == "logprobs_fwd":
            s["logprob"] = _f32(rows)
            s["top"] = _f32(rows, k) if k else None
            s["ids"] = torch.zeros(rows, k, dtype=torch.int32, device="cuda") if k else None
        else:
            out = _softmax(s["logits"].float() * case["scale"])
            s["lse"].copy_(out["lse"])
            if case["entropy"]:
                s["entropy"].copy_(out["entropy"])
            del out
            s["g"] = torch.randn(rows, generator=gen, device="cuda") / rows
            s["g"][s["tokens"] < 0] = 0.0
            s["ge"] = torch.randn(rows, generator=gen, device="cuda") / rows if case["entropy"] else None
            s["dlogits"] = _empty_rows(rows, vocab, pad, dt)
        return s
    sizes = _sizes(case)
    padded = [-(-n // BLOCK) * BLOCK for n in sizes]   # every tensor begins on a block of its own
    starts = [sum(padded[:i]) for i in range(len(padded))]
    total, split = sum(padded), sum(padded[:_decayed(case)])
    used = torch.zeros(total, dtype=torch.bool, device="cuda")
    s["starts"] = torch.tensor(starts, device="cuda")
    s["padded"] = torch.tensor(padded, device="cuda")
    ends = s["starts"] + torch.tensor(sizes, device="cuda")
    place = torch.arange(total, device="cuda")
    used = place < torch.repeat_interleave(ends, s["padded"], output_size=total)
    del place
    s["split"] = split
    weights = 0.02 * torch.randn(total, generator=gen, device="cuda") * used
    s["p"] = weights.to(DTYPE[case["dtype"]])
    s["master"] = weights if case["master"] else None
    # gradients of very different sizes, as rows of embeddings and norms have them
    size = torch.exp(2.0 * torch.randn(total // BLOCK, generator=gen, device="cuda")).repeat_interleave(BLOCK) * 1e-3
    s["g"] = (size * torch.randn(total, generator=gen, device="cuda") * used).to(DTYPE[case["gdtype"]])
    m = 0.3 * size * torch.randn(total, generator=gen, device="cuda") * used
    root = size * (0.5 + torch.rand(total, generator=gen, device="cuda")) * used
    if case["bits"] == 32:
        s["m"], s["v"] = m, root.square()
        s["ms"] = s["vs"] = None
    else:
        s["ms"], s["vs"] = _scales(m), _scales(root)
        s["m"] = (m.view(-1, BLOCK) / s["ms"][:, None]).view(-1).to(torch.float8_e4m3fn)
        s["v"] = (root.view(-1, BLOCK) / s["vs"][:, None]).view(-1).to(torch.float8_e4m3fn)
    s["sizes"], s["starts_list"], s["decayed"] = sizes, starts, _decayed(case)
    s["tensors"] = None
    return s


# ------------------------------------------------------------------ plain forms
def _norm_fwd(s):
    case = s["case"]
    x = s["x"].float()
    mean = x.mean(1, keepdim=True) if case["kind"] == "layer" else 0.0
    x = x - mean
    rstd = (x.square().mean(1, keepdim=True) + EPS).rsqrt()
    y = x * rstd * s["w"].float()
    if case["bias"]:
        y = y + s["b"].float()
    return {"y": y.to(s["x"].dtype), "rstd": rstd[:, 0], "mean": mean[:, 0] if case["kind"] == "layer" else None}


def _norm_bwd(s):
    case = s["case"]
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xh = s["x"].float()
    if case["kind"] == "layer":
        xh = xh - s["mean"][:, None]
    xh = xh * rstd
    u = dy * s["w"].float()
    dx = u - xh * (u * xh).mean(1, keepdim=True)
    if case["kind"] == "layer":
        dx = dx - u.mean(1, keepdim=True)
    s["dw"] += (dy * xh).sum(0)
    if case["bias"]:
        s["db"] += dy.sum(0)
    return {"dx": (dx * rstd).to(s["x"].dtype), "dw": s["dw"], "db": s["db"]}


def _softmax(x):
    """Log-sum-exp, entropy and log probabilities of rows of fp32 logits, at least one of them finite."""
    top = x.max(1, keepdim=True).values
    shifted = x - top
    e = torch.exp(shifted)
    total = e.sum(1, keepdim=True)
    log_total = torch.log(total)
    # an entry of -inf has probability zero and adds nothing to the entropy
    mean = (e * torch.clamp(shifted, min=-200.0)).sum(1) / total[:, 0]
    return {"lse": (top + log_total)[:, 0], "entropy": log_total[:, 0] - mean, "logp": shifted - log_total}


def _logprobs_fwd(s):
    case = s["case"]
    x, tokens, k = s["logits"].float(), s["tokens"].long(), case["k"]
    out = _softmax(x * case["scale"])
    given = torch.gather(out["logp"], 1, tokens.clamp(min=0)[:, None])[:, 0]
    got = {"logprob": torch.where(tokens < 0, torch.zeros_like(given), given), "lse": out["lse"],
           "entropy": out["entropy"] if case["entropy"] else None, "top": None, "ids": None}
    if k:
        ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k]  # equal values: lowest index first
        got["top"], got["ids"] = torch.gather(out["logp"], 1, ids), ids.to(torch.int32)
    return got


def _logprobs_bwd(s):
    case = s["case"]
    logp = s["logits"].float() * case["scale"] - s["lse"][:, None]
    p = torch.exp(logp)
    d = -s["g"][:, None] * p
    if case["entropy"]:
        d = d - s["ge"][:, None] * p * (torch.clamp(logp, min=-200.0) + s["entropy"][:, None])
    tokens = s["tokens"].long()
    d.scatter_add_(1, tokens.clamp(min=0)[:, None], torch.where(tokens < 0, torch.zeros_like(s["g"]), s["g"])[:, None])
    return {"dlogits": (d * case["scale"]).to(s["logits"].dtype)}


def _scales(x):
    """Power of two for each block that brings its largest magnitude into [128, 256)."""
    largest = x.abs().view(-1, BLOCK).amax(1)
    exponent = torch.frexp(largest).exponent - 1
    exponent = torch.where(largest > 0, exponent.clamp(min=-100), torch.full_like(exponent, -100))
    return ((exponent + (127 - 7)) << 23).to(torch.int32).view(torch.float32)


def _mix(x):
    """Scrambles 32-bit numbers held in int64 (two rounds of shift-xor and multiply)."""
    x = x ^ (x >> 16)
    x = (x * 0x7FEB352D) & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = (x * 0x846CA68B) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random_bits(s):
    """32 bits per element: a hash of seed, step, the tensor's number and the element's number in it."""
    count, total = s["starts"].numel(), s["m"].numel()
    key = _mix(torch.full((count,), (SEED + STEP * GOLDEN) & 0xFFFFFFFF, device="cuda"))
    key = _mix(key ^ torch.arange(1, count + 1, device="cuda"))
    place = torch.arange(total, device="cuda") - torch.repeat_interleave(s["starts"], s["padded"], output_size=total)
    return _mix((torch.repeat_interleave(key, s["padded"], output_size=total) + place * GOLDEN) & 0xFFFFFFFF)


def _to_codes(x, scale, bits16, keep):
    """x / scale rounded to e4m3 without bias: up with the probability of the fraction.  ``keep``: what is
    above zero stays above it."""
    y = (x.view(-1, BLOCK) / scale[:, None]).view(-1)
    z = y.abs()
    small = z < 2.0 ** -6                                     # e4m3's even spacing of 2^-9 begins here
    z = torch.where(small, z + 2.0 ** -6, z)
    z = (((z.view(torch.int32) + ((bits16 << 4) + 8).to(torch.int32)) >> 20) << 20).view(torch.float32)
    z = torch.where(small, z - 2.0 ** -6, z)
    if keep:
        z = torch.where(y > 0, z.clamp(min=2.0 ** -9), z)
    return torch.copysign(z, y).to(torch.float8_e4m3fn)


def _adamw_plain(s):
    case, g = s["case"], s["g"].float()
    eight = case["bits"] == 8
    if eight:
        m = s["m"].float().view(-1, BLOCK) * s["ms"][:, None]
        r = s["v"].float().view(-1, BLOCK) * s["vs"][:, None]
        m, v = m.view(-1), r.view(-1).square()
        # in 64 bits, rounded once: the roundings to 8 bits that follow go by values next to a border
        g64 = g.double()
        m = (BETA1 * m.double() + (1.0 - BETA1) * g64).float()
        v = (BETA2 * v.double() + (1.0 - BETA2) * g64 * g64).float()
        del g64
    else:
        m = s["m"] * BETA1 + (1.0 - BETA1) * g
        v = s["v"] * BETA2 + (1.0 - BETA2) * g.square()
    root = v.sqrt()
    step = m / (root / math.sqrt(1.0 - BETA2 ** STEP) + ADAM_EPS) * (LR / (1.0 - BETA1 ** STEP))
    p = s["master"] if case["master"] else s["p"].float()
    cut = s["split"]
    p = torch.cat([p[:cut] * (1.0 - LR * DECAY), p[cut:]]) - step
    del step
    if eight:
        bits = _random_bits(s)
        s["ms"].copy_(_scales(m))
        s["vs"].copy_(_scales(root))
        s["m"].copy_(_to_codes(m, s["ms"], bits & 0xFFFF, False))
        s["v"].copy_(_to_codes(root, s["vs"], bits >> 16, True))
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    if case["master"]:
        s["master"].copy_(p)
    s["p"].copy_(p.to(s["p"].dtype))
    return _state(s)


def _state(s):
    return {"p": s["p"], "master": s["master"], "m": s["m"], "v": s["v"], "ms": s["ms"], "vs": s["vs"]}


# ------------------------------------------------------------------ the framework's calls
def _own(s):
    case, b, ctx = s["case"], _lib(), _context()
    op = case["op"]
    if op == "norm_fwd":
        b.peagle_norm_fwd(ctx, b.NORM[case["kind"]], s["x"], s["w"], s["b"], EPS, s["y"], s["mean"], s["rstd"])
        return {"y": s["y"], "rstd": s["rstd"], "mean": s["mean"]}
    if op == "norm_bwd":
        b.peagle_norm_bwd(ctx, b.NORM[case["kind"]], s["x"], s["w"], s["mean"], s["rstd"], s["dy"], s["dx"], s["dw"], s["db"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    if op == "logprobs_fwd":
        b.peagle_token_logprobs_fwd(ctx, s["logits"], s["tokens"], case["scale"], s["logprob"], s["lse"], s["entropy"],
                                    s["top"], s["ids"])
        return {"logprob": s["logprob"], "lse": s["lse"], "entropy": s["entropy"], "top": s["top"], "ids": s["ids"]}
    if op == "logprobs_bwd":
        b.peagle_token_logprobs_bwd(ctx, s["logits"], s["tokens"], case["scale"], s["lse"], s["entropy"], s["g"], s["ge"],
                                    s["dlogits"])
        return {"dlogits": s["dlogits"]}
    if s["tensors"] is None:  # the list of tensors is put together once, as an optimizer does
        s["tensors"] = b.AdamWTensors([_one_tensor(s, i) for i in range(len(s["sizes"]))])
    b.peagle_adamw_step(ctx, s["tensors"], lr=LR, beta1=BETA1, beta2=BETA2, eps=ADAM_EPS, step=STEP, seed=SEED)
    return _state(s)


def _one_tensor(s, i):
    at, n = s["starts_list"][i], s["sizes"][i]
    part = slice(at, at + n)
    blocks = slice(at // BLOCK, at // BLOCK + -(-n // BLOCK))
    scaled = s["ms"] is not None
    return {"param": s["p"][part], "grad": s["g"][part], "m": s["m"][part], "v": s["v"][part],
            "master": s["master"][part] if s["master"] is not None else None,
            "m_scale": s["ms"][blocks] if scaled else None, "v_scale": s["vs"][blocks] if scaled else None,
            "weight_decay": DECAY if i < s["decayed"] else 0.0}


_PLAIN = {"norm_fwd": _norm_fwd, "norm_bwd": _norm_bwd, "logprobs_fwd": _logprobs_fwd, "logprobs_bwd": _logprobs_bwd,
          "adamw": _adamw_plain}


def run(s):
    if own:
        return _own(s)
    return _PLAIN[s["case"]["op"]](s)


# ------------------------------------------------------------------ the definitions in 64 bits
def exact(case, seed):
    """What ``run`` returns, from the formulas in 64 bits, a part of the rows at a time."""
    s = prepare(case, seed)
    op = case["op"]
    if op.startswith("norm"):
        return _exact_norm(case, s)
    if op.startswith("logprobs"):
        return _exact_logprobs(case, s)
    return _exact_adamw(case, s)


def _parts(rows, cols):
    size = max(1, 100_000_000 // max(1, cols))
    return [slice(i, min(rows, i + size)) for i in range(0, rows, size)]


def _exact_norm(case, s):
    rows, cols, layer = case["rows"], case["cols"], case["kind"] == "layer"
    w = s["w"].double()
    if case["op"] == "norm_fwd":
        ys, rs, ms = [], [], []
        for part in _parts(rows, cols):
            x = s["x"][part].double()
            var, mu = torch.var_mean(x, dim=1, correction=0)
            spread = var if layer else var + mu * mu            # mean square = variance + squared mean
            rstd = torch.pow(spread + EPS, -0.5)
            y = (x - mu[:, None]) if layer else x
            y = torch.einsum("rc,r,c->rc", y, rstd, w)
            ys.append(y + s["b"].double() if case["bias"] else y)
            rs.append(rstd)
            ms.append(mu)
        return {"y": torch.cat(ys), "rstd": torch.cat(rs), "mean": torch.cat(ms) if layer else None}
    dxs, dw, db = [], torch.zeros_like(w), torch.zeros_like(w)
    for part in _parts(rows, cols):
        r = s["rstd"][part].double()
        x = s["x"][part].double()
        x = x - s["mean"][part].double()[:, None] if layer else x
        dy = s["dy"][part].double()
        # dx = r u - r^3 x <u, x> / n - r <u> with u = w dy
        u = dy * w
        dx = u * r[:, None] - x * (torch.einsum("rc,rc->r", u, x) * r ** 3 / cols)[:, None]
        if layer:
            dx -= (u.sum(1) * r / cols)[:, None]
        dw += torch.einsum("rc,rc,r->c", dy, x, r)
        db += dy.sum(0)
        dxs.append(dx)
    return {"dx": torch.cat(dxs), "dw": dw, "db": db if case["bias"] else None}


def _exact_logprobs(case, s):
    rows, k, got = case["rows"], case["k"], {}
    for part in _parts(rows, case["vocab"]):
        z = s["logits"][part].double() * case["scale"]
        tok = s["tokens"][part].long()
        at = torch.arange(z.shape[0], device=z.device)
        if case["op"] == "logprobs_fwd":
            lse = torch.logsumexp(z, 1)
            one = {"lse": lse, "logprob": torch.where(tok < 0, 0.0, z[at, tok.clamp(min=0)] - lse)}
            if case["entropy"]:
                p = torch.exp(z - lse[:, None])
                one["entropy"] = -torch.xlogy(p, p).sum(1)
            if k:
                one["top"] = torch.topk(z, k, dim=1).values - lse[:, None]
        else:
            lse, g = s["lse"][part].double(), s["g"][part].double()
            p = torch.exp(z - lse[:, None])
            d = p * -g[:, None]
            if case["entropy"]:
                d -= (torch.xlogy(p, p) + p * s["entropy"][part].double()[:, None]) * s["ge"][part].double()[:, None]
            d[at, tok.clamp(min=0)] += torch.where(tok < 0, 0.0, g)
            one = {"dlogits": d * case["scale"]}
        for name, v in one.items():
            got.setdefault(name, []).append(v)
    got = {name: torch.cat(v) for name, v in got.items()}
    if case["op"] == "logprobs_fwd":
        # ids are whole numbers and follow from comparisons alone
        got = {"logprob": got["logprob"], "lse": got["lse"], "entropy": got.get("entropy"), "top": got.get("top"), "ids": None}
    return got


def _exact_adamw(case, s):
    g = s["g"].double()
    if case["bits"] == 8:
        m = s["m"].double() * s["ms"].double().repeat_interleave(BLOCK)
        v = (s["v"].double() * s["vs"].double().repeat_interleave(BLOCK)) ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    m += (g - m) * (1.0 - BETA1)
    v += (g * g - v) * (1.0 - BETA2)
    m_hat, v_hat = m / (1.0 - BETA1 ** STEP), v / (1.0 - BETA2 ** STEP)
    p = s["master"].double() if case["master"] else s["p"].double()
    p[:s["split"]] -= LR * DECAY * p[:s["split"]]
    p -= LR * m_hat / (torch.sqrt(v_hat) + ADAM_EPS)
    got = {"p": p, "master": p if case["master"] else None, "m": m, "v": v, "ms": None, "vs": None}
    if case["bits"] == 8:  # what the codes stand for, before their rounding to 8 bits
        for name, x in (("m", m), ("v", torch.sqrt(v))):
            largest = x.float().abs().view(-1, BLOCK).amax(1).double()
            scale = torch.exp2(torch.floor(torch.log2(largest)).clamp(min=-100.0) - 7.0)
            got[name + "s"], got[name] = scale, x / scale.repeat_interleave(BLOCK)
    return got
