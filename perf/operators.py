"""Dense layers of transformer blocks, in training and in serving, as programs call them: three operators of one block.

  ffn       the gated feed-forward block  y = (gate(x Wg) * (x Wu)) Wd : forward alone (serving: one token, a batch of
            sequences that each add a token, a prompt), or forward and the gradients of the input and the three weights
            (training)
  dropout   dropout whose mask comes from a counter-based generator and is never stored, forward (with the residual that
            follows it, if any) and backward
  int8      a dense layer on 8-bit integers: each token's row of x is quantised with a scale of its own, multiplied with
            weights that hold a scale for each output channel, and rescaled, with bias and activation

`run` computes them in plain torch operations where `own` is false, and through the framework's entry points where it is
true.  Sizes: whole ones of the powers of two that such blocks use, the classifier of 1024 features and 1000 classes at the
batch of 128 that the benchmark's models end in, and odd ones between.
"""
import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
_GATES = ("silu", "gelu", "gelu_tanh", "sigmoid", "relu")
_contexts = {}


def _context():
    """One context for the process, as a program would hold it."""
    if 0 not in _contexts:
        import paper_1901_05350_b200 as tfjsb

        _contexts[0] = tfjsb.Context(0)
    return _contexts[0]


# ---- the cases ---------------------------------------------------------------------------------------------


def _ffn(tokens, width, hidden, dtype="bf16", gate="silu", train=False):
    return {"kind": "ffn", "tokens": tokens, "width": width, "hidden": hidden, "dtype": dtype, "gate": gate, "train": train}


def _dropout(rows, positions, channels, dtype, rate, residual=False, shared=False):
    return {"kind": "dropout", "rows": rows, "positions": positions, "channels": channels, "dtype": dtype, "rate": rate,
            "residual": residual, "shared": shared}


def _int8(tokens, inner, outputs, dtype="bf16", bias=False, act="none"):
    return {"kind": "int8", "tokens": tokens, "inner": inner, "outputs": outputs, "dtype": dtype, "bias": bias, "act": act}


def listed():
    cases = [
        # answering one user: one token through a small block, where latency counts
        ("ffn_token", _ffn(1, 1024, 4096)),
        # a batch of sequences that each add one token: the weights are read for 24 rows
        ("ffn_tokens_24", _ffn(24, 2048, 8192, gate="gelu_tanh")),
        # a prompt of 4096 tokens before the first answer
        ("ffn_prompt", _ffn(4096, 2048, 8192)),
        # a training step of a small block on a packed batch: hidden width 8/3 of the model's, which is no whole multiple of anything
        ("ffn_train_ragged", _ffn(1000, 1024, 2730, gate="gelu", train=True)),
        # a training step of a large block
        ("ffn_train", _ffn(8192, 4096, 16384, train=True)),
        # training in the framework's own storage format
        ("ffn_train_fp32", _ffn(515, 512, 1365, dtype="fp32", train=True)),
        # dropout before a classifier, at the batch size and the classes of the benchmark's models
        ("dropout_classifier", _dropout(128, 1, 1000, "fp32", 0.25)),
        # dropout on a block's output, added to the residual stream of a large batch
        ("dropout_residual", _dropout(8, 2048, 4096, "bf16", 0.1, residual=True)),
        # one mask for all positions of a sequence (spatial dropout), a width that is no multiple of four
        ("dropout_shared", _dropout(64, 197, 771, "fp32", 0.5, shared=True)),
        # one token through a dense layer of 8-bit weights
        ("int8_token", _int8(1, 4096, 4096)),
        # the classifier of the benchmark's models on 8-bit weights
        ("int8_classifier", _int8(128, 1024, 1000, dtype="fp32", bias=True, act="relu6")),
        # a long prompt through the widest layer of a large block
        ("int8_prompt", _int8(8192, 4096, 16384)),
    ]
    return [dict(c, name=name) for name, c in cases]


def _log(rng, low, high):
    """A whole number spread evenly over the logarithm of low..high."""
    return min(high, max(low, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind = rng.choice(("ffn", "ffn", "dropout", "int8"))
    if kind == "ffn":
        dtype = rng.choice(("bf16", "bf16", "bf16", "fp32"))
        most = (8192, 4096, 16384) if dtype == "bf16" else (2048, 1024, 4096)
        tokens, width, hidden = _log(rng, 1, most[0]), _log(rng, 64, most[1]), _log(rng, 64, most[2])
        if rng.random() < 0.6:  # most blocks have widths that the tensor cores like
            width, hidden = -(-width // 64) * 64, -(-hidden // 64) * 64
        return _ffn(tokens, width, hidden, dtype, rng.choice(_GATES), rng.random() < 0.5)
    if kind == "dropout":
        rows, positions, channels = _log(rng, 1, 64), _log(rng, 1, 512), _log(rng, 1, 2048)
        residual, shared = rng.random() < 0.4, rng.random() < 0.3
        return _dropout(rows, positions, channels, rng.choice(("bf16", "fp32")), rng.choice((0.0, 0.1, 0.25, 0.5, 0.9)), residual, shared)
    return _int8(_log(rng, 1, 8192), _log(rng, 16, 8192), _log(rng, 16, 8192), rng.choice(("bf16", "fp32")), rng.random() < 0.5,
                 rng.choice(("none", "relu", "relu6")))


# ---- what a program has in hand ----------------------------------------------------------------------------


def _normal(gen, shape, std, dtype=torch.float32):
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def _noise_shape(case):
    """Shape of the mask: x's, or one row of it for all positions."""
    return (case["rows"], 1 if case["shared"] else case["positions"], case["channels"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    s = dict(case)
    if case["kind"] == "ffn":
        dtype, t, d, f = _DTYPES[case["dtype"]], case["tokens"], case["width"], case["hidden"]
        s["x"] = _normal(gen, (t, d), 1.0, dtype)  # the output of a norm
        s["w_gate"], s["w_up"] = (_normal(gen, (d, f), d ** -0.5, dtype) for _ in range(2))
        s["w_down"] = _normal(gen, (f, d), f ** -0.5, dtype)
        if case["train"]:
            s["dy"] = _normal(gen, (t, d), 1.0, dtype)
    elif case["kind"] == "dropout":
        dtype, shape = _DTYPES[case["dtype"]], (case["rows"], case["positions"], case["channels"])
        s["x"], s["dy"] = _normal(gen, shape, 1.0, dtype), _normal(gen, shape, 1.0, dtype)
        s["residual"] = _normal(gen, shape, 1.0, dtype) if case["residual"] else None
        s["seed"], s["offset"] = 0x9E3779B97F4A7C15 * (seed + 1) % 2 ** 64, 977 * seed + 5  # of the run, and of the step
    else:
        dtype, m, k, n = _DTYPES[case["dtype"]], case["tokens"], case["inner"], case["outputs"]
        s["x"] = _normal(gen, (m, k), 1.0, dtype)
        # weights laid out once: [outputs, inner], each output channel with the scale of its largest value, rows filled up with
        # zeros to a multiple of 16 bytes
        w = _normal(gen, (n, k), k ** -0.5)
        s["w_scale"] = w.abs().amax(1) / 127
        s["w"] = torch.zeros(n, -(-k // 16) * 16, dtype=torch.int8, device="cuda")
        s["w"][:, :k] = torch.round(w / s["w_scale"][:, None]).clamp(-127, 127)
        s["bias_values"] = _normal(gen, (n,), 0.1) if case["bias"] else None
    return s


# ---- plain forms -------------------------------------------------------------------------------------------


def _gate(name, g):
    """The gate's function of g, and its derivative."""
    if name == "silu":
        p = 1 / (1 + torch.exp(-g))
        return g * p, p * (1 + g * (1 - p))
    if name == "sigmoid":
        p = 1 / (1 + torch.exp(-g))
        return p, p * (1 - p)
    if name == "relu":
        return torch.where(g > 0, g, 0.0), (g > 0).to(g.dtype)
    if name == "gelu":
        p = 0.5 * torch.erfc(-g * math.sqrt(0.5))
        return g * p, p + g * torch.exp(-0.5 * g * g) * (1 / math.sqrt(2 * math.pi))
    a, b = math.sqrt(2 / math.pi), 0.044715  # gelu_tanh
    t = torch.tanh(a * (g + b * g * g * g))
    return 0.5 * g * (1 + t), 0.5 * (1 + t) + 0.5 * g * (1 - t * t) * a * (1 + 3 * b * g * g)


def _plain_ffn(s):
    dtype = s["x"].dtype
    x, wg, wu, wd = (s[k].float() for k in ("x", "w_gate", "w_up", "w_down"))
    g, u = x @ wg, x @ wu
    act, slope = _gate(s["gate"], g)
    h = act * u
    y = h @ wd
    if not s["train"]:
        return {"y": y.to(dtype)}
    dy = s["dy"].float()
    dh = dy @ wd.t()
    dg, du = dh * u * slope, dh * act
    return {"y": y.to(dtype), "dx": (dg @ wg.t() + du @ wu.t()).to(dtype), "dw_gate": (x.t() @ dg).to(dtype),
            "dw_up": (x.t() @ du).to(dtype), "dw_down": (h.t() @ dy).to(dtype)}


def _plain_words(count, seed, offset):
    """The first `count` 32-bit words of Philox-4x32 with ten rounds (Salmon, Moraes, Dror and Shaw, 2011): key = seed, counter =
    (index of the block of four words, offset).  64-bit integers hold the 32-bit words."""
    low = 0xFFFFFFFF
    block = torch.arange(-(-count // 4), device="cuda")
    zero = torch.zeros_like(block)
    c0, c1, c2, c3 = block & low, block >> 32, zero + (offset & low), zero + (offset >> 32)
    k0, k1 = seed & low, seed >> 32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57  # the low 64 bits of each product: all of it
        c0, c1, c2, c3 = ((p1 >> 32) & low) ^ c1 ^ k0, p1 & low, ((p0 >> 32) & low) ^ c3 ^ k1, p0 & low
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack((c0, c1, c2, c3), -1).reshape(-1)[:count]


def _plain_dropout(s):
    dtype, noise = s["x"].dtype, _noise_shape(s)
    words = _plain_words(math.prod(noise), s["seed"], s["offset"])
    keep = (words >= math.ceil(s["rate"] * 2 ** 32)).reshape(noise)  # word / 2^32 >= rate
    scale = 1 / (1 - s["rate"])
    y = torch.where(keep, s["x"].float() * scale, 0.0)
    if s["residual"] is not None:
        y = y + s["residual"].float()
    return {"y": y.to(dtype), "dx": torch.where(keep, s["dy"].float() * scale, 0.0).to(dtype)}


def _plain_int8(s):
    x = s["x"].double()  # whether a value lies above or below the middle between two integers
    largest = x.abs().amax(1, keepdim=True)
    q = torch.round(x * 127 / torch.where(largest > 0, largest, 1.0)).float()
    y = (q @ s["w"][:, : q.shape[1]].float().t()) * (largest.float() / 127) * s["w_scale"]
    if s["bias_values"] is not None:
        y = y + s["bias_values"]
    if s["act"] != "none":
        y = torch.where(y > 0, y, 0.0)
    if s["act"] == "relu6":
        y = torch.where(y < 6, y, 6.0)
    return {"y": y.to(s["x"].dtype)}


# ---- one pass ----------------------------------------------------------------------------------------------


def run(s):
    if not own:
        return {"ffn": _plain_ffn, "dropout": _plain_dropout, "int8": _plain_int8}[s["kind"]](s)
    c = _context()
    if s["kind"] == "ffn":
        weights = (s["w_gate"], s["w_up"], s["w_down"])
        if not s["train"]:
            return {"y": c.gated_ffn(s["x"], *weights, gate=s["gate"])}
        y, h, z = c.gated_ffn(s["x"], *weights, gate=s["gate"], save=True)
        dx, dw_gate, dw_up, dw_down = c.gated_ffn_backprop(s["x"], *weights, h, z, s["dy"], gate=s["gate"])
        return {"y": y, "dx": dx, "dw_gate": dw_gate, "dw_up": dw_up, "dw_down": dw_down}
    if s["kind"] == "dropout":
        noise = _noise_shape(s) if s["shared"] else None
        y = c.dropout(s["x"], s["rate"], s["seed"], offset=s["offset"], noise_shape=noise, residual=s["residual"])
        return {"y": y, "dx": c.dropout_backprop(s["dy"], s["rate"], s["seed"], offset=s["offset"], noise_shape=noise)}
    return {"y": c.dense_int8(s["x"], s["w"], s["w_scale"], bias=s["bias_values"], act=s["act"])}


def work(case):
    size = {"bf16": 2, "fp32": 4}[case["dtype"]]
    if case["kind"] == "ffn":
        t, d, f = case["tokens"], case["width"], case["hidden"]
        if case["train"]:  # x, dy, y, dx, weights and their gradients; three products forward, six backward
            return {"bytes": size * (4 * t * d + 6 * d * f), "flops": 18 * t * d * f}
        return {"bytes": size * (2 * t * d + 3 * d * f), "flops": 6 * t * d * f}
    if case["kind"] == "dropout":
        n = case["rows"] * case["positions"] * case["channels"]
        return {"bytes": size * n * (5 if case["residual"] else 4), "flops": n * (5 if case["residual"] else 4)}
    m, k, n = case["tokens"], case["inner"], case["outputs"]
    return {"bytes": size * (m * k + m * n) + n * k + 4 * n * (2 if case["bias"] else 1), "flops": 2 * m * k * n}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------


def _exact_gate(name, g):
    """The same two functions from torch's own special functions, in 64 bits."""
    if name == "relu":
        return g.clamp(min=0), torch.heaviside(g, torch.zeros_like(g))
    if name in ("silu", "sigmoid"):
        p = torch.special.expit(g)
        return (p, p * torch.special.expit(-g)) if name == "sigmoid" else (g * p, p + g * p * torch.special.expit(-g))
    if name == "gelu":
        return g * torch.special.ndtr(g), torch.special.ndtr(g) + g * torch.exp(-g ** 2 / 2) / math.sqrt(2 * math.pi)
    inner = math.sqrt(8 / math.pi) * (g + 0.044715 * g ** 3)  # 0.5 (1 + tanh(v)) = expit(2 v)
    p = torch.special.expit(inner)
    return g * p, p + g * p * torch.special.expit(-inner) * math.sqrt(8 / math.pi) * (1 + 3 * 0.044715 * g ** 2)


def _exact_keep(noise, rate, seed, offset):
    """The mask, with the products of 32-bit words taken in halves of 16 bits (no product exceeds 2^33)."""
    n = math.prod(noise)
    blocks = (n + 3) // 4
    word = lambda v: torch.full((blocks,), v, dtype=torch.int64, device="cuda")  # noqa: E731

    def high_low(a, m):
        lo, hi = (a & 0xFFFF) * m, (a >> 16) * m  # below 2^48 each
        total = (lo >> 16) + hi
        return (total >> 16) & 0xFFFFFFFF, ((total & 0xFFFF) << 16) | (lo & 0xFFFF)

    i = torch.arange(blocks, device="cuda")
    c = [i % 2 ** 32, i // 2 ** 32, word(offset % 2 ** 32), word(offset // 2 ** 32)]
    for r in range(10):
        keys = ((seed % 2 ** 32 + r * 0x9E3779B9) % 2 ** 32, (seed // 2 ** 32 + r * 0xBB67AE85) % 2 ** 32)
        a, b = high_low(c[0], 0xD2511F53), high_low(c[2], 0xCD9E8D57)
        c = [b[0] ^ c[1] ^ keys[0], b[1], a[0] ^ c[3] ^ keys[1], a[1]]
    words = torch.stack(c, 1).flatten()[:n]
    return (words.double() / 2.0 ** 32 >= rate).view(noise)


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "ffn":
        x, wg, wu, wd = (s[k].double() for k in ("x", "w_gate", "w_up", "w_down"))
        up = torch.mm(x, wu)
        act, slope = _exact_gate(case["gate"], torch.mm(x, wg))
        found = {"y": torch.mm(act * up, wd)}
        if case["train"]:
            dy = s["dy"].double()
            found["dw_down"] = torch.mm((act * up).T, dy)
            dh = torch.mm(dy, wd.T)
            dg, du = dh.mul(slope).mul_(up), dh.mul(act)
            found["dx"] = torch.mm(dg, wg.T).addmm_(du, wu.T)
            found["dw_gate"], found["dw_up"] = torch.mm(x.T, dg), torch.mm(x.T, du)
        return found
    if case["kind"] == "dropout":
        keep = _exact_keep(_noise_shape(case), case["rate"], s["seed"], s["offset"]).expand(s["x"].shape)
        y = s["x"].double().div(1 - case["rate"]).masked_fill(~keep, 0)
        return {"y": y if s["residual"] is None else y + s["residual"].double(),
                "dx": s["dy"].double().div(1 - case["rate"]).masked_fill(~keep, 0)}
    x = s["x"].double()
    step = x.abs().max(dim=1).values.div(127)
    q = torch.round(x * 127 / x.abs().max(dim=1).values.clamp(min=2.0 ** -149)[:, None])
    y = torch.mm(q, s["w"][:, : case["inner"]].double().T) * step[:, None] * s["w_scale"].double()[None, :]
    if case["bias"]:
        y += s["bias_values"].double()
    return {"y": y if case["act"] == "none" else y.clamp(0, 6 if case["act"] == "relu6" else math.inf)}
