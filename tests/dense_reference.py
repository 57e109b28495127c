"""Plain 64-bit statements of the dense layers of transformer blocks, from their formulas, and bounds for what rounding may do to
them.  Tensors in, tensors out; any device."""
import math

import torch

BF16, FP32 = 2.0 ** -8, 2.0 ** -24  # half a step, relative to the value


def unit(dtype):
    return BF16 if dtype == torch.bfloat16 else FP32


# ---- gated feed-forward block -------------------------------------------------------------------------------


def gate(name, g):
    """gate(g) and its derivative."""
    s = torch.special.expit
    if name == "silu":
        return g * s(g), s(g) * (1 + g * s(-g))
    if name == "sigmoid":
        return s(g), s(g) * s(-g)
    if name == "relu":
        return g.clamp(min=0), (g > 0).to(g.dtype)
    if name == "gelu":
        return g * torch.special.ndtr(g), torch.special.ndtr(g) + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)
    v = math.sqrt(2 / math.pi) * (g + 0.044715 * g ** 3)
    dv = math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * g ** 2)
    return g * (1 + torch.tanh(v)) / 2, (1 + torch.tanh(v)) / 2 + g * (1 - torch.tanh(v) ** 2) / 2 * dv


def gated_ffn(x, w_gate, w_up, w_down, name):
    x, w_gate, w_up, w_down = (t.double() for t in (x, w_gate, w_up, w_down))
    return (gate(name, x @ w_gate)[0] * (x @ w_up)) @ w_down


def gated_ffn_gradients(x, w_gate, w_up, w_down, dy, name):
    x, w_gate, w_up, w_down, dy = (t.double() for t in (x, w_gate, w_up, w_down, dy))
    g, u = x @ w_gate, x @ w_up
    a, slope = gate(name, g)
    dh = dy @ w_down.T
    dg, du = dh * u * slope, dh * a
    return dg @ w_gate.T + du @ w_up.T, x.T @ dg, x.T @ du, (a * u).T @ dy


def gated_ffn_bounds(x, w_gate, w_up, w_down, dy, name):
    """How far each element of (y, dx, dw_gate, dw_up, dw_down) may be off, by the roundings that the call makes.

    A sum of K products in the tensor core: each of its K / 16 additions of 16 products cuts the aligned terms and the sum towards
    zero, at most 17 steps of 2^-23 of the sum of magnitudes so far, so (K + 32) 2^-22 of the sum of all magnitudes covers it; CUDA-core
    sums round once a product and are covered too.  Slopes of the gates and their second derivatives are below 1.2, so an error e of
    g moves gate(g) and its slope by 1.2 e, and the functions themselves are good to 2^-19 of max(1, |g|).  h, dg and du are rounded
    once to the storage type, then the results."""
    r = unit(x.dtype)
    ax, ag, au, ad, ady = (t.double().abs() for t in (x, w_gate, w_up, w_down, dy))
    xg, xu = ax @ ag, ax @ au
    g, u = x.double() @ w_gate.double(), x.double() @ w_up.double()
    a, slope = (t.abs() for t in gate(name, g))
    c = lambda k: (k + 32) * 2.0 ** -22  # noqa: E731
    D, F, T = x.shape[1], w_gate.shape[1], x.shape[0]
    e_g, e_u = c(D) * xg, c(D) * xu
    e_a = 1.2 * e_g + 2.0 ** -19 * g.abs().clamp(min=1)
    e_h = (a + e_a) * (u.abs() + e_u) - a * u.abs() + r * (a + e_a) * (u.abs() + e_u)
    h = a * u.abs() + e_h
    outs = []

    def product(left, e_left, right, exact, k):
        """Bound of a product's result: errors of the left operand, of the sums, of the last rounding."""
        total = e_left @ right + c(k) * ((left + e_left) @ right)
        return total + r * (exact.abs() + total)

    outs.append(product(a * u.abs(), e_h, ad, gated_ffn(x, w_gate, w_up, w_down, name), F))
    dh = (dy.double() @ w_down.double().T).abs()
    e_dh = c(w_down.shape[1]) * (ady @ ad.T)
    both = lambda v, e: (dh + e_dh) * (v + e) * (1 + r) - dh * v  # noqa: E731
    e_slope = 1.2 * e_g + 2.0 ** -19 * g.abs().clamp(min=1)
    e_du = both(a, e_a)
    e_dg = both(u.abs() * slope, (u.abs() + e_u) * (slope + e_slope) - u.abs() * slope)
    dg, du = dh * u.abs() * slope, dh * a
    dx, dwg, dwu, dwd = gated_ffn_gradients(x, w_gate, w_up, w_down, dy, name)
    total = e_dg @ ag.T + e_du @ au.T + c(2 * F) * ((dg + e_dg) @ ag.T + (du + e_du) @ au.T)
    outs.append(total + r * (dx.abs() + total))
    outs.append(product(dg.T, e_dg.T, ax, dwg.T, T).T)
    outs.append(product(du.T, e_du.T, ax, dwu.T, T).T)
    outs.append(product((a * u.abs()).T, e_h.T, ady, dwd, T))
    assert h.shape == (T, F)
    return outs


# ---- dropout ------------------------------------------------------------------------------------------------


def philox(counter, key):
    """Philox-4x32-10 of tensors of 32-bit words (as int64): counter [..., 4], key (k0, k1)."""
    c = [counter[..., i].clone() for i in range(4)]
    mask = 0xFFFFFFFF

    def mul(a, m):  # in halves, so that nothing exceeds 2^49
        lo, hi = (a & 0xFFFF) * m, (a >> 16) * m
        total = (lo >> 16) + hi
        return (total >> 16) & mask, ((total & 0xFFFF) << 16) | (lo & 0xFFFF)

    for r in range(10):
        k0, k1 = (key[0] + r * 0x9E3779B9) & mask, (key[1] + r * 0xBB67AE85) & mask
        h0, l0 = mul(c[0], 0xD2511F53)
        h1, l1 = mul(c[2], 0xCD9E8D57)
        c = [h1 ^ c[1] ^ k0, l1, h0 ^ c[3] ^ k1, l0]
    return torch.stack(c, -1)


def words(first, count, seed, offset, device="cpu"):
    """Words first .. first + count - 1 of the stream (seed, offset)."""
    block = torch.arange(first // 4, (first + count + 3) // 4, device=device)
    zero = torch.zeros_like(block)
    counter = torch.stack((block & 0xFFFFFFFF, block >> 32, zero + (offset & 0xFFFFFFFF), zero + (offset >> 32)), -1)
    return philox(counter, (seed & 0xFFFFFFFF, seed >> 32)).reshape(-1)[first % 4:][:count]


def keep(shape, rate, seed, offset, device="cpu"):
    return (words(0, math.prod(shape), seed, offset, device) >= math.ceil(rate * 2 ** 32)).reshape(shape)


def dropout(x, rate, mask, residual=None):
    y = torch.where(mask, x.double() / (1 - rate), torch.zeros((), dtype=torch.float64, device=x.device))
    return y if residual is None else y + residual.double()


def dropout_bound(x, rate, mask, residual=None):
    """The scale is rounded once, the product (or product and sum) once, and the result once more into bfloat16."""
    y = dropout(x, rate, mask, residual).abs()
    e = 2.5 * FP32 * torch.where(mask, x.double().abs() / (1 - rate), torch.zeros_like(y)) + FP32 * y
    return e + (BF16 * (y + e) if x.dtype == torch.bfloat16 else 0) + 2.0 ** -149


# ---- 8-bit integers -------------------------------------------------------------------------------------------


def quantize(x):
    """q and scale of each row; the quotient in 64 bits decides, which no quotient of fp32 values is too close for: 127 x and (n + 1/2) m are
    multiples of 2^-25 of m at least 2^-25 m apart unless equal, and then 2^-53 of the quotient resolves them."""
    x = x.double()
    amax = x.abs().amax(1, keepdim=True)
    usable = torch.isfinite(amax) & (amax > 0)
    q = torch.round(torch.where(usable, x * 127 / torch.where(usable, amax, 1.0), 0.0))
    return q.to(torch.int64), (amax[:, 0] / 127)


def act(name, y):
    return y if name == "none" else y.clamp(min=0) if name == "relu" else y.clamp(0, 6)


def int8_product(q, scale, w, w_scale, bias, name):
    """The exact sums (whole numbers below 2^53), scaled in 64 bits; and how far fp32 arithmetic may be off: the sum's conversion, two products
    and the bias, each half a step."""
    total = q.double() @ w.double().T
    v = total * scale.double()[:, None] * w_scale.double()
    y = v if bias is None else v + bias.double()
    return act(name, y), 4 * FP32 * v.abs() + 1.5 * FP32 * y.abs() + 2.0 ** -140
