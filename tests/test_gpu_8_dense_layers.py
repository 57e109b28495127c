"""The dense layers of transformer blocks against their 64-bit statements, through the binding."""
import ctypes
import math

import pytest
import torch

import dense_reference as ref

pytestmark = pytest.mark.gpu

GATES = ["silu", "gelu", "gelu_tanh", "sigmoid", "relu"]
DTYPES = [torch.bfloat16, torch.float32]
ids = lambda v: str(v).replace("torch.", "") if isinstance(v, torch.dtype) else None  # noqa: E731


def normal(seed, shape, std=1.0, dtype=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def block(seed, t, d, f, o, dtype):
    return (normal(seed, (t, d), 1.0, dtype), normal(seed + 1, (d, f), d ** -0.5, dtype), normal(seed + 2, (d, f), d ** -0.5, dtype),
            normal(seed + 3, (f, o), f ** -0.5, dtype), normal(seed + 4, (t, o), 1.0, dtype))


def check_ffn(got, want, bound, dtype, what):
    got = got.double()
    off = (got - want).abs()
    assert torch.isfinite(got).all(), what
    worst = (off - bound).max().item()
    assert worst <= 0, (what, worst, off.max().item(), int((off - bound).argmax()))
    if want.numel() >= 4096:
        # two independent roundings to bfloat16 are 2^-8 sqrt(2 / 3) of the result in the mean at most; fp32 sums in segments of eight
        # additions cut towards zero are off by 8 * 2^-24 each, four products in a row by 1e-6
        rel = (off.norm() / want.norm()).item()
        assert rel <= (2.0 ** -8 if dtype == torch.bfloat16 else 2e-6), (what, rel)


# ---- gated feed-forward block -----------------------------------------------------------------------------------

SHAPES = [  # tokens, width, hidden, out width
    (1, 1, 1, 1), (1, 64, 64, 64), (2, 8, 16, 24), (3, 5, 7, 9), (5, 100, 60, 33), (8, 256, 512, 256), (9, 256, 512, 256), (16, 72, 200, 136),
    (31, 129, 257, 65), (64, 64, 2048, 64), (100, 1000, 24, 8), (127, 136, 328, 520), (128, 128, 128, 128), (129, 192, 320, 264),
    (255, 257, 259, 261), (256, 512, 512, 512), (300, 520, 1032, 72), (513, 264, 776, 1000), (1000, 384, 1030, 384),
]


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_ffn_forward_and_gradients(ctx, shape, dtype):
    gate = GATES[sum(shape) % 5]
    x, wg, wu, wd, dy = block(100 + sum(shape), *shape, dtype)
    want = [ref.gated_ffn(x, wg, wu, wd, gate), *ref.gated_ffn_gradients(x, wg, wu, wd, dy, gate)]
    bounds = ref.gated_ffn_bounds(x, wg, wu, wd, dy, gate)
    alone = ctx.gated_ffn(x, wg, wu, wd, gate=gate)
    ctx.check_device_status()
    check_ffn(alone, want[0], bounds[0], dtype, "y alone")
    y, h, z = ctx.gated_ffn(x, wg, wu, wd, gate=gate, save=True)
    grads = ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy, gate=gate)
    ctx.check_device_status()
    for got, w, b, what in zip((y, *grads), want, bounds, ("y", "dx", "dw_gate", "dw_up", "dw_down")):
        assert got.dtype == dtype
        check_ffn(got, w, b, dtype, what)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("gate", GATES)
def test_ffn_gates(ctx, gate, dtype):
    """Every gate, with projections as large as plus and minus 30."""
    x, wg, wu, wd, dy = block(7, 40, 96, 136, 48, dtype)
    x = x * 6
    want = [ref.gated_ffn(x, wg, wu, wd, gate), *ref.gated_ffn_gradients(x, wg, wu, wd, dy, gate)]
    bounds = ref.gated_ffn_bounds(x, wg, wu, wd, dy, gate)
    y, h, z = ctx.gated_ffn(x, wg, wu, wd, gate=gate, save=True)
    grads = ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy, gate=gate)
    for got, w, b, what in zip((y, *grads), want, bounds, ("y", "dx", "dw_gate", "dw_up", "dw_down")):
        check_ffn(got, w, b, dtype, what)
    few = ctx.gated_ffn(x[:4].contiguous(), wg, wu, wd, gate=gate)  # the form for single tokens
    check_ffn(few, want[0][:4], bounds[0][:4], dtype, "few")


# ---- dropout ------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape,noise", [
    ((1,), None), ((7,), None), ((8,), None), ((1000,), None), ((4097,), None), ((128, 1000), None), ((3, 5, 7), (3, 1, 7)), ((3, 5, 7), (1, 5, 1)),
    ((4, 33, 64), (4, 1, 64)), ((4, 33, 65), (4, 1, 65)), ((16, 300), (16, 1)), ((16, 300), (1, 300)), ((2, 3, 4, 5), (2, 1, 4, 1)),
    ((2, 1, 40, 9), (1, 1, 40, 9)), ((9, 8), (1, 1)), ((6, 11), (6, 11)), ((2, 70, 3, 50), (2, 70, 1, 50)), ((700, 3), (1, 3)),
    ((5, 3, 20, 37), (5, 3, 1, 37)), ((3, 40, 33), (1, 1, 33)), ((3, 4, 16, 50), (1, 4, 1, 50)), ((2, 100, 64), (2, 1, 64)), ((9, 197, 771), (9, 1, 771)),
], ids=str)
def test_dropout(ctx, shape, noise, dtype):
    x, r = normal(1, shape, 1.0, dtype), normal(2, shape, 1.0, dtype)
    seed, offset = 0xFEDCBA9876543210, 2 ** 33 + 17
    for rate in (0.0, 0.3, 0.99):
        mask = ref.keep(noise or shape, rate, seed, offset, "cuda").expand(shape)
        y = ctx.dropout(x, rate, seed, offset, noise_shape=noise)
        assert y.dtype == dtype and ((y.double() - ref.dropout(x, rate, mask)).abs() <= ref.dropout_bound(x, rate, mask)).all()
        assert torch.equal(y != 0, mask & (x != 0))
        assert torch.equal(ctx.dropout_backprop(x, rate, seed, offset, noise_shape=noise), y)
        z = ctx.dropout(x, rate, seed, offset, noise_shape=noise, residual=r)
        assert ((z.double() - ref.dropout(x, rate, mask, r)).abs() <= ref.dropout_bound(x, rate, mask, r)).all()


# ---- 8-bit integers -----------------------------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("rows,columns", [(1, 1), (1, 16), (3, 17), (5, 100), (128, 1024), (7, 2047), (4, 8192), (3, 9001), (2, 20000),
                                          (1500, 8), (1200, 24), (1300, 264), (1201, 1000), (1184, 2048), (1190, 2056), (1190, 4096), (1190, 4088), (1190, 5000), (1300, 33)])
def test_quantized_rows(ctx, rows, columns, dtype):
    x = normal(rows + columns, (rows, columns), 1.0, dtype)
    x[0, 0] = 4.0  # halves of the largest value lie on the middle between two integers
    x[0, columns // 2] = -2.0 if columns > 1 else 4.0
    q, scale = ctx.quantize_int8(x)
    want, want_scale = ref.quantize(x)
    assert q.shape == (rows, -(-columns // 16) * 16) and not q[:, columns:].any()
    assert torch.equal(q[:, :columns].to(torch.int64), want)
    assert torch.equal(scale, want_scale.float())


PRODUCTS = [  # M, K, N
    (1, 16, 1), (1, 16, 8), (1, 4112, 33), (1, 20000, 10), (1, 1024, 9000), (2, 48, 3), (5, 112, 33), (8, 256, 72), (16, 4096, 64), (17, 128, 128), (33, 1040, 130), (128, 1024, 1000), (129, 272, 257),
    (200, 2000, 136), (256, 512, 512), (300, 144, 1500), (1000, 640, 768),
]


@pytest.mark.parametrize("out_dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape", PRODUCTS, ids=str)
def test_int8_product(ctx, shape, out_dtype):
    M, K, N = shape
    gen = torch.Generator(device="cuda").manual_seed(M + K + N)
    a = torch.randint(-128, 128, (M, K), generator=gen, device="cuda").to(torch.int8)
    w = torch.randint(-128, 128, (N, K), generator=gen, device="cuda").to(torch.int8)
    sa, sw, bias = normal(1, (M,)).abs() * 0.01, normal(2, (N,)).abs() * 0.01, normal(3, (N,))
    for b, name in ((None, "none"), (bias, "relu"), (bias, "relu6")):
        y = ctx.matmul_int8(a, sa, w, sw, bias=b, act=name, out_dtype=out_dtype)
        ctx.check_device_status()
        want, bound = ref.int8_product(a, sa, w, sw, b, name)
        if out_dtype == torch.bfloat16:
            bound = bound + ref.BF16 * (want.abs() + bound)
        off = (y.double() - want).abs()
        assert y.dtype == out_dtype and (off <= bound).all(), (off - bound).max().item()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape", [(1, 64, 64), (1, 37, 5), (1, 5000, 700), (1, 131072, 9), (2, 131071, 16), (3, 1000, 200), (8, 100, 1000), (24, 512, 96), (128, 1024, 1000), (500, 333, 640)], ids=str)
def test_dense_int8(ctx, shape, dtype):
    M, K, N = shape
    x, bias = normal(4, (M, K), 1.0, dtype), normal(5, (N,), 0.1)
    w, w_scale = ctx.quantize_int8(normal(6, (N, K), K ** -0.5))
    y = ctx.dense_int8(x, w, w_scale, bias=bias, act="relu")
    ctx.check_device_status()
    q, scale = ref.quantize(x)
    want, bound = ref.int8_product(q, scale.float(), w[:, :K], w_scale, bias, "relu")
    if dtype == torch.bfloat16:
        bound = bound + ref.BF16 * (want.abs() + bound)
    assert y.dtype == dtype and ((y.double() - want).abs() <= bound).all()
    # the same as the two calls, bit for bit
    a, s = ctx.quantize_int8(x)
    assert torch.equal(y, ctx.matmul_int8(a, s, w, w_scale, bias=bias, act="relu", out_dtype=dtype))


# ---- every kernel shape -------------------------------------------------------------------------------------------

KERNELS = ["1,64,1,1", "1,128,1,1", "1,256,1,1", "2,128,1,1", "2,256,1,1", "2,256,1,2", "1,64,2,1", "1,128,2,1", "1,128,4,1", "1,64,8,1", "1,128,8,1"]


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("kernel", KERNELS)
def test_ffn_on_every_kernel(ctx, monkeypatch, kernel, dtype):
    """CTA group, columns of a tile, slices of K and parts of a tile's rows as the variable says, wherever a product allows it."""
    monkeypatch.setenv("TFJSB_DENSE_SHAPE", kernel)
    for shape in ((200, 600, 328, 136), (37, 1100, 513, 260)):
        gate = "silu"
        x, wg, wu, wd, dy = block(40, *shape, dtype)
        want = [ref.gated_ffn(x, wg, wu, wd, gate), *ref.gated_ffn_gradients(x, wg, wu, wd, dy, gate)]
        bounds = ref.gated_ffn_bounds(x, wg, wu, wd, dy, gate)
        y, h, z = ctx.gated_ffn(x, wg, wu, wd, gate=gate, save=True)
        grads = ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy, gate=gate)
        ctx.check_device_status()
        for got, w, b, what in zip((y, *grads), want, bounds, ("y", "dx", "dw_gate", "dw_up", "dw_down")):
            check_ffn(got, w, b, dtype, (what, shape))


@pytest.mark.parametrize("kernel", ["2,256,1,1", "2,256,1,2"])
@pytest.mark.parametrize("shape", [(2600, 72, 5000, 40), (5130, 1300, 136, 1024)], ids=str)
def test_ffn_with_several_rounds_of_tiles(ctx, monkeypatch, kernel, shape):
    """More tiles than CTA pairs: accumulators in turn, a last round of few tiles whose parts go to pairs of their own, rows that end in the
    first part of a tile."""
    monkeypatch.setenv("TFJSB_DENSE_SHAPE", kernel)
    x, wg, wu, wd, dy = block(50, *shape, torch.bfloat16)
    want = [ref.gated_ffn(x, wg, wu, wd, "gelu"), *ref.gated_ffn_gradients(x, wg, wu, wd, dy, "gelu")]
    bounds = ref.gated_ffn_bounds(x, wg, wu, wd, dy, "gelu")
    y, h, z = ctx.gated_ffn(x, wg, wu, wd, gate="gelu", save=True)
    grads = ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy, gate="gelu")
    ctx.check_device_status()
    for got, w, b, what in zip((y, *grads), want, bounds, ("y", "dx", "dw_gate", "dw_up", "dw_down")):
        check_ffn(got, w, b, torch.bfloat16, what)


@pytest.mark.parametrize("kernel", KERNELS)
def test_int8_on_every_kernel(ctx, monkeypatch, kernel):
    """Whole numbers: the sums have to be exact on each."""
    monkeypatch.setenv("TFJSB_DENSE_SHAPE", kernel)
    for M, K, N in ((300, 4208, 328), (37, 2064, 513), (1400, 272, 8200)):
        gen = torch.Generator(device="cuda").manual_seed(M)
        a = torch.randint(-128, 128, (M, K), generator=gen, device="cuda").to(torch.int8)
        w = torch.randint(-128, 128, (N, K), generator=gen, device="cuda").to(torch.int8)
        one_m, one_n = torch.ones(M, device="cuda"), torch.ones(N, device="cuda")
        y = ctx.matmul_int8(a, one_m, w, one_n, out_dtype=torch.float32)
        ctx.check_device_status()
        assert torch.equal(y, (a.double() @ w.double().T).float())
