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


# ---- refusals -----------------------------------------------------------------------------------------------------


def bf16(*shape):
    return torch.zeros(shape, dtype=torch.bfloat16, device="cuda")


def test_ffn_refusals(ctx, tfjsb):
    x, w, d = bf16(4, 16), bf16(16, 32), bf16(32, 24)
    before = ctx.launch_count
    for bad in [(x.float(), w, w, d), (x, w.float(), w, d), (x, w, bf16(16, 40), d), (x, w, w, bf16(16, 24)), (x[:, ::2], w, w, d), (x, w.t(), w, d),
                (x.cpu(), w, w, d), (x.half(), w, w, d), (x, w[0], w, d), (None, w, w, d)]:
        with pytest.raises((TypeError, ValueError)):
            ctx.gated_ffn(*bad)
    with pytest.raises(ValueError, match="gate must be one of"):
        ctx.gated_ffn(x, w, w, d, gate="tanh")
    with pytest.raises(ValueError):
        ctx.gated_ffn(x, w, w, d, out=bf16(4, 16))
    with pytest.raises(tfjsb.TfjsbError) as e:
        ctx.gated_ffn(x, w, w, bf16(32, 16), out=x)  # aliases its input
    assert e.value.status_name == "INVALID_ARG" and "overlaps" in str(e.value)
    y, h, z = ctx.gated_ffn(x, w, w, d, save=True)
    before = ctx.launch_count
    with pytest.raises(ValueError):
        ctx.gated_ffn_backprop(x, w, w, d, h[:-16].contiguous(), z, y)
    with pytest.raises(ValueError):
        ctx.gated_ffn_backprop(x, w, w, d, h, z, bf16(4, 16))
    assert ctx.launch_count == before


def test_ffn_refusals_of_the_library(ctx, tfjsb):
    lib = tfjsb.lib
    f = tfjsb.Ffn(4, 16, 32, 24, 1, 0)
    x, w, d, y, buf = bf16(4, 16), bf16(16, 32), bf16(32, 24), bf16(4, 24), torch.zeros(1 << 16, dtype=torch.uint8, device="cuda")
    p = lambda t, o=0: t.data_ptr() + o  # noqa: E731

    def call(x=p(x), y=p(y), h=None, z=None, work=p(buf), size=1 << 16):
        return lib.tfjsb_gated_ffn(ctx._h, ctypes.byref(f), x, p(w), p(w), p(d), y, h, z, work, size, None)

    before = ctx.launch_count
    assert call(h=p(buf, 32768)) == 1          # h without z
    assert call(size=16) == 1                  # a workspace that is too small
    assert call(x=None) == 1 and call(work=None) == 1
    assert call(x=p(x, 2)) == 1                # not 16-byte aligned
    assert call(y=p(x)) == 1 and call(work=p(x)) == 1
    assert b"overlaps" in lib.tfjsb_last_error(ctx._h)
    f.gate = 9
    assert call() == 1
    f.gate, f.hidden = 0, 0
    assert call() == 2
    assert ctx.launch_count == before


def test_dropout_refusals(ctx, tfjsb):
    x = torch.ones(4, 6, device="cuda")
    before = ctx.launch_count
    for rate in (-0.1, 1.0, 1.5, math.nan, 1 - 2.0 ** -40):
        with pytest.raises(tfjsb.TfjsbError) as e:
            ctx.dropout(x, rate, 1)
        assert e.value.status_name == "INVALID_ARG"
    with pytest.raises(tfjsb.TfjsbError) as e:
        ctx.dropout(x, 0.5, 1, noise_shape=(4, 2))
    assert e.value.status_name == "SHAPE"
    for bad in [dict(noise_shape=(4,)), dict(residual=torch.ones(4, 5, device="cuda")), dict(residual=x.bfloat16()), dict(out=torch.ones(6, 4, device="cuda")),
                dict(seed=-1), dict(seed=2 ** 64), dict(offset=2 ** 64), dict(seed=1.5)]:
        with pytest.raises((TypeError, ValueError)):
            ctx.dropout(x, 0.5, **{"seed": 1, **bad})
    for t in (x.double(), x.t(), x.cpu(), torch.ones(1, 1, 1, 1, 1, device="cuda"), torch.tensor(1.0, device="cuda")):
        with pytest.raises((TypeError, ValueError)):
            ctx.dropout(t, 0.5, 1)
    buf = torch.zeros(40, device="cuda")
    with pytest.raises(tfjsb.TfjsbError) as e:
        ctx.dropout(buf[:24], 0.5, 1, out=buf[4:28])  # overlaps x without being it
    assert e.value.status_name == "INVALID_ARG"
    assert ctx.launch_count == before


def test_int8_refusals(ctx, tfjsb):
    i8 = lambda *s: torch.zeros(s, dtype=torch.int8, device="cuda")  # noqa: E731
    one = lambda n: torch.ones(n, device="cuda")  # noqa: E731
    before = ctx.launch_count
    for args in [(i8(4, 20), one(4), i8(8, 20), one(8)), (i8(1, 131088), one(1), i8(1, 131088), one(1))]:
        with pytest.raises(tfjsb.TfjsbError) as e:
            ctx.matmul_int8(*args)
        assert e.value.status_name == "UNSUPPORTED"
    for args in [(i8(4, 16), one(4), i8(8, 32), one(8)), (i8(4, 16), one(5), i8(8, 16), one(8)), (i8(4, 16).float(), one(4), i8(8, 16), one(8)),
                 (i8(4, 16), one(4).bfloat16(), i8(8, 16), one(8)), (i8(16, 4).t(), one(4), i8(8, 16), one(8))]:
        with pytest.raises((TypeError, ValueError)):
            ctx.matmul_int8(*args)
    with pytest.raises((TypeError, ValueError)):
        ctx.matmul_int8(i8(4, 16), one(4), i8(8, 16), one(8), bias=one(4))
    with pytest.raises((TypeError, ValueError)):
        ctx.matmul_int8(i8(4, 16), one(4), i8(8, 16), one(8), out_dtype=torch.float16)
    with pytest.raises((TypeError, ValueError)):
        ctx.dense_int8(one(40).reshape(2, 20), i8(8, 20), one(8))  # rows of weights are to be filled up to 32
    with pytest.raises((TypeError, ValueError)):
        ctx.quantize_int8(one(8))
    with pytest.raises(KeyError):
        ctx.dense_int8(one(32).reshape(2, 16), i8(8, 16), one(8), act="tanh")
    with pytest.raises(tfjsb.TfjsbError) as e:
        ctx.quantize_int8(torch.zeros(1, 131073, device="cuda"))
    assert e.value.status_name == "UNSUPPORTED"
    assert ctx.launch_count == before


# ---- values that are not finite, empty tensors, what lies behind ----------------------------------------------------


def test_a_value_that_is_not_finite_stays_in_its_row(ctx):
    x, w, w_scale = normal(1, (40, 200)), *ctx.quantize_int8(normal(2, (72, 200)))
    want = ctx.dense_int8(x, w, w_scale)
    for rows in (40, 1):
        bad = x[:rows].clone()
        for i, v in enumerate((math.nan, math.inf, -math.inf)[:rows]):
            bad[i, 17 * i + 3] = v
        got = ctx.dense_int8(bad, w, w_scale)
        assert torch.isnan(got[:3]).all() and torch.equal(got[3:], want[3:rows])
    q, scale = ctx.quantize_int8(torch.tensor([[math.nan, math.inf, 1.0], [1.0, -math.inf, 2.0], [0.0, -0.0, 0.0], [1e-38, 0.0, -1e-38], [3e38, -1e38, 0.0]], device="cuda"))
    assert math.isnan(scale[0]) and scale[1] == math.inf and scale[2] == 0 and not q[:3].any()
    assert q[3, :3].tolist() == [127, 0, -127] and q[4, :3].tolist() == [127, -42, 0]
    for dtype in DTYPES:
        for tokens in (1, 20):
            a, wg, wu, wd, dy = block(3, tokens, 40, 72, 24, dtype)
            y = ctx.gated_ffn(a, wg, wu, wd)
            a[tokens // 2, 5] = math.nan
            z = ctx.gated_ffn(a, wg, wu, wd)
            keep = torch.arange(tokens, device="cuda") != tokens // 2
            assert torch.isnan(z[tokens // 2]).all() and torch.equal(z[keep], y[keep])
        v = normal(4, (1000,), 1.0, dtype)
        v[::3] = math.nan
        v[1::3] = math.inf
        mask = ref.keep((1000,), 0.5, 9, 0, "cuda")
        d = ctx.dropout(v, 0.5, 9)
        assert (d[~mask] == 0).all() and torch.equal(torch.isfinite(d[mask]), torch.isfinite(v[mask]))


def test_empty_tensors(ctx):
    for dtype in DTYPES:
        x, wg, wu, wd, _ = block(1, 3, 16, 24, 8, dtype)
        y, h, z = ctx.gated_ffn(x[:0], wg, wu, wd, save=True)
        assert y.shape == (0, 8) and ctx.gated_ffn(x[:0], wg, wu, wd).shape == (0, 8)
        dx, *dw = ctx.gated_ffn_backprop(x[:0], wg, wu, wd, h, z, y)
        assert dx.shape == (0, 16) and all(not g.any() for g in dw)
        assert ctx.dropout(x[:0], 0.5, 1).shape == (0, 16)
        q, s = ctx.quantize_int8(x[:0])
        assert q.shape == (0, 16) and s.shape == (0,)
        assert ctx.dense_int8(x[:0], *ctx.quantize_int8(x)).shape == (0, 3)
    assert ctx.matmul_int8(q, s, *ctx.quantize_int8(x)).shape == (0, 3)


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("columns", [40, 37])
def test_rows_behind_the_last_stay(ctx, columns, dtype):
    """Results into the front of a larger buffer: what lies behind is not touched."""
    for rows in (1, 5, 130):
        x, wg, wu, wd, _ = block(rows, rows, 48, 72, columns, dtype)
        q, s = ctx.quantize_int8(normal(1, (columns, 48)))
        for call in (lambda out: ctx.gated_ffn(x, wg, wu, wd, out=out), lambda out: ctx.dense_int8(x, q, s, out=out)):
            buf = torch.full((rows + 40, columns), 7.0, dtype=dtype, device="cuda")
            assert call(buf[:rows]).data_ptr() == buf.data_ptr()
            assert (buf[rows:] == 7).all() and torch.equal(buf[:rows], call(None))
        buf = torch.full((rows + 40, columns), 7.0, dtype=dtype, device="cuda")
        v = normal(2, (rows, columns), 1.0, dtype)
        ctx.dropout(v, 0.3, 4, out=buf[:rows])
        assert (buf[rows:] == 7).all() and torch.equal(buf[:rows], ctx.dropout(v, 0.3, 4))


def test_dropout_in_place(ctx):
    for dtype in DTYPES:
        x, r = normal(1, (33, 70), 1.0, dtype), normal(2, (33, 70), 1.0, dtype)
        want = ctx.dropout(x, 0.4, 11, residual=r)
        assert torch.equal(ctx.dropout(x.clone(), 0.4, 11, residual=r, out=(a := r.clone())), want) and torch.equal(a, want)
        b = x.clone()
        assert torch.equal(ctx.dropout(b, 0.4, 11, residual=r, out=b), want)


def test_gradients_that_are_not_wanted(ctx):
    for dtype in DTYPES:
        x, wg, wu, wd, dy = block(5, 70, 48, 100, 24, dtype)
        y, h, z = ctx.gated_ffn(x, wg, wu, wd, save=True)
        every = ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy)
        for want in range(16):
            flags = [bool(want >> i & 1) for i in range(4)]
            got = ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy, want=flags)
            for g, e, f in zip(got, every, flags):
                assert (g is None) if not f else torch.equal(g, e)


# ---- together, twice, elsewhere -------------------------------------------------------------------------------------


def training_step(ctx, x, wg, wu, wd, dy, seed):
    """A block's dense half: the feed-forward block, dropout of its output onto the residual stream, and back."""
    y, h, z = ctx.gated_ffn(x, wg, wu, wd, save=True)
    out = ctx.dropout(y, 0.1, seed, offset=3, residual=x)
    d = ctx.dropout_backprop(dy, 0.1, seed, offset=3)
    grads = ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, d)
    dx = ctx.dropout(grads[0], 0.0, 0, residual=dy)  # the residual's own gradient joins
    return out, dx, *grads[1:]


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_a_block_in_training(ctx, dtype):
    x, wg, wu, wd, dy = block(60, 300, 264, 520, 264, dtype)
    out, dx, *dw = training_step(ctx, x, wg, wu, wd, dy, 77)
    mask = ref.keep(x.shape, 0.1, 77, 3, "cuda")
    y = ref.gated_ffn(x, wg, wu, wd, "silu")
    d = ref.dropout(dy, 0.1, mask)
    wdx, *wdw = ref.gated_ffn_gradients(x, wg, wu, wd, d, "silu")
    # y is rounded once more on its way (to the storage type), d once; each rounding at most half a step of its value, so in the norm
    # three independent ones are 2^-8 in the mean (bfloat16), and 2e-6 as for the block alone (fp32)
    for got, want in zip((out, dx, *dw), (ref.dropout(y, 0.1, mask, x), wdx + dy.double(), *wdw)):
        rel = ((got.double() - want).norm() / want.norm()).item()
        assert rel <= (2.0 ** -8 if dtype == torch.bfloat16 else 2e-6), rel


def test_a_block_in_serving(ctx):
    """The same block on 8-bit weights, a token at a time and many: three dense layers and a product, against whole numbers in 64 bits."""
    x, wg, wu, wd, _ = block(61, 33, 256, 640, 256, torch.float32)
    layers = [ctx.quantize_int8(w.t().contiguous()) for w in (wg, wu, wd)]
    for rows in (1, 33):
        a = x[:rows].contiguous()
        g, u = (ctx.dense_int8(a, *layers[i], act="relu" if i == 0 else "none") for i in range(2))
        h = ctx.binary("mul", g, u)
        y = ctx.dense_int8(h, *layers[2])

        def dense(v, layer, act):
            q, s = ref.quantize(v)
            return ref.int8_product(q, s.float(), layer[0][:, :v.shape[1]], layer[1], None, act)[0].float()

        hw = dense(a, layers[0], "relu") * dense(a, layers[1], "none")
        # values of h next to the middle between two integers may be quantised to either, since h differs in its last bits: one step of
        # 1 / 127 of the row's largest value in some of 640 terms
        want = dense(hw, layers[2], "none")
        assert torch.allclose(h, hw, rtol=1e-6, atol=1e-7)
        assert ((y - want).norm() / want.norm()).item() <= 1e-3
        # and 8 bits are good for what they are good for
        exact = (torch.relu(a.double() @ wg.double()) * (a.double() @ wu.double())) @ wd.double()
        assert ((y.double() - exact).norm() / exact.norm()).item() <= 0.05


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_the_same_call_gives_the_same_bits(ctx, dtype):
    for shape in ((1, 100, 300, 50), (3, 512, 1024, 512), (70, 1000, 264, 1000), (300, 256, 520, 264)):
        x, wg, wu, wd, dy = block(9, *shape, dtype)
        q, s = ctx.quantize_int8(normal(1, (264, shape[1])))

        def everything():
            y, h, z = ctx.gated_ffn(x, wg, wu, wd, save=True)
            return (y, ctx.gated_ffn(x, wg, wu, wd), *ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy), ctx.dense_int8(x, q, s))

        first = everything()
        for _ in range(5):
            assert all(torch.equal(a, b) for a, b in zip(everything(), first))


def test_on_another_stream_and_after_work_on_it(ctx):
    x, wg, wu, wd, dy = block(62, 200, 264, 520, 264, torch.bfloat16)
    want = training_step(ctx, x, wg, wu, wd, dy, 5)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    big = torch.randn(4096, 4096, device="cuda")
    with torch.cuda.stream(side):
        for _ in range(5):
            big = big @ big * 1e-2
        late = x + 0 * big[:200, :264].to(x.dtype).nan_to_num(0, 0, 0)  # written at the end of that work
        got = training_step(ctx, late, wg, wu, wd, dy, 5)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_two_captured_graphs_and_eager_calls_between_them(ctx, dtype):
    """Each graph has its own workspaces; replays see what the inputs hold then."""
    sets = [list(block(63 + 10 * i, 70, 264, 520, 264, dtype)) for i in range(2)]
    layers = ctx.quantize_int8(normal(1, (40, 264)))

    def step(s):
        return (*training_step(ctx, *s, 5), ctx.dense_int8(s[0], *layers), ctx.gated_ffn(s[0][:1], *s[1:4]))

    for s in sets:
        step(s)
    torch.cuda.synchronize()
    graphs, outs = [], []
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(step(s))
        graphs.append(g)
    for turn in range(3):
        for s in sets:
            s[0].copy_(normal(100 + turn, s[0].shape, 1.0, dtype))
            s[4].copy_(normal(200 + turn, s[4].shape, 1.0, dtype))
        for i in (0, 1, 0):
            graphs[i].replay()
            step(sets[1 - i])
        torch.cuda.synchronize()
        for s, o in zip(sets, outs):
            assert all(torch.equal(a, b) for a, b in zip(step(s), o))
    ctx.check_device_status()


@pytest.mark.parametrize("gate", GATES)
def test_gradients_against_differences(ctx, gate):
    """The kernels' gradients against central differences of the 64-bit forward pass along random directions."""
    x, wg, wu, wd, dy = block(64, 24, 40, 56, 32, torch.float32)
    y, h, z = ctx.gated_ffn(x, wg, wu, wd, gate=gate, save=True)
    grads = ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy, gate=gate)
    inputs = [t.double() for t in (x, wg, wu, wd)]
    loss = lambda v: (ref.gated_ffn(*v, gate) * dy.double()).sum().item()  # noqa: E731
    for i, g in enumerate(grads):
        direction = normal(70 + i, inputs[i].shape).double()
        e = 1e-6
        ends = [loss([t + (s * e * direction if j == i else 0) for j, t in enumerate(inputs)]) for s in (1, -1)]
        slope = (ends[0] - ends[1]) / (2 * e)
        got = (g.double() * direction).sum().item()
        # differences are good to 1e-6 where no relu changes sides within them; the gradients to 2e-6 of their norm
        scale = (g.double().norm() * direction.norm()).item()
        assert abs(got - slope) <= 2e-5 * scale, (i, got, slope)


# ---- more than 2^31 elements ----------------------------------------------------------------------------------------


def test_dropout_of_more_than_2_31_elements(ctx):
    n, seed = 2 ** 31 + 4099, 12345
    x = torch.ones(n, dtype=torch.bfloat16, device="cuda")
    y = ctx.dropout(x, 0.5, seed, offset=1)
    for first in (0, 2 ** 31 - 2000, n - 4000):
        mask = ref.words(first, 4000, seed, 1, "cuda") >= 2 ** 31
        assert torch.equal(y[first:first + 4000] == 2, mask)
    y = ctx.dropout(x[: 2 ** 31 + 4096].view(-1, 4096), 0.5, seed, noise_shape=(2 ** 19 + 1, 1))
    rows = torch.tensor([0, 1, 2 ** 19 - 1, 2 ** 19], device="cuda")
    mask = ref.words(0, 2 ** 19 + 1, seed, 0, "cuda") >= 2 ** 31
    assert torch.equal((y[rows] == 2).all(1), mask[rows]) and torch.equal((y[rows] == 0).all(1), ~mask[rows])


def test_ffn_whose_hidden_values_are_more_than_2_31(ctx):
    t, d, f = 66000, 64, 32768
    x, wg, wu, wd, dy = block(80, t, d, f, d, torch.bfloat16)
    y, h, z = ctx.gated_ffn(x, wg, wu, wd, save=True)
    dx, _, _, _ = ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy, want=(True, False, False, False))
    ctx.check_device_status()
    for rows in (slice(0, 40), slice(65530, 65600), slice(t - 40, t)):
        args = (x[rows], wg, wu, wd)
        for got, want in ((y[rows], ref.gated_ffn(*args, "silu")), (dx[rows], ref.gated_ffn_gradients(*args, dy[rows], "silu")[0])):
            assert ((got.double() - want).norm() / want.norm()).item() <= 2.0 ** -8


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("gate", ["silu", "gelu", "gelu_tanh", "relu"])
def test_projections_that_are_enormous(ctx, gate, dtype):
    """g of 10^20, whose square is no fp32 number: the gates are g or 0 there, their slopes 1 or 0."""
    x, wg, wu, wd, dy = block(90, 50, 72, 136, 40, dtype)
    x, wu = x * 1e20, wu * 1e-20
    y, h, z = ctx.gated_ffn(x, wg, wu, wd, gate=gate, save=True)
    grads = ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy, gate=gate)
    for i, (got, want) in enumerate(zip((y, *grads), (ref.gated_ffn(x, wg, wu, wd, gate), *ref.gated_ffn_gradients(x, wg, wu, wd, dy, gate)))):
        if i == 3:  # dw_up = x^T du, du = dh gate(g): terms of 10^20 times 10^20, which neither type has numbers for
            assert (want.abs() > 3.4e38).any()
            continue
        assert torch.isfinite(got).all()
        assert ((got.double() - want).norm() / want.norm()).item() <= (2.0 ** -8 if dtype == torch.bfloat16 else 2e-6)


def test_what_was_saved_is_checked(ctx):
    x, wg, wu, wd, dy = block(91, 20, 16, 40, 24, torch.bfloat16)
    y, h, z = ctx.gated_ffn(x, wg, wu, wd, save=True)
    before = ctx.launch_count
    for bad_h, bad_z in [(h[:1].expand(h.shape), z), (h, z[:1].expand(z.shape)), (torch.stack((h, h), 1)[:, 0], z), (h.cpu(), z), (h.view(torch.int8), z), (z, h)]:
        with pytest.raises(ValueError):
            ctx.gated_ffn_backprop(x, wg, wu, wd, bad_h, bad_z, dy)
    for want in ((), (True,) * 3, (True,) * 5):
        with pytest.raises(ValueError):
            ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy, want=want)
    assert ctx.launch_count == before


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("columns,slices", [(c, s) for c in (64, 128, 256) for s in (3, 5, 6, 7)], ids=str)
def test_slices_whose_shares_differ(ctx, monkeypatch, columns, slices, dtype):
    """K cut in numbers that do not divide a tile's columns: some CTAs finish fewer of them, or none."""
    monkeypatch.setenv("TFJSB_DENSE_SHAPE", f"1,{columns},{slices},1")
    for shape in ((37, 2000, 456, 100), (130, 1900, 250, 72), (250, 328, 3000, 136)):
        x, wg, wu, wd, dy = block(400 + columns + slices, *shape, dtype)
        y, h, z = ctx.gated_ffn(x, wg, wu, wd, save=True)
        grads = ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy)
        ctx.check_device_status()
        want = [ref.gated_ffn(x, wg, wu, wd, "silu"), *ref.gated_ffn_gradients(x, wg, wu, wd, dy, "silu")]
        bounds = ref.gated_ffn_bounds(x, wg, wu, wd, dy, "silu")
        for got, w, b, what in zip((y, *grads), want, bounds, ("y", "dx", "dw_gate", "dw_up", "dw_down")):
            check_ffn(got, w, b, dtype, what)
    if dtype == torch.float32:
        q, s = ctx.quantize_int8(normal(1, (200, 5000)))
        a, sa = ctx.quantize_int8(normal(2, (70, 5000)))
        want, bound = ref.int8_product(a, sa, q, s, None, "none")
        assert ((ctx.matmul_int8(a, sa, q, s, out_dtype=torch.float32).double() - want).abs() <= bound).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape", [(2, 5, 17), (7, 1930, 36), (31, 410, 106), (64, 90, 2047), (300, 11, 33), (2000, 5, 100), (12000, 1, 16), (3, 3, 131072)], ids=str)
def test_int8_layers_of_one_kernel(ctx, shape, dtype):
    """Small layers quantise their rows and multiply them in one kernel: the same bits as the two calls."""
    m, n, k = shape
    x, bias = normal(1, (m, k), 1.0, dtype), normal(2, (n,))
    w, w_scale = ctx.quantize_int8(normal(3, (n, k)))
    q, scale = ctx.quantize_int8(x)
    before = ctx.launch_count
    y = ctx.dense_int8(x, w, w_scale, bias=bias, act="relu", out_dtype=torch.float32)
    assert ctx.launch_count == before + (1 if m * n <= 26000000 // (k + 2048) else 2)  # 31 x 410 x 106 is just beyond
    assert torch.equal(y, ctx.matmul_int8(q, scale, w, w_scale, bias=bias, act="relu", out_dtype=torch.float32))
    want, bound = ref.int8_product(q, scale, w, w_scale, bias, "relu")
    assert ((y.double() - want).abs() <= bound).all()


def test_two_threads_on_two_streams(ctx):
    """One context: calls share no memory, so two threads may make them at once."""
    import threading

    x, wg, wu, wd, dy = block(95, 100, 256, 520, 256, torch.bfloat16)
    want = training_step(ctx, x, wg, wu, wd, dy, 5)
    torch.cuda.synchronize()
    results = [[], []]

    def work(i):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(20):
                results[i].append(training_step(ctx, x, wg, wu, wd, dy, 5))
        stream.synchronize()

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert len(results[0]) == len(results[1]) == 20
    assert all(torch.equal(a, b) for r in results for got in r for a, b in zip(got, want))
