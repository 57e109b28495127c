"""More of the dense layers of transformer blocks on the GPU: what they promise beside their values, and kernels by name."""
import ctypes
import math
import threading

import pytest
import torch

import dense_reference as ref

pytestmark = pytest.mark.gpu

DTYPES = [torch.bfloat16, torch.float32]
ids = lambda v: str(v).replace("torch.", "") if isinstance(v, torch.dtype) else None  # noqa: E731


def normal(seed, shape, std=1.0, dtype=torch.float32):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(shape, generator=gen, device="cuda") * std).to(dtype)


def block(seed, t, d, f, o, dtype):
    return (normal(seed, (t, d), 1.0, dtype), normal(seed + 1, (d, f), d ** -0.5, dtype), normal(seed + 2, (d, f), d ** -0.5, dtype),
            normal(seed + 3, (f, o), f ** -0.5, dtype), normal(seed + 4, (t, o), 1.0, dtype))


def at_once(*work):
    """Each of `work` on a thread and a stream of its own; what they return."""
    results, errors = [None] * len(work), []
    start = threading.Barrier(len(work))

    def run(i):
        try:
            with torch.cuda.stream(torch.cuda.Stream()) as _:
                start.wait()
                results[i] = work[i]()
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001
            errors.append(e)

    torch.cuda.synchronize()
    threads = [threading.Thread(target=run, args=(i,)) for i in range(len(work))]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not errors, errors
    return results


# ---- several threads and streams ------------------------------------------------------------------------------------


def test_launches_of_several_threads_are_counted(ctx):
    x, wg, wu, wd, dy = block(1, 40, 72, 136, 72, torch.bfloat16)
    q, s = ctx.quantize_int8(normal(6, (40, 72)))

    def step():
        y, h, z = ctx.gated_ffn(x, wg, wu, wd, save=True)
        return (*ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, ctx.dropout(dy, 0.3, 1)), ctx.gated_ffn(x[:1], wg, wu, wd), ctx.dense_int8(x, q, s), y)

    before = ctx.launch_count
    want = step()
    each = ctx.launch_count - before
    before = ctx.launch_count
    got = at_once(*[lambda: [step() for _ in range(100)]] * 4)
    assert ctx.launch_count - before == 400 * each
    for steps in got:
        assert all(torch.equal(a, b) for one in steps for a, b in zip(one, want))
    ctx.check_device_status()


def test_different_layers_side_by_side(ctx):
    """Clusters, pairs and single CTAs of different products share the SMs."""
    cases = [block(10 + i, *shape, dtype) for i, (shape, dtype) in enumerate((
        ((600, 520, 1032, 520), torch.bfloat16), ((37, 2000, 456, 100), torch.bfloat16), ((300, 264, 520, 264), torch.float32)))]

    def train(case):
        x, wg, wu, wd, dy = case
        y, h, z = ctx.gated_ffn(x, wg, wu, wd, save=True)
        return (y, *ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy))

    want = [train(c) for c in cases]
    got = at_once(*[lambda c=c: [train(c) for _ in range(20)] for c in cases])
    for runs, expected in zip(got, want):
        assert all(torch.equal(a, b) for run in runs for a, b in zip(run, expected))
    ctx.check_device_status()


def test_messages_of_calls_that_fail_at_once(ctx, tfjsb):
    x, w, d = (torch.zeros(s, dtype=torch.bfloat16, device="cuda") for s in ((4, 16), (16, 32), (32, 16)))

    def failing(call, text):
        def run():
            for _ in range(2000):
                with pytest.raises(tfjsb.TfjsbError, match=text):
                    call()
        return run

    at_once(failing(lambda: ctx.gated_ffn(x, w, w, d, out=x), "overlaps x"), failing(lambda: ctx.dropout(x, 1.5, 1), "rate must be"),
            failing(lambda: ctx.dropout(x, 0.5, 1, noise_shape=(3, 16)), "each dimension of the mask"))


# ---- slopes of the gates, value by value ----------------------------------------------------------------------------


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("gate", ["silu", "gelu", "gelu_tanh", "sigmoid", "relu"])
def test_slopes_of_the_gates_far_out(ctx, gate, dtype):
    """One token whose x, u and gradient of h are 1 and whose g are the weights themselves: the gradient of w_gate is the slope, that of w_up the gate.

    g and what multiplies the slope are exact, so what is off is the functions': their arguments' rounding (half a step of v, which moves e^v by as
    much of itself, a few times; g^2 / 2 in place of v for the normal distribution) and a dozen operations, each half a step or an ulp of
    the terms that make the slope up.  bfloat16 rounds the gradient of g once more, and its exponential is off by 2 + 1.2 |v| ulps."""
    if dtype == torch.bfloat16 and gate == "gelu":
        pytest.skip("the gelu of bfloat16 results is good to 1e-7, not to a part of itself")
    reach = 8 if gate.startswith("gelu") else 40
    g = torch.arange(-reach * 16, reach * 16 + 1, device="cuda", dtype=torch.float64) / 16
    g = g.to(dtype).double().unique()  # 1/16 is finer than bfloat16 far out
    one = lambda *s: torch.ones(s, device="cuda", dtype=dtype)  # noqa: E731
    n = g.numel()
    x, wg, wu, wd = one(1, 1), g.to(dtype)[None].contiguous(), one(1, n), one(n, 1)
    _, h, z = ctx.gated_ffn(x, wg, wu, wd, gate=gate, save=True)
    _, slope, value, _ = ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, one(1, 1), gate=gate)
    ctx.check_device_status()
    a, want = ref.gate(gate, g)
    s = torch.special.expit
    if gate == "gelu":
        density, f = torch.exp(-g * g / 2) / math.sqrt(2 * math.pi), torch.special.erfc(-g / math.sqrt(2)) / 2
        # torch's ndtr is (1 + erf) / 2, which is good to 1e-16 and not to a part of itself: 1 % off at g = -7.8
        a, want = g * f, f + g * density
        v, terms = g * g, f + g.abs() * density
    elif gate == "gelu_tanh":
        v = math.sqrt(8 / math.pi) * (g + 0.044715 * g ** 3)
        a = g * s(v)  # tanh(v) + 1 has lost its bits far out
        factor = math.sqrt(8 / math.pi) * (1 + 3 * 0.044715 * g ** 2)
        want = s(v) + a * s(-v) * factor
        terms = s(v) + a.abs() * s(-v) * factor
    else:
        v = g
        terms = s(g) * (1 + g.abs() * s(-g)) if gate == "silu" else s(g) * s(-g) if gate == "sigmoid" else want
    off = (24 + 8 * v.abs()) * ref.FP32
    if dtype == torch.bfloat16:
        off = (64 + 16 * v.abs()) * ref.FP32
        bounds = off * terms + ref.BF16 * (want.abs() + off * terms), off * a.abs() + ref.BF16 * a.abs() * (1 + off)
    else:
        bounds = off * terms, off * a.abs()
    for got, right, bound, what in ((slope[0], want, bounds[0], "slope"), (value[0], a, bounds[1], "gate")):
        over = (got.double() - right).abs() - bound
        worst = over.argmax().item()
        assert over[worst].item() <= 0, (what, g[worst].item(), got[worst].item(), right[worst].item())


# ---- with and without what the gradient needs -----------------------------------------------------------------------


@pytest.mark.parametrize("tokens", [1, 2])
def test_a_token_or_two_without_a_gradient_are_rounded_once(ctx, tokens):
    """Sums of one term: g = x w_gate and u = x w_up are exact, gate(g) u and the product with w_down half a step of fp32 off each at most.  Then the call that
    keeps nothing rounds y to bfloat16, and the one that keeps h rounds h too."""
    columns = 4096
    x, wg, wu = normal(1, (tokens, 1), 1.0, torch.bfloat16), torch.ones(1, 1, dtype=torch.bfloat16, device="cuda"), normal(3, (1, 1), 1.0, torch.bfloat16)
    x = x.abs()  # on relu's linear side
    wd = normal(4, (1, columns), 1.0, torch.bfloat16)
    want = ref.gated_ffn(x, wg, wu, wd, "relu")
    few = ctx.gated_ffn(x, wg, wu, wd, gate="relu")
    kept, h, z = ctx.gated_ffn(x, wg, wu, wd, gate="relu", save=True)
    fp32 = 3 * ref.FP32
    assert ((few.double() - want).abs() <= (ref.BF16 + fp32) * want.abs()).all()
    assert ((kept.double() - want).abs() <= (2 * ref.BF16 + ref.BF16 ** 2 + 2 * fp32) * want.abs()).all()


@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_few_tokens_with_and_without_a_gradient(ctx, dtype):
    """The two forms against each other, and against the tokens' rows among more."""
    x, wg, wu, wd, dy = block(30, 12, 300, 520, 130, dtype)
    bound = ref.gated_ffn_bounds(x, wg, wu, wd, dy, "gelu")[0]
    all_of_them = ctx.gated_ffn(x, wg, wu, wd, gate="gelu")
    for tokens in range(1, 10):
        few, b = x[:tokens].contiguous(), bound[:tokens]
        alone, kept = ctx.gated_ffn(few, wg, wu, wd, gate="gelu").double(), ctx.gated_ffn(few, wg, wu, wd, gate="gelu", save=True)[0].double()
        assert ((alone - kept).abs() <= 2 * b).all() and ((alone - all_of_them[:tokens].double()).abs() <= 2 * b).all()


# ---- arguments ------------------------------------------------------------------------------------------------------


@pytest.mark.parametrize("call", ["dense_int8", "matmul_int8"])
def test_out_and_its_dtype_have_to_agree(ctx, call):
    x = normal(1, (5, 48))
    (w, sw), (a, sa) = ctx.quantize_int8(normal(2, (24, 48))), ctx.quantize_int8(x)
    run = (lambda **k: ctx.dense_int8(x, w, sw, **k)) if call == "dense_int8" else (lambda **k: ctx.matmul_int8(a, sa, w, sw, **k))
    assert run().dtype == (torch.float32 if call == "dense_int8" else torch.bfloat16)
    for given in DTYPES:
        want = run(out_dtype=given)
        assert want.dtype == given
        out = torch.empty_like(want)
        assert run(out=out) is out and torch.equal(out, want)
        assert torch.equal(run(out=torch.empty_like(want), out_dtype=given), want)
        other = DTYPES[1 - DTYPES.index(given)]
        before = ctx.launch_count
        with pytest.raises(TypeError, match="out_dtype"):
            run(out=out, out_dtype=other)
        with pytest.raises(TypeError, match="out must be a tensor"):
            run(out=out.tolist())
        assert ctx.launch_count == before


def test_errors_of_dropouts_gradient_name_its_arguments(ctx, tfjsb):
    dy = normal(1, (6, 10))
    buf = torch.zeros(80, device="cuda")
    for call, names in ((ctx.dropout, ("x", "out")), (ctx.dropout_backprop, ("dy", "dx"))):
        with pytest.raises(tfjsb.TfjsbError, match=f"that of {names[0]} or 1"):
            call(dy, 0.5, 1, noise_shape=(6, 2))
        with pytest.raises(tfjsb.TfjsbError, match=f"{names[1]} overlaps an input"):
            call(buf[:60], 0.5, 1, out=buf[4:64])
    assert torch.equal(ctx.dropout_backprop(dy, 0.5, 1, offset=7), ctx.dropout(dy, 0.5, 1, offset=7))
    assert torch.equal(ctx.dropout_backprop(dy, 0.5, 1, noise_shape=(6, 1), out=torch.empty_like(dy)), ctx.dropout(dy, 0.5, 1, noise_shape=(6, 1)))


def test_seeds_are_whole_numbers_of_any_kind(ctx):
    import numpy as np

    x = normal(1, (300,))
    want = ctx.dropout(x, 0.5, 3, offset=4)
    for seed, offset in ((3.0, 4), (3, 4.0), (np.int64(3), np.uint8(4)), (np.float32(3), 4), (torch.tensor(3), 4)):
        assert torch.equal(ctx.dropout(x, 0.5, seed, offset=offset), want)
        assert torch.equal(ctx.dropout_backprop(x, 0.5, seed, offset=offset), want)
    assert torch.equal(ctx.dropout(x, 0, True), x)
    for bad in (math.inf, -math.inf, math.nan, 1e30, 0.5, -1, 2 ** 64):
        with pytest.raises(ValueError, match="seed must be"):
            ctx.dropout(x, 0.5, bad)
        with pytest.raises(ValueError, match="offset must be"):
            ctx.dropout_backprop(x, 0.5, 1, offset=bad)


# ---- kernels by name ------------------------------------------------------------------------------------------------


def kernels(ctx, what):
    return [shape for name, shape in ctx.dense_kernels() if name == what]


def test_the_kernels_of_a_call_are_named(ctx, tfjsb):
    x, wg, wu, wd, dy = block(1, 40, 72, 136, 72, torch.bfloat16)
    y, h, z = ctx.gated_ffn(x, wg, wu, wd, save=True)
    assert [n for n, _ in ctx.dense_kernels()] == ["gated", "stored"]
    ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy)
    assert [n for n, _ in ctx.dense_kernels()] == ["gradient", "stored", "stored", "stored"]
    ctx.gated_ffn(x[:1], wg, wu, wd)
    assert ctx.dense_kernels() == []
    q, s = ctx.quantize_int8(normal(1, (200, 72)))
    ctx.dense_int8(x, q, s)
    assert [n for n, _ in ctx.dense_kernels()] == []  # small: one kernel on CUDA cores
    ctx.matmul_int8(*ctx.quantize_int8(x), q, s)
    assert [n for n, _ in ctx.dense_kernels()] == ["scaled"]
    short = ctypes.create_string_buffer(4)
    assert tfjsb.lib.tfjsb_dense_kernels(ctx._h, short, 4) == 0 and short.value == b"sca"
    assert tfjsb.lib.tfjsb_dense_kernels(ctx._h, None, 4) == tfjsb.lib.tfjsb_dense_kernels(None, short, 4) == 1


def check_block(ctx, shape, dtype, seed, gate="silu"):
    """Forward and gradients within their bounds; the kernels of both calls: (forward's, backward's)."""
    x, wg, wu, wd, dy = block(seed, *shape, dtype)
    y, h, z = ctx.gated_ffn(x, wg, wu, wd, gate=gate, save=True)
    forward = ctx.dense_kernels()
    grads = ctx.gated_ffn_backprop(x, wg, wu, wd, h, z, dy, gate=gate)
    backward = ctx.dense_kernels()
    ctx.check_device_status()
    want = [ref.gated_ffn(x, wg, wu, wd, gate), *ref.gated_ffn_gradients(x, wg, wu, wd, dy, gate)]
    for got, w, b, what in zip((y, *grads), want, ref.gated_ffn_bounds(x, wg, wu, wd, dy, gate), ("y", "dx", "dw_gate", "dw_up", "dw_down")):
        off = (got.double() - w).abs()
        assert got.dtype == dtype and torch.isfinite(got).all() and (off <= b).all(), (what, shape, (off - b).max().item())
        # in the norm: two independent roundings to bfloat16, or fp32 sums cut towards zero in segments of eight additions
        assert off.norm() <= (2.0 ** -8 if dtype == torch.bfloat16 else 2e-6) * w.norm(), (what, shape)
    assert [n for n, _ in forward] == ["gated", "stored"] and [n for n, _ in backward] == ["gradient", "stored", "stored", "stored"]
    return [k for _, k in forward], [k for _, k in backward]


LONG = 2520  # 40 k-blocks, the last one not whole: two to eight slices of four k-blocks or more, none without any
# products whose K is long: tokens, width, hidden, out width, and where they are among the six of check_block
SLICED = {"gated": ((150, LONG, 200, 72), [0]), "stored and dx": ((150, 200, LONG, 200), [1, 4]), "gradient": ((150, 72, 200, LONG), [2]),
          "weights": ((LONG, 100, 200, 200), [3, 5]), "few rows, gated": ((37, LONG, 200, 72), [0]), "few rows, stored": ((37, 100, LONG, 200), [1, 4]),
          "few rows, gradient": ((37, 72, 200, LONG), [2])}


@pytest.mark.parametrize("slices", [2, 3, 4, 5, 6, 7, 8])
@pytest.mark.parametrize("dtype,columns", [(torch.bfloat16, 64), (torch.bfloat16, 128), (torch.bfloat16, 256), (torch.float32, 128)], ids=str)
@pytest.mark.parametrize("what", list(SLICED))
def test_every_product_in_slices(ctx, monkeypatch, what, dtype, columns, slices):
    shape, places = SLICED[what]
    if columns == 64 and "gated" in what:
        pytest.skip("a gated tile of 64 columns has 32 of each weight, half a box")
    if columns == 256 and slices == 7 and what == "gated":
        pytest.skip("seven slices' sums of 128 rows of g and u have 196 KiB, more than the stages that they take the place of")
    kernel = f"1,{columns},{slices},1"
    monkeypatch.setenv("TFJSB_DENSE_SHAPE", kernel)
    forward, backward = check_block(ctx, shape, dtype, 500 + columns + slices)
    assert [(forward + backward)[i] for i in places] == [kernel] * len(places)


@pytest.mark.parametrize("kernel", ["1,64,1,1", "1,128,1,1", "1,256,1,1", "2,128,1,1", "2,256,1,1", "2,256,1,2"])
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
def test_every_product_on_every_unsliced_kernel(ctx, monkeypatch, kernel, dtype):
    """Fp32 products have tiles of 128 columns alone; tiles of 64 are not for the gated one."""
    if dtype == torch.float32 and kernel.split(",")[1] != "128":
        pytest.skip("fp32 products have 128 columns a tile")
    monkeypatch.setenv("TFJSB_DENSE_SHAPE", kernel)
    for shape in ((200, 600, 328, 136), (37, 1100, 513, 260)):
        forward, backward = check_block(ctx, shape, dtype, 600)
        assert (forward + backward)[1 if kernel.startswith("1,64") else 0:] == [kernel] * (5 if kernel.startswith("1,64") else 6)


@pytest.mark.parametrize("columns", [64, 128, 256])
@pytest.mark.parametrize("slices", [1, 2, 3, 4, 5, 6, 7, 8])
def test_int8_products_in_slices(ctx, monkeypatch, columns, slices):
    """Whole numbers: the sums have to be exact."""
    kernel = f"1,{columns},{slices},1"
    monkeypatch.setenv("TFJSB_DENSE_SHAPE", kernel)
    for M, K, N in ((150, 5040, 200), (37, 5056, 130)):  # 40 k-blocks of 128
        gen = torch.Generator(device="cuda").manual_seed(M + slices)
        a, w = (torch.randint(-128, 128, (rows, K), generator=gen, device="cuda").to(torch.int8) for rows in (M, N))
        y = ctx.matmul_int8(a, torch.ones(M, device="cuda"), w, torch.ones(N, device="cuda"), out_dtype=torch.float32)
        assert kernels(ctx, "scaled") == [kernel]
        ctx.check_device_status()
        assert torch.equal(y, (a.double() @ w.double().T).float())


# ---- several tiles a CTA --------------------------------------------------------------------------------------------

# Tokens, width, hidden, out width; which of the six products have 1.4 rounds of tiles or more on CTA pairs and on single CTAs.  264 and 328 are five and six
# k-blocks, three segments of two: a tile begins on the other accumulator than the one before it.
ROUNDS = [((2600, 264, 2300, 328), [0, 2]), ((2600, 2100, 264, 2100), [1, 4]), ((264, 2600, 2300, 2100), [3, 5])]


@pytest.mark.parametrize("kernel", ["1,128,1,1", "2,128,1,1"])
@pytest.mark.parametrize("dtype", DTYPES, ids=ids)
@pytest.mark.parametrize("shape,places", ROUNDS, ids=str)
def test_rounds_of_tiles(ctx, monkeypatch, shape, places, dtype, kernel):
    """Accumulators and segments of sums in turn from tile to tile, one tile's epilogue beside the next one's sums, for every product."""
    monkeypatch.setenv("TFJSB_DENSE_SHAPE", kernel)
    group = int(kernel[0])
    t, d, f, o = shape
    tiles = lambda m, n, columns=128: -(-m // (128 * group)) * -(-n // columns)  # noqa: E731
    # in the order of the two calls' products: gated, y; gradients of g and u, w_down, x, w_gate and w_up
    counts = [tiles(t, f, 64), tiles(t, o), tiles(t, f), tiles(f, o), tiles(t, d), 2 * tiles(d, f)]
    slots = torch.cuda.get_device_properties(0).multi_processor_count // group
    assert all(counts[i] >= 1.4 * slots for i in places), counts
    forward, backward = check_block(ctx, shape, dtype, 700, "gelu")
    assert forward + backward == [kernel] * 6


@pytest.mark.parametrize("shape", [(2048, 1024, 4096, 1024), (1999, 1000, 2600, 900)], ids=str)
def test_ordinary_fp32_blocks_of_several_rounds(ctx, shape):
    """The kernels that the call takes by itself."""
    check_block(ctx, shape, torch.float32, 800)


# ---- the longest sums -----------------------------------------------------------------------------------------------


def sparse(rows, columns, places, value):
    """Zeros but for `value` at `places`."""
    m = torch.zeros(rows, columns, dtype=torch.bfloat16, device="cuda")
    for r, c in places:
        m[r, c] = value
    return m


@pytest.mark.parametrize("what", ["width", "hidden"])
def test_sums_of_2_30_terms(ctx, what):
    """A handful of CTAs sum for half a second, the longest that a wait may take without progress: the epilogue waits for all of it, and the kernel after
    it, which begins on the other SMs, for its end.  All terms but a few are zero, so the sums are exact."""
    n, tokens, few = 2 ** 30, 3, 8
    at = [0, 1, 12345, n // 8 - 1, n // 8, n // 2 + 77, n - 65, n - 1]
    if what == "width":  # g = x w_gate
        x = sparse(tokens, n, [(t, k) for t in range(tokens) for k in at], 1.0)
        wg, wu = sparse(n, few, [(k, c) for k in at for c in range(few)], 1.0), sparse(n, few, [(at[-1], c) for c in range(few)], 1.0)
        wd = sparse(few, few, [(c, c) for c in range(few)], 0.5)
        y, want = ctx.gated_ffn(x, wg, wu, wd, gate="relu"), 0.5 * len(at)
    else:  # y = h w_down
        x = sparse(tokens, few, [(t, 0) for t in range(tokens)], 1.0)
        wg, wd = sparse(few, n, [(0, k) for k in at], 2.0), sparse(n, few, [(k, c) for k in at for c in range(few)], 1.0)
        wu = wg
        y, want = ctx.gated_ffn(x, wg, wu, wd, gate="relu"), 4.0 * len(at)
    ctx.check_device_status()
    assert ctx.dense_kernels()[0 if what == "width" else 1][1].split(",")[2] == "8"
    assert y.shape == (tokens, few) and (y == want).all(), y
    del x, wg, wu, wd
    torch.cuda.empty_cache()
