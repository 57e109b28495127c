"""Pins of the 64-bit statements that the dense layers are tested against (CPU)."""
import math

import pytest
import torch

import dense_reference as ref


@pytest.mark.parametrize("counter,key,want", [
    # known answers published with the generator
    ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
    ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
    ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1)),
])
def test_philox_known_answers(counter, key, want):
    assert tuple(ref.philox(torch.tensor(counter), key).tolist()) == want


def test_words_are_one_stream_however_it_is_cut():
    all_of_it = ref.words(0, 103, 12345678901234567890, 2 ** 40 + 3)
    for first, count in ((0, 1), (1, 7), (4, 4), (50, 53), (102, 1)):
        assert torch.equal(ref.words(first, count, 12345678901234567890, 2 ** 40 + 3), all_of_it[first:first + count])
    assert not torch.equal(all_of_it, ref.words(0, 103, 12345678901234567890, 3))


@pytest.mark.parametrize("rate", [0.0, 0.1, 0.5, 0.9])
def test_the_share_that_is_kept(rate):
    n = 200_000
    kept = ref.keep((n,), rate, 7, 0).double().mean().item()
    assert abs(kept - (1 - rate)) <= 5 * math.sqrt(max(rate * (1 - rate), 1e-12) / n)


@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh", "sigmoid", "relu"])
def test_gates_against_torch_and_their_slopes_against_differences(name):
    g = torch.linspace(-6, 6, 1001, dtype=torch.float64)
    f = torch.nn.functional
    theirs = {"silu": f.silu, "gelu": f.gelu, "gelu_tanh": lambda v: f.gelu(v, approximate="tanh"), "sigmoid": torch.sigmoid, "relu": torch.relu}[name]
    a, slope = ref.gate(name, g)
    assert torch.allclose(a, theirs(g), rtol=1e-12, atol=1e-14)
    away = g.abs() > 1e-3
    d = (ref.gate(name, g + 1e-5)[0] - ref.gate(name, g - 1e-5)[0]) / 2e-5
    assert torch.allclose(slope[away], d[away], rtol=1e-6, atol=1e-8)


@pytest.mark.parametrize("name", ["silu", "gelu", "gelu_tanh", "sigmoid", "relu"])
def test_gradients_against_autograd(name):
    gen = torch.Generator().manual_seed(3)
    x, wg, wu, wd, dy = (torch.randn(s, generator=gen, dtype=torch.float64) for s in ((5, 7), (7, 9), (7, 9), (9, 4), (5, 4)))
    leaves = [t.clone().requires_grad_() for t in (x, wg, wu, wd)]
    ref.gated_ffn(*leaves, name).backward(dy)
    for got, leaf in zip(ref.gated_ffn_gradients(x, wg, wu, wd, dy, name), leaves):
        assert torch.allclose(got, leaf.grad, rtol=1e-10, atol=1e-12)


def test_quantized_rows():
    x = torch.tensor([[1.0, 0.5, -0.25, 0.0], [0.0, 0.0, 0.0, 0.0], [-127.0, 63.5, 62.5, 0.5]])
    q, scale = ref.quantize(x)
    assert q.tolist() == [[127, 64, -32, 0], [0, 0, 0, 0], [-127, 64, 62, 0]]  # 63.5, 31.75, halves to even
    assert torch.equal(scale, torch.tensor([1 / 127, 0.0, 1.0], dtype=torch.float64))
    bad = torch.tensor([[1.0, math.inf], [math.nan, 2.0]])
    q, scale = ref.quantize(bad)
    assert q.abs().sum() == 0 and scale[0] == math.inf and math.isnan(scale[1])
