"""CPU: the oracles of dropout and of the gated feed-forward block against published vectors, torch's autograd and
differences."""
import math

import numpy as np
import pytest
import torch

from oracle import dropout_numpy as dn
from oracle import gated_ffn as gf


@pytest.mark.parametrize("counter,key,want", [
    # known answers published with the generator
    ([0, 0, 0, 0], [0, 0], [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]),
    ([0xFFFFFFFF] * 4, [0xFFFFFFFF] * 2, [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]),
    ([0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344], [0xA4093822, 0x299F31D0],
     [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]),
])
def test_generator_gives_the_published_words(counter, key, want):
    assert [int(w) for w in dn.philox4x32_10(counter, key)] == want


def test_lanes_are_the_halves_of_the_blocks_words():
    seed, seq = 0x123456789ABCDEF, 0xFEDCBA987654321
    got = dn.lanes(3, 21, seed, seq)
    for r in range(3):
        for c in range(21):
            w = dn.philox4x32_10([c // 8, r, seq & 0xFFFFFFFF, seq >> 32], [seed & 0xFFFFFFFF, seed >> 32])
            assert got[r, c] == (int(w[(c % 8) // 2]) >> (16 * (c % 2))) & 0xFFFF


def test_drop_rate_and_mean():
    n = 1 << 18
    for p in (0.1, 0.5, 0.9):
        keep = dn.keep_mask(64, n // 64, p, 7, 9)
        # five standard deviations of a binomial count
        assert abs(keep.mean() - (1 - p)) < 5 * math.sqrt(p * (1 - p) / n) + 1 / 65536
        assert abs(dn.scale(p) * (1 - dn.threshold(p) / 65536) - 1) < 1e-12
    assert dn.keep_mask(4, 100, 0.0, 1, 2).all() and not dn.keep_mask(4, 100, 1.0, 1, 2).any()
    assert dn.scale(1.0) == 0.0


def make(m, k, f, seed):
    g = torch.Generator().manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, dtype=torch.float64)
    return rnd(m, k), rnd(f, k) / math.sqrt(k), rnd(f, k) / math.sqrt(k), rnd(m, f)


@pytest.mark.parametrize("name", ["relu", "silu", "gelu"])
@pytest.mark.parametrize("p", [0.0, 0.3])
def test_gradients_are_those_of_autograd_and_of_differences(name, p):
    x, wg, wu, dh = make(5, 7, 9, 11)
    x32, wg32, wu32, dh32 = (t.float() for t in (x, wg, wu, dh))
    x, wg, wu, dh = (t.double() for t in (x32, wg32, wu32, dh32))
    got = gf.backward(x32, wg32, wu32, dh32, name, p, 5, 6).value
    leaves = [t.clone().requires_grad_() for t in (x, wg, wu)]
    gate = leaves[0] @ leaves[1].t()
    a = {"relu": torch.relu, "silu": torch.nn.functional.silu, "gelu": torch.nn.functional.gelu}[name](gate)
    factor = torch.from_numpy(dn.keep_mask(5, 9, p, 5, 6)).double() * dn.scale(p)
    h = a * (leaves[0] @ leaves[2].t()) * factor
    h.backward(dh)
    assert torch.allclose(h.detach(), gf.forward(x32, wg32, wu32, name, p, 5, 6).value["h"], rtol=1e-12, atol=1e-14)
    for t, n in zip(leaves, ("dx", "dwg", "dwu")):
        assert torch.allclose(t.grad, got[n], rtol=1e-11, atol=1e-13)

    def loss(x, wg, wu):
        a, _ = gf.act(x @ wg.t(), name)
        return float((a * (x @ wu.t()) * factor * dh).sum())

    g = torch.Generator().manual_seed(3)
    step = 1e-5
    for i, n in enumerate(("dx", "dwg", "dwu")):
        v = torch.randn(got[n].shape, generator=g, dtype=torch.float64)
        args = [x, wg, wu]
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + step * v, args[i] - step * v
        diff = (loss(*up) - loss(*down)) / (2 * step)
        # a central difference of step 1e-5 leaves a third-order term of about 1e-10 and cancellation of about 1e-10
        assert abs(diff - float((got[n] * v).sum())) < 1e-7
