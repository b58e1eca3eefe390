"""Pins of the oracles behind the 8-bit blocks and the sampler: hand-worked cases, invariants, torch's own e4m3."""
import numpy as np
import pytest
import torch

from oracle import blocks as OB
from oracle import sampling as OS


def test_e4m3_rounding_matches_torch_and_its_own_values():
    rng = np.random.default_rng(0)
    a = np.concatenate([rng.normal(size=4000) * 10.0 ** rng.integers(-4, 3, 4000), OB.E4M3, -OB.E4M3,
                        (OB.E4M3[1:] + OB.E4M3[:-1]) / 2]).astype(np.float32)
    a = a[np.abs(a) <= 448]
    want = torch.from_numpy(a).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(OB.to_e4m3(a), want)
    assert np.array_equal(OB.from_e4m3(want), torch.from_numpy(want).view(torch.float8_e4m3fn).double().numpy())
    assert OB.E4M3[-1] == 448 and OB.to_e4m3([1e9, -1e9]).tolist() == [0x7e, 0xfe]


def test_rms_norm_and_activations_by_hand():
    n = OB.rms_norm([[3.0, 4.0]], [1.0, 2.0], 0.0)
    assert np.allclose(n, [[3 / np.sqrt(12.5), 8 / np.sqrt(12.5)]])
    assert OB.row_scales(np.zeros((1, 3)))[0] == 2.0 ** -100 / 448
    v = np.array([-1000.0, -1.0, 0.0, 1.0, 1000.0])
    assert np.allclose(OB.activation(v, "relu"), [0, 0, 0, 1, 1000])
    assert np.allclose(OB.activation(v, "gelu"), [0, -0.15865525393145707, 0, 0.8413447460685429, 1000])
    assert np.allclose(OB.activation(v, "silu"), [0, -0.2689414213699951, 0, 0.7310585786300049, 1000])
    assert np.allclose(OB.activation(v, "gelu_tanh"), [0, -0.15880800939172324, 0, 0.8411919906082768, 1000])


def test_sampling_by_hand():
    x = np.log([0.1, 0.4, 0.2, 0.3])
    keep = lambda **a: OS.kept_tokens(x, None, **({"T": 1.0, "k": 0, "p": 1.0, "q": 0.0} | a))[0].tolist()  # noqa: E731
    assert keep() == [0, 1, 2, 3]
    assert keep(k=2) == [1, 3]
    assert keep(p=0.39) == [1] and keep(p=0.5) == [1, 3] and keep(p=0.75) == [1, 2, 3]
    assert keep(k=2, p=0.5) == [1]                          # 0.4 of 0.7 reaches half
    assert keep(q=0.6) == [1, 3] and keep(q=5.0) == [1]
    assert keep(T=0.0) == [1]
    assert keep(p=0.0) == [1]
    tok, logq = OS.sample_row(x, None, 1.0, 0, 1.0, 0.0, [0.0, 0.05, 0.1000001, 0.49, 0.51, 0.69, 0.71, 0.9999999])
    assert tok.tolist() == [0, 0, 1, 1, 2, 2, 3, 3]
    assert np.allclose(logq, np.log([0.1, 0.1, 0.4, 0.4, 0.2, 0.2, 0.3, 0.3]))
    # ties go to the lower token, masked tokens have no say
    y = np.array([1.0, np.nan, 1.0, 1.0, -np.inf])
    allow = np.array([1, 0, 1, 1, 1], bool)
    assert OS.kept_tokens(y, allow, 1.0, 2, 1.0, 0.0)[0].tolist() == [0, 2]
    assert OS.kept_tokens(y, np.zeros(5, bool), 1.0, 0, 1.0, 0.0) is None
    assert OS.kept_tokens([0.0, np.inf, np.inf], None, 1.0, 0, 1.0, 0.0)[0].tolist() == [1, 2]


@pytest.mark.parametrize("T,k,p,q", [(1.0, 0, 1.0, 0.0), (0.7, 5, 0.8, 0.0), (1.4, 0, 0.6, 0.05)])
def test_even_numbers_draw_the_distribution(T, k, p, q):
    rng = np.random.default_rng(1)
    x = rng.normal(size=40) * 2
    tokens, w = OS.kept_tokens(x, None, T, k, p, q)
    u = (np.arange(20000) + 0.5) / 20000
    got = np.bincount(OS.sample_row(x, None, T, k, p, q, u)[0], minlength=40) / u.size
    want = np.zeros(40)
    want[tokens] = w / w.sum()
    assert np.abs(got - want).max() <= 1 / u.size            # an even grid misses an interval's length by at most one step
