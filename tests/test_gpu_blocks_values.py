"""The values of the blocks' operators, one by one.

Products here are exact (a row of x times a unit row of w), so an activation's argument is the bf16 number itself."""
import numpy as np
import pytest
import torch

from oracle import blocks as OB

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn


@pytest.fixture(scope="module")
def api():
    from paper_2608_00938_b200 import api as _api
    return _api


def values():
    """Every bf16 number of 2^-20 <= |v| <= 64."""
    v = torch.arange(1 << 16, dtype=torch.int32).to(torch.int16).view(BF).float()
    return v[torch.isfinite(v) & (v.abs() <= 64) & (v.abs() >= 2.0 ** -20)].to(BF)


def activated(api, v, act, kind, M):
    """act of each of v through the product: rows of up to M values (one a row), column 0 and a later one."""
    outs = []
    for i in range(0, v.numel(), M):
        part = v[i:i + M]
        x = torch.zeros(M, 64, device=DEV, dtype=BF)
        x[:part.numel(), 5] = part.to(DEV)
        w = torch.zeros(256, 64, device=DEV, dtype=BF)
        w[:, 5] = 1.0
        y = torch.empty(M, 256, device=DEV, dtype=kind)
        api.grace_linear_act(x, w, y, act=act)
        assert torch.equal(y[:, 0], y[:, 201])
        outs.append(y[:part.numel(), 0].double().cpu())
    return torch.cat(outs).numpy()


@pytest.mark.parametrize("M", [100, 4096])
def test_gelu_to_bf16_has_one_rounding(api, M):
    """v Phi(v) = max(v, 0) - a Phi(-a), a = |v|.  Phi(-a) is 2 to a polynomial within 6e-6 of it up to a = 9, whose fp32 value is off by
    2^-19 in the last step (it is below 64) and by 9 times half a step of 8 in the one before: 6e-6 of 2^P, and 2^-22 for the exponential: 2^-16
    in all.  Beyond a = 9 what is left is below 2^-54.  Then one rounding to bf16."""
    v = values()
    x = v.double().numpy()
    ref = OB.activation(x, "gelu")
    tail = np.abs(np.maximum(x, 0) - ref)                     # a Phi(-a)
    off = 2.0 ** -16 * tail + 2.0 ** -24 * np.abs(ref) + 2.0 ** -54
    got = activated(api, v, "gelu", BF, M)
    lo, hi = (torch.from_numpy(t).float().to(BF).double().numpy() for t in (ref - off, ref + off))   # (2^-24: this conversion's own)
    wrong = (got < lo) | (got > hi)
    assert not wrong.any(), (int(wrong.sum()), x[wrong][:5], got[wrong][:5], ref[wrong][:5])


@pytest.mark.parametrize("M", [100, 4096])
def test_gelu_to_fp32_keeps_its_tail(api, M):
    """Phi(-a) as 2 to a polynomial of degree 12: fit, fp32 Horner steps and exponential within 2^-20.3 up to a = 2, 2^-18.5 up to 5 and 2^-15.7 up
    to 8.6, beyond which what is left is below 2^-54.  Then a product and a sum in one rounding."""
    v = values()
    x = v.double().numpy()
    ref = OB.activation(x, "gelu")
    a = np.abs(x)
    tail = np.abs(np.maximum(x, 0) - ref)
    off = np.where(a <= 2, 2.0 ** -20.3, np.where(a <= 5, 2.0 ** -18.5, 2.0 ** -15.7)) * tail + np.where(a > 8.5, 2.0 ** -54, 0.0)
    err = np.abs(activated(api, v, "gelu", F32, M) - ref)
    bound = off + 2.0 ** -24 * (np.abs(ref) + off)
    i = (err / bound).argmax()
    assert (err <= bound).all(), (x[i], err[i], ref[i])


@pytest.mark.parametrize("kind", [BF, F32])
@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("M", [100, 4096])
def test_logistic_forms(api, M, act, kind):
    """v / (1 + 2^s): s passes two roundings (silu) or five (tanh's, of a cube) of 2^-24 each, the exponential is good to 2^-22, the
    reciprocal to 2^-23, five more roundings.  Held at s = 60: results below 64 2^-60 = 2^-54 are that far from 0 at the most."""
    v = values()
    x = v.double().numpy()
    ref = OB.activation(x, act)
    z = x if act == "silu" else 2 * np.sqrt(2 / np.pi) * (x + 0.044715 * x ** 3)
    off = ((2 if act == "silu" else 5) * np.abs(z) / (1 + np.exp(np.clip(z, -700, 700))) + 4 + 2 + 5) * 2.0 ** -24 * np.abs(ref) + 2.0 ** -53
    err = np.abs(activated(api, v, act, kind, M) - ref)
    bound = off + (2.0 ** -8 if kind == BF else 2.0 ** -24) * (np.abs(ref) + off)
    i = (err / bound).argmax()
    assert (err <= bound).all(), (x[i], err[i], ref[i])


@pytest.mark.parametrize("D", [16384, 8191, 4096, 1024, 1023])
def test_norm_divides_by_the_scale(api, D):
    """y = n / y_scale, rounded once more, for n exactly gamma (rows of ones): values next to e4m3's borders."""
    rng = np.random.default_rng(D)
    for stream in (F32, BF):
        for _ in range(6):
            most = np.float32(rng.uniform(0.5, 40))
            scale = np.float32(most / np.float32(448))
            middles = (OB.E4M3[1:] + OB.E4M3[:-1]) / 2
            near = np.float32(rng.choice(middles, D) * float(scale))
            near = np.clip((near.view(np.int32) + rng.integers(-4, 5, D).astype(np.int32)).view(np.float32), None, most) * rng.choice(np.float32([-1, 1]), D)
            near[rng.integers(D)] = most
            gamma = torch.tensor(near, dtype=F32, device=DEV)
            x = torch.ones(3, D, device=DEV, dtype=stream)
            out, s = torch.empty(3, D, device=DEV, dtype=E4M3), torch.empty(3, device=DEV)
            api.grace_rms_norm(x, gamma, out, 0.0, scale=s)
            assert (s.cpu().numpy() == scale).all()
            want = OB.to_e4m3((near / scale).astype(np.float32))
            got = out.view(torch.uint8).cpu().numpy()
            assert (got == want).all(), int((got != want).sum())


def test_norm_whose_scale_is_infinite(api):
    """A gain that overflows takes its own element, not the row's others."""
    x = torch.full((2, 512), 1e-3, device=DEV)
    x[0, 7] = 20.0
    gamma = torch.ones(512, device=DEV)
    gamma[7] = 3e38
    out, s = torch.empty(2, 512, device=DEV, dtype=E4M3), torch.empty(2, device=DEV)
    api.grace_rms_norm(x, gamma, out, scale=s)
    assert s[0].item() == float("inf") and torch.isfinite(s[1])
    q = out.float()
    assert torch.isnan(q[0, 7]) and (q[0, :7] == 0).all() and (q[0, 8:] == 0).all()
    assert q[1, 7] == 448


def test_a_single_row_of_any_stride(api):
    """One row out of a wider matrix: its stride says nothing."""
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    wide = torch.randn(1, 520, device=DEV, generator=g).to(BF).as_strided((1, 512), (513, 1))
    w = torch.randn(64, 512, device=DEV, generator=g).to(BF)
    y = torch.empty(1, 64, device=DEV)
    api.grace_linear_act(wide, w, y)
    assert (y.double() - wide.double() @ w.double().T).abs().max() <= 2.0 ** -19 * (wide.double().abs() @ w.double().abs().T).max()
