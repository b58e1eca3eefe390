"""grace_sample where a limit or a number lies next to a border of the running sums: the tokens have to be those of the
definition in 64-bit arithmetic on whichever side of the border the fp32 argument falls, in every form of the kernel (a warp a row:
V <= 2048 and more than 592 rows; 4, 8 or 32 warps a row otherwise)."""
import numpy as np
import pytest
import torch

from test_gpu_sample import DEV, api, check, logits_for, numbers  # noqa: F401

pytestmark = pytest.mark.gpu


def beside(value, steps):
    """The fp32 number nearest to `value`, `steps` numbers further, within (0, 1)."""
    v = np.float32(value)
    for _ in range(abs(int(steps))):
        v = np.nextafter(v, np.float32(1 if steps > 0 else 0))
    return float(np.clip(v, np.float32(2.0 ** -24), np.float32(1 - 2.0 ** -24)))


def test_top_p_beside_a_border_under_many_light_tokens(api):
    """31 of 32 heavy tokens weigh top_p of the whole but for a few parts in a million, and so do 2015 light ones together, each below
    half a step of a sum that holds a heavy one (an fp32 sum in order stays 32)."""
    R, V = 700, 2048
    x = torch.zeros(R, V, device=DEV)
    x[:, 32:] = -16.636
    u = torch.full((R, 2), 0.98)
    u[:, 1] = 0.9687                                         # (30 kept tokens or 31 turn on this one)
    start = np.float32(31 / 32 * (1 - 3.62e-6))
    p = [float(start + np.float32((i - 350) * 2.0 ** -24)) for i in range(R)]
    check(api, x, u, R, 1, k=[2047] * R, p=p)
    check(api, x, u, R, 1, p=p)
    check(api, x, u, R, 1, p=p, q=[1e-8] * R)


@pytest.mark.parametrize("B,V", [(640, 300), (640, 1500), (640, 2048), (300, 900), (40, 3000), (12, 12000), (8, 30000)])
@pytest.mark.parametrize("masked", [False, True])
def test_top_p_beside_a_border(api, B, V, masked):
    rng = np.random.default_rng(V)
    x = logits_for(V + 1, B, V, std=1.5)
    allow = rng.random((B, V)) < 0.4 if masked else None
    xd = x.double().cpu().numpy()
    for k, T in ((0, 1.0), (V // 4, 1.3)):
        p = []
        for r in range(B):
            a = xd[r] if allow is None else xd[r][allow[r]]
            w = np.exp((np.sort(a)[::-1] - a.max()) / float(np.float32(T)))
            if k:
                w = w[:k]
            run = np.cumsum(w) / w.sum()
            p.append(beside(run[rng.integers(0, max(1, len(run) - 2))], rng.integers(-1, 2)))
        lists = dict(k=[k] * B, T=[T] * B, p=p)
        u = numbers(V, B, 2)
        u[:, 0] = 1 - 2.0 ** -24                             # the last kept token
        check(api, x, u, B, 1, allow=allow, **lists)
        check(api, x, u, B, 1, allow=allow, **(lists | dict(q=[0.02] * B)))


@pytest.mark.parametrize("R,V,draws", [(640, 257, 1), (640, 2048, 1), (640, 2000, 12), (300, 700, 1), (30, 5000, 1), (3, 2048, 600), (6, 40000, 1)])
def test_numbers_beside_a_border(api, R, V, draws):
    rng = np.random.default_rng(V + draws)
    x = logits_for(V, R, V, std=2.0)
    xd = x.double().cpu().numpy()
    u = torch.empty(R, draws)
    for r in range(R):
        run = np.cumsum(np.exp(xd[r] - xd[r].max()))
        run /= run[-1]
        for d in range(draws):
            u[r, d] = beside(run[rng.integers(0, V - 1)], rng.integers(-1, 2))
    check(api, x, u, 1, R)


def test_rows_decided_in_64_bits_repeat(api):
    """Rows that 64 bits decide, on two streams: no result depends on the order in which threads add to a list."""
    R, V = 1500, 2048
    rng = np.random.default_rng(3)
    x = logits_for(5, R, V, std=0.5)
    xd = x.double().cpu().numpy()
    run = np.cumsum(np.exp(-np.sort(-xd, 1)), 1)
    run /= run[:, -1:]
    p = torch.tensor([beside(run[r, rng.integers(0, V - 2)], 0) for r in range(R)], device=DEV)
    u = torch.full((R, 1), 1 - 2.0 ** -24, device=DEV)
    outs, streams = [], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            sc, lq, tk = torch.empty(R, device=DEV), torch.empty(R, device=DEV), torch.empty(R, device=DEV, dtype=torch.int32)
            api.grace_sample(x, u, sc, tk, R, 1, top_p=p, out_logq=lq)
            outs.append((sc, lq, tk))
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))


@pytest.mark.parametrize("R", [5, 640])
def test_logits_and_temperatures_next_to_nothing(api, R):
    """Differences of subnormal size weigh by themselves, not by what an overflowing 1 / T leaves of them; a temperature below 1e-36 counts as that."""
    V = 300
    x = -torch.rand(R, V, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))
    u = numbers(1, R, 3)
    check(api, x * 3e-35, u, 1, R, T=[1e-35])
    check(api, x * 3e-36, u, 1, R, T=[1e-36], p=[0.9])
    check(api, x * 1e-38, u, 1, R, T=[1e-36], k=[200])
    score, token = torch.empty(R, 3, device=DEV), torch.empty(R, 3, device=DEV, dtype=torch.int32)
    tokens = []
    for T in (1e-36, 1e-37, 1e-40):
        api.grace_sample(x * 3e-36, u.to(DEV), score, token, 1, R, temperature=torch.tensor([T], device=DEV))
        tokens.append(token.clone())
    assert torch.equal(tokens[0], tokens[1]) and torch.equal(tokens[0], tokens[2])
