"""grace_sample's warp-a-row form (V <= 2048, more than 592 rows: a batch of beams) on the rows where lists overflow, ties are
split and values are not finite, and top-p together with min-p in every form: a list that min-p has shortened while top-p's share is
one of the whole row."""
import numpy as np
import pytest
import torch

from test_gpu_sample import BF, DEV, F32, api, check, logits_for, numbers  # noqa: F401

pytestmark = pytest.mark.gpu


def one(limits, B=1):
    return {name: [value] * B for name, value in limits.items()}


BOTH = [dict(p=0.95, q=0.1), dict(p=0.9, q=0.01, T=1.5), dict(p=0.5, q=0.02), dict(p=0.95, q=0.05, k=2000), dict(p=0.999, q=0.3), dict(p=0.0, q=0.5), dict(p=0.9, q=1.0)]


@pytest.mark.parametrize("limits", BOTH, ids=lambda d: ",".join(f"{k}={v}" for k, v in d.items()))
@pytest.mark.parametrize("M,V", [(610, 300), (610, 2048), (3, 200), (5, 1500), (4, 2048), (3, 5000), (2, 12000), (2, 30000), (1, 65536)])
def test_top_p_with_min_p(api, M, V, limits):
    for kind in (F32, BF):
        check(api, logits_for(V, M, V, kind=kind), numbers(V, M, 2), 1, M, **one(limits))
    allow = np.random.default_rng(V).random((M, V)) < 0.3
    check(api, logits_for(V, M, V), numbers(V, M, 1), 1, M, allow=allow, **one(limits))
    allow = np.random.default_rng(V).random((M, V)) < 0.9
    check(api, logits_for(V, M, V), numbers(V, M, 1), 1, M, allow=allow, **one(limits))


def many(rows, R):
    """The rows over and over, R in all."""
    return torch.tensor(np.asarray(rows)[np.arange(R) % len(rows)], dtype=F32, device=DEV)


TIES = [dict(), dict(k=1), dict(kshare=0.5), dict(kshare=0.2, p=0.5), dict(p=0.5), dict(p=0.25, T=2.0), dict(q=1.0), dict(T=0.0), dict(p=0.5, q=1.0), dict(p=0.9, q=0.3),
        dict(p=0.7, q=0.36)]


def ties(V, R, limits, allow=None):
    rng = np.random.default_rng(V)
    rows = np.stack([np.zeros(V), np.where(np.arange(V) % 3 == 0, 1.0, 0.0), rng.integers(0, 4, V).astype(float), np.where(rng.random(V) < 0.5, 0.0, -0.0),
                     np.where(np.arange(V) == V - 1, 5.0, -5.0), np.full(V, torch.finfo(F32).min), np.where(rng.random(V) < 0.1, 1.0, rng.normal(size=V) * 1e-3)])
    limits = dict(limits)
    if "kshare" in limits:
        limits["k"] = max(1, int(limits.pop("kshare") * V))
    return many(rows, R), numbers(V, R, 2), limits


@pytest.mark.parametrize("limits", TIES, ids=lambda d: ",".join(f"{k}={v}" for k, v in d.items()) or "none")
@pytest.mark.parametrize("R,V", [(609, 260), (609, 1025), (609, 2048), (7, 50), (7, 2048), (7, 6000), (7, 30000)])
def test_ties(api, R, V, limits):
    x, u, lim = ties(V, R, limits)
    check(api, x, u, 1, R, **one(lim))
    for density in (0.3, 0.9):
        check(api, x, u, 1, R, allow=np.random.default_rng(R).random((R, V)) < density, **one(lim))


@pytest.mark.parametrize("V", [300, 1001, 2048])
def test_lightest_tokens(api, V):
    """One heavy token and many whose weights are next to nothing one by one, and together what top_p still wants: most of the row stays,
    in one or two steps of the histogram."""
    rng = np.random.default_rng(V)
    powers = np.array([3.0, 8.0, 12.0, 17.0, 19.0, 20.5, 20.99, 21.01, 21.9, 22.1, 23.0])
    x = -np.log(2.0) * powers[:, None] * np.ones((1, V)) + rng.normal(size=(11, V)) * 1e-4
    x[np.arange(11), rng.integers(0, V, 11)] = 0.0
    R = 605
    logits = many(x, R)
    light = np.exp(logits.double().cpu().numpy()).sum(1) - 1.0
    u = torch.tensor([[0.3, 0.9993, 0.9999, 0.9999995]] * R, dtype=F32)
    for share in (0.1, 0.9):
        p = [(1.0 + share * w) / (1.0 + w) for w in light]
        check(api, logits, u, R, 1, p=p)
        check(api, logits, u, R, 1, p=p, k=[V - 3] * R)
        check(api, logits, u, R, 1, p=p, allow=rng.random((R, V)) < 0.95)


@pytest.mark.parametrize("V", [300, 2048])
def test_infinities_lowest_values_and_nan(api, V):
    x = logits_for(4, 8, V)
    x[0, [5, 80, 299]] = float("inf")
    x[1] = -float("inf")
    x[2] = -float("inf")
    x[2, 17] = -2.0
    x[3, 10:] = torch.finfo(F32).min
    x[4] = torch.finfo(F32).max
    x[5, ::2] = -float("inf")
    x[6] *= 1e20
    R = 616
    x = x.repeat(R // 8, 1)
    u = numbers(2, R, 2)
    allow = np.random.default_rng(5).random((R, V)) < 0.7
    for limits in (dict(), dict(k=2), dict(k=V - 20), dict(p=0.6), dict(q=0.1), dict(T=0.0), dict(T=1e-30), dict(T=1e32), dict(p=0.7, q=0.2), dict(T=float("nan"))):
        check(api, x, u, 1, R, **one(limits))
        check(api, x, u, 1, R, allow=allow, **one(limits))
    x = logits_for(9, R, V)
    bad = (3, 100, 615)
    for r in bad:
        x[r, V // 2] = float("nan")
    check(api, x, u, 1, R, p=[0.9], nan_rows=bad)
    check(api, x, u, 1, R, allow=np.ones((R, V), bool), k=[5], nan_rows=bad)
