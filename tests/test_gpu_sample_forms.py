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
