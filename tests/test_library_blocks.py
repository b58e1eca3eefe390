"""CPU-only checks of the C entries of the norm, the product with an epilogue and the sampler: every refusal is made on the
host, before anything is launched (the pointers here are never followed), and the weights' e4m3 form is the oracle's."""
import numpy as np
import pytest

from oracle import blocks as OB

OK, INVALID, SHAPE = 0, 1, 2
P = 1 << 20                                                  # a well aligned address that nothing follows


@pytest.fixture(scope="module")
def api():
    from paper_2608_00938_b200 import build
    build()
    from paper_2608_00938_b200 import api as _api
    return _api


def _norm(api, **a):
    a = dict(x_f32=None, x_bf16=P, ldx=64, delta=None, ldd=0, x_out=None, ldxo=0, gamma=P, y_bf16=P, y_e4m3=None, ldy=64,
             scale=None, R=4, D=64, eps=1e-6) | a
    return api._rms_norm(*(a[k] for k in ("x_f32", "x_bf16", "ldx", "delta", "ldd", "x_out", "ldxo", "gamma", "y_bf16", "y_e4m3", "ldy",
                                          "scale", "R", "D", "eps")), None)


@pytest.mark.parametrize("bad,code", [
    (dict(x_bf16=None), INVALID), (dict(x_f32=P), INVALID), (dict(gamma=None), INVALID), (dict(y_bf16=None), INVALID),
    (dict(y_e4m3=P, scale=P), INVALID), (dict(y_bf16=None, y_e4m3=P), INVALID), (dict(scale=P), INVALID), (dict(delta=P, ldd=64), INVALID),
    (dict(x_out=P, ldxo=64), INVALID), (dict(delta=P, ldd=63, x_out=P, ldxo=64), INVALID), (dict(delta=P, ldd=64, x_out=P, ldxo=63), INVALID),
    (dict(delta=P, ldd=64, x_out=P, ldxo=72), INVALID),      # in place with another stride
    (dict(R=0), INVALID), (dict(R=-1), INVALID), (dict(D=0), INVALID), (dict(ldx=63), INVALID), (dict(ldy=63), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(x_bf16=P + 1), INVALID), (dict(gamma=P + 2), INVALID),
    (dict(D=16385, ldx=16385, ldy=16385), SHAPE),
])
def test_norm_refuses(api, bad, code):
    assert _norm(api, **bad) == code


def _linear(api, e4m3, **a):
    a = dict(x=P, ldx=64, xs=None, w=P, ldw=64, ws=None, bias=None, act=0, res=None, ldr=0, yb=P, yf=None, ldy=32, M=8, N=32, K=64) | a
    if e4m3:
        return api._linear_act_e4m3(*(a[k] for k in ("x", "ldx", "xs", "w", "ldw", "ws", "bias", "act", "res", "ldr", "yb", "yf", "ldy", "M", "N", "K")), None)
    return api._linear_act(*(a[k] for k in ("x", "ldx", "w", "ldw", "bias", "act", "res", "ldr", "yb", "yf", "ldy", "M", "N", "K")), None)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("bad,code", [
    (dict(x=None), INVALID), (dict(w=None), INVALID), (dict(yb=None), INVALID), (dict(yf=P), INVALID), (dict(M=0), INVALID),
    (dict(N=0), INVALID), (dict(K=0), INVALID), (dict(M=-5), INVALID), (dict(act=-1), INVALID), (dict(act=5), INVALID), (dict(x=P + 8), INVALID),
    (dict(w=P + 2), INVALID), (dict(ldx=68), INVALID), (dict(ldw=60), INVALID), (dict(ldx=48), INVALID), (dict(ldy=31), INVALID),
    (dict(yb=P + 1), INVALID), (dict(res=P, ldr=31), INVALID), (dict(res=P + 1, ldr=32), INVALID), (dict(res=P, ldr=40), INVALID),
    (dict(bias=P + 2), INVALID), (dict(K=60), SHAPE),
])
def test_linear_act_refuses(api, e4m3, bad, code):
    assert _linear(api, e4m3, **bad) == code


def test_linear_act_e4m3_wants_sixteen(api):
    assert _linear(api, True, K=56) == SHAPE                 # 8 bf16 are 16 bytes, 8 e4m3 are not
    assert _linear(api, True, ldx=72) == INVALID
    assert _linear(api, True, xs=P + 1) == INVALID and _linear(api, True, ws=P + 2) == INVALID


def _sample(api, **a):
    a = dict(lf=P, lb=None, ld=100, allow=None, score=None, lse=None, T=None, k=None, p=None, q=None, u=P, B=2, M=3, V=100, draws=1,
             os=P, oq=None, op=None, ot=P, st=None) | a
    return api._sample(*(a[k] for k in ("lf", "lb", "ld", "allow", "score", "lse", "T", "k", "p", "q", "u", "B", "M", "V", "draws",
                                        "os", "oq", "op", "ot", "st")), None)


@pytest.mark.parametrize("bad,code", [
    (dict(lf=None), INVALID), (dict(lb=P), INVALID), (dict(u=None), INVALID), (dict(os=None), INVALID), (dict(ot=None), INVALID),
    (dict(B=0), INVALID), (dict(M=0), INVALID), (dict(V=0), INVALID), (dict(draws=0), INVALID), (dict(draws=-1), INVALID), (dict(ld=99), INVALID),
    (dict(lf=P + 2), INVALID), (dict(lf=None, lb=P + 1), INVALID), (dict(allow=P + 4), INVALID), (dict(T=P + 1), INVALID), (dict(k=P + 2), INVALID),
    (dict(u=P + 3), INVALID), (dict(V=65537, ld=65537), SHAPE), (dict(B=65536, M=32768), SHAPE),
])
def test_sample_refuses(api, bad, code):
    assert _sample(api, **bad) == code


def test_quantized_rows_are_the_oracles(api):
    rng = np.random.default_rng(3)
    w = (rng.normal(size=(7, 33)) * 10.0 ** rng.integers(-6, 4, (7, 1))).astype(np.float32)
    w[2] = 0.0
    q, scale = api.grace_quantize_rows_e4m3(w)
    want = np.maximum(np.abs(w).max(1), np.float32(2.0 ** -100)) / np.float32(448)
    assert np.array_equal(scale, want.astype(np.float32))
    assert np.array_equal(q, OB.to_e4m3((w / scale[:, None]).astype(np.float32)))
    assert not q[2].any()
    for bad in (np.nan, np.inf, -np.inf):
        w2 = w.copy()
        w2[1, 5] = bad
        with pytest.raises(api.GraceError):
            api.grace_quantize_rows_e4m3(w2)
    with pytest.raises(ValueError):
        api.grace_quantize_rows_e4m3(w[0])


INT_MAX = 2 ** 31 - 1


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("sizes", [
    dict(M=65535 * 128 + 1, N=255, ldy=255),                 # more row tiles than a grid takes, too few columns for the persistent kernel
    dict(M=65535 * 128 + 1), dict(M=INT_MAX), dict(N=INT_MAX - 200, ldy=INT_MAX), dict(M=1, K=INT_MAX - 15, ldx=INT_MAX - 15, ldw=INT_MAX - 15),
])
def test_linear_act_refuses_sizes_whose_tiles_it_cannot_count(api, e4m3, sizes):
    assert _linear(api, e4m3, **sizes) == SHAPE


def test_norm_and_sample_refuse_sizes_that_they_cannot_count(api):
    assert _norm(api, R=INT_MAX) == SHAPE and _norm(api, R=INT_MAX - 2) == SHAPE
    assert _sample(api, draws=2 ** 30 + 1) == SHAPE and _sample(api, draws=INT_MAX) == SHAPE
    assert _sample(api, st=P + 2) == INVALID
