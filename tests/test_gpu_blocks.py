"""GPU parity of grace_rms_norm and grace_linear_act against their definitions in fp64, at the sizes, strides and values where
they can go wrong.

Tolerances, derived.  A rounding to a type is off by at most half a step: bf16 2^-8, e4m3 2^-4 (and half its least step, 2^-10,
near zero), fp32 2^-24 of the value.  Norm: the sum of squares passes at most 8 + 4 + 9 additions on its way (relative 21 x
2^-24, halved by the root), the root, the gain and the scale are a handful of fp32 roundings: 2^-19 covers them.  Product: its
accumulation as in the other GEMM tests, 2^-19 of the sum of absolute products; the activations' slopes are at most 1.13; gelu of a
bf16 result is a fit within 7.5e-5 of a Phi(-a) <= 0.17; the others a few fp32 roundings (2^-20 of the value); scale, bias and
residual two more (2^-22 of their absolute sum)."""
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


def f64(t):
    return t.detach().double().cpu().numpy()


def gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def strided(t, ld, offset=0):
    """The rows of t with stride ld in a buffer that starts `offset` elements behind an aligned address; (view, whole buffer)."""
    R, D = t.shape
    buf = torch.empty(offset + R * ld + 64, dtype=torch.float32, device=DEV).fill_(7.0).to(t.dtype)
    view = buf[offset:offset + R * ld].view(R, ld)[:, :D]
    view.copy_(t)
    return view, buf


def assert_rows_only(view, buf, before, what):
    """Nothing of the buffer but the view's rows has changed."""
    a, b = buf.clone(), before.clone()
    R, D = view.shape
    off = view.storage_offset()
    for x in (a, b):
        x[off:off + R * view.stride(0)].view(R, view.stride(0))[:, :D].zero_()
    assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), f"{what}: wrote outside its rows"


def check_norm(api, x, delta, gamma, out_type, eps=1e-6, ldx=None, offset=0, in_place=False):
    R, D = x.shape
    ld = ldx or D
    xv, xb = strided(x, ld, offset)
    dv = None if delta is None else strided(delta, ld, offset)[0]
    gv = torch.empty(D + 8, device=DEV)[offset % 4:][:D]
    gv.copy_(gamma)
    out, ob = strided(torch.zeros(R, D, device=DEV).to(out_type), ld, offset)
    xo, xob = (xv, xb) if in_place or delta is None else strided(torch.zeros_like(x), ld, offset)
    scale = torch.full((R + 4,), -3.0, device=DEV)
    before = (xb.clone(), ob.clone(), xob.clone())
    api.grace_rms_norm(xv, gv, out, eps, delta=dv, x_out=None if delta is None or in_place else xo,
                       scale=scale[:R] if out_type == E4M3 else None)
    torch.cuda.synchronize()
    s = x if delta is None else (x.float() + delta.float()).to(x.dtype)
    if delta is not None:
        assert torch.equal(xo.contiguous(), s), "stream"
        assert_rows_only(xo, xob, before[2], "x_out")
    if delta is None or not in_place:
        assert torch.equal(xv.contiguous().view(torch.uint8), x.contiguous().view(torch.uint8)), "x was written"
    assert_rows_only(out, ob, before[1], "out")
    ref = OB.rms_norm(f64(s), f64(gamma), eps)
    if out_type == BF:
        err = np.abs(f64(out) - ref)
        assert (err <= (2.0 ** -8 + 2.0 ** -19) * np.abs(ref) + 1e-38).all(), err.max()
        return
    want = OB.row_scales(ref)
    got = f64(scale[:R])
    assert (np.abs(got - want) <= 2.0 ** -18 * want).all()
    assert (f64(scale[R:]) == -3.0).all()
    q = f64(out)
    assert np.abs(q).max() <= 448
    nonzero = np.abs(ref).max(1) > 2.0 ** -99
    assert (np.abs(q[nonzero]).max(1) == 448).all()
    n = ref / want[:, None]
    assert (np.abs(q - n) <= (2.0 ** -4 + 2.0 ** -17) * np.abs(n) + 2.0 ** -10 * 1.001).all()


@pytest.mark.parametrize("out_type", [BF, E4M3])
@pytest.mark.parametrize("stream", [BF, F32])
@pytest.mark.parametrize("R,D", [(1, 1), (3, 7), (5, 8), (1, 512), (9, 200), (37, 512), (6, 768), (5, 1000), (4, 1024), (3, 1032), (130, 2048),
                                 (3, 2056), (2, 4096), (2, 4104), (2, 16384), (1, 16383), (4099, 64)])
def test_norm_matches_fp64(api, R, D, stream, out_type):
    g = gen(R * 100003 + D)
    x = (torch.randn(R, D, device=DEV, generator=g) * 3).to(stream)
    delta = torch.randn(R, D, device=DEV, generator=g).to(BF)
    gamma = 1 + 0.3 * torch.randn(D, device=DEV, generator=g)
    check_norm(api, x, delta, gamma, out_type)
    check_norm(api, x, delta, gamma, out_type, in_place=True)
    check_norm(api, x, None, gamma, out_type)


@pytest.mark.parametrize("out_type", [BF, E4M3])
@pytest.mark.parametrize("stream", [BF, F32])
@pytest.mark.parametrize("D,ld,offset", [(512, 520, 0), (512, 513, 0), (512, 512, 1), (512, 1024, 8), (40, 48, 3), (33, 64, 0), (2048, 2049, 5)])
def test_norm_takes_any_stride_and_alignment(api, D, ld, offset, stream, out_type):
    g = gen(D + ld)
    x, delta = (torch.randn(11, D, device=DEV, generator=g)).to(stream), torch.randn(11, D, device=DEV, generator=g).to(BF)
    gamma = torch.randn(D, device=DEV, generator=g)
    for in_place in (False, True):
        check_norm(api, x, delta, gamma, out_type, ldx=ld, offset=offset, in_place=in_place)


def test_norm_in_one_call_or_two_gives_the_same_bits(api):
    g = gen(5)
    for stream in (BF, F32):
        x, delta = (torch.randn(70, 512, device=DEV, generator=g)).to(stream), torch.randn(70, 512, device=DEV, generator=g).to(BF)
        gamma = torch.randn(512, device=DEV, generator=g)
        one, two = torch.empty(70, 512, device=DEV, dtype=E4M3), torch.empty(70, 512, device=DEV, dtype=E4M3)
        s1, s2 = torch.empty(70, device=DEV), torch.empty(70, device=DEV)
        api.grace_rms_norm(x, gamma, one, delta=delta, x_out=torch.empty_like(x), scale=s1)
        added = (x.float() + delta.float()).to(stream)
        api.grace_rms_norm(added, gamma, two, scale=s2)
        assert torch.equal(one.view(torch.uint8), two.view(torch.uint8)) and torch.equal(s1, s2)


def test_norm_of_extreme_rows(api):
    x = torch.randn(8, 512, device=DEV, generator=gen(6))
    x[0] = 0.0
    x[1] *= 1e-30                                            # below what eps leaves
    x[2] *= 1e15
    x[3, 77] = float("nan")
    x[4, 5] = float("inf")
    gamma = torch.ones(512, device=DEV)
    for stream in (F32, BF):
        xs = x.to(stream)
        out, scale, y = torch.empty(8, 512, device=DEV, dtype=E4M3), torch.empty(8, device=DEV), torch.empty(8, 512, device=DEV, dtype=BF)
        api.grace_rms_norm(xs, gamma, out, scale=scale)
        api.grace_rms_norm(xs, gamma, y)
        assert (f64(out[0]) == 0).all() and scale[0] > 0 and (f64(y[0]) == 0).all()
        assert torch.isnan(scale[3]) and torch.isnan(y[3]).all() and torch.isnan(scale[4])
        fine = [1, 2, 5, 6, 7]
        ref = OB.rms_norm(f64(xs[fine]), np.ones(512), 1e-6)
        assert (np.abs(f64(y[fine]) - ref) <= 2.0 ** -7.9 * np.abs(ref) + 1e-38).all()
        assert torch.isfinite(scale[fine]).all()
    # a row behind the last stays as it was
    out = torch.full((9, 512), 3.0, device=DEV, dtype=BF)
    api.grace_rms_norm(x[5:7], gamma, out[:2])
    assert (out[2:] == 3.0).all()


def test_norm_refuses(api):
    x, gamma = torch.zeros(4, 64, device=DEV), torch.ones(64, device=DEV)
    out = torch.zeros(4, 64, device=DEV, dtype=BF)
    ok = dict(x=x, gamma=gamma, out=out)
    for bad in (dict(x=x.half()), dict(x=x[0]), dict(gamma=gamma[:32]), dict(gamma=gamma.double()), dict(out=out[:3]), dict(out=out.float()),
                dict(out=out.to(E4M3)), dict(scale=torch.zeros(4, device=DEV)), dict(x_out=x), dict(delta=x), dict(delta=out[:, :32]),
                dict(x=x.cpu()), dict(x=x.t()), dict(delta=out, x_out=out), dict(out=out.to(E4M3), scale=torch.zeros(3, device=DEV))):
        with pytest.raises(ValueError):
            api.grace_rms_norm(**(ok | bad))
    with pytest.raises(api.GraceError):
        api.grace_rms_norm(x, gamma, out, eps=-1.0)


# ------------------------------------------------------------------------------------------
# product with an epilogue
# ------------------------------------------------------------------------------------------
def operands(g, M, N, K, e4m3):
    x, w = torch.randn(M, K, device=DEV, generator=g), torch.randn(N, K, device=DEV, generator=g) * K ** -0.5
    if not e4m3:
        return x.to(BF), w.to(BF), None, None
    xs, ws = x.abs().amax(1) / 448, w.abs().amax(1) / 448
    return (x / xs[:, None]).to(E4M3), (w / ws[:, None]).to(E4M3), xs, ws


def check_linear(api, M, N, K, e4m3, act, bias, residual, y_type, seed=0, ld_y=None, offset=0, in_place=False, ld_x=None, scales=True):
    g = gen(seed + M * 7 + N * 3 + K)
    x, w, xs, ws = operands(g, M, N, K, e4m3)
    if not scales:
        xs = ws = None
    if ld_x:
        x, w = (torch.zeros(t.shape[0], ld_x, device=DEV).to(t.dtype)[:, :K].copy_(t) for t in (x, w))
    b = torch.randn(N, device=DEV, generator=g) if bias else None
    r = (torch.randn(M, N, device=DEV, generator=g) * 2).to(y_type) if residual else None
    ld = ld_y or N
    y, yb = strided(r if in_place else torch.zeros(M, N, device=DEV).to(y_type), ld, offset)
    rv = y if in_place else (None if r is None else strided(r, ld, offset)[0])
    before = yb.clone()
    api.grace_linear_act(x, w, y, bias=b, act=act, residual=rv, x_scale=xs, w_scale=ws)
    torch.cuda.synchronize()
    assert api.grace_wait_timeouts() == 0
    assert_rows_only(y, yb, before, "y")
    xd, wd = x.double(), w.double()
    if xs is not None:
        xd, wd = xd * xs[:, None].double(), wd * ws[:, None].double()
    v, sums = (xd @ wd.T), (xd.abs() @ wd.abs().T)
    if b is not None:
        v = v + b.double()
        sums = sums + b.double().abs() * 2.0 ** -3
    v, sums = f64(v), f64(sums)
    a = OB.activation(v, act)
    ref = a if r is None else a + f64(r)
    tol = 1.13 * 2.0 ** -19 * sums + 2.0 ** -20 * np.abs(a) + 2.0 ** -22 * (np.abs(a) + np.abs(ref))
    if act == "gelu":
        tol = tol + (7.5e-5 * 0.17 if y_type == BF else 2.0 ** -22 * np.abs(v))
    tol = tol + (2.0 ** -8 if y_type == BF else 2.0 ** -24) * (np.abs(ref) + tol) + 1e-30
    err = np.abs(f64(y) - ref)
    i = np.unravel_index((err / tol).argmax(), err.shape)
    assert (err <= tol).all(), f"|err| {err[i]:.3g} at {i}, bound {tol[i]:.3g}, ref {ref[i]:.4g}"


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("M,N,K", [
    (1, 1, 16), (1, 2048, 512), (3, 5, 48), (16, 2048, 512), (16, 512, 2048), (127, 65, 112), (128, 64, 4096), (129, 130, 64), (300, 1000, 528),
    (513, 512, 512), (700, 33, 8192), (1023, 257, 320),
    (1024, 256, 64), (1025, 257, 80), (1500, 2048, 512), (2049, 300, 208), (3000, 1001, 1040), (40000, 512, 128), (20000, 264, 144),
])
def test_linear_matches_fp64(api, M, N, K, e4m3):
    for i, (act, bias, residual, y) in enumerate([("none", False, False, BF), ("gelu", True, False, BF), ("none", True, True, BF), ("silu", True, True, F32)]):
        check_linear(api, M, N, K, e4m3, act, bias, residual, y, seed=i)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("y", [BF, F32])
@pytest.mark.parametrize("act", ["none", "relu", "gelu", "gelu_tanh", "silu"])
def test_linear_activations(api, act, y, e4m3):
    for M, N, K in ((200, 96, 256), (1100, 320, 128)):
        for bias in (False, True):
            for residual in (False, True):
                check_linear(api, M, N, K, e4m3, act, bias, residual, y)


@pytest.mark.parametrize("y", [BF, F32])
@pytest.mark.parametrize("M,N,K,ld,offset", [(200, 100, 64, 104, 0), (200, 100, 64, 101, 0), (200, 100, 64, 100, 1), (1200, 520, 128, 528, 0),
                                             (1200, 520, 128, 521, 0), (1200, 520, 128, 520, 3), (1300, 261, 96, 264, 0), (1300, 261, 96, 272, 8)])
def test_linear_rows_of_any_stride_and_alignment(api, M, N, K, ld, offset, y):
    for in_place in (False, True):
        check_linear(api, M, N, K, False, "gelu_tanh", True, True, y, ld_y=ld, offset=offset, in_place=in_place)
        check_linear(api, M, N, K, True, "none", True, True, y, ld_y=ld, offset=offset, in_place=in_place, ld_x=K + 16)
    check_linear(api, M, N, K, False, "silu", False, False, y, ld_y=ld, offset=offset, ld_x=K + 8)
    check_linear(api, M, N, K, True, "silu", False, False, y, ld_y=ld, offset=offset, scales=False)


@pytest.mark.parametrize("e4m3", [False, True])
@pytest.mark.parametrize("M,N,K", [(5, 70, 80), (260, 200, 1024), (1500, 600, 400), (2500, 257, 2000)])
def test_linear_of_small_integers_is_exact(api, M, N, K, e4m3):
    g = gen(M)
    kind = E4M3 if e4m3 else BF
    x = torch.randint(-2, 3, (M, K), device=DEV, generator=g).float()
    w = torch.randint(-2, 3, (N, K), device=DEV, generator=g).float()
    b = torch.randint(-50, 51, (N,), device=DEV, generator=g).float()
    r = torch.randint(-50, 51, (M, N), device=DEV, generator=g).float()
    y = torch.empty(M, N, device=DEV)
    one = dict(x_scale=torch.full((M,), 2.0, device=DEV), w_scale=torch.full((N,), 0.5, device=DEV)) if e4m3 else {}
    api.grace_linear_act(x.to(kind), w.to(kind), y, bias=b, act="relu", residual=r, **one)
    assert torch.equal(y, (x @ w.T + b).clamp_min(0) + r)


@pytest.mark.parametrize("M,N", [(1, 40), (16, 64), (130, 500), (200, 2000), (700, 1000), (1000, 8000), (1100, 300), (2500, 512)])
@pytest.mark.parametrize("e4m3,K", [(False, 16384), (True, 32768), (False, 1096), (False, 2120), (True, 6160)])
def test_long_sums_do_not_drift(api, M, N, e4m3, K):
    """Products of positive numbers, whose running sums grow evenly (a step adds 16 or 32 products of mean 1).  An accumulator that cuts
    off what it cannot hold loses at most a last place, 2^-23 of the sum so far, at each of a segment's steps; there are 128 at the
    most and the sums so far are half the segment's on average: 64 x 2^-23 of it, and an eighth more for the evenness.  The sums of
    16 segments at the most, of four CTAs and the epilogue are rounded to nearest: 24 x 2^-24.  (1024 steps without segments: 512
    x 2^-23 by the same count.)"""
    g = gen(M + N)
    kind = E4M3 if e4m3 else BF
    x = (torch.rand(M, K, device=DEV, generator=g) + 0.5).to(kind)
    w = (torch.rand(N, K, device=DEV, generator=g) + 0.5).to(kind)
    y = torch.empty(M, N, device=DEV)
    api.grace_linear_act(x, w, y)
    want = x.double() @ w.double().T
    assert float(((y.double() - want).abs() / want).max()) <= 84 * 2.0 ** -23


def test_linear_of_large_values(api):
    """Activations far out: no NaN from an overflowing exponential, zero or the value itself."""
    v = torch.tensor([-1e30, -3e4, -300.0, -90.0, -41.0, -20.0, -16.0, -6.0, 0.0, 6.0, 16.0, 41.0, 90.0, 300.0, 3e4, 1e30], device=DEV).to(BF)
    for M in (16, 1040):
        x = torch.zeros(M, 64, device=DEV, dtype=BF)
        x[:16, 0] = v
        w = torch.zeros(256, 64, device=DEV, dtype=BF)
        w[:, 0] = 1.0
        for act in ("gelu", "gelu_tanh", "silu"):
            for kind in (BF, F32):
                y = torch.empty(M, 256, device=DEV, dtype=kind)
                api.grace_linear_act(x, w, y, act=act)
                ref = OB.activation(np.clip(f64(v), -1e6, 1e6), act)
                ref = np.where(f64(v) > 1e5, f64(v), np.where(f64(v) < -1e5, 0.0, ref))
                got = f64(y[:16, 7])
                assert np.isfinite(got).all()
                assert (np.abs(got - ref) <= 2.0 ** -7.9 * np.abs(ref) + 2e-5).all(), (act, got, ref)


def test_linear_columns_of_infinite_biases(api):
    """A bias of -inf takes a column out: the smooth activations' limits are 0 (silu's and tanh's forms stop at 64 2^-60 = 2^-54)."""
    for M in (40, 1200):
        x, w, _, _ = operands(gen(4), M, 300, 160, False)
        b = torch.zeros(300, device=DEV)
        b[7::10], b[3::50] = -float("inf"), float("inf")
        for act in ("relu", "gelu", "gelu_tanh", "silu"):
            for kind in (BF, F32):
                y = torch.empty(M, 300, device=DEV, dtype=kind)
                api.grace_linear_act(x, w, y, bias=b, act=act)
                assert (y[:, 7::10].abs() <= 2.0 ** -53).all() and (y[:, 3::50] == float("inf")).all(), (act, kind)
                rest = torch.isfinite(b)
                assert torch.isfinite(y[:, rest]).all()


def test_linear_keeps_a_bad_row_to_itself(api):
    for e4m3 in (False, True):
        for M in (40, 1200):
            x, w, xs, ws = operands(gen(3), M, 300, 160, e4m3)
            if e4m3:
                xs[5] = float("nan")
            else:
                x[5, 3] = float("nan")
            for act in ("none", "relu", "gelu", "gelu_tanh", "silu"):
                for kind in (BF, F32):
                    y = torch.empty(M, 300, device=DEV, dtype=kind)
                    api.grace_linear_act(x, w, y, act=act, x_scale=xs, w_scale=ws)
                    bad = torch.isnan(y)
                    assert bad[5].all() and int(bad.sum()) == 300, (act, kind)


def test_linear_refuses(api):
    x, w, y = (torch.zeros(s, device=DEV, dtype=BF) for s in ((8, 64), (32, 64), (8, 32)))
    ok = dict(x=x, w=w, y=y)
    one = torch.ones(8, device=DEV)
    for bad in (dict(x=x.float()), dict(w=w.float()), dict(w=w[:, :32]), dict(y=y[:, :16]), dict(y=y.half()), dict(bias=one), dict(bias=torch.ones(32, device=DEV).double()),
                dict(residual=y.float()), dict(residual=y[:4]), dict(act="tanh"), dict(x_scale=one), dict(x=x.to(E4M3)), dict(x=x.cpu()), dict(y=y.t()),
                dict(x=x.to(E4M3), w=w.to(E4M3), x_scale=one[:4])):
        with pytest.raises(ValueError):
            api.grace_linear_act(**(ok | bad))
    with pytest.raises(api.GraceError):
        api.grace_linear_act(x[:, :60], w[:, :60], y)        # K % 8
    with pytest.raises(api.GraceError):
        api.grace_linear_act(x[:, 1:57], w[:, 1:57], y)      # rows that do not start on 16 bytes


def test_norm_and_product_in_a_graph_on_another_stream(api):
    """Captured and replayed with new contents, eager calls of the same shapes in between on another stream."""
    M, D, N = 1100, 256, 512
    g = gen(9)
    x, delta = torch.randn(M, D, device=DEV, generator=g).to(BF), torch.randn(M, D, device=DEV, generator=g).to(BF)
    gamma, bias = 1 + 0.1 * torch.randn(D, device=DEV, generator=g), torch.randn(N, device=DEV, generator=g)
    w, ws = (torch.randn(N, D, device=DEV, generator=g) / 16).to(E4M3), torch.ones(N, device=DEV)

    def buffers():
        return dict(xo=torch.empty_like(x), q=torch.empty(M, D, device=DEV, dtype=E4M3), s=torch.empty(M, device=DEV), y=torch.empty(M, N, device=DEV, dtype=BF))

    def run(b):
        api.grace_rms_norm(x, gamma, b["q"], delta=delta, x_out=b["xo"], scale=b["s"])
        api.grace_linear_act(b["q"], w, b["y"], bias=bias, act="gelu", x_scale=b["s"], w_scale=ws)

    cap, eager = buffers(), buffers()
    run(eager)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.stream(side):
        run(cap)
        with torch.cuda.graph(graph, stream=side):
            run(cap)
    torch.cuda.synchronize()
    for i in range(3):
        x.copy_(torch.randn(M, D, device=DEV, generator=g))
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graph.replay()
        run(eager)
        torch.cuda.synchronize()
        for k in cap:
            assert torch.equal(cap[k].contiguous().view(torch.uint8), eager[k].contiguous().view(torch.uint8)), (i, k)
