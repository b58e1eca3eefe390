"""GPU parity of grace_sample against the oracle's definition in fp64: the drawn tokens are equal, whatever the limits, ties,
masks and sizes; scores are the one fp32 expression of the ranking calls; log q within what fp32 sums allow (the weights' sum and
its logarithm: a few 2^-20; the exponent's rounding 2^-23 of |log q|)."""
import numpy as np
import pytest
import torch

from oracle import sampling as OS

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def api():
    from paper_2608_00938_b200 import api as _api
    return _api


def pack(allow):
    """bool [R, V] -> int64 words [R, ceil(V/64)] on the device; the bits behind V are set: they have no say."""
    R, V = allow.shape
    words = (V + 63) // 64
    full = np.ones((R, words * 64), np.uint64)
    full[:, :V] = allow
    return torch.from_numpy((full.reshape(R, words, 64) << np.arange(64, dtype=np.uint64)).sum(2, dtype=np.uint64).view(np.int64)).to(DEV)


def check(api, logits, u, B, M, allow=None, T=None, k=None, p=None, q=None, ld=None, offset=0, nan_rows=()):
    """logits fp32 or bf16 tensor [R, V] on the device; T, k, p, q: lists of B numbers or None."""
    R, V = logits.shape
    draws = u.shape[1]
    ld = ld or V
    buf = torch.full((offset + R * ld + 8,), 99.0, device=DEV, dtype=logits.dtype)
    rows = buf[offset:offset + R * ld].view(R, ld)[:, :V]
    rows.copy_(logits)
    score, lse = torch.randn(R, device=DEV), torch.randn(R, device=DEV)
    dev = lambda a, t: None if a is None else torch.tensor(a, dtype=t, device=DEV)  # noqa: E731
    out = [torch.full((R * draws + 3,), -7.0, device=DEV) for _ in range(2)] + [torch.full((R * draws + 3,), -7, device=DEV, dtype=torch.int32) for _ in range(2)]
    status = torch.zeros(1, device=DEV, dtype=torch.int32)
    api.grace_sample(rows, u.to(DEV), out[0][:-3].view(B, -1), out[2][:-3].view(B, -1), B, M, allow_bits=None if allow is None else pack(allow), row_score=score,
                     row_lse=lse, temperature=dev(T, F32), top_k=dev(k, torch.int32), top_p=dev(p, F32), min_p=dev(q, F32), out_logq=out[1][:-3].view(B, -1),
                     out_parent=out[3][:-3].view(B, -1), d_status=status)
    torch.cuda.synchronize()
    assert all((o[-3:] == -7).all() for o in out), "wrote behind its outputs"
    assert bool(status.item() & 2) == bool(len(nan_rows)), status
    x = logits.double().cpu().numpy()
    x32 = logits.float().cpu().numpy()
    un = u.double().cpu().numpy()
    f32 = lambda v, default: float(np.float32(default if v is None else v))  # noqa: E731
    sc, ls = score.cpu().numpy(), lse.cpu().numpy()
    got = [o[:-3].view(R, draws).cpu().numpy() for o in out]
    for r in range(R):
        b = r // M
        one = lambda a, default: default if a is None else a[b]  # noqa: E731
        a = None if allow is None else allow[r]
        if r in nan_rows:
            tok, logq = np.zeros(draws, np.int64), np.full(draws, -np.inf)
        else:
            tok, logq = OS.sample_row(x[r], a, f32(one(T, 1.0), 1.0), one(k, 0), f32(one(p, 1.0), 1.0), f32(one(q, 0.0), 0.0), un[r])
        assert np.array_equal(got[2][r], tok), (r, got[2][r], tok)
        assert (got[3][r] == r % M).all()
        dead = np.isneginf(logq)
        want = np.where(dead, np.float32(-np.inf), sc[r] + (x32[r][tok] - ls[r]))
        assert np.array_equal(got[0][r], want.astype(np.float32), equal_nan=True), r
        assert np.array_equal(np.isneginf(got[1][r]), dead)
        assert (np.abs(got[1][r][~dead] - logq[~dead]) <= 2.0 ** -17 + 2.0 ** -22 * np.abs(logq[~dead])).all(), r


def logits_for(seed, R, V, std=3.0, kind=F32):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return (torch.randn(R, V, device=DEV, generator=g) * std).to(kind)


def numbers(seed, R, draws):
    g = torch.Generator()
    g.manual_seed(seed)
    return torch.rand(R, draws, generator=g)


LIMITS = [dict(), dict(T=0.7), dict(k=1), dict(k=17), dict(p=0.9), dict(p=0.3, T=1.5), dict(q=0.05), dict(k=40, p=0.8, q=0.02, T=0.8), dict(T=0.0, k=5, p=0.5),
          dict(p=0.0), dict(k=100000, p=1.0, q=0.0), dict(q=2.0), dict(p=0.999, T=4.0)]


@pytest.mark.parametrize("limits", LIMITS, ids=lambda d: ",".join(f"{k}={v}" for k, v in d.items()) or "none")
@pytest.mark.parametrize("B,M,V", [(1, 1, 1), (1, 3, 2), (2, 2, 63), (1, 5, 64), (3, 40, 257), (2, 350, 300), (1, 7, 1000), (2, 9, 2048), (2, 301, 2047), (1, 3, 2049),
                                   (1, 2, 5001), (1, 2, 8193), (1, 2, 16384), (1, 2, 20001), (1, 1, 65536)])
def test_dense_rows_match_the_definition(api, B, M, V, limits):
    lists = {name: [value] * B for name, value in limits.items()}
    for kind, draws in ((F32, 1), (BF, 3)):
        check(api, logits_for(V + M, B * M, V, kind=kind), numbers(V, B * M, draws), B, M, **lists)


@pytest.mark.parametrize("density", [0.0, 0.004, 0.05, 0.3, 0.8, 1.0])
@pytest.mark.parametrize("B,M,V", [(2, 3, 64), (1, 30, 200), (2, 301, 2048), (1, 5, 2048), (1, 3, 5000), (1, 2, 16384), (1, 2, 40000), (1, 2, 65472)])
def test_masked_rows_match_the_definition(api, B, M, V, density):
    rng = np.random.default_rng(V + int(density * 1000))
    R = B * M
    allow = rng.random((R, V)) < density
    allow[0] = False                                         # a row that the mask leaves empty
    if R > 1:
        allow[1] = False
        allow[1, rng.integers(V)] = True                     # and one with a single token
    logits = logits_for(V, R, V)
    # what the mask hides has no say: NaN, infinities, the type's lowest value
    hidden = torch.from_numpy(~allow).to(DEV)
    junk = torch.tensor([float("nan"), float("inf"), -float("inf"), torch.finfo(F32).min, torch.finfo(F32).max], device=DEV)
    logits = torch.where(hidden, junk[torch.randint(0, 5, (R, V), device=DEV)], logits)
    for limits in (dict(), dict(p=0.9, T=0.8), dict(k=7, p=0.9, q=0.01), dict(T=0.0)):
        check(api, logits, numbers(V, R, 2), B, M, allow=allow, **{n: [v] * B for n, v in limits.items()})
    check(api, logits.to(BF), numbers(V + 1, R, 1), B, M, allow=allow, p=[0.95] * B)


@pytest.mark.parametrize("V", [300, 1001, 2048, 5000, 16384])
def test_top_p_that_reaches_into_the_lightest(api, V):
    """One heavy token and many whose weights are next to nothing one by one, and together what top_p still wants."""
    rng = np.random.default_rng(V)
    powers = np.array([8.0, 12.0, 17.0, 19.0, 20.5, 20.99, 21.01, 21.9, 22.1, 23.0])
    x = -np.log(2.0) * powers[:, None] * np.ones((1, V)) + rng.normal(size=(10, V)) * 1e-4
    x[np.arange(10), rng.integers(0, V, 10)] = 0.0
    logits = torch.tensor(x, dtype=F32, device=DEV)
    u = torch.tensor([[0.3, 0.9993, 0.9999, 0.9999995]] * 10, dtype=F32)
    light = np.exp(x).sum(1) - 1.0
    for share in (0.1, 0.5, 0.9):                            # of the light ones' weight
        p = [(1.0 + share * w) / (1.0 + w) for w in light]
        check(api, logits, u, 10, 1, p=p)
        check(api, logits, u, 10, 1, p=p, allow=rng.random((10, V)) < 0.95)


@pytest.mark.parametrize("V", [50, 700, 2048, 6000, 30000])
def test_ties(api, V):
    """Equal logits: the whole row, two values, few values, signed zeros; the lower token goes first."""
    rng = np.random.default_rng(V)
    rows = np.stack([np.zeros(V), np.where(np.arange(V) % 3 == 0, 1.0, 0.0), rng.integers(0, 4, V).astype(float), np.where(rng.random(V) < 0.5, 0.0, -0.0),
                     np.where(np.arange(V) == V - 1, 5.0, -5.0), np.full(V, torch.finfo(F32).min)])
    logits = torch.tensor(rows, dtype=F32, device=DEV)
    u = numbers(V, 6, 4)
    for limits in (dict(), dict(k=1), dict(k=V // 2), dict(k=V // 5 + 1, p=0.5), dict(p=0.5), dict(p=0.25, T=2.0), dict(q=1.0), dict(T=0.0)):
        check(api, logits, u, 1, 6, **{n: [v] for n, v in limits.items()})


def test_rows_of_infinities_and_lowest_values(api):
    V = 300
    x = logits_for(4, 8, V)
    x[0, [5, 80, 299]] = float("inf")
    x[1] = -float("inf")
    x[2] = -float("inf")
    x[2, 17] = -2.0
    x[3, 10:] = torch.finfo(F32).min                              # the mask value of other programs
    x[4] = torch.finfo(F32).max
    x[5, ::2] = -float("inf")
    x[6] *= 1e20
    u = numbers(2, 8, 5)
    for limits in (dict(), dict(k=2), dict(k=200), dict(p=0.6), dict(q=0.1), dict(T=0.0), dict(T=1e-30), dict(T=1e-42), dict(T=1e32), dict(T=float("nan"))):
        check(api, x, u, 1, 8, **{n: [v] for n, v in limits.items()})
        check(api, x, u, 1, 8, allow=np.ones((8, V), bool), **{n: [v] for n, v in limits.items()})


def test_nan_rows_are_flagged_and_alone(api):
    for V in (100, 3000, 20000):
        x = logits_for(V, 6, V)
        x[2, V // 2] = float("nan")
        check(api, x, numbers(1, 6, 2), 2, 3, p=[0.9, 0.9], nan_rows=(2,))
        check(api, x, numbers(1, 6, 2), 2, 3, allow=np.ones((6, V), bool), nan_rows=(2,))
        allow = np.ones((6, V), bool)
        allow[2, V // 2] = False
        check(api, x, numbers(1, 6, 2), 2, 3, allow=allow)


@pytest.mark.parametrize("V,draws", [(64, 2048), (1000, 333), (2048, 32), (2048, 9), (9000, 1000), (33000, 65)])
def test_many_draws_and_their_borders(api, V, draws):
    """Numbers over the whole of [0, 1), its ends included."""
    u = numbers(V, 2, draws)
    u[0, :4] = torch.tensor([0.0, 1.0 - 2.0 ** -24, 2.0 ** -30, 0.5])
    u[1] = (torch.arange(draws) + 0.5) / draws
    check(api, logits_for(V, 2, V), u, 1, 2)
    check(api, logits_for(V, 2, V), u, 1, 2, T=[0.9], p=[0.97])
    # borders that numbers hit exactly: 2^n equal weights
    check(api, torch.zeros(2, 64, device=DEV), torch.arange(128).view(2, 64).float() / 128, 1, 2)


def test_limits_belong_to_requests(api):
    B, M, V = 5, 60, 1500
    check(api, logits_for(8, B * M, V), numbers(8, B * M, 1), B, M, T=[1.0, 0.0, 0.5, 2.0, 1.0], k=[0, 3, 50, 0, 1], p=[1.0, 0.5, 0.9, 0.8, 0.2], q=[0.0, 0.0, 0.05, 0.0, 0.9])


@pytest.mark.parametrize("V,ld,offset", [(300, 304, 0), (300, 301, 0), (300, 300, 1), (301, 512, 3), (2500, 2501, 2), (18000, 18001, 1)])
@pytest.mark.parametrize("kind", [F32, BF])
def test_rows_of_any_stride_and_alignment(api, V, ld, offset, kind):
    check(api, logits_for(V, 7, V, kind=kind), numbers(3, 7, 2), 1, 7, p=[0.9], ld=ld, offset=offset)
    check(api, logits_for(V, 7, V, kind=kind), numbers(3, 7, 2), 1, 7, allow=np.random.default_rng(1).random((7, V)) < 0.2, ld=ld, offset=offset)


def test_offsets_beyond_32_bits(api):
    """Rows whose elements lie more than 2^32 bytes and 2^31 elements into the tensor."""
    V, ld, R = 200, 1 << 24, 160
    buf = torch.empty(R * ld, device=DEV, dtype=BF)
    rows = buf.view(R, ld)[:, :V]
    x = logits_for(1, R, V, kind=BF)
    rows.copy_(x)
    u = numbers(1, R, 1)
    score, token = torch.empty(R, device=DEV), torch.empty(R, device=DEV, dtype=torch.int32)
    api.grace_sample(rows, u.to(DEV), score, token, 1, R)
    want = [OS.sample_row(x[r].double().cpu().numpy(), None, 1.0, 0, 1.0, 0.0, u[r].double().numpy())[0][0] for r in range(R)]
    assert token.cpu().numpy().tolist() == want
    del buf, rows
    torch.cuda.empty_cache()


def test_sample_refuses(api):
    x, u = torch.zeros(6, 100, device=DEV), torch.zeros(6, 2, device=DEV)
    sc, tk = torch.zeros(12, device=DEV), torch.zeros(12, device=DEV, dtype=torch.int32)
    ok = dict(logits=x, u=u, out_score=sc, out_token=tk, B=2, M=3)
    two = torch.ones(2, device=DEV)
    for bad in (dict(logits=x.half()), dict(logits=x[0]), dict(B=3), dict(u=u[:5]), dict(u=u[0]), dict(u=u.double()), dict(out_score=sc[:11]), dict(out_token=tk.long()),
                dict(out_token=sc), dict(allow_bits=torch.zeros(6, 1, device=DEV, dtype=torch.int64)), dict(temperature=two[:1]), dict(top_k=two), dict(top_p=two.double()),
                dict(min_p=two.cpu()), dict(row_score=two), dict(row_lse=two), dict(out_logq=two), dict(out_parent=tk[:3]), dict(logits=x.cpu()), dict(u=u.t().contiguous().t())):
        with pytest.raises(ValueError):
            api.grace_sample(**(ok | bad))
    with pytest.raises(api.GraceError):
        api.grace_sample(torch.zeros(6, 65537, device=DEV), u, sc, tk, 2, 3)
    with pytest.raises(api.GraceError):
        api.grace_sample(x, torch.zeros(6, 0, device=DEV), sc[:0], tk[:0], 2, 3)


def test_sampled_step_from_the_blocks_to_the_beam(api):
    """What a sampled decode step runs: add and norm to 8 bits, feed-forward up with GELU and down into the stream, norm, logits, the
    catalog's bits, a draw per row, the beams' new nodes; every stage against its definition on what the stage in front left.  Then the
    same in a graph, replayed with other numbers."""
    import synth
    from oracle import blocks as OB
    from oracle.sid_trie import SidTrie
    rng = synth.rng_for(3, 77)
    B, M, V, L, D, F = 3, 50, 256, 3, 128, 512
    R = B * M
    sids = synth.catalog(rng, 9000, V, L)
    trie = SidTrie(sids, V)
    bits, base, _ = api.grace_trie_build_dense(sids, V)
    dt = api.make_trie(torch.from_numpy(bits.view(np.int64)).to(DEV), torch.from_numpy(base).to(DEV), V, L, trie.num_nodes)
    none = api.make_matcher(api.MATCH_NONE)
    first = rng.integers(0, sids.shape[0], R)
    node = torch.tensor([trie.walk(sids[i, :1]) for i in first], dtype=torch.int32, device=DEV)
    node[7] = -1                                             # a dead beam
    key = torch.from_numpy((sids[first, 0].astype(np.int64) + 1)).to(DEV)
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    n = lambda *s: torch.randn(*s, device=DEV, generator=g)  # noqa: E731
    x0, delta, gam = n(R, D).to(BF), n(R, D).to(BF), [1 + 0.1 * n(D) for _ in range(2)]
    up, ups = api.grace_quantize_rows_e4m3((n(F, D) / D ** 0.5).cpu().numpy())
    up, ups = torch.from_numpy(up).to(DEV).view(torch.float8_e4m3fn), torch.from_numpy(ups).to(DEV)
    down, b_up, b_down, w_out = (n(D, F) / F ** 0.5).to(BF), n(F), n(D), (n(V, D) * 0.3).to(BF)
    x1, x2 = torch.empty_like(x0), torch.empty_like(x0)
    q, s = torch.empty(R, D, device=DEV, dtype=torch.float8_e4m3fn), torch.empty(R, device=DEV)
    h, hn, logits = torch.empty(R, F, device=DEV, dtype=BF), torch.empty(R, D, device=DEV, dtype=BF), torch.empty(R, V, device=DEV)
    allow = torch.empty(R, V // 64, device=DEV, dtype=torch.int64)
    u, score0 = torch.rand(R, 1, device=DEV, generator=g), -torch.rand(R, device=DEV, generator=g)
    T, p = torch.full((B,), 0.8, device=DEV), torch.full((B,), 0.9, device=DEV)
    score, logq = torch.empty(B, M, device=DEV), torch.empty(B, M, device=DEV)
    token, parent = torch.empty(B, M, device=DEV, dtype=torch.int32), torch.empty(B, M, device=DEV, dtype=torch.int32)
    new_node, new_key = torch.empty(R, device=DEV, dtype=torch.int32), torch.empty(R, device=DEV, dtype=torch.int64)
    status = torch.zeros(1, device=DEV, dtype=torch.int32)

    def step():
        api.grace_rms_norm(x0, gam[0], q, delta=delta, x_out=x1, scale=s)
        api.grace_linear_act(q, up, h, bias=b_up, act="gelu", x_scale=s, w_scale=ups)
        api.grace_linear_act(h, down, x2, bias=b_down, residual=x1)
        api.grace_rms_norm(x2, gam[1], hn)
        api.grace_linear_act(hn, w_out, logits)
        api.grace_gtm_allow_bits(node, key, dt, none, allow, B, M, 1, status)
        api.grace_sample(logits, u, score, token, B, M, allow_bits=allow, row_score=score0, temperature=T, top_p=p, out_logq=logq, out_parent=parent, d_status=status)
        api.grace_beam_update(parent, token, score, node, key, dt, new_node, new_key, B, M, M, 1, status)

    f = lambda t: t.double().cpu().numpy()  # noqa: E731

    def verify():
        torch.cuda.synchronize()
        assert status.item() == 0
        assert torch.equal(x1, (x0.float() + delta.float()).to(BF))
        ref = OB.activation(f(q) * f(s)[:, None] @ (f(up) * f(ups)[:, None]).T + f(b_up), "gelu")
        assert np.abs(f(h) - ref).max() <= 2.0 ** -8 * np.abs(ref).max() + 1e-4
        ref = f(h) @ f(down).T + f(b_down) + f(x1)
        assert np.abs(f(x2) - ref).max() <= 2.0 ** -8 * np.abs(ref).max() + 1e-4
        child = np.zeros((R, V), bool)
        for r, nd in enumerate(node.cpu().numpy()):
            if nd >= 0:
                child[r] = [trie.child(int(nd), v) >= 0 for v in range(V)]
        x = f(logits)
        for r in range(R):
            tok, lq = OS.sample_row(x[r], child[r], float(np.float32(0.8)), 0, float(np.float32(0.9)), 0.0, f(u[r]))
            assert token.view(-1)[r].item() == tok[0]
            assert logq.view(-1)[r].item() == pytest.approx(lq[0], abs=1e-5)
            want = -1 if np.isneginf(lq[0]) else trie.child(int(node[r]), int(tok[0]))
            assert new_node[r].item() == want
        assert new_node[7].item() == -1 and score.view(-1)[7].item() == -np.inf

    step()
    verify()
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        with torch.cuda.graph(graph, stream=side):
            step()
    for i in range(2):
        u.copy_(torch.rand(R, 1, device=DEV, generator=g))
        graph.replay()
        verify()


def test_two_streams_and_repeats_give_the_same_bits(api):
    """Calls under way at once share nothing, and no result depends on the order of threads."""
    R, V = 3000, 2048
    x = logits_for(3, R, V)
    u = numbers(3, R, 1).to(DEV)
    p = torch.full((1,), 0.92, device=DEV)
    outs = []
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i in range(6):
        with torch.cuda.stream(streams[i % 2]):
            sc, lq, tk = torch.empty(R, device=DEV), torch.empty(R, device=DEV), torch.empty(R, device=DEV, dtype=torch.int32)
            api.grace_sample(x, u, sc, tk, 1, R, top_p=p, out_logq=lq)
            outs.append((sc, lq, tk))
    torch.cuda.synchronize()
    for o in outs[1:]:
        assert all(torch.equal(a, b) for a, b in zip(o, outs[0]))
