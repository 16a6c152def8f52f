"""Tokens drawn from logits, against the definition in 64 bits: the same token wherever the random number is not next to a border between two."""
import numpy as np
import pytest

import drafts_reference as drafts
from test_gpu_parity import dev, g, host  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

F32 = np.float32


def _row(r, V, kind):
    if kind == "equal":
        return np.full(V, 1.5, F32)
    if kind == "levels":  # a few values: ties everywhere
        return r.integers(-4, 3, V).astype(F32)
    if kind == "peaked":
        x = r.standard_normal(V).astype(F32)
        x[r.integers(0, V, max(1, V // 50))] += F32(12)
        return x
    if kind == "masked":  # most are no candidates
        x = r.standard_normal(V).astype(F32) * 3
        x[r.random(V) < 0.9] = -np.inf
        x[r.random(V) < 0.3] = np.nan
        x[r.integers(0, V)] = F32(0.25)
        return x
    if kind == "wide":  # spread far beyond what has any weight
        return (r.standard_normal(V) * 1e4).astype(F32)
    return (r.standard_normal(V) * (0.5 if kind == "flat" else 3)).astype(F32)


KINDS = ["normal", "flat", "peaked", "levels", "masked", "equal", "wide"]


def _check(g, x, u, T=None, k=None, p=None, m=None, gpu_x=None):
    t = lambda a, dt: None if a is None else dev(np.asarray(a, dt))  # noqa: E731
    tokens, probs = g.sample_tokens(dev(x) if gpu_x is None else gpu_x, dev(u), temperature=t(T, F32), top_k=t(k, np.int32), top_p=t(p, F32), min_p=t(m, F32))
    tokens, probs = host(tokens), host(probs)
    for i in range(len(x)):
        at = lambda a, none, dt: none if a is None else dt(a[i])  # noqa: E731
        token, share, gap = drafts.sample(x[i], F32(u[i]), at(T, 1.0, F32), at(k, 0, int), at(p, 1.0, F32), at(m, 0.0, F32))
        # Weights are whole numbers of 2^-44 of the largest's, sums exact, so a border is off by 2^-45 a token at most, 2^18 of them 2^-27, of which
        # a sum that is 1 at least is as much; random numbers of the tests are kept further from borders than that where several tokens are kept
        if gap < 2.0 ** -26:
            continue
        assert tokens[i] == token, (i, tokens[i], token, gap)
        assert abs(probs[i] - share) <= 2.0 ** -24 * share + 2.0 ** -26, (i, probs[i], share)
    return tokens, probs


# fewer tokens than a workgroup has threads, one more, odd ones, several a thread
@pytest.mark.parametrize("V", [1, 2, 63, 100, 1024, 1025, 5003, 32000])
@pytest.mark.parametrize("dt", [np.float32, np.float16])
def test_every_filter(g, V, dt):
    r = np.random.default_rng(V)
    rows, params = [], []
    for kind in KINDS:
        for T in (1.0, 0.6, 1.7, 0.0):
            for k, p, m in ((0, 1, 0), (1, 1, 0), (5, 1, 0), (0, 0.9, 0), (0, 0.3, 0), (0, 1, 0.1), (40, 0.8, 0.01), (V // 2, 0.95, 0.001), (V + 3, 0.999, 0), (-1, 0.0, 2.0), (7, -1.0, -1.0)):
                rows.append(_row(r, V, kind))
                params.append((T, k, p, m))
    with np.errstate(over="ignore"):
        x = np.array(rows).astype(dt)
    T, k, p, m = zip(*params)
    tokens, _ = _check(g, x, r.random(len(x)).astype(F32), T, k, p, m)
    assert ((tokens >= 0) & (tokens < V)).all()


@pytest.mark.parametrize("dt", [np.float32, np.float16])
def test_the_most_tokens(g, dt):
    """As many as there may be: flat, where every border is close to the next, equal (2^18 ties), and peaked"""
    r = np.random.default_rng(1)
    V = 1 << 18
    x = np.array([_row(r, V, kind) for kind in ("flat", "equal", "peaked", "levels", "normal", "flat")]).astype(dt)
    for k, p, m in ((None, None, None), ([1000] * 6, [0.9] * 6, None), (None, [0.5] * 6, None), ([200000] * 6, [0.99] * 6, [0.05] * 6)):
        _check(g, x, r.random(6).astype(F32), [1.0, 1.0, 0.7, 1.0, 1.3, 2.0], k, p, m)


# 2, 4 and 8 workgroups a row
@pytest.mark.parametrize("rows,V", [(12, 65536), (12, 70000), (12, 150001), (60, 66000), (128, 65537)])
@pytest.mark.parametrize("dt", [np.float32, np.float16])
def test_rows_over_several_workgroups(g, rows, V, dt):
    r = np.random.default_rng(V)
    size = g.lib().gpusq_sample_tokens_workspace_bytes(rows, V)
    assert size > 0
    params = [(1.0, 0, 1, 0), (0.7, 50, 1, 0), (1.3, 0, 0.9, 0), (1, 700, 0.95, 0.01), (1, 3000, 1, 0), (0, 5, 0.5, 0.2), (1, 0, 1, 0.05), (1, V - 3, 0.999, 0), (1, 0, 0.01, 0), (0.5, 1, 1, 0), (1, 2, 0, 2)]
    for n, kind in enumerate(KINDS + ["none", "infinite"]):
        x = np.array([_row(r, V, kind if kind in KINDS else "normal") for _ in range(rows)])
        if kind == "none":
            x[:] = -np.inf
            x[::2, 5] = np.nan
        if kind == "infinite":
            x[:, r.integers(0, V, 9)] = np.inf
        T, k, p, m = zip(*[params[(n + i) % len(params)] for i in range(rows)])
        with np.errstate(over="ignore"):
            x = x.astype(dt)
        u = r.random(rows).astype(F32)
        tokens, _ = _check(g, x, u, T, k, p, m)
        t = lambda a, d: dev(np.asarray(a, d))  # noqa: E731
        ws = torch.full((size,), 255, dtype=torch.uint8, device="cuda")
        again, _ = g.sample_tokens(dev(x), dev(u), temperature=t(T, F32), top_k=t(k, np.int32), top_p=t(p, F32), min_p=t(m, F32), workspace=ws)
        assert np.array_equal(host(again), tokens)


def test_infinite_logits_are_cut_like_others(g):
    """Tokens of +infinity weigh 1 each: by k, by share, by index"""
    x = np.zeros((8, 300), F32)
    x[:, [7, 50, 60, 299]] = np.inf
    u = np.array([0.0, 0.3, 0.6, 0.99, 0.99, 0.99, 1.0, 0.99], F32)
    k, p = np.array([0, 0, 0, 0, 2, 0, 3, 3], np.int32), np.array([1, 1, 1, 1, 1, 0.5, 1, 0.1], F32)
    tokens, probs = g.sample_tokens(dev(x), dev(u), top_k=dev(k), top_p=dev(p))
    assert host(tokens).tolist() == [7, 50, 60, 299, 50, 50, 60, 7] and host(probs).tolist() == [0.25, 0.25, 0.25, 0.25, 0.5, 0.5, F32(1) / F32(3), 1]


def test_ties_go_to_the_lowest_index(g):
    V = 4096
    x = np.zeros((6, V), F32)
    x[:, 100] = x[:, 7] = x[:, 3000] = 2.0
    x[5, 50] = -0.0
    u = np.array([0.0, 0.49, 0.51, 0.99, 0.999, 0.0], F32)
    tokens, probs = g.sample_tokens(dev(x), dev(u), top_k=dev(np.array([2, 2, 2, 1, 3, 0], np.int32)), temperature=dev(np.array([1, 1, 1, 1, 1, -1], F32)))
    assert host(tokens).tolist() == [7, 7, 100, 7, 3000, 7] and host(probs)[:4].tolist() == [0.5, 0.5, 0.5, 1.0]
    # -0 and 0 are ties
    x = np.full((2, 3), -np.inf, F32)
    x[0, :2], x[1, 1:] = (-0.0, 0.0), (0.0, -0.0)
    tokens, _ = g.sample_tokens(dev(x), dev(np.array([0.7, 0.7], F32)), top_k=dev(np.array([1, 1], np.int32)))
    assert host(tokens).tolist() == [0, 1]
    # equal tokens and a share of them: as many as it takes
    x = np.zeros((4, 10), F32)
    tokens, probs = g.sample_tokens(dev(x), dev(np.full(4, 0.999, F32)), top_p=dev(np.array([0.25, 0.5, 0.5000001, 0.05], F32)))
    assert host(tokens).tolist() == [2, 4, 5, 0] and np.allclose(host(probs), [1 / 3, 1 / 5, 1 / 6, 1], rtol=2.0 ** -24, atol=0)


def test_rows_without_an_answer_and_infinite_logits(g):
    inf, nan = np.inf, np.nan
    x = np.array([[-inf, -inf, nan], [nan, nan, nan], [1, inf, inf], [-inf, 3, nan], [65504, -65504, 65504], [-inf, -inf, -3e38]], F32)
    tokens, probs = g.sample_tokens(dev(x), dev(np.array([0.3, 0.3, 0.6, 0.9, 0.2, 0.5], F32)))
    assert host(tokens).tolist() == [-1, -1, 2, 1, 0, 2] and host(probs).tolist() == [0, 0, 0.5, 1, 0.5, 1]
    # temperatures that are none; random numbers at and beyond the ends
    x = np.array([[1, 2, 2, 0]] * 6, F32)
    tokens, _ = g.sample_tokens(dev(x), dev(np.array([0.9, 0.9, 0.9, 0.0, 1.0, 5.0], F32)), temperature=dev(np.array([nan, 0, -1, 1, 1, 1], F32)))
    assert host(tokens).tolist() == [1, 1, 1, 0, 3, 3]
    tokens, _ = g.sample_tokens(dev(x), dev(np.full(6, 0.5, F32)), temperature=dev(np.array([1e-38, 1e38, inf, 1e-45, 1, 1], F32)), top_p=dev(np.array([nan] * 6, F32)))
    assert host(tokens).tolist() == [2, 2, 2, 2, 1, 1]


@pytest.mark.parametrize("dt", [np.float32, np.float16])
def test_strides_and_offsets(g, dt):
    """Rows with others' values between them, that begin at any value"""
    r = np.random.default_rng(2)
    whole = (r.standard_normal((9, 2100)) * 2).astype(dt)
    whole[:, :3] = whole[:, 1900:] = 50  # would be drawn
    on_gpu = dev(whole)
    for a, b in ((3, 1900), (4, 1003), (5, 6)):
        _check(g, whole[:, a:b], r.random(9).astype(F32), gpu_x=on_gpu[:, a:b])
    _check(g, whole[4:5, 3:70], r.random(1).astype(F32), gpu_x=on_gpu[4:5, 3:70])
    _check(g, whole[:, 7:8], r.random(9).astype(F32), gpu_x=on_gpu[:, 7:8])


def test_shares(g):
    """Over many random numbers tokens come as often as their weights say: the counts within five standard deviations"""
    r = np.random.default_rng(3)
    x = np.log(np.array([5, 1, 3, 0.5, 0.25, 8], F32))
    n = 20000
    tokens, probs = g.sample_tokens(dev(np.tile(x, (n, 1)).astype(F32)), dev(r.random(n).astype(F32)), top_p=dev(np.full(n, 0.95, F32)))
    w = np.array([5, 1, 3, 0, 0, 8]) / 17  # 17 of 17.75 is more than 0.95, 16 is less
    count = np.bincount(host(tokens), minlength=6)
    assert (np.abs(count - n * w) <= 5 * np.sqrt(n * w * (1 - w)) + 1e-9).all()
    assert np.allclose(host(probs), w[host(tokens)], rtol=1e-6)


def test_replayed_from_a_graph_and_twice_the_same(g):
    r = np.random.default_rng(4)
    x = [dev((r.standard_normal((5, 9001)) * 2).astype(F32)) for _ in range(3)]
    u, p, k = dev(r.random(5).astype(F32)), dev(np.full(5, 0.9, F32)), dev(np.array([0, 5, 50, 500, 5000], np.int32))
    call = lambda t: g.sample_tokens(t, u, top_k=k, top_p=p)  # noqa: E731
    eager = [call(t) for t in x]
    for t, e in zip(x, eager):
        assert all(torch.equal(a, b) for a, b in zip(call(t), e))
    buf, graph = x[0].clone(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = call(buf)
    for i in (1, 2, 0, 1):
        buf.copy_(x[i])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, eager[i]))


def test_refusals(g):
    x, u = torch.zeros((3, 8), device="cuda"), torch.zeros(3, device="cuda")
    for call in (lambda: g.sample_tokens(x.double(), u), lambda: g.sample_tokens(x, u[:2]), lambda: g.sample_tokens(x.t(), torch.zeros(8, device="cuda")), lambda: g.sample_tokens(x.cpu(), u),
                 lambda: g.sample_tokens(x, u, top_k=u), lambda: g.sample_tokens(x, u, top_p=0.9), lambda: g.sample_tokens(x, u, temperature=u.cpu()), lambda: g.sample_tokens(x, u.half())):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(g.GpusqError):
        g.sample_tokens(torch.zeros((3, 0), device="cuda"), u)
    for bad in (torch.zeros((3, (1 << 18) + 1), device="cuda"), torch.zeros((1, 9), device="cuda").expand(3, 9)):
        with pytest.raises(g.GpusqError) as e:
            g.sample_tokens(bad, u)
        assert e.value.status == g.ERR_SHAPE


@pytest.mark.parametrize("dt", [np.float32, np.float16])
@pytest.mark.parametrize("V", [1, 5, 1000, 33001, 70001])
def test_greedy_rows(g, V, dt):
    """The first of the greatest: zeros of either sign, ties, what is no number in front of it, infinities, nothing at all"""
    r = np.random.default_rng(V)
    x = np.round(r.standard_normal((9, V)) * 2).astype(dt)  # (many equal ones)
    x[1] = np.where(r.random(V) < 0.5, dt(0.0), dt(-0.0))
    x[2] = -np.inf
    x[3] = np.nan
    x[4, : V // 2] = np.nan
    x[5, r.integers(0, V, 3)] = np.inf
    x[6, : V - 1] = -np.inf
    x[7, :] = -65504
    tokens, probs = g.sample_tokens(dev(x), dev(r.random(9).astype(F32)), temperature=dev(np.array([0, 0, 0, 0, -1, 0, 0, 0, np.nan], F32)), top_k=dev(np.full(9, 3, np.int32)))
    numbers = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    exp = np.where(numbers.max(-1) == -np.inf, -1, numbers.argmax(-1))
    assert np.array_equal(host(tokens), exp) and np.array_equal(host(probs), (exp >= 0).astype(F32))


def test_on_another_stream(g):
    r = np.random.default_rng(0)
    x, u = dev(r.standard_normal((5, 70000)).astype(F32)), dev(r.random(5).astype(F32))
    T, k, p = dev(np.array([1, 0, 0.5, 2, 1], F32)), dev(np.array([0, 0, 40, 2000, 1], np.int32)), dev(np.array([0.9, 1, 1, 0.8, 1], F32))
    want = [host(t) for t in g.sample_tokens(x, u, temperature=T, top_k=k, top_p=p)]
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        got = g.sample_tokens(x, u, temperature=T, top_k=k, top_p=p)
        torch.cuda.current_stream().synchronize()
    assert all(np.array_equal(a, host(b)) for a, b in zip(want, got))
