"""The decoder's operators together, as pipeline.DecoderLayer runs them: against the layer's definition in 64 bits, and replayed from a graph."""
import numpy as np
import pytest

import decoder_reference as ref
from test_gpu_parity import dev, g, host  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

D, H, KV, HD, HIDDEN, B, S, SD, GROUP, PAGES = 256, 8, 2, 64, 512, 3, 50, 192, 64, 12


def _rms(x):
    y = x.float()
    return (y * torch.rsqrt((y * y).mean(-1, keepdim=True) + 1e-6)).half()


@pytest.fixture(scope="module")
def setup(g):
    from paper_2305_10727_amd.pipeline import DecoderLayer
    r = np.random.default_rng(0)
    layer = DecoderLayer(D, H, KV, HD, HIDDEN, B, S, SD, PAGES, group=GROUP)
    W = {n: (r.standard_normal(shape) * 0.06).astype(np.float32) for n, shape in layer.widths.items()}
    Ws = (r.standard_normal((2 * KV * HD, SD)) * 0.06).astype(np.float32)
    layer.prepare_weights({n: dev(w) for n, w in W.items()}, dev(Ws))
    a = np.arange(64)[:, None] * 10000.0 ** (-np.arange(0, HD, 2) / HD)
    st = dict(layer=layer, W=W, cos=np.cos(a).astype(np.float32), sin=np.sin(a).astype(np.float32), states=r.standard_normal((B, S, SD)).astype(np.float16),
              bias=(r.standard_normal(2 * KV * HD) * 0.1).astype(np.float32), weights=[(1 + 0.1 * r.standard_normal(HD)).astype(np.float32) for _ in range(2)],
              table=r.permutation(PAGES)[:2 * B].reshape(B, 2).astype(np.int32), state_lens=np.array([S, 17, 1], np.int32))
    layer.see(dev(st["states"]), dev(st["bias"]))
    return st


def _inputs(st, start, n, seed):
    """n new tokens of each sequence behind `start` earlier ones"""
    t = np.tile(np.arange(start, start + n, dtype=np.int32), B)
    seq = np.repeat(np.arange(B), n)
    x = np.random.default_rng(seed).standard_normal((B * n, D)).astype(np.float16)
    return dict(x=dev(x), positions=dev(t), slots=dev((st["table"][seq, t // 64] * 64 + t % 64).astype(np.int32)), kv_lens=dev(np.full(B, start + n, np.int32)))


def _step(st, i):
    return st["layer"].forward(i["x"], (_rms, _rms, _rms), (dev(st["cos"]), dev(st["sin"])), i["positions"], i["slots"], dev(st["table"]), i["kv_lens"],
                               head_weights=[dev(w) for w in st["weights"]], state_lens=dev(st["state_lens"]))


def _defined(st, i, n, start):
    """The layer in 64 bits, on the values that weights, cache and states' keys and values stand for"""
    W = {}
    for name, w in st["W"].items():
        c, s = ref.groups_int4(w, GROUP)
        W[name] = c.astype(np.float64) * s.astype(np.float64).repeat(GROUP, 1)
    rms = lambda v: v / np.sqrt((v * v).mean(-1, keepdims=True) + 1e-6)  # noqa: E731
    x, pos = host(i["x"]).astype(np.float64), host(i["positions"])
    qkv = (rms(x) @ W["qkv"].T).reshape(B * n, H + 2 * KV, HD)
    q = ref.norm_rope(qkv[:, :H], True, st["weights"][0], 1e-6, st["cos"][pos], st["sin"][pos], HD, False)
    K, V = ref.read_pages(host(st["layer"].cache), HD)
    kv = host(st["layer"].states_kv.Y).astype(np.float64).reshape(B, S, 2 * KV, HD)
    a = np.zeros((B * n, H, HD))
    for b in range(B):
        k, v = (p[st["table"][b]].transpose(0, 2, 1, 3).reshape(128, KV, HD)[:start + n] for p in (K, V))
        seen = np.arange(start + n)[None] <= start + np.arange(n)[:, None]
        for h in range(H):
            a[b * n:(b + 1) * n, h] = ref.attend(q[b * n:(b + 1) * n, h], k[:, h * KV // H], v[:, h * KV // H], seen, HD ** -0.5)[0]
    x = x + a.reshape(B * n, -1) @ W["out"].T
    q = (rms(x) @ W["query"].T).reshape(B * n, H, HD)
    for b in range(B):
        seen = np.broadcast_to(np.arange(S)[None] < st["state_lens"][b], (n, S))
        for h in range(H):
            a[b * n:(b + 1) * n, h] = ref.attend(q[b * n:(b + 1) * n, h], kv[b, :, h * KV // H], kv[b, :, KV + h * KV // H], seen, HD ** -0.5)[0]
    x = x + a.reshape(B * n, -1) @ W["states_out"].T
    y = rms(x) @ W["fc1"].T
    from scipy.special import ndtr
    return x + (y * ndtr(y)) @ W["fc2"].T


def test_a_chunk_and_tokens_behind_it(setup):
    """A prompt's chunk, then single tokens that see it in the cache.  Between the definition and the kernels lie some twenty roundings to
    fp16 of operands and results, of 2^-11 each, none of which grows on its way (norms, weighted means and linear layers of norm about one)."""
    start = 0
    for seed, n in enumerate((20, 1, 1, 5)):
        i = _inputs(setup, start, n, seed)
        y = host(_step(setup, i)).astype(np.float64)
        exp = _defined(setup, i, n, start)
        assert np.sqrt(((y - exp) ** 2).mean() / (exp ** 2).mean()) <= 20 * 2.0 ** -11 / np.sqrt(3)
        assert np.abs(y - exp).max() <= 20 * 2.0 ** -11 * np.abs(exp).max()
        start += n


def test_replayed_from_a_graph(setup):
    i = _inputs(setup, 27, 1, 9)
    layer = setup["layer"]
    args = (i["x"], (_rms, _rms, _rms), (dev(setup["cos"]), dev(setup["sin"])), i["positions"], i["slots"], dev(setup["table"]), i["kv_lens"])
    kw = dict(head_weights=[dev(w) for w in setup["weights"]], state_lens=dev(setup["state_lens"]))
    layer.capture(*args, **kw)
    for step in range(4):
        new = _inputs(setup, 27 + step, 1, 20 + step)
        for name in i:
            i[name].copy_(new[name])
        before = layer.cache.clone()
        got = layer.replay().clone()
        torch.cuda.synchronize()
        kept = layer.cache.clone()
        layer.cache.copy_(before)
        eager = layer.forward(*args, **kw)
        torch.cuda.synchronize()
        assert torch.equal(got, eager) and torch.equal(kept, layer.cache)


def test_weights_prepared_again_behind_a_capture(g, setup):
    """A captured step follows the layer's weights as an eager one does, and keeps the tensors that it was captured with"""
    from paper_2305_10727_amd.pipeline import DecoderLayer
    layer = DecoderLayer(D, H, KV, HD, HIDDEN, B, S, SD, PAGES, group=GROUP)

    def prepare(seed):
        r = np.random.default_rng(seed)
        layer.prepare_weights({n: dev((r.standard_normal(shape) * 0.06).astype(np.float32)) for n, shape in layer.widths.items()},
                              dev((r.standard_normal((2 * KV * HD, SD)) * 0.06).astype(np.float32)))
        layer.see(dev(setup["states"]), dev(setup["bias"]))

    def arguments():
        i = _inputs(setup, 0, 1, 40)
        return (i["x"], (_rms, _rms, _rms), (dev(setup["cos"]), dev(setup["sin"])), i["positions"], i["slots"], dev(setup["table"]), i["kv_lens"]), \
            dict(head_weights=[dev(w) for w in setup["weights"]], state_lens=dev(setup["state_lens"]))

    prepare(50)
    args, kw = arguments()
    layer.capture(*args, **kw)
    del args, kw
    results = []
    for seed in (50, 51, 52):
        prepare(seed)
        filler = [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in (64, 512, 4096, 16384, 65536, 1 << 20) for _ in range(8)]  # NaN where something was freed
        got = layer.replay().clone()
        torch.cuda.synchronize()
        args, kw = arguments()
        eager = layer.forward(*args, **kw)
        assert torch.equal(got, eager)
        results.append(got)
        del filler
    assert not torch.equal(results[0], results[1]) and not torch.equal(results[1], results[2])


def test_packed_weights_go_where_they_are_told_to(g):
    codes, scales = g.quantize_groups_int4(torch.randn((36, 256), device="cuda"), 64)
    packed = g.pack_int4_groups(codes, scales, 64)
    out = torch.zeros_like(packed)
    assert g.pack_int4_groups(codes, scales, 64, out=out) is out and torch.equal(out, packed)
    for bad in (out[:-16], out.to(torch.int8), out.cpu()):
        with pytest.raises(ValueError):
            g.pack_int4_groups(codes, scales, 64, out=bad)


def test_what_a_later_call_would_refuse_is_not_in_the_cache(setup):
    """Tokens that the sequences cannot share, a table or lengths of another batch or type: refused before anything is written"""
    layer, good = setup["layer"], _inputs(setup, 3, 2, 30)
    before = layer.cache.clone()
    table, state_lens = dev(setup["table"]), dev(setup["state_lens"])

    def step(i, table=table, state_lens=state_lens, kv_lens=good["kv_lens"]):
        return layer.forward(i["x"], (_rms, _rms, _rms), (dev(setup["cos"]), dev(setup["sin"])), i["positions"], i["slots"], table, kv_lens, state_lens=state_lens)

    for bad in (lambda: step({n: t[:4].contiguous() for n, t in good.items()}), lambda: step(good, table=table[:2].contiguous()), lambda: step(good, table=table.long()),
                lambda: step(good, state_lens=state_lens[:1].contiguous()), lambda: step(good, kv_lens=good["kv_lens"].cpu())):
        with pytest.raises(ValueError):
            bad()
        assert torch.equal(before, layer.cache)
    step(good)
    assert not torch.equal(before, layer.cache)
    layer.cache.copy_(before)
