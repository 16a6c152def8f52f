"""Host-only checks of the decoder's operators: arguments that are refused before anything is launched, sizes of buffers, the places of the
4-bit formats.  No kernel is launched here."""
import ctypes
import os
import subprocess
import sys

import numpy as np
import pytest

import decoder_reference as ref
from test_abi_host import ROOT, lib  # noqa: F401

OK, ERR_NULL, ERR_SHAPE, ERR_ALIGN, ERR_UNSUPPORTED = range(5)
P, ODD = 0x10000, 0x10008  # never dereferenced: every call below fails validation first


@pytest.fixture(scope="module")
def g():
    pytest.importorskip("torch")
    from paper_2305_10727_amd import gpusq
    gpusq.lib()
    return gpusq


def _refuses(g, name, good, changes):
    """good: arguments by name, in order; changes: (status, {name: value})"""
    fn = getattr(g.lib(), name)
    for status, change in changes:
        assert set(change) <= set(good)
        assert fn(*{**good, **change}.values()) == status, (name, change)


def test_linear_int4(g):
    base = dict(W=P, group=64, codes=P, scales=P, N=64, K=128, stream=None)
    _refuses(g, "gpusq_quantize_groups_int4", base, [
        (ERR_NULL, dict(W=None)), (ERR_NULL, dict(codes=None)), (ERR_NULL, dict(scales=None)), (ERR_SHAPE, dict(N=0)), (ERR_SHAPE, dict(K=96)), (ERR_SHAPE, dict(K=-128)),
        (ERR_SHAPE, dict(N=2**31)), (ERR_UNSUPPORTED, dict(group=16)), (ERR_UNSUPPORTED, dict(group=0)), (ERR_ALIGN, dict(W=ODD)), (ERR_ALIGN, dict(codes=ODD)), (ERR_ALIGN, dict(scales=ODD))])
    base = dict(codes=P, scales=P, group=64, packed=P, N=64, K=128, stream=None)
    _refuses(g, "gpusq_pack_int4_groups", base, [(ERR_NULL, dict(packed=None)), (ERR_SHAPE, dict(K=32)), (ERR_UNSUPPORTED, dict(group=256)), (ERR_ALIGN, dict(packed=ODD))])
    base = dict(X=P, W=P, group=32, bias=P, Y=P, out_dt=g.F16, M=3, N=64, K=128, epilogue=g.EPI_BIAS, stream=None)
    _refuses(g, "gpusq_linear_int4", base, [
        (ERR_NULL, dict(X=None)), (ERR_NULL, dict(W=None)), (ERR_NULL, dict(Y=None)), (ERR_NULL, dict(bias=None)), (ERR_SHAPE, dict(M=0)), (ERR_SHAPE, dict(M=2**31)),
        (ERR_SHAPE, dict(M=16 * 65535 + 1)), (ERR_SHAPE, dict(K=100)), (ERR_UNSUPPORTED, dict(N=62)), (ERR_UNSUPPORTED, dict(out_dt=g.I8)), (ERR_UNSUPPORTED, dict(epilogue=5)),
        (ERR_UNSUPPORTED, dict(group=8)), (ERR_ALIGN, dict(X=ODD)), (ERR_ALIGN, dict(W=ODD)), (ERR_ALIGN, dict(Y=ODD)), (ERR_ALIGN, dict(bias=ODD))])
    size = g.lib().gpusq_int4_groups_packed_bytes
    assert size(64, 128, 32) == 4 * (1024 + 128) and size(65, 129 * 32, 32) == 5 * 33 * 1152 and size(16, 192, 64) == 2 * (1024 + 64) and size(16, 128, 128) == 1024 + 32
    assert size(64, 100, 32) == 0 and size(64, 128, 48) == 0 and size(0, 128, 32) == 0


def test_qk_norm_rope(g):
    base = dict(qkv=P, dt=g.F16, row_stride=512, tokens=3, heads=4, kv_heads=2, head_dim=64, norm=1, qw=P, kw=P, eps=1e-6, cos=P, sin=P, positions=P, rows=9, rot=64, interleaved=0,
                q=P, k=P, v=P, cache=P, slots=P, pages=4, stream=None)
    _refuses(g, "gpusq_qk_norm_rope", base, [
        (ERR_NULL, dict(qkv=None)), (ERR_NULL, dict(q=None)), (ERR_NULL, dict(slots=None)), (ERR_NULL, dict(cos=None)), (ERR_NULL, dict(sin=None)), (ERR_NULL, dict(positions=None)),
        (ERR_NULL, dict(cache=None, k=None, v=None)), (ERR_UNSUPPORTED, dict(cache=None)), (ERR_SHAPE, dict(tokens=0)), (ERR_SHAPE, dict(heads=3)), (ERR_SHAPE, dict(kv_heads=0)),
        (ERR_SHAPE, dict(row_stride=504)), (ERR_UNSUPPORTED, dict(row_stride=516)), (ERR_SHAPE, dict(rot=72)), (ERR_SHAPE, dict(rot=-8)), (ERR_UNSUPPORTED, dict(rot=20)),
        (ERR_SHAPE, dict(rows=0)), (ERR_SHAPE, dict(pages=0)), (ERR_SHAPE, dict(pages=2**25)), (ERR_UNSUPPORTED, dict(dt=g.I8)), (ERR_UNSUPPORTED, dict(eps=-1.0)),
        (ERR_UNSUPPORTED, dict(eps=float("nan"))), (ERR_UNSUPPORTED, dict(head_dim=60)), (ERR_UNSUPPORTED, dict(head_dim=264, row_stride=4096)), (ERR_ALIGN, dict(qkv=ODD)),
        (ERR_ALIGN, dict(q=ODD)), (ERR_ALIGN, dict(k=ODD)), (ERR_ALIGN, dict(v=ODD)), (ERR_ALIGN, dict(cache=ODD)), (ERR_ALIGN, dict(qw=ODD)), (ERR_ALIGN, dict(kw=ODD)),
        (ERR_ALIGN, dict(cos=ODD)), (ERR_ALIGN, dict(sin=ODD)), (ERR_ALIGN, dict(slots=P + 2)), (ERR_ALIGN, dict(positions=P + 1))])


def test_attention_kv4(g):
    base = dict(q=P, cache=P, table=P, lens=P, cu=P, out=P, ws=P, tokens=5, batch=2, max_q=3, max_pages=100, pages=300, heads=8, kv_heads=2, head_dim=128, scale=0.0, stream=None)
    _refuses(g, "gpusq_attention_kv4", base, [
        (ERR_NULL, dict(q=None)), (ERR_NULL, dict(cache=None)), (ERR_NULL, dict(table=None)), (ERR_NULL, dict(lens=None)), (ERR_NULL, dict(out=None)), (ERR_NULL, dict(ws=None)),
        (ERR_SHAPE, dict(heads=7)), (ERR_SHAPE, dict(tokens=0)), (ERR_SHAPE, dict(batch=0)), (ERR_SHAPE, dict(max_q=6)), (ERR_SHAPE, dict(cu=None)), (ERR_SHAPE, dict(max_pages=0)),
        (ERR_SHAPE, dict(max_pages=2**25)), (ERR_SHAPE, dict(pages=0)), (ERR_SHAPE, dict(tokens=2**29)), (ERR_UNSUPPORTED, dict(head_dim=12)), (ERR_UNSUPPORTED, dict(scale=-1.0)),
        (ERR_UNSUPPORTED, dict(scale=float("nan"))), (ERR_UNSUPPORTED, dict(scale=float("inf"))), (ERR_ALIGN, dict(q=ODD)), (ERR_ALIGN, dict(cache=ODD)), (ERR_ALIGN, dict(out=ODD)),
        (ERR_ALIGN, dict(ws=ODD)), (ERR_ALIGN, dict(table=P + 2)), (ERR_ALIGN, dict(lens=P + 2)), (ERR_ALIGN, dict(cu=P + 2))])
    size = g.lib().gpusq_attention_kv4_workspace_bytes
    assert size(1, 1, 1, 1, 8, 2, 128) == 0 and size(1, 1, 1, 2000, 8, 2, 128) % (8 * 130 * 4) == 0 < size(1, 1, 1, 2000, 8, 2, 128)
    assert size(0, 1, 1, 1, 8, 2, 128) == 0 and size(1, 1, 1, 2000, 8, 3, 128) == 0
    assert g.lib().gpusq_kv4_page_bytes(2, 128) == 2 * 9216 and g.lib().gpusq_kv4_page_bytes(1, 40) == 4608 and g.lib().gpusq_kv4_page_bytes(3, 136) == 3 * 18432
    assert g.lib().gpusq_kv4_page_bytes(0, 128) == 0 and g.lib().gpusq_kv4_page_bytes(2, 260) == 0


def test_cross_attention(g):
    base = dict(q=P, k=P, v=P, lens=P, mask=P, out=P, ws=P, batch=1, q_len=1, kv_len=5000, heads=8, kv_heads=2, head_dim=64, qb=512, qt=512, qh=64, kb=640000, kt=128, kh=64, vb=640000,
                vt=128, vh=64, scale=0.0, stream=None)
    _refuses(g, "gpusq_cross_attention", base, [
        (ERR_NULL, dict(q=None)), (ERR_NULL, dict(k=None)), (ERR_NULL, dict(v=None)), (ERR_NULL, dict(out=None)), (ERR_NULL, dict(ws=None)), (ERR_SHAPE, dict(heads=9)),
        (ERR_SHAPE, dict(batch=0)), (ERR_SHAPE, dict(q_len=0)), (ERR_SHAPE, dict(kv_len=0)), (ERR_SHAPE, dict(kv_len=2**31 - 1)), (ERR_SHAPE, dict(batch=2**20, q_len=2**20)),
        (ERR_SHAPE, dict(qt=-8)), (ERR_SHAPE, dict(vb=2**41)), (ERR_ALIGN, dict(kt=132)), (ERR_ALIGN, dict(vh=60)), (ERR_ALIGN, dict(qb=4)), (ERR_UNSUPPORTED, dict(head_dim=4)),
        (ERR_UNSUPPORTED, dict(scale=-0.1)), (ERR_ALIGN, dict(q=ODD)), (ERR_ALIGN, dict(k=ODD)), (ERR_ALIGN, dict(v=ODD)), (ERR_ALIGN, dict(out=ODD)), (ERR_ALIGN, dict(lens=P + 1))])
    size = g.lib().gpusq_cross_attention_workspace_bytes
    assert size(64, 1, 577, 16, 16, 64) == 0 and size(1, 1, 5000, 8, 2, 64) > 0 and size(1, 1, 0, 8, 2, 64) == 0


def test_floats_reach_their_parameters_among_the_others():
    """The extension module passes floats in registers of their own: a C function of mixed parameters sees each where it stands"""
    torch = pytest.importorskip("torch")
    from paper_2305_10727_amd import _fastcall, gpusq
    seen = []
    proto = ctypes.CFUNCTYPE(ctypes.c_int, *([ctypes.c_long] * 3), ctypes.c_float, *([ctypes.c_long] * 6), ctypes.c_float, ctypes.c_long)
    fn = proto(lambda *a: seen.append(a) or 0)
    _fastcall.setup(lambda: 0, lambda d: 77, gpusq._raise)
    try:
        call = _fastcall.FastCall("mixed", ctypes.cast(fn, ctypes.c_void_p).value, "iiifiiiiiifs")
        call(1, 2, 3, 0.5, 4, 5, 6, 7, 8, 9, -1.0)
    finally:
        _fastcall.setup(torch._C._cuda_getDevice, gpusq._stream_of, gpusq._raise)
    assert seen == [(1, 2, 3, 0.5, 4, 5, 6, 7, 8, 9, -1.0, 77)]
    with pytest.raises(TypeError):
        call(1, 2, 3, "x", 4, 5, 6, 7, 8, 9, 1.0)
    with pytest.raises(ValueError):
        _fastcall.FastCall("three", 1, "fff")


@pytest.mark.parametrize("D", [8, 64, 80, 128, 136, 256])
def test_every_place_of_a_page_is_used_once(D):
    """Of a page's nibbles and scales no two values share one, none is left over, and a token's key bytes and 16-bit value places are its own"""
    p = ref.Places(D)
    nibbles = np.concatenate([(p.k_byte * 2 + p.k_shift // 4).ravel(), (p.v_byte * 2 + p.v_shift // 4).ravel()])
    scales = np.concatenate([p.k_scale.ravel(), p.v_scale.ravel()])
    taken = np.concatenate([nibbles, *[scales * 4 + i for i in range(4)]])
    assert np.array_equal(np.sort(taken), np.arange(2 * p.bytes))
    for byte, unit in ((p.k_byte, 1), (p.v_byte, 2)):
        owner = {}
        for t in range(64):
            for at in set((byte[t] // unit).tolist()):
                assert owner.setdefault(at, t) == t


def test_formats_read_back():
    r = np.random.default_rng(0)
    for D in (40, 128, 200):
        x = r.standard_normal((2, 3, 64, D)).astype(np.float32)
        c, s = ref.cache_codes(x)
        assert abs(c).max() == 7
        K, V = ref.read_pages(ref.write_pages(c, s, -c, s, D), D)
        exp = c * s.astype(np.float64).repeat(32, -1)[..., :D]
        assert np.array_equal(K, exp) and np.array_equal(V, -exp)
        assert np.array_equal(exp.astype(np.float16).astype(np.float64), exp)  # fp16 numbers
        assert (np.abs(exp - x) <= 0.56 * s.astype(np.float64).repeat(32, -1)[..., :D]).all()


def test_plans_of_attention(tmp_path):
    """Who takes which columns of an attention, walked on the host with the code the kernels read it with (attend_plan_walk.cpp)"""
    exe = str(tmp_path / "walk")
    build = subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                            "-I", os.path.join(ROOT, "paper_2305_10727_amd", "csrc"), os.path.join(ROOT, "tests", "attend_plan_walk.cpp"), "-o", exe],
                           capture_output=True, text=True)
    assert build.returncode == 0, build.stderr
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and run.stdout == "ok\n", run.stdout


def test_states_that_a_loop_cannot_look_beyond(g):
    """The most states: what the loops over the keys look ahead of a tile stays a number of 31 bits"""
    base = dict(q=P, k=P, v=P, lens=None, mask=None, out=P, ws=P, batch=1, q_len=100, kv_len=2**31 - 129, heads=1, kv_heads=1, head_dim=64, qb=64, qt=64, qh=64, kb=0, kt=0, kh=64, vb=0,
                vt=0, vh=64, scale=-1.0, stream=None)
    _refuses(g, "gpusq_cross_attention", base, [(ERR_UNSUPPORTED, dict()), (ERR_SHAPE, dict(kv_len=2**31 - 128)), (ERR_SHAPE, dict(kv_len=2**31 - 65))])


def test_a_layer_keeps_its_weights_where_they_are(g, monkeypatch):
    """A captured step of pipeline.DecoderLayer has the addresses of its weights: preparing others does not move them"""
    torch = pytest.importorskip("torch")
    from paper_2305_10727_amd import pipeline
    layer = pipeline.DecoderLayer(64, 2, 1, 32, 128, 1, 8, 64, 1, device="cpu")
    monkeypatch.setattr(layer.states_kv, "prepare_weights", lambda W: None)
    monkeypatch.setattr(g, "quantize_groups_int4", lambda W, group: (W, W))
    monkeypatch.setattr(g, "pack_int4_groups", lambda codes, scales, group, out=None: torch.empty(codes.numel(), dtype=torch.uint8) if out is None else out)
    weights = {n: torch.zeros(shape) for n, shape in layer.widths.items()}
    layer.prepare_weights(weights, None)
    first = dict(layer.packed)
    layer.prepare_weights(weights, None)
    assert set(first) == set(layer.widths) and all(layer.packed[n] is first[n] for n in first)


def test_what_no_launch_counts_is_refused(g):
    """A launch has 2^32 - 1 threads: one more workgroup than that is a shape that is refused, one less meets the next check"""
    base = dict(q=ODD, cache=P, table=P, lens=P, cu=None, out=P, ws=P, tokens=65535, batch=65535, max_q=1, max_pages=1, pages=300, heads=128, kv_heads=128, head_dim=64, scale=0.0, stream=None)
    _refuses(g, "gpusq_attention_kv4", base, [(ERR_ALIGN, dict()), (ERR_SHAPE, dict(tokens=65536, batch=65536)),
                                              (ERR_SHAPE, dict(tokens=2**24, batch=1, cu=P, heads=1, kv_heads=1, max_pages=2000)),  # the join's rows
                                              (ERR_ALIGN, dict(tokens=2**24 - 1, batch=1, cu=P, heads=1, kv_heads=1, max_pages=2000))])
    base = dict(q=ODD, k=P, v=P, lens=None, mask=None, out=P, ws=P, batch=65535, q_len=1, kv_len=40, heads=128, kv_heads=128, head_dim=64, qb=8192, qt=8192, qh=64, kb=0, kt=64, kh=64, vb=0,
                vt=64, vh=64, scale=0.0, stream=None)
    _refuses(g, "gpusq_cross_attention", base, [(ERR_ALIGN, dict()), (ERR_SHAPE, dict(batch=65536))])
    base = dict(W=ODD, group=64, codes=P, scales=P, N=2**20 - 1, K=2**15, stream=None)
    _refuses(g, "gpusq_quantize_groups_int4", base, [(ERR_ALIGN, dict()), (ERR_SHAPE, dict(N=2**20))])
    base = dict(codes=ODD, scales=P, group=64, packed=P, N=2**20 - 16, K=2**15, stream=None)
    _refuses(g, "gpusq_pack_int4_groups", base, [(ERR_ALIGN, dict()), (ERR_SHAPE, dict(N=2**20 - 15))])
    assert g.lib().gpusq_attention_kv4_workspace_bytes(1, 1, 1, 2**25 - 2, 8, 2, 128) > 0 == g.lib().gpusq_attention_kv4_workspace_bytes(1, 1, 1, 2**25 - 1, 8, 2, 128)


def test_rows_whose_last_steps_pass_31_bits(g):
    """The longest rows of a 4-bit layer: a workgroup's 64 steps of 128 behind the last one are still numbers of 31 bits"""
    base = dict(X=ODD, W=P, group=32, bias=None, Y=P, out_dt=g.F16, M=1, N=4, K=2**31 - 8224, epilogue=0, stream=None)
    assert -(-base["K"] // 128) * 128 + 63 * 128 + 96 < 2**31
    _refuses(g, "gpusq_linear_int4", base, [(ERR_ALIGN, dict()), (ERR_SHAPE, dict(K=2**31 - 8192)), (ERR_SHAPE, dict(K=2**31 - 32))])


@pytest.mark.parametrize("name,sizes", [("attention_kv4", (1, 2**30, 2**30, 2000, 65536, 1, 64)), ("attention_kv4", (2**31 - 1, 1, 1, 2**20, 65536, 32768, 256)),
                                        ("attention_kv4", (1, 1, 2, 2000, 8, 2, 64)), ("cross_attention", (2**30, 2**30, 5000, 65536, 1, 64)),
                                        ("cross_attention", (1, 1, 2**31 - 1, 8, 2, 64))])
def test_workspaces_of_sizes_that_are_refused(g, name, sizes):
    """0 for what the call would refuse, without a product that passes 64 bits (a divisor that wrapped to 0 would end the process: asked in one of its own)"""
    ask = "import sys; sys.path.insert(0, %r)\nfrom paper_2305_10727_amd import gpusq\nprint(gpusq.lib().gpusq_%s_workspace_bytes%r)" % (ROOT, name, sizes)
    run = subprocess.run([sys.executable, "-c", ask], capture_output=True, text=True, timeout=300)
    assert run.returncode == 0 and run.stdout == "0\n", run


def test_strides_of_dimensions_of_one(g):
    torch = pytest.importorskip("torch")
    t = torch.zeros(64).as_strided((1, 3, 1, 8), (5, 16, 7, 1))
    assert g._strides(t) == (0, 16, 0, 1) and g._strides(torch.zeros(())) == ()
    with pytest.raises(TypeError):
        g._strides(3)
