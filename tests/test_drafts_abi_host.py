"""Host-only checks of the operators that answer with drafted tokens: arguments that are refused before anything is launched, sizes of buffers.  No kernel is
launched here."""
import ctypes
import os
import subprocess

import pytest

from test_decoder_abi_host import ERR_ALIGN, ERR_NULL, ERR_SHAPE, ERR_UNSUPPORTED, ODD, P, ROOT, _refuses, g  # noqa: F401


def test_plans(tmp_path):
    """How products, rows of logits and caches are cut, walked on the host with the code the kernels read it with (drafts_plan_walk.cpp)"""
    exe = str(tmp_path / "walk")
    build = subprocess.run(["g++", "-O2", "-std=c++17", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                            "-I", os.path.join(ROOT, "paper_2305_10727_amd", "csrc"), os.path.join(ROOT, "tests", "drafts_plan_walk.cpp"), "-o", exe],
                           capture_output=True, text=True)
    assert build.returncode == 0, build.stderr
    run = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert run.returncode == 0 and run.stdout == "ok\n", run.stdout


def test_a_trees_workspace(g):
    """Of sizes that the call would refuse: 0"""
    size = g.lib().gpusq_attention_tree_kv4_workspace_bytes
    assert size(63, 1, 63, 1025, 32, 8, 128) > 0 == size(63, 1, 64, 1025, 32, 8, 128) == size(63, 1, 63, 2**25 - 1, 32, 8, 128) == size(63, 1, 63, 1025, 31, 8, 128)


def test_attention_tree_kv4(g):
    base = dict(q=P, cache=P, table=P, lens=P, cu=P, tree=P, words=2, out=P, ws=P, tokens=70, batch=2, max_q=40, max_pages=100, pages=300, heads=8, kv_heads=2, head_dim=128, scale=0.0,
                stream=None)
    _refuses(g, "gpusq_attention_tree_kv4", base, [
        (ERR_NULL, dict(q=None)), (ERR_NULL, dict(cache=None)), (ERR_NULL, dict(table=None)), (ERR_NULL, dict(lens=None)), (ERR_NULL, dict(out=None)), (ERR_NULL, dict(tree=None)),
        (ERR_NULL, dict(ws=None)), (ERR_SHAPE, dict(words=1)), (ERR_SHAPE, dict(words=0)), (ERR_SHAPE, dict(words=2**31)), (ERR_SHAPE, dict(max_q=71, words=3)), (ERR_SHAPE, dict(cu=None)),
        (ERR_SHAPE, dict(tokens=2**30, max_q=2**30, words=2**25, heads=1, kv_heads=1)), (ERR_SHAPE, dict(heads=7)), (ERR_SHAPE, dict(max_pages=0)), (ERR_SHAPE, dict(pages=0)),
        (ERR_UNSUPPORTED, dict(head_dim=12)), (ERR_UNSUPPORTED, dict(scale=-1.0)), (ERR_ALIGN, dict(tree=P + 2)), (ERR_ALIGN, dict(q=ODD)), (ERR_ALIGN, dict(ws=ODD)), (ERR_ALIGN, dict(cu=P + 2))])


def test_draft_tree(g):
    base = dict(parents=P, lens=P, cu=P, table=P, tree=P, positions=P, slots=P, tokens=70, batch=2, max_q=40, max_pages=100, stream=None)
    _refuses(g, "gpusq_draft_tree", base, [
        (ERR_NULL, dict(parents=None)), (ERR_NULL, dict(lens=None)), (ERR_NULL, dict(tree=None)), (ERR_NULL, dict(table=None)), (ERR_SHAPE, dict(tokens=0)), (ERR_SHAPE, dict(batch=0)),
        (ERR_SHAPE, dict(batch=2**24)), (ERR_SHAPE, dict(max_q=0)), (ERR_SHAPE, dict(max_q=71)), (ERR_SHAPE, dict(cu=None)), (ERR_UNSUPPORTED, dict(tokens=600, max_q=513)),
        (ERR_SHAPE, dict(max_pages=0)), (ERR_SHAPE, dict(max_pages=2**25)), (ERR_ALIGN, dict(parents=P + 2)), (ERR_ALIGN, dict(lens=P + 1)), (ERR_ALIGN, dict(cu=P + 2)),
        (ERR_ALIGN, dict(table=P + 2)), (ERR_ALIGN, dict(tree=P + 2)), (ERR_ALIGN, dict(positions=P + 2)), (ERR_ALIGN, dict(slots=P + 2))])


def test_accept_drafts(g):
    two = (ctypes.c_void_p * 2)(P, P + 2**20)
    at = lambda *p: ctypes.addressof(kept.setdefault(p, (ctypes.c_void_p * len(p))(*p)))  # noqa: E731
    kept = {}
    base = dict(drafted=P, sampled=P, parents=P, lens=P, cu=P, table=P, caches=ctypes.addressof(two), layers=2, path=P, accepted=P, answers=P, new=P, tokens=70, batch=2, max_q=40, max_pages=9,
                pages=16, kv_heads=2, head_dim=128, stream=None)
    size = 16 * 2 * 9216
    _refuses(g, "gpusq_accept_drafts", base, [
        (ERR_NULL, dict(drafted=None)), (ERR_NULL, dict(sampled=None)), (ERR_NULL, dict(parents=None)), (ERR_NULL, dict(lens=None)), (ERR_NULL, dict(path=None)), (ERR_NULL, dict(accepted=None)),
        (ERR_NULL, dict(answers=None)), (ERR_NULL, dict(new=None)), (ERR_NULL, dict(caches=None)), (ERR_NULL, dict(table=None)), (ERR_NULL, dict(caches=at(P, None))),
        (ERR_SHAPE, dict(tokens=0)), (ERR_SHAPE, dict(max_q=71)), (ERR_SHAPE, dict(cu=None)), (ERR_UNSUPPORTED, dict(tokens=600, max_q=513)), (ERR_SHAPE, dict(layers=-1)), (ERR_SHAPE, dict(layers=1025)),
        (ERR_SHAPE, dict(kv_heads=0)), (ERR_UNSUPPORTED, dict(head_dim=100)), (ERR_SHAPE, dict(max_pages=0)), (ERR_SHAPE, dict(pages=0)), (ERR_SHAPE, dict(pages=2**25)),
        (ERR_SHAPE, dict(kv_heads=65535)), (ERR_SHAPE, dict(batch=2**23, tokens=2**23 * 40, cu=P)), (ERR_UNSUPPORTED, dict(caches=at(P, P))), (ERR_UNSUPPORTED, dict(caches=at(P, P + size - 16))),
        (ERR_UNSUPPORTED, dict(caches=at(P + size - 16, P))), (ERR_ALIGN, dict(caches=at(P, P + size + 8))), (ERR_ALIGN, dict(drafted=P + 2)), (ERR_ALIGN, dict(sampled=P + 2)),
        (ERR_ALIGN, dict(parents=P + 2)), (ERR_ALIGN, dict(lens=P + 2)), (ERR_ALIGN, dict(cu=P + 2)), (ERR_ALIGN, dict(table=P + 2)), (ERR_ALIGN, dict(path=P + 2)), (ERR_ALIGN, dict(accepted=P + 2)),
        (ERR_ALIGN, dict(answers=P + 2)), (ERR_ALIGN, dict(new=P + 2)),
        (ERR_SHAPE, dict(layers=0, caches=None, tokens=41, max_q=42)), (ERR_ALIGN, dict(layers=0, caches=None, table=None, path=P + 2))])


def test_linear_int8_tokens(g):
    base = dict(X=P, dt=g.F16, Wq=P, w_scale=P, bias=P, Y=P, out_dt=g.F16, ws=P, M=3, N=64, K=128, epilogue=g.EPI_BIAS, stream=None)
    _refuses(g, "gpusq_linear_int8_tokens", base, [
        (ERR_NULL, dict(X=None)), (ERR_NULL, dict(Wq=None)), (ERR_NULL, dict(w_scale=None)), (ERR_NULL, dict(bias=None)), (ERR_NULL, dict(Y=None)), (ERR_NULL, dict(ws=None)), (ERR_SHAPE, dict(M=0)),
        (ERR_SHAPE, dict(N=0)), (ERR_SHAPE, dict(K=0)), (ERR_SHAPE, dict(K=132112)), (ERR_SHAPE, dict(M=64 * 65535 + 1)), (ERR_SHAPE, dict(N=2**24 + 4)), (ERR_SHAPE, dict(M=2**21, N=2**20)),
        (ERR_UNSUPPORTED, dict(K=120)), (ERR_UNSUPPORTED, dict(N=62)), (ERR_UNSUPPORTED, dict(dt=g.I8)), (ERR_UNSUPPORTED, dict(out_dt=g.I32)), (ERR_UNSUPPORTED, dict(epilogue=4)),
        (ERR_ALIGN, dict(X=ODD)), (ERR_ALIGN, dict(Wq=ODD)), (ERR_ALIGN, dict(w_scale=ODD)), (ERR_ALIGN, dict(bias=ODD)), (ERR_ALIGN, dict(Y=ODD)), (ERR_ALIGN, dict(ws=ODD))])
    size = g.lib().gpusq_linear_int8_tokens_workspace_bytes
    assert size(3, 128) >= 3 * 128 + 12 and size(0, 128) == 0 and size(3, 132112) == 0 and size(3, -1) == 0 and size(2**31, 16) == 0 and size(5, 16) % 16 == 0


def test_sample_tokens(g):
    base = dict(logits=P, dt=g.F32, stride=1000, random=P, T=P, k=P, p=P, m=P, tokens=P, probs=P, ws=P, rows=3, V=999, stream=None)
    _refuses(g, "gpusq_sample_tokens", base, [
        (ERR_NULL, dict(logits=None)), (ERR_NULL, dict(random=None)), (ERR_NULL, dict(tokens=None)), (ERR_NULL, dict(probs=None)), (ERR_SHAPE, dict(rows=0)), (ERR_SHAPE, dict(V=0)),
        (ERR_SHAPE, dict(V=1001)), (ERR_SHAPE, dict(V=2**18 + 1, stride=2**19)), (ERR_SHAPE, dict(stride=2**31)), (ERR_SHAPE, dict(rows=2**22)), (ERR_UNSUPPORTED, dict(dt=g.I8)),
        (ERR_ALIGN, dict(logits=P + 2)), (ERR_ALIGN, dict(logits=P + 1, dt=g.F16)), (ERR_ALIGN, dict(random=P + 2)), (ERR_ALIGN, dict(T=P + 2)), (ERR_ALIGN, dict(k=P + 2)), (ERR_ALIGN, dict(p=P + 2)),
        (ERR_ALIGN, dict(m=P + 2)), (ERR_ALIGN, dict(tokens=P + 2)), (ERR_ALIGN, dict(probs=P + 2)), (ERR_ALIGN, dict(ws=ODD)), (ERR_NULL, dict(V=200000, stride=200000, ws=None))])
    size = g.lib().gpusq_sample_tokens_workspace_bytes
    assert size(1, 200000) > 0 and size(1, 200000) % 16 == 0 and size(1000, 200000) == 0 and size(1, 1000) == 0 and size(0, 1000) == 0 and size(1, 2**18 + 1) == 0


def test_results_in_one_allocation(g):
    """Types and sizes as asked for, each at a multiple of 16 bytes, none over another"""
    torch = pytest.importorskip("torch")
    like = torch.zeros(1)
    wanted = [(torch.int32, 3, 5), (torch.float32, 7), (torch.int32, 0), (torch.uint8, 33), (torch.float16, 2, 1, 3, 1), (torch.int64, 1)]
    got = g._empties(like, *wanted)
    assert isinstance(got, tuple) and len(got) == len(wanted)
    for i, (t, (dtype, *sizes)) in enumerate(zip(got, wanted)):
        assert t.dtype is dtype and list(t.shape) == sizes and t.is_contiguous() and t.data_ptr() % 16 == 0 and t.device == like.device
        t.fill_(i + 1)
    assert all((t == i + 1).all() for i, t in enumerate(got))
    kept = got[3]
    del got, t
    assert (kept.clone() == 4).all()
    for bad in ((), (torch.int32,), ((torch.int32,),), ((3, 4),), ([torch.int32, 3],), ((torch.int32, 1, 1, 1, 1, 1),), ((torch.int32, "3"),), ((torch.int32, 1),) * 9):
        with pytest.raises(TypeError):
            g._empties(like, *bad)
    for bad in ((torch.int32, -1), (torch.int32, 2**40, 2**40)):
        with pytest.raises((ValueError, TypeError)):
            g._empties(like, (torch.int32, 2), bad)
    with pytest.raises(TypeError):
        g._empties(3, (torch.int32, 2))
