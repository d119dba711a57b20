"""Paged sequences and prepared projections without a GPU: the page lists and attention passes under
sanitizers, and the refusals of every entry point, which come before any device work."""
import ctypes
import os

import pytest
import torch

from paper_2609_23286_amd import rv
from test_sanitizers import NATIVE, ROOT, SAN, build_and_run

vp = ctypes.c_void_p
A = vp(4096)   # a device address that nothing reads
B = vp(4104)   # not 16-byte aligned
INF, NAN = float("inf"), float("nan")


def test_page_lists_and_passes_under_sanitizers(tmp_path):
    exe = str(tmp_path / "seq_logic_check")
    build_and_run(["g++", "-std=c++17", *SAN, "-o", exe, os.path.join(NATIVE, "seq_logic_check.cpp"),
                   os.path.join(ROOT, "paper_2609_23286_amd", "csrc", "rv_seq.cpp")], exe, "sequence logic OK")


def prep(n_q=4, n_kv=2, norm=2, axes=2, eps=1e-5, base=100.0, vecs=(None,) * 4):
    return rv.rv_qkv_prep(n_q, n_kv, norm, axes, eps, base, *vecs)


def forward(p, q=A, qs=256, k=A, ks=128, v=A, vs=128, dtype=0, n=10, pos=A, Q=A, K=A, V=A):
    return rv.lib().rv_prepare_qkv(None if p is None else ctypes.byref(p), q, qs, k, ks, v, vs, dtype, n, pos, Q, K, V,
                                   None)


def backward(p, q=A, qs=256, k=A, ks=128, dtype=0, n=10, pos=A, dQ=A, dK=A, dV=A, dq=A, dqs=256, dk=A, dks=128, dv=A,
             dvs=128, sums=(None,) * 4):
    return rv.lib().rv_prepare_qkv_bwd(None if p is None else ctypes.byref(p), q, qs, k, ks, dtype, n, pos, dQ, dK, dV,
                                       dq, dqs, dk, dks, dv, dvs, *sums, None)


def message():
    return rv.lib().rv_last_error().decode()


BAD_PREPS = [
    (lambda: None, "NULL"),
    (lambda: prep(n_q=0), "head counts"),
    (lambda: prep(n_kv=0), "head counts"),
    (lambda: prep(n_q=1025), "head counts"),
    (lambda: prep(norm=3), "norm"),
    (lambda: prep(norm=-1), "norm"),
    (lambda: prep(axes=3), "n_axes"),
    (lambda: prep(axes=-1), "n_axes"),
    (lambda: prep(eps=-1e-5), "eps"),
    (lambda: prep(eps=NAN), "eps"),
    (lambda: prep(eps=INF), "eps"),
    (lambda: prep(base=0.5), "base"),
    (lambda: prep(base=NAN), "base"),
    (lambda: prep(base=INF), "base"),
    (lambda: prep(norm=0, vecs=(4096, None, None, None)), "belong to a norm"),
    (lambda: prep(vecs=(None, None, 4104, None)), "aligned"),
]


@pytest.mark.parametrize("i", range(len(BAD_PREPS)))
def test_bad_preparations_are_refused(i):
    make, words = BAD_PREPS[i]
    for call in (forward, backward):
        assert call(make()) == rv.RV_ERR_INVALID
        assert words in message()


@pytest.mark.parametrize("bad,words", [
    (dict(n=-1), "n_tokens"), (dict(dtype=2), "dtype"), (dict(pos=None), "pos"), (dict(q=None), "q is required"),
    (dict(k=None), "k is required"), (dict(qs=255), "row stride"), (dict(ks=120), "row stride"),
    (dict(qs=257), "16 bytes"), (dict(q=B), "16 bytes"), (dict(k=B), "16 bytes")])
def test_bad_rows_are_refused(bad, words):
    for call in (forward, backward):
        assert call(prep(), **bad) == rv.RV_ERR_INVALID
        assert words in message()


@pytest.mark.parametrize("bad,words", [
    (dict(v=None), "both"), (dict(V=None), "both"), (dict(vs=64), "row stride"), (dict(v=B), "16 bytes"),
    (dict(Q=None), "Q and K"), (dict(K=None), "Q and K"), (dict(Q=B), "aligned"), (dict(V=B), "aligned")])
def test_bad_forward_arguments_are_refused(bad, words):
    assert forward(prep(), **bad) == rv.RV_ERR_INVALID
    assert words in message()


@pytest.mark.parametrize("bad,words", [
    (dict(dV=None), "both"), (dict(dv=None), "both"), (dict(dQ=None), "dQ and dK"), (dict(dK=None), "dQ and dK"),
    (dict(dq=None), "dq is required"), (dict(dk=None), "dk is required"), (dict(dqs=128), "row stride"),
    (dict(dvs=100), "row stride"), (dict(dQ=B), "aligned"), (dict(dk=B), "16 bytes")])
def test_bad_backward_arguments_are_refused(bad, words):
    assert backward(prep(), **bad) == rv.RV_ERR_INVALID
    assert words in message()
    assert backward(prep(norm=0), sums=(A, None, None, None)) == rv.RV_ERR_INVALID
    assert "belong to a norm" in message()


def test_nothing_to_do_is_fine():
    assert forward(prep(), n=0, q=None, k=None, v=None, pos=None, Q=None, K=None, V=None) == rv.RV_OK
    assert backward(prep(), n=0, q=None, k=None, pos=None, dQ=None) == rv.RV_OK


def test_an_uninitialised_device_is_refused():
    """The arguments pass; there is no device here, or rv_init has not run on it."""
    if torch.cuda.is_available():
        pytest.skip("there is a device")
    assert forward(prep()) in (rv.RV_ERR_INVALID, rv.RV_ERR_HIP) and message()
    assert backward(prep()) in (rv.RV_ERR_INVALID, rv.RV_ERR_HIP)
    h = vp()
    assert rv.lib().rv_pool_create(16, 64, 10, 4, 1000, ctypes.byref(h)) == rv.RV_ERR_HIP and not h.value


@pytest.mark.parametrize("args", [(0, 64, 1, 1, 1), (1025, 64, 1, 1, 1), (16, 128, 1, 1, 1), (16, 64, 0, 1, 1),
                                  (16, 64, 1, 0, 1), (16, 64, 1, 1, 0), (16, 64, 1, 1, (1 << 30) + 1),
                                  (16, 64, 1, 1 << 30, 1 << 30)])
def test_bad_pools_are_refused(args):
    h = vp(1)
    assert rv.lib().rv_pool_create(*args, ctypes.byref(h)) == rv.RV_ERR_INVALID
    assert message() and not h.value
    assert rv.lib().rv_pool_create(*args, None) == rv.RV_ERR_INVALID


def test_calls_without_a_pool_are_refused():
    L, one = rv.lib(), (ctypes.c_int * 1)(0)
    rows = (ctypes.c_int64 * 1)(0)
    assert L.rv_pool_destroy(None) == rv.RV_OK
    assert L.rv_pool_free_pages(None) == -1 and L.rv_pool_len(None, 0) == -1
    assert L.rv_pool_open(None, ctypes.byref(ctypes.c_int())) == rv.RV_ERR_INVALID
    assert L.rv_pool_fork(None, 0, 0, 1, one, None) == rv.RV_ERR_INVALID
    assert L.rv_pool_close(None, 1, one) == rv.RV_ERR_INVALID
    assert L.rv_pool_truncate(None, 0, 0) == rv.RV_ERR_INVALID
    assert L.rv_pool_append(None, 1, one, A, A, one, None) == rv.RV_ERR_INVALID
    assert L.rv_pool_gather(None, 1, one, rows, rows, A, A, None) == rv.RV_ERR_INVALID
    assert L.rv_pool_compact(None, 1, one, rows, rows, A, None) == rv.RV_ERR_INVALID
    assert L.rv_attend_seqs(None, 1, one, one, A, A, A, 16, A, A, None) == rv.RV_ERR_INVALID
    assert L.rv_admit_seqs(None, 1, one, A, A, A, A, 10, None, 1, A, A, None) == rv.RV_ERR_INVALID
    assert L.rv_mem_stage_qkv(None, ctypes.byref(prep()), A, 256, A, 128, A, 128, 0, 10, A, A, None) == rv.RV_ERR_INVALID


def test_the_binding_refuses_what_the_library_cannot_see():
    with pytest.raises(ValueError, match="norm"):
        rv.QKVPrep(4, 2, norm="batch")
    with pytest.raises(TypeError, match="q_weight"):
        rv.QKVPrep(4, 2, q_weight=torch.ones(64, dtype=torch.float64))
    with pytest.raises(ValueError, match="device tensor"):
        rv.QKVPrep(4, 2, q_weight=torch.ones(64))
    for bad, words in ((torch.zeros(3, 256), "device tensor"), ("q", "expected a torch tensor")):
        with pytest.raises((ValueError, TypeError), match=words):
            rv._rows(bad, 4, "q")
    with pytest.raises(ValueError, match="2 values for 3"):
        rv._ints([1, 2], 3, "n_rows")
