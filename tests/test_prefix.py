"""Decode attention over shared prefixes on the CPU: its fp64 reference against the one without
sharing, and the refusals of the C ABI and of the binding before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

from oracle import paged
from paper_2608_04771_gb300 import build as B
from paper_2608_04771_gb300 import reco


@pytest.fixture(scope="module")
def L():
    B.build()
    return reco.lib()


# ---------------------------------------------------------------- the reference
def test_reference_is_the_decode_over_copies():
    """The same batch with every sequence's prefix copied into pages of its own."""
    rng = np.random.default_rng(1)
    page, per, d, group, shared = 4, 5, 6, [3, 3, 1, 3, 3, 3], [6, 6, 2, 0, 0, 0]
    n_pages = 40
    K, V = rng.standard_normal((2, n_pages, 2, page, d)), rng.standard_normal((2, n_pages, 2, page, d))
    table = rng.permutation(n_pages)[:6 * per].reshape(6, per)
    lens = np.array(shared)[None, :, None] + rng.integers(0, 9, (2, 6, 2))
    q, kn, vn = rng.standard_normal((2, 6, 6, d)), rng.standard_normal((2, 6, 2, d)), rng.standard_normal((2, 6, 2, d))
    K2, V2 = K.copy(), V.copy()
    for pool in (K2, V2):
        for j in range(6):
            pool[:, table[1, j // page], :, j % page] = pool[:, table[0, j // page], :, j % page]
    assert paged.prefix_lead(group) == [0, 0, 2, 3, 3, 3]
    a, b = lens.copy(), lens.copy()
    hidden = table.copy()
    hidden[1, 0] = 10 ** 6  # a whole page of the prefix: not looked at
    got = paged.prefix_decode(K, V, hidden, a, q, kn, vn, 0.4, group, shared)
    want = paged.decode(K2, V2, table, b, q, kn, vn, 0.4)
    for x, y in zip(got, want):
        assert np.abs(x - y).max() < 1e-12
    assert np.array_equal(a, b)


# ---------------------------------------------------------------- refusals
def _kv(**kw):
    a = dict(k=16, v=32, table=64, n_layers=2, B=3, H_q=8, H_kv=2, n_pages=20, max_pages=6, page=16, d=128,
             dtype=reco.RECO_BF16)
    a.update(kw)
    return reco.reco_paged_kv(*(a[f] for f, _ in reco.reco_paged_kv._fields_))


@pytest.mark.parametrize("kw,text,status", [
    (dict(group=None), b"NULL group", reco.RECO_EINVAL), (dict(shared=None), b"NULL group", reco.RECO_EINVAL),
    (dict(group=18), b"aligned", reco.RECO_EINVAL), (dict(shared=17), b"aligned", reco.RECO_EINVAL),
    (dict(q=None), b"NULL", reco.RECO_EINVAL), (dict(lens=None), b"NULL", reco.RECO_EINVAL),
    (dict(out=None), b"NULL", reco.RECO_EINVAL), (dict(k_new=16), b"k_new", reco.RECO_EINVAL),
    (dict(q=24), b"aligned", reco.RECO_EINVAL), (dict(out=20), b"aligned", reco.RECO_EINVAL),
    (dict(lse=17), b"aligned", reco.RECO_EINVAL), (dict(out_dtype=7), b"out_dtype", reco.RECO_EINVAL),
    (dict(scale=float("nan")), b"scale", reco.RECO_EINVAL), (dict(ws=None), b"workspace", reco.RECO_EINVAL),
    (dict(ws=128), b"aligned", reco.RECO_EINVAL), (dict(ws_bytes=-1), b"workspace", reco.RECO_EINVAL),
    (dict(kv=dict(H_q=34)), b"at most 16", reco.RECO_EUNSUPPORTED), (dict(kv=dict(d=96)), b"head dim", reco.RECO_EUNSUPPORTED),
    (dict(kv=dict(k=0)), b"NULL", reco.RECO_EINVAL), (dict(kv=dict(page=24)), b"page", reco.RECO_EUNSUPPORTED)])
def test_arguments_that_are_refused(L, kw, text, status):
    a = dict(kv={}, q=16, k_new=None, v_new=None, lens=16, group=16, shared=16, scale=0.1, out=16, out_dtype=0, lse=None,
             ws=256, ws_bytes=0)
    a.update(kw)
    p = lambda x: None if x is None else ctypes.c_void_p(x)  # noqa: E731
    n = reco.reco_paged_workspace_bytes(reco.RECO_OP_PAGED_PREFIX, _kv()) + a["ws_bytes"]
    st = L.reco_paged_prefix_attn(ctypes.byref(_kv(**a["kv"])), p(a["q"]), p(a["k_new"]), p(a["v_new"]), p(a["lens"]),
                                  p(a["group"]), p(a["shared"]), a["scale"], p(a["out"]), a["out_dtype"], p(a["lse"]),
                                  p(a["ws"]), n, None)
    assert st == status and text in L.reco_last_error(), (st, L.reco_last_error())


def test_workspace_size(L):
    size = lambda **kw: reco.reco_paged_workspace_bytes(reco.RECO_OP_PAGED_PREFIX, _kv(k=0, v=0, table=0, **kw))  # noqa: E731
    heads = 2 * 3 * 8
    assert size() >= reco.reco_paged_workspace_bytes(reco.RECO_OP_PAGED_DECODE, _kv()) + 2 * heads * 128 * 4
    assert size(B=4000, H_q=32) >= 2 * 2 * 4000 * 32 * 128 * 4 and size(d=64) < size()
    with pytest.raises(reco.RecoError) as e:
        size(H_q=34)
    assert e.value.status == reco.RECO_EUNSUPPORTED
    with pytest.raises(reco.RecoError):
        reco.reco_workspace_bytes(reco.RECO_OP_PAGED_PREFIX, reco.reco_kv(16, 32, 1, 1, 2, 1, 64, 64, 0))


def test_more_rows_than_a_call_counts_are_refused(L):
    """The work of the own rows is counted in 32 bits: 24 a tile of 128 float32 rows with more than eight heads, 15 with
    fewer, 8 in bf16; the descriptor's own limit of 2^34 rows leaves room for all but the first."""
    big = dict(n_layers=1, B=2 ** 10, H_kv=1, n_pages=1000, max_pages=2 ** 15, page=256)
    for H_q, dtype, fine in ((9, reco.RECO_F32, False), (8, reco.RECO_F32, True), (16, reco.RECO_BF16, True)):
        for shrink in (0, 1):
            kv = _kv(H_q=H_q, dtype=dtype, **{**big, "B": big["B"] * 2 - 1 if not shrink else big["B"]})
            size = ctypes.c_size_t()
            st = L.reco_paged_workspace_bytes(reco.RECO_OP_PAGED_PREFIX, ctypes.byref(kv), ctypes.byref(size))
            assert st == (reco.RECO_OK if fine or shrink else reco.RECO_EUNSUPPORTED), (H_q, dtype, shrink)
    kv = _kv(H_q=9, dtype=reco.RECO_F32, **{**big, "B": 2047})
    p = ctypes.c_void_p(256)
    st = L.reco_paged_prefix_attn(ctypes.byref(kv), p, None, None, p, p, p, 0.1, p, reco.RECO_F32, None, p, 1 << 40, None)
    assert st == reco.RECO_EUNSUPPORTED and b"more than one call counts" in L.reco_last_error()


def test_binding_refuses_tensors_the_library_would_misread():
    K, table = torch.zeros(2, 5, 2, 16, 64), torch.zeros(3, 4, dtype=torch.int32)
    kv = reco.make_paged_kv(K, K.clone(), table, 4)
    q, new, lens = torch.zeros(2, 3, 4, 64), torch.zeros(2, 3, 2, 64), torch.zeros(2, 3, 2, dtype=torch.int32)
    one = torch.zeros(3, dtype=torch.int32)
    good = dict(kv=kv, q=q, k_new=new, v_new=new, lens=lens, group=one, shared=one, scale=0.1, out=torch.zeros_like(q),
                lse=torch.zeros(2, 3, 4), ws=torch.zeros(256, dtype=torch.uint8))
    for bad in (dict(q=q[:, :2]), dict(q=q.bfloat16()), dict(v_new=None), dict(lens=lens[0]), dict(group=one[:2]),
                dict(group=one.long()), dict(shared=one.float()), dict(shared=torch.zeros(6, dtype=torch.int32)[::2]),
                dict(out=q[0]), dict(lse=torch.zeros(2, 3, 4).double()), dict(ws=torch.zeros(256)), {}):
        with pytest.raises(ValueError):  # the last one: a cache on the host
            reco.reco_paged_prefix_attn(**{**good, **bad})
