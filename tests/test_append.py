"""The append to a paged cache on the CPU: its fp64 reference against the rotation's properties, and
the refusals of the C ABI and of the binding before anything is launched."""
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
@pytest.mark.parametrize("interleaved", [False, True])
def test_reference_rotation_is_a_complex_product(interleaved):
    rng = np.random.default_rng(1)
    x, f = rng.standard_normal((3, 10)), rng.random(4)
    y = paged.rotate(x, 7, f, interleaved)
    pair = (lambda t: t[:, 0:8:2] + 1j * t[:, 1:8:2]) if interleaved else (lambda t: t[:, :4] + 1j * t[:, 4:8])
    assert np.abs(pair(y) - pair(x) * np.exp(7j * f)).max() < 1e-12
    assert np.array_equal(y[:, 8:], x[:, 8:]) and np.array_equal(paged.rotate(x, 0, f, interleaved), x)
    # products of rotated rows go by the difference of their positions
    z = rng.standard_normal((3, 10))
    dot = lambda s, t: (paged.rotate(x, s, f, interleaved) * paged.rotate(z, t, f, interleaved)).sum(1)  # noqa: E731
    assert np.abs(dot(105, 100) - dot(5, 0)).max() < 1e-11


def test_reference_append_by_hand():
    K = np.zeros((1, 3, 1, 4, 2))
    V = np.zeros_like(K)
    table, lens = np.array([[2, 0], [1, -1]]), np.array([[[3], [0]]])
    k = np.arange(8.0).reshape(1, 4, 1, 2)
    paged.append(K, V, table, lens, k, -k, [0, 2, 3])  # token 3 is nobody's
    assert lens.tolist() == [[[5], [1]]]
    assert K[0, 2, 0, 3].tolist() == [0, 1] and K[0, 0, 0, 0].tolist() == [2, 3] and K[0, 1, 0, 0].tolist() == [4, 5]
    assert V[0, 0, 0, 0].tolist() == [-2, -3] and np.count_nonzero(K) == 5


# ---------------------------------------------------------------- refusals
def _kv(**kw):
    a = dict(k=16, v=32, table=64, n_layers=2, B=3, H_q=8, H_kv=2, n_pages=20, max_pages=6, page=16, d=128,
             dtype=reco.RECO_BF16)
    a.update(kw)
    return reco.reco_paged_kv(*(a[f] for f, _ in reco.reco_paged_kv._fields_))


def _call(L, **kw):
    a = dict(kv=_kv(), k=(64, 512, 256, 128), v=(64, 512, 256, 128), q=None, q_out=None, T=4, starts=16, pos=16,
             inv_freq=16, rot=128, interleaved=0, lens=16, ws=256, ws_bytes=8192)
    a.update(kw)
    p = lambda x: None if x is None else ctypes.c_void_p(x)  # noqa: E731
    r = lambda x: None if x is None else ctypes.byref(reco.reco_rows(*x))  # noqa: E731
    return L.reco_paged_append(ctypes.byref(a["kv"]), r(a["k"]), r(a["v"]), r(a["q"]), r(a["q_out"]), a["T"], p(a["starts"]),
                               p(a["pos"]), p(a["inv_freq"]), a["rot"], a["interleaved"], p(a["lens"]), p(a["ws"]),
                               a["ws_bytes"], None)


ROWS = (64, 512, 256, 128)


@pytest.mark.parametrize("kw,text", [
    (dict(k=None), b"NULL k"), (dict(v=None), b"NULL v"), (dict(k=(0, 512, 256, 128)), b"NULL k"),
    (dict(k=(72, 512, 256, 128)), b"k and its strides"), (dict(v=(64, 508, 256, 128)), b"v and its strides"),
    (dict(v=(64, 512, 252, 128)), b"v and its strides"), (dict(k=(64, 512, 256, 124)), b"k and its strides"),
    (dict(q=ROWS), b"q and q_out"), (dict(q_out=ROWS), b"q and q_out"), (dict(q=ROWS, q_out=(68, 512, 256, 128)), b"q_out and"),
    (dict(q=(64, 512, 256, 4), q_out=ROWS), b"q and its"), (dict(q=(0, 512, 256, 128), q_out=ROWS), b"NULL q"),
    (dict(T=-1), b"T = -1"), (dict(T=2 ** 30 + 1), b"T = "), (dict(starts=None), b"NULL"), (dict(lens=None), b"NULL"),
    (dict(starts=18), b"aligned"), (dict(lens=17), b"aligned"), (dict(pos=18), b"aligned"), (dict(inv_freq=19), b"aligned"),
    (dict(pos=None), b"NULL pos"), (dict(inv_freq=None), b"NULL pos or inv_freq"), (dict(rot=-16), b"rot"),
    (dict(rot=144), b"rot"), (dict(rot=8), b"rot"), (dict(rot=100), b"rot"), (dict(interleaved=2), b"interleaved"),
    (dict(ws=None), b"workspace"), (dict(ws=128), b"aligned"), (dict(ws_bytes=8191), b"workspace")])
def test_append_arguments_that_are_refused(L, kw, text):
    assert _call(L, **kw) == reco.RECO_EINVAL and text in L.reco_last_error(), L.reco_last_error()


@pytest.mark.parametrize("bad,status", [
    (dict(H_q=7), reco.RECO_EINVAL), (dict(k=0), reco.RECO_EINVAL), (dict(table=66), reco.RECO_EINVAL),
    (dict(d=96), reco.RECO_EUNSUPPORTED), (dict(page=48), reco.RECO_EUNSUPPORTED), (dict(n_pages=1 << 25), reco.RECO_EUNSUPPORTED)])
def test_descriptors_that_are_refused(L, bad, status):
    assert _call(L, kv=_kv(**bad)) == status


def test_more_tokens_than_a_call_counts_are_refused(L):
    kv = _kv(n_layers=1000, B=3, H_q=2, H_kv=1)
    assert _call(L, kv=kv, T=2 ** 30, k=(64, 0, 0, 0), v=(64, 0, 0, 0)) == reco.RECO_EUNSUPPORTED and b"2^36" in L.reco_last_error()


def test_nothing_to_append_is_no_launch(L):
    """T = 0 returns before anything is launched (there is no GPU here), with views that point nowhere."""
    assert _call(L, T=0, k=(0, 0, 0, 0), v=(0, 0, 0, 0), pos=None, inv_freq=None) == reco.RECO_OK
    assert _call(L, T=0, ws_bytes=10) == reco.RECO_EINVAL


def test_workspace_size(L):
    size = reco.reco_paged_workspace_bytes(reco.RECO_OP_PAGED_APPEND, _kv(H_q=200, H_kv=2, k=0, v=0, table=0))
    assert size <= 8192 and size % 256 == 0
    with pytest.raises(reco.RecoError):
        reco.reco_workspace_bytes(reco.RECO_OP_PAGED_APPEND, reco.reco_kv(16, 32, 1, 1, 2, 1, 64, 64, 0))


def test_binding_refuses_tensors_the_library_would_misread():
    K, table = torch.zeros(2, 5, 2, 16, 64), torch.zeros(3, 4, dtype=torch.int32)
    kv = reco.make_paged_kv(K, K.clone(), table, 4)
    qkv = torch.zeros(2, 7, 8, 64)
    q, k, v = qkv.split([4, 2, 2], dim=2)
    good = dict(kv=kv, k=k, v=v, starts=torch.zeros(4, dtype=torch.int32), lens=torch.zeros(2, 3, 2, dtype=torch.int32),
                ws=torch.zeros(8192, dtype=torch.uint8), pos=torch.zeros(7, dtype=torch.int32), inv_freq=torch.zeros(32),
                q=q, q_out=torch.zeros(2, 7, 4, 64))
    for bad in (dict(k=k[:, :6]), dict(k=k[0]), dict(v=v.bfloat16()), dict(k=k.transpose(2, 3).contiguous().transpose(2, 3)),
                dict(q=q[:1]), dict(q=None), dict(q_out=None), dict(q_out=torch.zeros(2, 7, 4, 32)), dict(pos=None),
                dict(pos=torch.zeros(6, dtype=torch.int32)), dict(pos=torch.zeros(7)), dict(starts=torch.zeros(3, dtype=torch.int32)),
                dict(inv_freq=torch.zeros(32).double()), dict(lens=torch.zeros(2, 3, 1, dtype=torch.int32)),
                dict(ws=torch.zeros(8192)), {}):  # the last one: a cache on the host
        with pytest.raises(ValueError):
            reco.reco_paged_append(**{**good, **bad})
