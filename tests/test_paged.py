"""The paged cache on the CPU: its fp64 reference against closed forms, torch and the contiguous
oracle, and the refusals of the C ABI and of the binding before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

import oracle
from oracle import paged
from paper_2608_04771_gb300 import build as B
from paper_2608_04771_gb300 import reco


@pytest.fixture(scope="module")
def L():
    B.build()
    return reco.lib()


def _cache(rng, Ly=2, Bn=2, H=2, G=3, page=4, per=3, d=8):
    """A small cache with shuffled pages (the reference takes any page size)."""
    n_pages = Bn * per + 1
    K, V = rng.standard_normal((Ly, n_pages, H, page, d)), rng.standard_normal((Ly, n_pages, H, page, d))
    table = rng.permutation(n_pages)[:Bn * per].reshape(Bn, per)
    q = rng.standard_normal((Ly, Bn, H * G, d))
    return K, V, table, q


def _rows(pool, table, ly, b, h):
    return pool[ly, table[b], h].reshape(-1, pool.shape[-1])


# ---------------------------------------------------------------- the reference
def test_reference_decode_is_the_contiguous_oracles():
    rng = np.random.default_rng(1)
    K, V, table, q = _cache(rng)
    lens = np.array([[[1, 5], [12, 7]], [[4, 3], [8, 9]]])
    out, lse, *_ = paged.decode(K, V, table, lens.copy(), q, None, None, 0.3)
    for ly, b, hq in np.ndindex(2, 2, 6):
        h = hq // 3
        n = lens[ly, b, h]
        k, v = _rows(K, table, ly, b, h)[:n], _rows(V, table, ly, b, h)[:n]
        o, z = oracle.decode_unit(q[ly, b, hq].astype(np.float32), k.astype(np.float32), v.astype(np.float32), n, 0.3)
        assert np.abs(out[ly, b, hq] - o).max() < 1e-5 and abs(lse[ly, b, hq] - z) < 1e-5


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (3, 2), (5, 12), (100, 0), (4, 1)])
def test_reference_decode_is_torchs_masked_attention(window, sinks):
    rng = np.random.default_rng(2)
    K, V, table, q = _cache(rng)
    lens = np.array([[[0, 5], [11, 7]], [[4, 3], [8, 9]]])
    kn, vn = rng.standard_normal((2, 2, 2, 8)), rng.standard_normal((2, 2, 2, 8))
    W = rng.random((2, 2, 2, 12))
    W0, K0, lens0 = W.copy(), K.copy(), lens.copy()
    out, _, _, seen, _ = paged.decode(K, V, table, lens, q, kn, vn, 0.5, window, sinks, W)
    assert np.array_equal(lens, lens0 + 1)
    for ly, b, h in np.ndindex(2, 2, 2):
        n = lens[ly, b, h]
        k, v = torch.from_numpy(_rows(K, table, ly, b, h)[:n]), torch.from_numpy(_rows(V, table, ly, b, h)[:n])
        assert np.array_equal(k[n - 1].numpy(), kn[ly, b, h]) and np.array_equal(v[n - 1].numpy(), vn[ly, b, h])
        assert np.array_equal(k[:n - 1].numpy(), _rows(K0, table, ly, b, h)[:n - 1])
        j = torch.arange(n)
        mask = torch.ones(n, dtype=bool) if window == 0 else (j < sinks) | (j >= n - window)
        qq = torch.from_numpy(q[ly, b, 3 * h:3 * h + 3])
        want = torch.nn.functional.scaled_dot_product_attention(qq, k, v, attn_mask=mask.expand(3, n), scale=0.5)
        assert np.abs(out[ly, b, 3 * h:3 * h + 3] - want.numpy()).max() < 1e-12
        assert (seen[ly, b, 3 * h:3 * h + 3] == int(mask.sum())).all()
        p = torch.softmax((qq @ k.T * 0.5).masked_fill(~mask, -torch.inf), 1).mean(0).numpy()
        want_w = W0[ly, b, h].copy()
        want_w[n - 1] = 0.0
        want_w[:n] += p
        assert np.abs(W[ly, b, h] - want_w).max() < 1e-12


def test_reference_weights_of_one_token_sum_to_one():
    rng = np.random.default_rng(3)
    K, V, table, q = _cache(rng)
    lens = np.full((2, 2, 2), 9)
    W = np.zeros((2, 2, 2, 12))
    paged.decode(K, V, table, lens, q, None, None, 1.0, 4, 2, W)
    assert np.allclose(W.sum(-1), 1.0) and (W[..., 2:5] == 0).all() and (W[..., 9:] == 0).all()


def test_reference_eviction_by_hand():
    K = np.arange(2 * 4, dtype=float).reshape(1, 2, 1, 4, 1)  # pages hold 0..3 and 4..7
    V = -K.copy()
    table = np.array([[1, 0]])  # rows 0..7 hold 4 5 6 7 0 1 2 3
    W = np.array([[[[9.0, 1.0, 3.0, 3.0, 2.0, 5.0, 0.0, 7.0]]]])
    lens = np.array([[[7]]])
    # 7 rows to 4, one sink and one latest row: of 1, 3, 3, 2, 5 the two largest, the tie to the lower index
    kept = paged.evict(K, V, W, table, lens, [4], 1, 1)
    assert kept[0, 0, 0].tolist() == [0, 2, 5, 6] and lens.item() == 4
    assert _rows(K, table, 0, 0, 0)[:4, 0].tolist() == [4.0, 6.0, 1.0, 2.0]
    assert _rows(V, table, 0, 0, 0)[:4, 0].tolist() == [-4.0, -6.0, -1.0, -2.0]
    assert W[0, 0, 0, :4].tolist() == [9.0, 3.0, 5.0, 0.0]
    assert paged.evict(K, V, W, table, lens, [4], 1, 1) == {}  # within its budget: nothing


# ---------------------------------------------------------------- refusals
def _kv(**kw):
    a = dict(k=16, v=32, table=64, n_layers=2, B=3, H_q=8, H_kv=2, n_pages=20, max_pages=6, page=16, d=128,
             dtype=reco.RECO_BF16)
    a.update(kw)
    return reco.reco_paged_kv(*(a[f] for f, _ in reco.reco_paged_kv._fields_))


def test_workspace_sizes(L):
    size = lambda op, **kw: reco.reco_paged_workspace_bytes(op, _kv(**kw))  # noqa: E731
    dec, wts = size(reco.RECO_OP_PAGED_DECODE), size(reco.RECO_OP_PAGED_WEIGHTS)
    assert dec > 0 and wts - dec >= 2 * 3 * 8 * (6 * 16 + 1) * 4  # logits and normalisers of a token
    assert size(reco.RECO_OP_PAGED_EVICT) >= 2 * 3 * 2 * (6 * 16 + 1) * 4
    assert size(reco.RECO_OP_PAGED_DECODE, k=0, v=0, table=0) == dec  # only sizes are read
    # beyond 32 bits: 28 x 8 x 28 heads of 131072 rows
    big = dict(n_layers=28, B=8, H_q=28, H_kv=4, max_pages=8192, n_pages=9000)
    assert size(reco.RECO_OP_PAGED_WEIGHTS, **big) > 28 * 8 * 28 * 131072 * 4
    for op in (reco.RECO_OP_PAGED_DECODE, reco.RECO_OP_PAGED_WEIGHTS):  # no size for heads that the call refuses
        for H_q in (34, 2 ** 31 - 2):
            with pytest.raises(reco.RecoError) as e:
                size(op, H_q=H_q)
            assert e.value.status == reco.RECO_EUNSUPPORTED
    with pytest.raises(reco.RecoError) as e:
        size(reco.RECO_OP_DECODE)
    assert e.value.status == reco.RECO_EINVAL
    with pytest.raises(reco.RecoError):
        reco.reco_workspace_bytes(reco.RECO_OP_PAGED_DECODE, reco.reco_kv(16, 32, 1, 1, 2, 1, 64, 64, 0))


@pytest.mark.parametrize("bad,status", [
    (dict(n_layers=0), reco.RECO_EINVAL), (dict(B=0), reco.RECO_EINVAL), (dict(H_kv=0), reco.RECO_EINVAL),
    (dict(H_q=0), reco.RECO_EINVAL), (dict(H_q=7), reco.RECO_EINVAL), (dict(n_pages=0), reco.RECO_EINVAL),
    (dict(max_pages=0), reco.RECO_EINVAL), (dict(dtype=2), reco.RECO_EINVAL), (dict(k=0), reco.RECO_EINVAL),
    (dict(v=0), reco.RECO_EINVAL), (dict(table=0), reco.RECO_EINVAL), (dict(k=8), reco.RECO_EINVAL),
    (dict(v=40), reco.RECO_EINVAL), (dict(table=66), reco.RECO_EINVAL), (dict(d=96), reco.RECO_EUNSUPPORTED),
    (dict(page=8), reco.RECO_EUNSUPPORTED), (dict(page=48), reco.RECO_EUNSUPPORTED),
    (dict(page=512), reco.RECO_EUNSUPPORTED), (dict(page=0), reco.RECO_EUNSUPPORTED),
    (dict(page=-16), reco.RECO_EUNSUPPORTED), (dict(n_layers=70000, B=70000), reco.RECO_EUNSUPPORTED),
    (dict(n_layers=100, B=400), reco.RECO_EUNSUPPORTED), (dict(max_pages=1 << 27), reco.RECO_EUNSUPPORTED),
    (dict(B=8192, max_pages=1 << 16), reco.RECO_EUNSUPPORTED),
    (dict(n_pages=1 << 25), reco.RECO_EUNSUPPORTED)])
def test_descriptors_that_are_refused(L, bad, status):
    kv, vp, big = _kv(**bad), ctypes.c_void_p, 1 << 40
    ws = vp(256)
    assert L.reco_paged_decode_attn(ctypes.byref(kv), vp(16), None, None, vp(16), 0.1, 0, 0, vp(16), 0, None, ws, big,
                                    None) == status
    assert L.reco_paged_decode_attn_weights(ctypes.byref(kv), vp(16), None, None, vp(16), 0.1, 0, 0, vp(16), 0, None,
                                            vp(16), ws, big, None) == status
    assert L.reco_paged_evict(ctypes.byref(kv), vp(16), vp(16), vp(16), 1, 0, None, ws, big, None) == status
    assert reco.lib().reco_last_error()


@pytest.mark.parametrize("kw,text,status", [
    (dict(q=None), b"NULL", reco.RECO_EINVAL), (dict(lens=None), b"NULL", reco.RECO_EINVAL),
    (dict(out=None), b"NULL", reco.RECO_EINVAL), (dict(k_new=16), b"k_new", reco.RECO_EINVAL),
    (dict(v_new=16), b"k_new", reco.RECO_EINVAL), (dict(q=24), b"aligned", reco.RECO_EINVAL),
    (dict(out=20), b"aligned", reco.RECO_EINVAL), (dict(k_new=16, v_new=24), b"aligned", reco.RECO_EINVAL),
    (dict(lens=18), b"aligned", reco.RECO_EINVAL), (dict(lse=17), b"aligned", reco.RECO_EINVAL),
    (dict(weights=24), b"aligned", reco.RECO_EINVAL), (dict(out_dtype=7), b"out_dtype", reco.RECO_EINVAL),
    (dict(window=-1), b"window", reco.RECO_EINVAL), (dict(window=5, sinks=-1), b"sinks", reco.RECO_EINVAL),
    (dict(sinks=4), b"window", reco.RECO_EINVAL), (dict(scale=float("nan")), b"scale", reco.RECO_EINVAL),
    (dict(ws=None), b"workspace", reco.RECO_EINVAL), (dict(ws=128), b"aligned", reco.RECO_EINVAL),
    (dict(ws_bytes=-1), b"workspace", reco.RECO_EINVAL), (dict(H_q=34), b"at most 16", reco.RECO_EUNSUPPORTED)])
def test_decode_arguments_that_are_refused(L, kw, text, status):
    a = dict(q=16, k_new=None, v_new=None, lens=16, scale=0.1, window=0, sinks=0, out=16, out_dtype=0, lse=None,
             weights=16, ws=256, ws_bytes=0, H_q=8)
    a.update(kw)
    kv = _kv(H_q=a["H_q"])
    p = lambda x: None if x is None else ctypes.c_void_p(x)  # noqa: E731
    for wts in (False, True):
        if "weights" in kw and not wts:
            continue
        op = reco.RECO_OP_PAGED_WEIGHTS if wts else reco.RECO_OP_PAGED_DECODE
        n = reco.reco_paged_workspace_bytes(op, _kv()) + a["ws_bytes"]
        args = [ctypes.byref(kv), p(a["q"]), p(a["k_new"]), p(a["v_new"]), p(a["lens"]), a["scale"], a["window"],
                a["sinks"], p(a["out"]), a["out_dtype"], p(a["lse"])] + ([p(a["weights"])] if wts else []) + \
            [p(a["ws"]), n, None]
        st = (L.reco_paged_decode_attn_weights if wts else L.reco_paged_decode_attn)(*args)
        assert st == status and text in L.reco_last_error(), (wts, st, L.reco_last_error())


def test_weights_need_an_array(L):
    vp = ctypes.c_void_p
    st = L.reco_paged_decode_attn_weights(ctypes.byref(_kv()), vp(16), None, None, vp(16), 0.1, 0, 0, vp(16), 0, None,
                                          None, vp(256), 1 << 40, None)
    assert st == reco.RECO_EINVAL and b"weights" in L.reco_last_error()


@pytest.mark.parametrize("kw,text", [
    (dict(weights=None), b"NULL"), (dict(lens=None), b"NULL"), (dict(budget=None), b"NULL"),
    (dict(weights=18), b"aligned"), (dict(budget=18), b"aligned"), (dict(kept=18), b"aligned"), (dict(w=-1), b"w = "),
    (dict(sinks=-1), b"sinks"), (dict(w=97), b"w = "), (dict(w=90, sinks=7), b"together"),
    (dict(w=1, sinks=2 ** 31 - 1), b"together"), (dict(ws=None), b"workspace"), (dict(short=1), b"workspace")])
def test_evict_arguments_that_are_refused(L, kw, text):
    a = dict(weights=16, lens=16, budget=16, w=4, sinks=2, kept=None, ws=256, short=0)
    a.update(kw)
    kv = _kv()
    p = lambda x: None if x is None else ctypes.c_void_p(x)  # noqa: E731
    n = reco.reco_paged_workspace_bytes(reco.RECO_OP_PAGED_EVICT, kv) - a["short"]
    st = L.reco_paged_evict(ctypes.byref(kv), p(a["weights"]), p(a["lens"]), p(a["budget"]), a["w"], a["sinks"],
                            p(a["kept"]), p(a["ws"]), n, None)
    assert st == reco.RECO_EINVAL and text in L.reco_last_error()


def test_binding_refuses_tensors_the_library_would_misread():
    K = torch.zeros(2, 5, 2, 16, 64)
    table = torch.zeros(3, 4, dtype=torch.int32)
    for bad in (dict(V=K[:, :4]), dict(V=K.bfloat16()), dict(K=K.transpose(0, 1), V=K.transpose(0, 1)),
                dict(table=table.long()), dict(table=table[:, ::2]), dict(table=table[0]),
                dict(K=K[0], V=K[0])):
        a = dict(K=K, V=K, table=table)
        a.update(bad)
        with pytest.raises(ValueError):
            reco.make_paged_kv(a["K"], a["V"], a["table"], 4)
    with pytest.raises(TypeError):
        reco.make_paged_kv(K.half(), K.half(), table, 4)
    kv = reco.make_paged_kv(K, K.clone(), table, 4)
    assert (kv.n_layers, kv.n_pages, kv.H_kv, kv.page, kv.d, kv.B, kv.max_pages) == (2, 5, 2, 16, 64, 3, 4)
    q, new, lens = torch.zeros(2, 3, 4, 64), torch.zeros(2, 3, 2, 64), torch.zeros(2, 3, 2, dtype=torch.int32)
    out, lse, wts = torch.zeros_like(q), torch.zeros(2, 3, 4), torch.zeros(2, 3, 2, 64)
    ws = torch.zeros(256, dtype=torch.uint8)
    good = dict(kv=kv, q=q, k_new=new, v_new=new, lens=lens, scale=0.1, out=out, lse=lse, ws=ws)
    for bad in (dict(q=q[:, :2]), dict(q=q.bfloat16()), dict(q=q.transpose(0, 1).contiguous().transpose(0, 1)),
                dict(k_new=new[..., :32]), dict(v_new=None), dict(lens=lens.long()), dict(lens=lens[0]),
                dict(out=out[0]), dict(lse=lse.double()), dict(ws=ws.float()), {}):
        with pytest.raises(ValueError):  # the last one: a cache on the host
            reco.reco_paged_decode_attn(**{**good, **bad})
        with pytest.raises(ValueError):
            reco.reco_paged_decode_attn_weights(weights=wts, **{**good, **bad})
    with pytest.raises(ValueError):
        reco.reco_paged_decode_attn_weights(weights=wts[..., :63], **good)
    ev = dict(kv=kv, weights=wts, lens=lens, budget=torch.zeros(3, dtype=torch.int32), w=1, sinks=0, kept_idx=None, ws=ws)
    for bad in (dict(weights=wts.double()), dict(budget=torch.zeros(2, dtype=torch.int32)), dict(lens=lens[:1]),
                dict(kept_idx=wts), {}):
        with pytest.raises(ValueError):
            reco.reco_paged_evict(**{**ev, **bad})
