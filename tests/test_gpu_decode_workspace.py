"""One workspace for decode calls over contiguous caches of different sizes, heads, types and head dimensions,
batches that grow and shrink: as with a workspace of their own, bit for bit."""
import numpy as np
import pytest
import torch

from paper_2608_04771_gb300 import reco

pytestmark = pytest.mark.gpu
DEV = "cuda"
BF, F32 = torch.bfloat16, torch.float32

# (layers, B, H_q, H_kv, d, dtype, shortest and longest unit): few long units cut into many pieces; hundreds of
# units cut where the warps' ranges end; halves of more than eight heads; float32
SHAPES = [
    (1, 2, 28, 4, 128, BF, 6000, 9000),
    (7, 32, 28, 4, 128, BF, 280, 700),
    (7, 8, 28, 4, 128, BF, 280, 700),
    (1, 2, 14, 2, 128, F32, 5000, 7000),
    (5, 40, 12, 1, 64, BF, 300, 600),
    (10, 30, 6, 2, 64, F32, 150, 400),
    (6, 20, 32, 2, 128, BF, 600, 900),
    (10, 40, 4, 2, 128, BF, 1, 200),
]
ORDER = [0, 1, 0, 2, 1, 3, 5, 6, 1, 4, 7, 1, 6, 5, 3, 0]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    from paper_2608_04771_gb300 import build
    build.build()
    reco.lib()


def _inputs(i):
    Ly, B, Hq, H, d, dt, lo, hi = SHAPES[i]
    g = torch.Generator(device=DEV)
    g.manual_seed(500 + i)
    rand = lambda *s: torch.randn(s, generator=g, device=DEV).to(dt)  # noqa: E731
    lens = np.random.default_rng(500 + i).integers(lo, hi + 1, (Ly, B, H)).astype(np.int32)
    K, V = rand(Ly, B, H, hi + 1, d), rand(Ly, B, H, hi + 1, d)
    return K, V, torch.from_numpy(lens).to(DEV), rand(Ly, B, Hq, d), rand(Ly, B, H, d), rand(Ly, B, H, d)


def _decode(inputs, i, ws):
    K, V, lens, q, kn, vn = inputs
    kv = reco.make_kv(K, V, q.shape[2])
    lens = lens.clone()
    out, lse = torch.full(q.shape, 7.0, device=DEV), torch.full(q.shape[:3], 7.0, device=DEV)
    reco.reco_decode_attn(kv, q, kn, vn, lens, q.shape[3] ** -0.5, out, lse,
                          reco.workspace(reco.RECO_OP_DECODE, kv, 0, DEV) if ws is None else ws)
    reco.reco_check()
    return out, lse, lens


def test_growing_and_shrinking_calls_share_a_workspace():
    made = {i: _inputs(i) for i in set(ORDER)}
    want = {i: _decode(made[i], i, None) for i in made}
    size = max(reco.reco_workspace_bytes(reco.RECO_OP_DECODE, reco.make_kv(m[0], m[1], m[3].shape[2])) for m in made.values())
    ws = torch.zeros(size, dtype=torch.uint8, device=DEV)
    for step, i in enumerate(ORDER):
        got = _decode(made[i], i, ws)
        for name, a, b in zip(("out", "lse", "lens"), got, want[i]):
            assert torch.equal(a, b), (step, i, name)


def test_the_answers_it_compares_with_are_right():
    """The calls with a workspace of their own against float64 attention."""
    for i in (1, 4, 5):
        K, V, lens, q, kn, vn = _inputs(i)
        K0, V0 = K.clone(), V.clone()
        out, lse, _ = _decode((K, V, lens, q, kn, vn), i, None)
        Ly, B, Hq, H, d = *q.shape[:3], K.shape[2], q.shape[3]
        for ly, b, h in [(0, 0, 0), (Ly - 1, B - 1, H - 1), (Ly // 2, B // 2, H // 2)]:
            n = int(lens[ly, b, h])
            k = torch.cat([K0[ly, b, h, :n], kn[ly, b, h][None]]).double()
            v = torch.cat([V0[ly, b, h, :n], vn[ly, b, h][None]]).double()
            x = q[ly, b, h * (Hq // H):(h + 1) * (Hq // H)].double() @ k.T * d ** -0.5
            # bf16: the probabilities enter their product in two parts of 8 bits each, 2^-17; float32 chains of
            # d products and of (n / 8 + 64) additions, 2^-24 of the largest sum of products each
            big = float((q[ly, b].double().abs().amax() * k.abs().sum(1).max()) * d ** -0.5)
            rel = 2 * (d + 6) * 2.0 ** -24 * big + 2.0 ** -21 + (64 + n / 8) * 2.0 ** -24 + 2.0 ** -17
            p = torch.softmax(x, 1)
            err = (out[ly, b, h * (Hq // H):(h + 1) * (Hq // H)].double() - p @ v).abs()
            assert (err <= rel * (p @ v.abs()) + 2.0 ** -24).all()
            z = torch.logsumexp(x, 1)
            assert ((lse[ly, b, h * (Hq // H):(h + 1) * (Hq // H)].double() - z).abs() <= rel + 2.0 ** -23 * z.abs()).all()
