"""Products with packed rows over the whole range of the floats: vectors and scales so large or small that only their products are ordinary numbers."""
import numpy as np
import pytest
import torch

from oracle import lowbit as lb
from paper_1901_08924_b200 import lpc

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}


def _ctx():
    return lpc.Context(None, None, lpc.LOGISTIC, 0.0, 1, 1, 4, lpc.CLIP_NONE, 1.0, 3)


def _on_device(k, d):
    return torch.from_numpy(lb.pack_rows(k).view(np.int32)).to(DEV), torch.from_numpy(d).to(DEV)


# exponents of the vector and of the scale.  The result is a whole number below 2^15 times 2^(a + b), a normal number, and all its partial sums are too
FORWARD = [(t, a, b) for t in ("f32", "bf16") for a, b in
           ((-20, 106), (-20, 20), (-60, 127), (-100, 124), (-126, 124), (-132, 124), (0, 100), (0, -100), (60, -120), (110, -126), (120, -140), (100, 0))]
FORWARD += [("f32", -149, 120), ("f16", -24, 30), ("f16", -24, 24), ("f16", 10, -20), ("f16", 10, -140)]


@pytest.mark.parametrize("x_type,a,b", FORWARD)
@pytest.mark.parametrize("G", [32, 128, 256])
def test_forward_products_of_far_apart_magnitudes(x_type, a, b, G):
    # one or several groups in 128 columns; the last column's code is the largest
    R, K = 70, 300
    rng = np.random.default_rng(200 + a)
    k = rng.integers(-8, 8, (R, K))
    k[0] = 7
    d = np.full((R, -(-K // G)), 2.0 ** b).astype(np.float32)
    codes, delta = _on_device(k, d)
    ctx = _ctx()
    for M in (1, 7, 12, 20):
        x = rng.integers(-8, 9, (M, K)).astype(np.float64)
        x[0, :] = 8
        want = torch.from_numpy(np.ldexp(x @ k.T, a + b)).float().to(TYPES[x_type])
        X = torch.from_numpy(np.ldexp(x, a)).to(TYPES[x_type]).to(DEV)
        assert (X.double().cpu().numpy() == np.ldexp(x, a)).all()
        got = ctx.packed_matvec(codes, delta, K, X, G)
        ctx.sync_status()
        assert torch.equal(got.cpu(), want), (M, (got.cpu().double() - want.double()).abs().max())
    ctx.close()


@pytest.mark.parametrize("x_type", ["f32", "bf16"])
@pytest.mark.parametrize("G", [32, 64, 128])
def test_magnitudes_that_change_along_a_row(x_type, G):
    # every 128 columns have their own, and the scales make up for it: sums of whole numbers times 2^-3
    R, K = 50, 128 * 9 + 40
    rng = np.random.default_rng(5)
    a = rng.integers(-110, 111, -(-K // 128))
    a[:3] = (-100, 100, 0)
    k = rng.integers(-8, 8, (R, K))
    groups = -(-K // G)
    d = np.ldexp(1.0, -3 - a[np.arange(groups) * G // 128])[None].repeat(R, 0).astype(np.float32)
    codes, delta = _on_device(k, d)
    ctx = _ctx()
    for M in (1, 3, 16):
        x = rng.integers(-8, 9, (M, K)).astype(np.float64)
        X = torch.from_numpy(np.ldexp(x, a[np.arange(K) // 128])).to(TYPES[x_type]).to(DEV)
        got = ctx.packed_matvec(codes, delta, K, X, G)
        ctx.sync_status()
        assert torch.equal(got.cpu(), torch.from_numpy((x @ k.T) / 8).float().to(TYPES[x_type]))
    ctx.close()


@pytest.mark.parametrize("x_type", ["f32", "bf16"])
def test_what_overflows_is_infinite_with_its_sign(x_type):
    # 2^126 times a scale of 4 and a code of 7 or -8; a code of 0 leaves nothing of it
    K = 128
    k = np.zeros((3, K), np.int64)
    k[0, 5], k[1, 5] = 7, -8
    codes, delta = _on_device(k, np.full((3, 1), 4.0, np.float32))
    X = torch.zeros((1, K), dtype=TYPES[x_type], device=DEV)
    X[0, 5] = 2.0 ** 126
    ctx = _ctx()
    got = ctx.packed_matvec(codes, delta, K, X, 128).float().cpu()
    ctx.sync_status()
    assert got[0, 0] == float("inf") and got[0, 1] == -float("inf") and got[0, 2] == 0
    ctx.close()
