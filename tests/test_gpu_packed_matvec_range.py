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


def _plain_t(k, d, G, dy):
    """dY W in 64 bits, from dY delta rounded to fp32 as the header says."""
    W = np.zeros((dy.shape[0], k.shape[1]))
    with np.errstate(over="ignore", invalid="ignore"):
        for c in range(k.shape[1]):
            W[:, c] = (dy.astype(np.float32) * d[:, c // G][None]).astype(np.float64) @ k[:, c].astype(np.float64)
    return W


@pytest.mark.parametrize("x_type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("G", [32, 64, 128])
@pytest.mark.parametrize("sign", [1.0, -1.0])
def test_transposed_products_next_to_the_largest_float(x_type, G, sign):
    # (2 - 2^-10) 2^127 is a float, above the largest bfloat16.  Rows 0 and 1 leave half of it
    R, K, M = 20, 150, 3
    k = np.zeros((R, K), np.int64)
    k[:2] = 1
    k[0, 1::2] = k[1, 1::2] = -1
    e = 100 if x_type != "f16" else 10
    d = np.zeros((R, -(-K // G)), np.float32)
    d[:2] = (2 - 2.0 ** -10) * 2.0 ** (127 - e)
    codes, delta = _on_device(k, d)
    dy = np.zeros((M, R))
    dy[1, 0], dy[1, 1] = 2.0 ** e, -2.0 ** (e - 1)
    dy[2, 0], dy[2, 1] = -2.0 ** e, 2.0 ** (e - 1)
    dy *= sign
    ctx = _ctx()
    got = ctx.packed_matvec_t(codes, delta, K, torch.from_numpy(dy).to(TYPES[x_type]).to(DEV), G)
    ctx.sync_status()
    assert torch.equal(got.cpu(), torch.from_numpy(_plain_t(k, d, G, dy)).float().to(TYPES[x_type]))
    ctx.close()


@pytest.mark.parametrize("x_type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("G", [32, 64, 128])
def test_infinities_of_both_signs_in_the_transposed_product(x_type, G):
    R, K, M = 40, 200, 17
    rng = np.random.default_rng(3)
    k = rng.integers(-8, 8, (R, K))
    d = np.full((R, -(-K // G)), 0.5, np.float32)
    d[7] = np.inf
    dy = rng.integers(-8, 9, (M, R)).astype(np.float64)
    dy[:, 7] = 1
    k[7] = 1
    dy[1, 7], dy[4, 7] = -3, 0   # times an infinite scale: nothing is NaN
    dy[5, 11], dy[6, 11], dy[9, 11], dy[10, 39] = np.inf, -np.inf, np.nan, -np.inf
    codes, delta = _on_device(k, d)
    ctx = _ctx()
    for rows in (slice(0, M), slice(5, 7)):
        for scale in (np.inf, 0.25):
            d[7] = scale
            delta[7] = float(scale)
            got = ctx.packed_matvec_t(codes, delta, K, torch.from_numpy(dy[rows]).to(TYPES[x_type]).to(DEV), G)
            ctx.sync_status()
            want = torch.from_numpy(_plain_t(k, d, G, dy[rows])).float().to(TYPES[x_type])
            assert torch.equal(got.cpu().isnan(), want.isnan()) and torch.equal(got.cpu().nan_to_num(5.0), want.nan_to_num(5.0))
    ctx.close()


@pytest.mark.parametrize("x_type,a,b", [(t, a, b) for t in ("f32", "bf16") for a, b in ((-20, 106), (-100, 120), (-132, 124), (0, 100), (0, -100), (100, -120), (120, -140), (-100, -30))]
                         + [("f16", -24, 120), ("f16", 10, -100)])
@pytest.mark.parametrize("G", [32, 128])
def test_transposed_products_of_far_apart_magnitudes(x_type, a, b, G):
    R, K = 300, 70
    rng = np.random.default_rng(200 + a)
    k = rng.integers(-8, 8, (R, K))
    codes, delta = _on_device(k, np.full((R, -(-K // G)), 2.0 ** b).astype(np.float32))
    ctx = _ctx()
    for M in (1, 7, 12, 20):
        y = rng.integers(-8, 9, (M, R)).astype(np.float64)
        got = ctx.packed_matvec_t(codes, delta, K, torch.from_numpy(np.ldexp(y, a)).to(TYPES[x_type]).to(DEV), G)
        ctx.sync_status()
        assert torch.equal(got.cpu(), torch.from_numpy(np.ldexp(y @ k, a + b)).float().to(TYPES[x_type]))
    ctx.close()


@pytest.mark.parametrize("x_type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("G", [32, 128])
def test_what_a_value_counts_to_beside_larger_ones(x_type, G):
    """Forward: a value counts to 2^-23 of itself (fp32) and 2^-39 of the largest of its 128 columns, whose code is zero here, so that nothing hides what the small
    ones lose; the sums add n 2^-23 of the sum of magnitudes, scale and factors four roundings, and the output's type its own half step."""
    R, K, M = 60, 500, 9
    rng = np.random.default_rng(8)
    spread = 45 if x_type != "f16" else 20
    x = rng.standard_normal((M, K)) * 2.0 ** -rng.uniform(0, spread, (M, K))
    X = torch.from_numpy(x).to(TYPES[x_type])
    x = X.double().numpy()
    k = rng.integers(-8, 8, (R, K))
    top = np.zeros((M, K))
    for s in range(0, K, 128):
        cols = slice(s, min(s + 128, K))
        top[:, cols] = np.abs(x[:, cols]).max(1, keepdims=True)
        k[:, s + np.argsort(-np.abs(x[:, cols]).max(0))[:20]] = 0   # the largest ones' codes
    d = rng.uniform(0.5, 2, (R, -(-K // G))).astype(np.float32)
    codes, delta = _on_device(k, d)
    W = k * d.astype(np.float64).repeat(G, 1)[:, :K]
    lost = np.zeros_like(x) + (2.0 ** -23 * np.abs(x) if x_type == "f32" else 0) + (2.0 ** -39 * top if x_type != "f16" else 0)
    want, size = x @ W.T, np.abs(x) @ np.abs(W).T
    bound = lost @ np.abs(W).T + (K + 4) * 2.0 ** -23 * size
    half = torch.finfo(TYPES[x_type]).eps / 2
    ctx = _ctx()
    got = ctx.packed_matvec(codes, delta, K, X.to(DEV), G).double().cpu().numpy()
    ctx.sync_status()
    assert (np.abs(got - want) <= bound + half * (np.abs(want) + bound) + (2.0 ** -25 if x_type == "f16" else 0)).all()
    ctx.close()


@pytest.mark.parametrize("x_type", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("G", [32, 64, 128])
def test_what_a_product_counts_to_where_sums_cancel(x_type, G):
    """Transposed: dY delta, rounded to fp32 (2^-24), counts to 2^-18 of itself for the 16-bit types.  Pairs of rows with opposite codes and nearly equal scales
    leave little, so that the output's own rounding does not hide it."""
    R, K, M = 24, 200, 16
    rng = np.random.default_rng(9)
    k = rng.integers(-7, 8, (R, K))
    k[1::2] = -k[::2]
    d = rng.uniform(0.5, 1, (R, -(-K // G))).astype(np.float32)
    d[1::2] = d[::2] * (1 + 2.0 ** -12 * rng.uniform(0, 1, d[::2].shape)).astype(np.float32)
    dy = torch.from_numpy(rng.standard_normal((M, R)) * 2.0 ** -rng.uniform(0, 10, (M, R))).to(TYPES[x_type])
    dy[:, 1::2] = dy[:, ::2]
    y = dy.double().numpy()
    W = k * d.astype(np.float64).repeat(G, 1)[:, :K]
    want, size = y @ W, np.abs(y) @ np.abs(W)
    bound = ((2.0 ** -18 if x_type != "f32" else 0) + 2.0 ** -24 + (3 * R + 3) * 2.0 ** -23) * size
    half = torch.finfo(TYPES[x_type]).eps / 2
    codes, delta = _on_device(k, d)
    ctx = _ctx()
    got = ctx.packed_matvec_t(codes, delta, K, dy.to(DEV), G).double().cpu().numpy()
    ctx.sync_status()
    assert (np.abs(got - want) <= bound + half * (np.abs(want) + bound) + (2.0 ** -25 if x_type == "f16" else 0)).all()
    ctx.close()
