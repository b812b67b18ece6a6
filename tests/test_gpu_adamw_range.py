"""The AdamW step at the ends of its ranges: second moments below the normal floats, gradients far above one, values of tiny moments."""
import numpy as np
import pytest
import torch

import test_gpu_adamw as base
from oracle import lowbit as lb
from paper_1901_08924_b200 import lpc

pytestmark = pytest.mark.gpu
DEV = "cuda"
F = np.float32


@pytest.mark.parametrize("beta2", [0.999, 0.9999, 1 - 2.0 ** -23])
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("n,lead,nan", [(4096, 0, False), (4099, 1, False), (4096, 0, True), (301, 0, True)])
def test_roots_of_second_moments_below_the_normal_floats(beta2, bits, n, lead, nan):
    # the bias factor of the first step, 1 / sqrt(1 - beta2), is up to 2,896, and lifts the root of a second moment that is no normal float to where eps shows it.  The
    # weights are zero, so that the update is all there is.  m' (beta1 = 0: the gradient), the root (its moment is a multiple of 2^-149: at least 2^10 of them here, so
    # 2^-11 of it, half of that in the root, 2^-12 of what the root is of the divisor) and ten roundings of 2^-23
    eps = 1e-10
    rng = np.random.default_rng(1)
    v = 2.0 ** rng.uniform(-139, -120, n)
    g = (np.sqrt(v / (1 - beta2)) * rng.choice([-1, 1], n)).astype(F)
    ctx = base._ctx()
    opt = lpc.AdamW(ctx, n, None, bits, (0.0, beta2), eps)
    p, state = base._dev(np.zeros(n, F), lead), opt.init_state()
    at = rng.integers(0, n, 5) if nan else []
    sent = g.copy()
    sent[at] = np.nan
    opt.step(p, base._dev(sent, lead), state, 1, 1.0)
    assert ctx.status() == (lpc.ERR_NONFINITE if nan else lpc.OK)
    p = p.double().cpu().numpy()
    assert not p[at].any()   # left as they are
    g = g.astype(np.float64)
    root = np.abs(g)   # sqrt(v') / sqrt(1 - beta2)
    want = -g / (root + eps)
    # v' is rounded to a multiple of 2^-149 three times (g^2, times 1 - beta2, the sum): 1.5 of them at most, and g^2 itself
    v_true = (1 - beta2) * g * g
    off = 0.5 * (1.5 * 2.0 ** -149 / v_true + 0.5 * 2.0 ** -149 / (g * g))
    bound = np.abs(want) * (off * root / (root + eps) + 10 * 2.0 ** -23)
    bound[at] = np.inf
    assert (np.abs(p - want) <= bound).all()
    assert (root / eps).max() > (2.0 ** -23 if beta2 > 0.999 else 0)   # the roots do show
    opt.close(), ctx.close()


@pytest.mark.parametrize("size", [2.0 ** 16, 2.0 ** 40, 2.0 ** 60])
@pytest.mark.parametrize("offs", [None, base.TENSORS[2]])
def test_large_gradients_with_8_bit_moments(size, offs):
    # blocks of m above 2^14 and of v above 2^30, where one power of two is no factor of its own any more
    n, lr, seed = 5003, 1e-3, 77
    segs = base._segs(offs, n)
    p, g, m, v = base._inputs(n, 3)
    g, m, v = g.numpy() * F(size), m * F(size), v * F(size) * F(size)
    wd, ls = [0.1] * (len(segs) - 1), [1.0] * (len(segs) - 1)
    ctx = base._ctx(seed=seed)
    opt = lpc.AdamW(ctx, n, offs, 8, (base.B1, base.B2), base.EPS, 0.1)
    codes, exps, vals = base._state8(m, v, segs, seed)
    state = (base._dev(codes["m"]), base._dev(codes["v"]), base._dev(exps))
    assert exps[:, 0].max() > 127 + 14 and exps[:, 1].max() > 127 + 30 - (2 if size < 2 ** 20 else 0)
    got = opt.state_values(state)
    for x, which in zip(got, "mv"):
        assert (x.double().cpu().numpy() == vals[which]).all()
    dp = base._dev(p)
    opt.step(dp, base._dev(g), state, 4, lr)
    want, st = base._oracle8(p, g, vals["m"], vals["v"], segs, seed, 4, lr, wd, ls)
    ctx.sync_status()
    assert base._near(dp, want, p, lr, 0.1)
    for i, which in enumerate("mv"):
        assert (state[i].cpu().numpy() == st[which][0]).all() and (state[2].cpu().numpy()[:, i] == st[which][1]).all()
    opt.close(), ctx.close()


@pytest.mark.parametrize("n", [256, 5003])
def test_values_of_tiny_moments_round_to_the_nearest(n):
    # every code of blocks with every small exponent: what bfloat16 holds comes out as it is, the rest as its nearest neighbour
    ctx = base._ctx()
    opt = lpc.AdamW(ctx, n, None, 8)
    blocks = -(-n // 256)
    every = np.tile(np.arange(256, dtype=np.uint8), blocks)
    codes = {"m": every, "v": every}
    for first in list(range(1, 60, blocks)) + [100, 127, 200]:
        e = (first + np.arange(blocks)).astype(np.uint8)
        exps = np.stack([e, e], 1)
        got = opt.state_values((base._dev(codes["m"]), base._dev(codes["v"]), base._dev(exps)))
        ctx.sync_status()
        for x, which in zip(got, "mv"):
            value = lb.decode(which, codes[which].reshape(-1, 256), e).ravel()[:n]
            want = torch.from_numpy(value).float().bfloat16()   # no code is near a tie that the first rounding could move: both keep to even
            assert torch.equal(x.cpu(), want), (first, which)
    opt.close(), ctx.close()


def test_an_eps_that_the_approximate_quotient_cannot_divide_by_is_refused():
    n = 512
    ctx = base._ctx()
    for eps in (2.0 ** 126, 2.0 ** 127):
        with pytest.raises(lpc.LpcError) as e:
            lpc.AdamW(ctx, n, None, 8, (0.9, 0.999), eps)
        assert e.value.code == lpc.ERR_INVALID_ARG
    for bits, eps in ((8, 2.0 ** 125), (32, 2.0 ** 127)):
        # beta1 = 0 and a gradient of 2^60: the update is 2^60 / (eps + 2^60), far below eps
        opt = lpc.AdamW(ctx, n, None, bits, (0.0, 0.999), eps)
        p = torch.zeros(n, device=DEV)
        opt.step(p, torch.full((n,), 2.0 ** 60, device=DEV), opt.init_state(), 1, 1.0)
        ctx.sync_status()
        assert ((p.double() * eps / 2.0 ** 60 + 1).abs() <= 2.0 ** -20).all()
        opt.close()
    ctx.close()
