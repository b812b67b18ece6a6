"""Steps on the messages of many workers: whole groups of eight (four for the widths that are known at run time only), groups and a rest, and hundreds."""
import numpy as np
import pytest
import torch

import test_gpu_adamw as base
from oracle import lowbit as lb
from paper_1901_08924_b200 import lpc, synth

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _check(N, b, bits, n, offs, mu):
    segs, t = base._segs(offs, n), 9
    ctx = base._ctx(N, b)
    U = synth.gradient_vectors(N, n, "gauss", seed=b, device=DEV)
    M = 0.3 * synth.gradient_vectors(1, n, "gauss", seed=99, device=DEV)[0] if mu else None
    codes, delta, _ = ctx.quantize_pack(U, 3, seg_offsets=offs)
    woff, _ = lpc.packed_layout(n, b, offs)
    words = codes.cpu().numpy().view(np.uint32)
    k = np.concatenate([[lb.stream_indices(words[i, woff[s]:woff[s + 1]], b, segs[s + 1] - segs[s]) for i in range(N)] for s in range(len(segs) - 1)], 1)
    d = np.repeat(delta.cpu().numpy(), np.diff(segs), 1)
    g = base._dev(lb.average_of_messages(k, d, N, None if M is None else M.cpu().numpy()))
    p, _, m, v = base._inputs(n, 6)
    runs = []
    for packed in (True, False):
        opt = lpc.AdamW(ctx, n, offs, bits, (base.B1, base.B2), base.EPS, 0.1)
        dp = base._dev(p)
        if bits == 32:
            state = (base._dev(m), base._dev(v), None)
        else:
            c8, e8, _ = base._state8(m, v, segs, 11)
            state = (base._dev(c8["m"]), base._dev(c8["v"]), base._dev(e8))
        if packed:
            opt.unpack_average_step(codes, delta, dp, state, t, 1e-2, mu=M)
        else:
            opt.step(dp, g, state, t, 1e-2)
        runs.append((dp, *[s for s in state if s is not None]))
        opt.close()
    ctx.sync_status()
    for x, y in zip(*runs):
        assert torch.equal(x, y)
    assert not torch.equal(runs[0][0].cpu(), torch.from_numpy(p))
    ctx.close()


@pytest.mark.parametrize("b", [1, 2, 3, 4, 5, 8, 12, 16, 32])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("N,offs,mu", [(8, base.TENSORS[3], True), (9, None, False), (16, base.TENSORS[2], True), (17, base.TENSORS[3], False), (12, base.TENSORS[2], False), (27, None, True)])
def test_whole_groups_of_workers_and_a_rest(N, offs, mu, b, bits):
    _check(N, b, bits, 5003, offs, mu)


@pytest.mark.parametrize("b", [2, 4, 6, 8])
@pytest.mark.parametrize("N", [100, 1024])
def test_hundreds_of_workers(N, b):
    _check(N, b, 8 if N == 100 else 32, 2100, [0, 2052, 2100], True)
