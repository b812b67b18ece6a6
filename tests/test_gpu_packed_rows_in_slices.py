"""A matrix of more rows than a context has workers: packed slice by slice into one array, used as one."""
import numpy as np
import pytest
import torch

from oracle import lowbit as lb
from paper_1901_08924_b200 import lpc, synth

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("G", [32, 128])
def test_rows_beyond_the_most_workers_of_a_context(G):
    R, K, most = 2500, 300, 1024
    offs = [min(i * G, K) for i in range(-(-K // G) + 1)]
    W = synth.gradient_vectors(R, K, "gauss", seed=4, device=DEV)
    codes = torch.zeros((R, (K + 31) // 32 * 4), dtype=torch.int32, device=DEV)
    delta = torch.zeros((R, len(offs) - 1), device=DEV)
    full, rest = (lpc.Context(None, None, lpc.LOGISTIC, 0.0, n, 1, 4, lpc.CLIP_NONE, 1.0, 3) for n in (most, R % most))
    for k, first in enumerate(range(0, R, most)):
        part = slice(first, min(first + most, R))
        (full if first + most <= R else rest).quantize_pack(W[part], k, seg_offsets=offs, codes_out=codes[part], delta_out=delta[part])
    full.sync_status(), rest.sync_status()
    Wq = torch.from_numpy(lb.unpack_rows(codes.cpu().numpy().view(np.uint32), delta.cpu().numpy(), K, G)).to(DEV)
    step = delta.double().repeat_interleave(G, 1)[:, :K]
    assert ((Wq - W.double()).abs() <= step * (1 + 1e-6)).all()
    # a slice's rounding is its own: the same rows twice, at two k's, differ
    twice = [full.quantize_pack(W[:most], k, seg_offsets=offs)[0] for k in (0, 1)]
    assert torch.equal(twice[0], codes[:most]) and not torch.equal(twice[1], codes[:most])
    x, dy = torch.randn(3, K, device=DEV), torch.randn(3, R, device=DEV)
    for got, a, b in ((rest.packed_matvec(codes, delta, K, x, G), x.double(), Wq.t()), (rest.packed_matvec_t(codes, delta, K, dy, G), dy.double(), Wq)):
        assert ((got.double() - a @ b).abs() <= (a.shape[1] + 4) * 2.0 ** -23 * (a.abs() @ b.abs())).all()
    full.close(), rest.close()
    with pytest.raises(lpc.LpcError):
        lpc.Context(None, None, lpc.LOGISTIC, 0.0, most + 1, 1, 4, lpc.CLIP_NONE, 1.0, 3)
