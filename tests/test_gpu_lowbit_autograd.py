"""AdamW steps and products with packed rows beside torch's autograd: what would lose a gradient is refused, what is written counts as written."""
import pytest
import torch

from paper_1901_08924_b200 import lpc, synth

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _context(N=1, b=4):
    return lpc.Context(None, None, lpc.LOGISTIC, 0.0, N, 1, b, lpc.CLIP_NONE, 1.0, 5)


def test_products_refuse_what_autograd_would_record():
    R, K, M = 8, 256, 2
    ctx = _context(R)
    codes, delta, _ = ctx.quantize_pack(synth.gradient_vectors(R, K, "gauss", seed=1, device=DEV), 1)
    X, dY = torch.randn(M, K, device=DEV), torch.randn(M, R, device=DEV)
    want, want_t = ctx.packed_matvec(codes, delta, K, X, 0), ctx.packed_matvec_t(codes, delta, K, dY, 0)
    for leaf, call in ((X, lambda x: ctx.packed_matvec(codes, delta, K, x, 0)), (dY, lambda y: ctx.packed_matvec_t(codes, delta, K, y, 0))):
        x = leaf.clone().requires_grad_()
        for arg in (x, x * 2):
            with pytest.raises(AssertionError, match="autograd"):
                call(arg)
        expect = want if leaf is X else want_t
        assert torch.equal(call(x.detach()), expect)
        with torch.no_grad():
            assert torch.equal(call(x), expect)
    with pytest.raises(AssertionError, match="autograd"):
        ctx.packed_matvec(codes, delta.clone().requires_grad_(), K, X, 0)
    with pytest.raises(AssertionError, match="autograd"):
        ctx.packed_matvec(codes, delta, K, X, 0, out=torch.zeros_like(want).requires_grad_())
    ctx.sync_status()
    ctx.close()
