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


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("packed", [False, True])
def test_a_backward_pass_notices_that_its_weights_were_stepped(bits, packed):
    n = 1000
    ctx = _context()
    opt = lpc.AdamW(ctx, n, None, bits)
    flat = torch.randn(n, device=DEV)
    p = flat.requires_grad_()
    copy = torch.zeros(n, dtype=torch.bfloat16, device=DEV)
    state = opt.init_state()
    U = synth.gradient_vectors(1, n, "gauss", seed=3, device=DEV)
    codes, delta, _ = ctx.quantize_pack(U, 1)

    def step(t):
        if packed:
            opt.unpack_average_step(codes, delta, p, state, t, 0.1, copy_out=copy)
        else:
            opt.step(p, U[0], state, t, 0.1, copy_out=copy)

    (p * p).sum().backward()   # before a step: as ever
    assert torch.equal(p.grad, 2 * p.detach())
    loss, x = (p * p).sum(), torch.ones(n, dtype=torch.bfloat16, device=DEV, requires_grad=True)
    used = (copy * x).sum()
    before = [s._version for s in state if s is not None]
    step(1)
    for late in (loss, used):
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            late.backward()
    assert all(s._version > b for s, b in zip([s for s in state if s is not None], before))
    # weights that are views of one vector, in a backward pass of their own
    part = flat.detach()[:10]
    late = (part * torch.ones(10, device=DEV, requires_grad=True)).sum()
    step(2)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        late.backward()
    with torch.inference_mode():   # such tensors have no count
        q = torch.ones(n, device=DEV)
    opt.step(q, U[0], opt.init_state(), 1, 0.1)
    ctx.sync_status()
    opt.close(), ctx.close()


def test_a_backward_pass_notices_that_an_output_was_written_again():
    R, K = 8, 256
    ctx = _context(R)
    codes, delta, _ = ctx.quantize_pack(synth.gradient_vectors(R, K, "gauss", seed=1, device=DEV), 1)
    X, dY = torch.randn(2, K, device=DEV), torch.randn(2, R, device=DEV)
    out, out_t = ctx.packed_matvec(codes, delta, K, X, 0), ctx.packed_matvec_t(codes, delta, K, dY, 0)
    late = [(o * torch.ones_like(o).requires_grad_()).sum() for o in (out, out_t)]
    ctx.packed_matvec(codes, delta, K, 2 * X, 0, out=out)
    ctx.packed_matvec_t(codes, delta, K, 2 * dY, 0, out=out_t)
    opt = lpc.AdamW(ctx, R, None, 8)
    m, v = torch.zeros(R, dtype=torch.bfloat16, device=DEV), torch.zeros(R, dtype=torch.bfloat16, device=DEV)
    late.append((m * torch.ones_like(m).requires_grad_()).sum())
    opt.state_values(opt.init_state(), out=(m, v))
    for x in late:
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            x.backward()
    ctx.sync_status()
    opt.close(), ctx.close()
