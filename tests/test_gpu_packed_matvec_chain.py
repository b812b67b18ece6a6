"""Products with packed rows right behind the kernels that write what they read, and before those that write it again."""
import pytest
import torch

from paper_1901_08924_b200 import lpc

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("x_type", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("G", [32, 64, 128])
def test_codes_and_vectors_rewritten_in_place(G, x_type):
    # weights -> codes -> Y -> dX -> the next weights and vectors, all in the same memory and without a pause, against the same calls with one between each two
    R, K, M, rounds = 256, 2048, 3, 40
    ctx = lpc.Context(None, None, lpc.LOGISTIC, 0.0, R, 1, 4, lpc.CLIP_NONE, 1.0, 3)
    offs = list(range(0, K + 1, G))
    gen = torch.Generator(device=DEV).manual_seed(1)
    Ws = [torch.randn(R, K, generator=gen, device=DEV) for _ in range(4)]
    Xs = [torch.randn(M, K, generator=gen, device=DEV).to(x_type) for _ in range(3)]
    codes, delta, clipped = ctx.quantize_pack(Ws[0], 0, seg_offsets=offs)
    Y, dX = torch.empty(M, R, dtype=x_type, device=DEV), torch.empty(M, K, dtype=x_type, device=DEV)

    def run(pause):
        out = []
        for k in range(rounds):
            ctx.quantize_pack(Ws[k % 4], k, seg_offsets=offs, codes_out=codes, delta_out=delta, clipped_out=clipped)
            pause()
            ctx.packed_matvec(codes, delta, K, Xs[k % 3], G, out=Y)
            pause()
            ctx.packed_matvec_t(codes, delta, K, Y, G, out=dX)
            pause()
            out.append((Y.clone(), dX.clone()))
            pause()
        return out

    apart = run(torch.cuda.synchronize)
    for _ in range(3):
        together = run(lambda: None)
        ctx.sync_status()
        for k, (a, b) in enumerate(zip(apart, together)):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]), k
    assert len({float(y.float().sum()) for y, _ in apart}) == rounds
    ctx.close()
