"""Products of two contexts from two host threads at once."""
import threading

import pytest
import torch

from paper_1901_08924_b200 import lpc

pytestmark = pytest.mark.gpu
DEV = "cuda"


@pytest.mark.parametrize("G", [32, 128])
def test_calls_that_want_different_amounts_of_shared_memory(G):
    # the same kernel for 9, 12 and 16 vectors, with 75 to 83 KB
    R, K, rounds = 16, 16384, 6000
    gen = torch.Generator(device=DEV).manual_seed(1)
    codes = torch.randint(-2 ** 31, 2 ** 31, (R, K // 8), generator=gen, device=DEV).int()
    delta = torch.rand((R, K // G), generator=gen, device=DEV)
    work = []
    for M in (9, 16, 12):
        stream = torch.cuda.Stream()
        ctx = lpc.Context(None, None, lpc.LOGISTIC, 0.0, 1, 1, 4, lpc.CLIP_NONE, 1.0, 3, stream)
        x, y = torch.randn((M, K), generator=gen, device=DEV).bfloat16(), torch.empty((M, R), dtype=torch.bfloat16, device=DEV)
        torch.cuda.synchronize()
        work.append((ctx, x, y, ctx.packed_matvec(codes, delta, K, x, G)))
    torch.cuda.synchronize()
    failed = []

    def run(ctx, x, y, want):
        try:
            for i in range(rounds):
                ctx.packed_matvec(codes, delta, K, x, G, out=y)
                if i % 100 == 99:
                    ctx.sync_status()
        except Exception as e:
            failed.append(repr(e))

    threads = [threading.Thread(target=run, args=w) for w in work]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failed
    for ctx, x, y, want in work:
        assert torch.equal(y, want)
        ctx.close()
