"""Every variant of the products with packed rows: the launch rules choose one by the sizes, the group, the type and the number of vectors.

On 148 SMs the shapes below reach all of them.  Forward, 16 x 130: one warp per row tile, two column tiles of 8 warps, four column tiles; 16 x 16,400 and
20,000 x 8,200: two warps that share rows, two column tiles of 16 warps.  Transposed, 16 x 130: two blocks of 128 columns a CTA or one, as few rows have it; 1,000 x 1,000:
one.  Each with groups of 32, 64 and 128 columns, three types and every number of vectors at which the rules change."""
import numpy as np
import pytest
import torch

from paper_1901_08924_b200 import lpc

pytestmark = pytest.mark.gpu
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
VECTORS = (1, 2, 3, 4, 5, 8, 9, 12, 16, 17, 33)


def _pack(k):
    """The words of signed 4-bit indices (rows, cols)."""
    rows, cols = k.shape
    full = torch.zeros((rows, (cols + 31) // 32 * 32), dtype=torch.int64, device=DEV)
    full[:, :cols] = k + 8
    words = (full.view(rows, -1, 8) << torch.arange(0, 32, 4, device=DEV)).sum(2)
    return torch.where(words >= 1 << 31, words - (1 << 32), words).int()


@pytest.mark.parametrize("x_type", list(TYPES))
@pytest.mark.parametrize("G", [32, 64, 96, 128, 0])
@pytest.mark.parametrize("R,K", [(16, 130), (16, 16400), (1000, 1000), (20000, 8200)])
def test_every_variant_is_exact(R, K, G, x_type):
    # at most 20,000 products of 8 * 8 / 4, multiples of 1/16: below 2^23 of them, so every sum is exact, and is rounded to the type once
    gen = torch.Generator(device=DEV).manual_seed(R + K)
    k = torch.randint(-8, 8, (R, K), generator=gen, device=DEV)
    groups = -(-K // G) if G else 1
    delta = torch.exp2(torch.randint(-4, -1, (R, groups), generator=gen, device=DEV).float())
    codes = _pack(k)
    W = k.double() * delta.double().repeat_interleave(G or K, 1)[:, :K]
    del k
    ctx = lpc.Context(None, None, lpc.LOGISTIC, 0.0, 1, 1, 4, lpc.CLIP_NONE, 1.0, 3)
    for M in VECTORS:
        for call, n, A in ((ctx.packed_matvec, K, W.t()), (ctx.packed_matvec_t, R, W)):
            x = torch.randint(-8, 9, (M, n), generator=gen, device=DEV).to(TYPES[x_type])
            got = call(codes, delta, K, x, G)
            ctx.sync_status()
            assert torch.equal(got, (x.double() @ A).float().to(x.dtype)), (M, call.__name__)
    ctx.close()


@pytest.mark.parametrize("x_type", list(TYPES))
@pytest.mark.parametrize("R,K,G", [(4096, 4096, 64), (4096, 4096, 32), (16384, 16384, 128)])
def test_large_products_of_normal_values(R, K, G, x_type):
    # the bound of tests/test_gpu_packed_matvec.py for sums in any order, with what a factor counts to: 2^-18 transposed for the 16-bit types, 2^-23 for fp32
    gen = torch.Generator(device=DEV).manual_seed(7)
    k = torch.randint(-8, 8, (R, K), generator=gen, device=DEV, dtype=torch.int8)
    delta = torch.rand((R, K // G), generator=gen, device=DEV) * 0.02
    codes = torch.cat([_pack(k[i:i + 1024].long()) for i in range(0, R, 1024)])
    ctx = lpc.Context(None, None, lpc.LOGISTIC, 0.0, 1, 1, 4, lpc.CLIP_NONE, 1.0, 3)
    half = torch.finfo(TYPES[x_type]).eps / 2
    for M in (1, 16):
        for transposed in (False, True):
            n, want_n = (R, K) if transposed else (K, R)
            x = torch.randn((M, n), generator=gen, device=DEV).to(TYPES[x_type])
            got = (ctx.packed_matvec_t if transposed else ctx.packed_matvec)(codes, delta, K, x, G).double()
            ctx.sync_status()
            want, size = (torch.zeros((M, want_n), dtype=torch.float64, device=DEV) for _ in range(2))
            for i in range(0, R, 2048):
                W = k[i:i + 2048].double() * delta[i:i + 2048].double().repeat_interleave(G, 1)
                if transposed:
                    want += x[:, i:i + 2048].double() @ W
                    size += x[:, i:i + 2048].double().abs() @ W.abs()
                else:
                    want[:, i:i + 2048], size[:, i:i + 2048] = x.double() @ W.t(), x.double().abs() @ W.abs().t()
            factor = 2.0 ** -18 if transposed and x_type != "f32" else 2.0 ** -22
            bound = ((n + 4) * 2.0 ** -23 + factor) * size
            assert ((got - want).abs() <= bound + half * (want.abs() + bound) + 2.0 ** -24).all()
            assert torch.linalg.norm(got - want) <= torch.linalg.norm(half * want) + (2.0 ** -21 + factor) * torch.linalg.norm(size)
    ctx.close()
