"""A context whose stream is not torch's current one: where results come from, and in which order they are written."""
import pytest
import torch

from paper_1901_08924_b200 import lpc, synth

pytestmark = pytest.mark.gpu
DEV = "cuda"


def _context(stream, N=4, b=4):
    return lpc.Context(None, None, lpc.LOGISTIC, 0.0, N, 1, b, lpc.CLIP_NONE, 1.0, 5, stream)


def test_results_take_no_memory_that_the_current_stream_may_still_use():
    N, K, M = 4, 1 << 16, 3
    side = torch.cuda.Stream()
    ctx = _context(side, N)
    opt = lpc.AdamW(ctx, K, None, 8)
    U = synth.gradient_vectors(N, K, "gauss", seed=1, device=DEV)
    X = torch.ones(M, K, dtype=torch.bfloat16, device=DEV)
    torch.cuda.synchronize()
    codes, delta, _ = ctx.quantize_pack(U, 1)
    state = opt.init_state()
    Y = ctx.packed_matvec(codes, delta, K, X, 0)
    torch.cuda.synchronize()
    calls = {"codes": lambda: ctx.quantize_pack(U, 1)[0], "product": lambda: ctx.packed_matvec_t(codes, delta, K, Y, 0), "values": lambda: opt.state_values(state)[0],
             "sums": lambda: ctx.server_reduce(codes, K, lpc.SCHEME_SERVER_SUM, 1)[0], "counts": lambda: ctx.message_entropy(codes, K, host_counts=False)[0],
             "moments": lambda: opt.init_state()[0]}
    for name, call in calls.items():
        like = call()
        shape, dtype = like.shape, like.dtype
        del like
        torch.cuda.synchronize()
        mine = [torch.empty(shape, dtype=dtype, device=DEV) for _ in range(4)]   # blocks of the current stream, given back
        where = {t.data_ptr() for t in mine}
        del mine
        torch.cuda.synchronize()
        got = [call() for _ in range(4)]
        torch.cuda.synchronize()
        assert not where & {t.data_ptr() for t in got}, name
    ctx.sync_status()
    opt.close(), ctx.close()


@pytest.mark.parametrize("bits", [32, 8])
def test_moments_are_zero_before_the_first_step(bits):
    # the current stream is busy; the context's is not, and steps at once
    n = 100_000
    g, want = synth.gradient_vectors(1, n, "gauss", seed=2, device=DEV)[0], torch.ones(n, device=DEV)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ctx = _context(side, 1)
    opt = lpc.AdamW(ctx, n, None, bits)
    with torch.cuda.stream(side):
        state = opt.init_state()
        opt.step(want, g, state, 1, 0.1)
    p = torch.ones(n, device=DEV)
    full = [torch.full_like(s, 99) for s in state[:2]]
    torch.cuda.synchronize()
    del full
    torch.cuda._sleep(200_000_000)   # a tenth of a second
    other = opt.init_state()
    opt.step(p, g, other, 1, 0.1)
    side.synchronize()
    assert torch.equal(p, want)
    seen = [t.clone() for t in other if t is not None]   # on the current stream, which waited
    torch.cuda.synchronize()
    assert torch.equal(seen[0], state[0]) and torch.equal(seen[1], state[1])
    ctx.sync_status()
    opt.close(), ctx.close()


def test_the_current_streams_own_work_on_new_moments_comes_behind_their_zeros():
    n = 1 << 20
    side = torch.cuda.Stream()
    ctx = _context(side, 1)
    opt = lpc.AdamW(ctx, n)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)
    m, v, _ = opt.init_state()
    m += 3
    torch.cuda.synchronize()
    assert (m == 3).all() and (v == 0).all()
    opt.close(), ctx.close()


def test_a_capture_that_forks_to_the_contexts_stream():
    # the current stream is captured, the context's joins it: results come from the graph's own memory, whatever stream they belong to
    N, K, M = 4, 4096, 3
    main, side = torch.cuda.Stream(), torch.cuda.Stream()
    ctx = _context(side, N)
    opt = lpc.AdamW(ctx, K)
    U = synth.gradient_vectors(N, K, "gauss", seed=1, device=DEV)
    X, p, state = torch.ones(M, K, device=DEV), torch.ones(K, device=DEV), opt.init_state()
    torch.cuda.synchronize()
    ctx.quantize_pack(U, 0)   # the quantizer plans a layout when it first sees it, and allocates
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=main):
        side.wait_stream(main)
        codes, delta, _ = ctx.quantize_pack(U, 1)
        Y = ctx.packed_matvec(codes, delta, K, X, 0)
        dX = ctx.packed_matvec_t(codes, delta, K, Y, 0)
        opt.unpack_average_step(codes, delta, p, state, 1, 0.1)
        main.wait_stream(side)
        total = dX.sum()
        del codes, delta
        again = Y * 2
    X.copy_(torch.randn(M, K, device=DEV))
    torch.cuda.synchronize()
    for _ in range(3):
        p.fill_(1), state[0].zero_(), state[1].zero_()
        torch.cuda.synchronize()
        graph.replay()
    torch.cuda.synchronize()
    got = [t.clone() for t in (Y, dX, again, total, p)]
    q, fresh = torch.ones(K, device=DEV), opt.init_state()
    torch.cuda.synchronize()
    codes, delta, _ = ctx.quantize_pack(U, 1)
    Y = ctx.packed_matvec(codes, delta, K, X, 0)
    dX = ctx.packed_matvec_t(codes, delta, K, Y, 0)
    opt.unpack_average_step(codes, delta, q, fresh, 1, 0.1)
    ctx.sync_status()
    for a, b in zip(got, (Y, dX, Y * 2, dX.sum(), q)):
        assert torch.equal(a, b)
    del graph
    opt.close(), ctx.close()
