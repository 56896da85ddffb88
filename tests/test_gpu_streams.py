"""The calls of the first dense stage's training step on another stream than the current one, while the current one is held up: what a
call makes for itself must not be read before it is written, nor lie in memory that queued work still uses.  Integers: exact."""
import numpy as np
import pytest
import torch

import oracle as orc

pytestmark = pytest.mark.gpu

HELD = 100_000_000  # cycles, some 50 ms


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2207_12000_b200 import binding
    return binding


def integers(*shape, seed=0):
    return torch.from_numpy(np.random.default_rng(seed).integers(-3, 4, size=shape).astype(np.float32)).cuda()


def leave_a_block_in_use(shape, dtype=torch.float32):
    """Hands a block of this size back to the allocator which the held-up current stream is still to fill with NaN."""
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    t = torch.empty(shape, dtype=dtype, device="cuda")
    torch.cuda._sleep(HELD)
    t.fill_(float("nan"))


def wide(t):
    return t.detach().cpu().double().numpy()


@pytest.mark.parametrize("result", ("made", "given"))
def test_int64_indices_are_converted_before_they_are_read(B, result):
    n, F, H, rows = 5000, 32, 64, 3000
    hop, dY, Wt = integers(n, F, seed=1), integers(1, rows, H, seed=2), integers(H, F, seed=3)
    side = torch.cuda.Stream()
    for seed in range(3):
        batch = np.random.default_rng(seed).integers(0, n, size=rows)
        want_grad, want = orc.lc_first_layer_grad([wide(hop)], batch, wide(dY), None, 0), wide(hop)[batch] @ wide(Wt).T
        batch = torch.from_numpy(batch).cuda()
        out, room = torch.empty((H, F), device="cuda"), torch.empty(B.gnnpre_lc_first_layer_grad_workspace(1, rows, F, H), dtype=torch.uint8, device="cuda")
        Y = torch.empty((1, rows, H), device="cuda")
        torch.cuda.synchronize()
        torch.cuda._sleep(HELD)
        got = B.gnnpre_lc_first_layer_grad([hop], batch, dY, stream=side, check=False, **({"out": out, "workspace": room} if result == "given" else {}))
        torch.cuda._sleep(HELD)
        fwd = B.gnnpre_lc_first_layer([hop], batch, Wt, stream=side, check=False, **({"out": Y} if result == "given" else {}))
        torch.cuda.synchronize()
        assert np.array_equal(wide(got), want_grad)
        assert np.array_equal(wide(fwd)[0], want)


def test_results_that_a_call_makes_do_not_lie_in_memory_that_is_still_used(B):
    side = torch.cuda.Stream()
    table, ids = integers(700, 1024, seed=1), torch.arange(3000, device="cuda") % 700
    G = integers(700, 1024, seed=2)
    d_out, hop, dY, Wt = integers(3000, 1024, seed=3), integers(3000, 512, seed=4), integers(1, 3000, 256, seed=5), integers(256, 512, seed=6)
    calls = [((3000, 1024), lambda: B.gnnpre_embedding_lookup(table, ids, stream=side)),
             ((700, 1024), lambda: B.gnnpre_orthogonalize(G, stream=side, check=False)),
             ((700, 1024), lambda: B.gnnpre_embedding_grad(d_out, ids, 700, stream=side)),
             ((256, 512), lambda: B.gnnpre_lc_first_layer_grad([hop], None, dY, stream=side, check=False)),
             ((1, 3000, 256), lambda: B.gnnpre_lc_first_layer([hop], None, Wt, stream=side, check=False))]
    want = [table[ids], B.gnnpre_orthogonalize(G),
            torch.from_numpy(orc.embedding_grad(wide(d_out), ids.cpu().numpy(), 700, 1.0)).float().cuda(),
            (dY[0].double().T @ hop.double()).float(), (hop.double() @ Wt.double().T).float()[None]]
    for _, call in calls:  # (a kernel's first launch may wait for the device)
        call()
    for (shape, call), right in zip(calls, want):
        leave_a_block_in_use(shape)
        got = call()
        torch.cuda.synchronize()
        assert torch.equal(got, right)


def test_calls_on_two_streams_side_by_side(B):
    """Neither call brings a workspace, and the first one's is free for the taking when the second one asks."""
    side = torch.cuda.Stream()
    rows, dim, count = 4000, 64, 300_000
    table_ids = [np.random.default_rng(s).integers(0, rows, size=count) for s in (1, 2)]
    ids = [torch.from_numpy(i).cuda() for i in table_ids]
    d_out = [integers(count, dim, seed=s) for s in (3, 4)]
    hop, dY = integers(60_000, 128, seed=5), [integers(1, 60_000, 128, seed=s) for s in (6, 7)]
    G = [integers(1500, 1600, seed=s) for s in (8, 9)]
    grads, weights, updates = ([torch.empty(s, device="cuda") for _ in range(2)] for s in ((rows, dim), (128, 128), (1500, 1600)))
    alone = [B.gnnpre_orthogonalize(g) for g in G]
    for _ in range(5):
        torch.cuda.synchronize()
        for i, stream in enumerate((None, side)):
            B.gnnpre_embedding_grad(d_out[i], ids[i], rows, out=grads[i], stream=stream)
        for i, stream in enumerate((None, side)):
            B.gnnpre_lc_first_layer_grad([hop], None, dY[i], out=weights[i], stream=stream, check=False)
        for i, stream in enumerate((None, side)):
            B.gnnpre_orthogonalize(G[i], out=updates[i], stream=stream, check=False)
        torch.cuda.synchronize()
        for i in range(2):
            assert np.array_equal(wide(grads[i]), orc.embedding_grad(wide(d_out[i]), table_ids[i], rows, 1.0))
            assert np.array_equal(wide(weights[i]), wide(dY[i])[0].T @ wide(hop))
            assert torch.equal(updates[i], alone[i])


def test_another_librarys_stream(B):
    """An object that has a handle only: what the calls make is ordered with it as with torch's own."""
    class Handle:
        def __init__(self, cuda_stream):
            self.cuda_stream = cuda_stream

    side = torch.cuda.Stream()
    table, ids, batch = integers(50, 12, seed=1), torch.arange(300, device="cuda") % 50, torch.arange(40, device="cuda")
    G, dY = integers(30, 20, seed=2), integers(1, 40, 16, seed=3)
    for stream in (None, side, Handle(side.cuda_stream)):
        torch.cuda._sleep(HELD // 10)
        rows = B.gnnpre_embedding_lookup(table, ids, stream=stream)
        grad = B.gnnpre_lc_first_layer_grad([table], batch, dY, stream=stream)
        update = B.gnnpre_orthogonalize(G, stream=stream)
        torch.cuda.synchronize()
        assert torch.equal(rows, table[ids]) and np.array_equal(wide(grad), wide(dY)[0].T @ wide(table)[:40])
        assert torch.equal(update, B.gnnpre_orthogonalize(G))
