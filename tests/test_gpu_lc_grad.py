"""gnnpre_lc_first_layer_grad against the oracle.

Integers whose sums fp32 holds are compared bit for bit: gather, mask, operand layouts and the shares of the batch.  On normal inputs
the error is bounded by the terms' absolute values: a term's operands enter whole, the dropped products are below 2^-23 of it;
inside the tensor core a term meets at most 32 sums that are cut at 2^-23 of their size; the sums of 64 rows are then added,
rounded to nearest (2^-24), at most once per 64 rows and hop within a share and at most 192 times between shares.
"""
import numpy as np
import pytest
import torch

import gnnpre_inputs as gi
import oracle as orc

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2207_12000_b200 import binding
    return binding


def padded(M, pad, rows_too=0, fill=float("nan")):
    """Device copy of a host array, its rows inside longer ones full of `fill`."""
    M = torch.as_tensor(np.ascontiguousarray(M))
    *lead, r, c = M.shape
    buf = torch.full((*lead, r + rows_too, c + pad), fill, dtype=torch.float32, device="cuda")
    view = buf[..., :r, :c]
    view.copy_(M)
    return view


def aligned(M):
    """The same with rows that start on 16-byte boundaries (hop matrices)."""
    return padded(M, 4 + -M.shape[1] % 4)


SHAPES = [
    # n, F, H, batch size (None = every row), hops
    (1000, 32, 16, 128, 1), (64, 16, 128, 32, 1), (40, 5, 32, 1, 2), (5000, 100, 256, 4096, 3), (3000, 128, 256, 1000, 2),
    (777, 13, 48, 300, 2), (2000, 602, 64, 517, 1), (517, 40, 80, None, 2), (900, 300, 192, 333, 1), (400, 129, 144, 31, 9),
    (60000, 100, 256, 50001, 3), (30, 1, 16, 33, 1), (2000, 2500, 256, 70, 1), (300, 20, 240, 20000, 1)]


def case(n, F, H, bs, K, seed, integers):
    rng = np.random.default_rng(seed)
    draw = (lambda *s: rng.integers(-3, 4, size=s).astype(np.float32)) if integers else (lambda *s: rng.standard_normal(s, dtype=np.float32))
    rows = n if bs is None else bs
    hops = [draw(n, F) for _ in range(K)]
    dY, Y = draw(K, rows, H), draw(K, rows, H)
    if bs is None:
        return hops, None, dY, Y
    batch = rng.integers(0, n, size=bs)
    if bs > 20:  # padding, on both sides of the matrix, with what must not be looked at
        batch[rng.random(bs) < 0.05] = -1
        batch[rng.random(bs) < 0.05] = n
        batch[5], batch[6] = np.iinfo(np.int32).max, np.iinfo(np.int32).min
        dY[:, (batch < 0) | (batch >= n)] = np.nan
    return hops, batch, dY, Y


@pytest.mark.parametrize("n,F,H,bs,K", SHAPES)
def test_exact_on_integers(B, n, F, H, bs, K):
    hops, batch, dY, Y = case(n, F, H, bs, K, n + F, True)
    mask = 0b1010110110
    d_hops = [aligned(h) for h in hops]
    d_batch = None if batch is None else torch.from_numpy(batch.astype(np.int32)).cuda()
    want = orc.lc_first_layer_grad(hops, batch, dY, Y, mask)
    # what lies where the mask leaves nothing is not looked at either
    dY_masked = dY.copy()
    for k in range(K):
        if mask >> k & 1:
            dY_masked[k][Y[k] <= 0] = np.inf
    got = B.gnnpre_lc_first_layer_grad(d_hops, d_batch, padded(dY_masked, 3, 1), Y=padded(Y, 1, 2), relu_mask=mask)
    assert got.shape == (H, F) and np.array_equal(got.cpu().double().numpy(), want)
    # hops side by side, a strided result, added to what is there
    side = np.concatenate(list(dY_masked), axis=1), np.concatenate(list(Y), axis=1)
    old = np.random.default_rng(1).integers(-5, 6, size=(H, F)).astype(np.float32)
    out = padded(old, 3)
    B.gnnpre_lc_first_layer_grad(d_hops, d_batch, padded(side[0], 2), Y=padded(side[1], 2), relu_mask=mask, concat=True, out=out, accumulate=True)
    assert np.array_equal(out.cpu().double().numpy(), want + old)
    assert torch.isnan(out._base[:, F:]).all()


@pytest.mark.parametrize("n,F,H,bs,K", SHAPES)
def test_normal_inputs_within_the_bound(B, n, F, H, bs, K):
    hops, batch, dY, Y = case(n, F, H, bs, K, n + H, False)
    dY *= np.float32(1e-20)  # any scale fits
    mask = 0b11110
    got = B.gnnpre_lc_first_layer_grad([aligned(h) for h in hops], None if batch is None else torch.from_numpy(batch).cuda(),
                                       torch.from_numpy(dY).cuda(), Y=torch.from_numpy(Y).cuda(), relu_mask=mask)
    want, size = orc.lc_first_layer_grad(hops, batch, dY, Y, mask, want_abs=True)
    rows = n if bs is None else bs
    bound = (33 * 2.0 ** -23 + (K * (rows / 64 + 1) + 192) * 2.0 ** -24) * size
    err = np.abs(got.cpu().double().numpy() - want)
    assert (err <= bound).all(), float((err / np.maximum(bound, 1e-300)).max())
    # and far below what one product of bf16 or tf32 numbers would give: 2^-18 of the result's size
    assert np.linalg.norm(err) <= 2.0 ** -18 * np.linalg.norm(want)


def test_is_the_forward_calls_gradient(B):
    """The layer is linear in its weight where the signs of Y do not change: <dY, Y(W + D) - Y(W)> = <dW, D>.  Integers: exact."""
    rng = np.random.default_rng(5)
    hops = [aligned(rng.integers(0, 4, size=(700, 36)).astype(np.float32)) for _ in range(2)]
    W, D = (torch.from_numpy(rng.integers(lo, 5, size=(48, 36)).astype(np.float32)).cuda() for lo in (0, 0))
    W[::3] *= -1  # outputs that are never positive, before and after
    D[::3] *= -1
    batch = torch.from_numpy(rng.integers(0, 700, size=501).astype(np.int32)).cuda()
    mask = 0b10
    Y, Y2 = (B.gnnpre_lc_first_layer(hops, batch, w, relu_mask=mask) for w in (W, W + D))
    dY = torch.from_numpy(rng.integers(-3, 4, size=(2, 501, 48)).astype(np.float32)).cuda()
    same = (Y > 0) == (Y2 > 0)
    dY[~same] = 0  # (rows of zeros that D brings above zero)
    dW = B.gnnpre_lc_first_layer_grad(hops, batch, dY, Y=Y, relu_mask=mask)
    assert float(((Y2 - Y).double() * dY.double()).sum()) == float((dW.double() * D.double()).sum())


def test_empty_batch_and_no_relu(B):
    hop = aligned(np.ones((10, 7), dtype=np.float32))
    none = torch.empty((1, 0, 16), device="cuda")
    batch = torch.empty(0, dtype=torch.int32, device="cuda")
    assert (B.gnnpre_lc_first_layer_grad([hop], batch, none) == 0).all()
    kept = torch.full((16, 7), 2.0, device="cuda")
    assert (B.gnnpre_lc_first_layer_grad([hop], batch, none, out=kept, accumulate=True) == 2).all()
    dY = torch.ones((1, 10, 16), device="cuda")
    assert (B.gnnpre_lc_first_layer_grad([hop], None, dY) == 10).all()
    batch = torch.full((10,), -1, dtype=torch.int32, device="cuda")
    assert (B.gnnpre_lc_first_layer_grad([hop], batch, dY) == 0).all()


def test_not_finite_operands_reach_their_sums(B):
    hop = aligned(np.ones((40, 20), dtype=np.float32))
    dY = torch.ones((1, 40, 16), device="cuda")
    dY[0, 7, 3] = float("nan")
    hop[9, 4] = float("inf")
    got = B.gnnpre_lc_first_layer_grad([hop], None, dY)
    bad = torch.zeros((16, 20), dtype=torch.bool, device="cuda")
    bad[3], bad[:, 4] = True, True
    assert not torch.isfinite(got[bad]).any() and (got[~bad] == 40).all()


def test_reproducible_in_a_graph_and_on_a_stream(B):
    hops, batch, dY, Y = case(3000, 77, 96, 5000, 2, 3, False)
    args = [aligned(h) for h in hops], torch.from_numpy(batch.astype(np.int32)).cuda(), torch.from_numpy(dY).cuda()
    y = torch.from_numpy(Y).cuda()
    first = B.gnnpre_lc_first_layer_grad(*args, Y=y, relu_mask=2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    assert torch.equal(B.gnnpre_lc_first_layer_grad(*args, Y=y, relu_mask=2, stream=side), first)
    out = torch.empty_like(first)
    room = torch.empty(B.gnnpre_lc_first_layer_grad_workspace(2, 5000, 77, 96), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.gnnpre_lc_first_layer_grad(*args, Y=y, relu_mask=2, out=out, workspace=room, check=False)
    for _ in range(2):
        out.fill_(7.0), room.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, first)


def test_waits_that_run_out_are_reported_and_leave_the_device_usable(B):
    hop, dY = aligned(np.ones((1000, 150), dtype=np.float32)), torch.ones((1000, 144), device="cuda")
    assert B.gnnpre_lc_grad_selftest_wait_timeout(hop, dY, polls=50) == -8
    assert (B.gnnpre_lc_first_layer_grad([hop], None, dY[None]) == 1000).all()


def test_a_training_step_of_the_first_stage(B):
    """Categories to features, hops, first stage, its gradients and an orthogonalised update, each against the oracle on what the
    step before it gave."""
    rng = np.random.default_rng(3)
    g = gi.rmat(3000, 9000, 4, directed_candidates=False)
    kinds, F, H, K = 200, 44, 64, 2
    table = torch.from_numpy(rng.standard_normal((kinds, F), dtype=np.float32)).cuda()
    ids_np = rng.integers(-1, kinds, size=g.n)
    ids = torch.from_numpy(ids_np).cuda()
    X0 = B.gnnpre_embedding_lookup(table, ids, scale=0.5)
    plan = B.gnnpre_build_plan(g.rowptr.cuda(), g.colidx.cuda(), B.GNNPRE_OP_GCN_SYM, F)
    hops, _ = B.gnnpre_propagate(plan, X0, K)
    batch_np = rng.permutation(g.n)[:700]
    batch = torch.from_numpy(batch_np.astype(np.int32)).cuda()
    Wt = torch.from_numpy((rng.standard_normal((H, F)) / np.sqrt(F)).astype(np.float32)).cuda()
    Y = B.gnnpre_lc_first_layer(hops, batch, Wt, relu_mask=0b10, precision=B.GNNPRE_LC_TF32X3)
    dY = torch.from_numpy(rng.standard_normal((K, 700, H), dtype=np.float32) / 700).cuda()
    dW = B.gnnpre_lc_first_layer_grad(hops, batch, dY, Y=Y, relu_mask=0b10)
    wide = lambda t: t.cpu().numpy()  # noqa: E731
    want, size = orc.lc_first_layer_grad([wide(h) for h in hops], batch_np, wide(dY), wide(Y), 0b10, want_abs=True)
    assert (np.abs(wide(dW).astype(np.float64) - want) <= (33 * 2.0 ** -23 + (K * 12 + 192) * 2.0 ** -24) * size).all()
    update = B.gnnpre_orthogonalize(dW, scale=0.2)
    ortho = orc.orthogonalize(wide(dW), 5, tuple(float(np.float32(c)) for c in (3.4445, -4.7750, 2.0315)), 1e-7, float(np.float32(0.2)))
    assert np.linalg.norm(wide(update) - ortho) <= 2.0 ** -12 * np.linalg.norm(ortho)
    Wt -= update
    # back to the table: dX_k = dZ_k W_1 (the first stage itself, with the weight's other side), through the hops (the GCN filter is
    # symmetric), to the categories
    dZ = torch.where((Y > 0) | (torch.arange(K, device="cuda") == 0)[:, None, None], dY, 0.0)
    every = [torch.zeros((g.n, H), device="cuda").index_copy_(0, batch.long(), dZ[k]) for k in range(K)]
    back = B.gnnpre_lc_first_layer(every, None, (Wt + update).t().contiguous()[:32], precision=B.GNNPRE_LC_TF32X3)
    d1, _ = B.gnnpre_propagate(B.gnnpre_build_plan(g.rowptr.cuda(), g.colidx.cuda(), B.GNNPRE_OP_GCN_SYM, 32), back[0].contiguous(), 1)
    d2, _ = B.gnnpre_propagate(B.gnnpre_build_plan(g.rowptr.cuda(), g.colidx.cuda(), B.GNNPRE_OP_GCN_SYM, 32), back[1].contiguous(), 2)
    dX0 = d1[0] + d2[1]
    d_table = B.gnnpre_embedding_grad(dX0, ids, kinds, scale=0.5)
    want, size, terms = orc.embedding_grad(wide(dX0), ids_np, kinds, 0.5, want_abs=True)
    assert (np.abs(wide(d_table).astype(np.float64) - want) <= (terms[:, None] + 3) * 2.0 ** -24 * size + 2.0 ** -24 * np.abs(want)).all()
    # the step descends: <d_table, D> is the change of <dY, Y> along D in the columns that were carried back, to rounding
    D = torch.zeros_like(table)
    D[:, :32] = d_table
    D *= 1e-2 / D.norm()
    W_old = Wt + update
    lin = lambda t: sum((torch.where((Y[k] > 0) | (k == 0), (h[batch.long()].double() @ W_old.double().t()), 0.0) * dY[k].double()).sum()  # noqa: E731
                        for k, h in enumerate(B.gnnpre_propagate(plan, B.gnnpre_embedding_lookup(t, ids, scale=0.5), K)[0]))
    slope = float(lin(table + D) - lin(table - D)) / 2
    assert abs(slope - float((d_table.double() * D[:, :32].double()).sum())) <= 1e-4 * abs(slope)
    plan.close()


def test_int64_indices_beyond_32_bits_are_padding(B):
    """2^32 + 5 and the like name no row, whatever their lower half is."""
    rng = np.random.default_rng(9)
    n, F, H = 50, 20, 32
    hop = rng.integers(-3, 4, size=(n, F)).astype(np.float32)
    batch = np.array([3, (1 << 32) + 5, 7, -(1 << 32) + 2, (1 << 33), -(1 << 40), 49, 50, -1, np.iinfo(np.int64).max, np.iinfo(np.int64).min])
    dY = rng.integers(-3, 4, size=(1, batch.size, H)).astype(np.float32)
    got = B.gnnpre_lc_first_layer_grad([aligned(hop)], torch.from_numpy(batch).cuda(), torch.from_numpy(dY).cuda())
    assert np.array_equal(got.cpu().double().numpy(), orc.lc_first_layer_grad([hop], batch, dY, None, 0))


def test_one_term_is_off_by_little_more_than_a_rounding(B):
    """A batch of one row: every element of the gradient is one product of two 24-bit numbers.  The products left out are below 2^-24 of
    it; of the six sums inside the tensor core only the last is of the result's size, and cut at 2^-23 of it: 2^-22 covers both."""
    rng = np.random.default_rng(2)
    F, H = 1000, 256
    x = (rng.choice([-1, 1], F) * (1 + rng.random(F)) * 2.0 ** rng.integers(-30, 30, F)).astype(np.float32)
    dy = (rng.choice([-1, 1], H) * (1 + rng.random(H)) * 2.0 ** rng.integers(-30, 30, H)).astype(np.float32)
    x[:8] = dy[:8] = [np.float32(1 + 2.0 ** -7 - 2.0 ** -23 * k) for k in range(1, 9)]  # long second and third parts
    x[8:16] = dy[8:16] = [np.float32(1 + 2.0 ** -8 + 2.0 ** -16 + s * 2.0 ** -23) for s in range(-4, 4)]
    got = B.gnnpre_lc_first_layer_grad([aligned(x[None])], None, torch.from_numpy(dy.reshape(1, 1, H)).cuda())
    want = np.outer(dy.astype(np.float64), x.astype(np.float64))
    off = np.abs(got.cpu().double().numpy() - want) / np.abs(want)
    assert off.max() <= 2.0 ** -22, off.max() * 2.0 ** 23


def test_the_largest_numbers_are_finite(B):
    top = np.finfo(np.float32).max
    x = np.array([[top, -top, 3.39e38, 3.3953e38, -3.38953e38, 1.0, 2.0 ** -100, 0.0]], dtype=np.float32)
    dy = np.zeros((1, 1, 16), dtype=np.float32)
    dy[0, 0, :4] = [1.0, -1.0, 0.5, 2.0 ** -20]
    got = B.gnnpre_lc_first_layer_grad([torch.from_numpy(x).cuda()], None, torch.from_numpy(dy).cuda()).cpu().double().numpy()
    want = np.outer(dy[0, 0].astype(np.float64), x[0].astype(np.float64))
    assert (np.abs(got - want) <= 2.0 ** -22 * np.abs(want)).all()


def test_hops_of_one_node(B):
    """A matrix of one row has no pitch to speak of: torch may say 0, or the length of an odd row."""
    dY = torch.ones((1, 1, 16), device="cuda")
    for F in (1, 7, 100, 602):
        x = torch.arange(1, F + 1, device="cuda", dtype=torch.float32)
        for hop in (x[None], x[None].expand(1, F), x.as_strided((1, F), (0, 1))):
            got = B.gnnpre_lc_first_layer_grad([hop], None, dY)
            assert torch.equal(got, x.expand(16, F))


@pytest.mark.parametrize("pad", (0, 4, 3))
@pytest.mark.parametrize("n,F,H,bs,K", [(700, 36, 16, 300, 2), (700, 130, 48, 299, 3), (500, 20, 144, 1000, 9), (900, 100, 256, 777, 3), (90, 8, 256, 1, 2)])
def test_layouts_of_the_gradient_are_exact_on_integers(B, n, F, H, bs, K, pad):
    """[K, B, H] and hops side by side, rows that start on 16-byte boundaries (pad 0 and 4: the copy engine's tiles, whose outermost stride
    is then smaller than a row) and rows that do not; padding rows and masked elements hold what must not be looked at."""
    hops, batch, dY, Y = case(n, F, H, bs, K, n + F + pad, True)
    mask = 0b101010110
    for k in range(K):
        if mask >> k & 1:
            dY[k][(Y[k] <= 0) & np.isfinite(dY[k])] = np.inf
    with np.errstate(invalid="ignore"):
        want = orc.lc_first_layer_grad(hops, batch, dY, Y, mask)
    d_hops, d_batch = [aligned(h) for h in hops], torch.from_numpy(batch).cuda()
    place = (lambda M: padded(M, pad)) if pad else (lambda M: torch.from_numpy(np.ascontiguousarray(M)).cuda())
    got = B.gnnpre_lc_first_layer_grad(d_hops, d_batch, place(dY), Y=place(Y), relu_mask=mask)
    assert np.array_equal(got.cpu().double().numpy(), want)
    side = [np.concatenate(list(t), axis=1) for t in (dY, Y)]
    got = B.gnnpre_lc_first_layer_grad(d_hops, d_batch, place(side[0]), Y=place(side[1]), relu_mask=mask, concat=True)
    assert np.array_equal(got.cpu().double().numpy(), want)


@pytest.mark.parametrize("K,H", [(1, 64), (2, 16), (3, 144), (9, 256)])
def test_the_forward_calls_own_output_side_by_side(B, K, H):
    rng = np.random.default_rng(K)
    hops = [rng.integers(-2, 3, size=(600, 24)).astype(np.float32) for _ in range(K)]
    batch = rng.integers(-1, 600, size=433)
    Wt = rng.integers(-2, 3, size=(H, 24)).astype(np.float32)
    mask = (1 << K) - 2
    d_hops, d_batch = [aligned(h) for h in hops], torch.from_numpy(batch).cuda()
    Y = B.gnnpre_lc_first_layer(d_hops, d_batch, torch.from_numpy(Wt).cuda(), relu_mask=mask, concat=True)
    dY = rng.integers(-3, 4, size=(433, K * H)).astype(np.float32)
    got = B.gnnpre_lc_first_layer_grad(d_hops, d_batch, torch.from_numpy(dY).cuda(), Y=Y, relu_mask=mask, concat=True)
    split = lambda M: list(M.reshape(433, K, H).transpose(1, 0, 2))  # noqa: E731
    assert np.array_equal(got.cpu().double().numpy(), orc.lc_first_layer_grad(hops, batch, split(dY), split(Y.cpu().numpy()), mask))
