"""gnnpre_embedding_lookup and gnnpre_embedding_grad against the oracle.

Bounds.  A lookup is one fp32 product (2^-24 relative) and one rounding to the output's type (half a step: eps / 2 relative, or
half the smallest subnormal).  A gradient adds c terms in fp32: at most c roundings of 2^-24, each of a partial sum bounded by the
sum of the terms' absolute values; then one product with the scale (2^-24) and, for a 16-bit table, one rounding to it.
Integers small enough for fp32 to hold every partial sum are compared bit for bit.
"""
import numpy as np
import pytest
import torch

import oracle as orc

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_SUBNORMAL = {F32: 2.0 ** -150, BF16: 2.0 ** -134, F16: 2.0 ** -25}


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2207_12000_b200 import binding
    return binding


def wide(t):
    return t.detach().cpu().double().numpy()


def matrix(rows, cols, dtype, seed, pad=0, offset=0, integers=False):
    """Rows of a wider buffer that starts `offset` elements into its memory; what lies between the rows is NaN."""
    gen = torch.Generator().manual_seed(seed)
    v = torch.randint(-4, 5, (rows, cols), generator=gen).float() if integers else torch.randn((rows, cols), generator=gen)
    buf = torch.full((rows * (cols + pad) + offset,), float("nan"), dtype=dtype, device="cuda")
    m = buf[offset:].view(rows, cols + pad)[:, :cols]
    m.copy_(v.to(dtype))
    return m


def draw_ids(count, rows, how, seed, dtype):
    rng = np.random.default_rng(seed)
    if how == "uniform":
        ids = rng.integers(0, rows, size=count)
    elif how == "one":
        ids = np.full(count, rows - 1)
    elif how == "padding":
        ids = np.full(count, -1)
    elif how == "descending":
        ids = np.sort(rng.integers(0, rows, size=count))[::-1].copy()
    else:  # frequent and rare ones, and some outside on both sides
        ids = np.minimum(np.exp(rng.random(count) * np.log(rows + 1)).astype(np.int64) - 1, rows - 1)
        ids[rng.random(count) < 0.1] = -1
        ids[rng.random(count) < 0.05] = rows
        ids[rng.random(count) < 0.02] = np.iinfo(np.int32).max if dtype is torch.int32 else 1 << 40
        ids[rng.random(count) < 0.02] = np.iinfo(np.int32).min if dtype is torch.int32 else -(1 << 33)
    return torch.from_numpy(ids).to(dtype).cuda(), ids


@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("rows,dim,count,pad,offset", [
    (1, 1, 1, 0, 0), (7, 3, 5, 0, 0), (1000, 602, 37, 0, 0), (1000, 602, 37, 6, 0), (513, 128, 4096, 0, 0), (300, 100, 777, 4, 4),
    (300, 100, 777, 1, 1), (64, 17, 50000, 15, 0), (64, 256, 30001, 0, 2), (5, 1030, 9, 0, 0), (2000, 64, 70000, 0, 0)])
def test_lookup(B, dtype, rows, dim, count, pad, offset):
    for wide_ids in (torch.int32, torch.int64):
        table = matrix(rows, dim, dtype, dim, pad, offset)
        ids, ids_np = draw_ids(count, rows, "mixed", count, wide_ids)
        out = matrix(count, dim, dtype, 1, pad, offset)
        before = out._base.clone()
        got = B.gnnpre_embedding_lookup(table, ids, scale=1.7, out=out)
        assert got is out
        want = orc.embedding_lookup(wide(table), ids_np, float(np.float32(1.7)))
        err = np.abs(wide(out) - want)
        assert (err <= (torch.finfo(dtype).eps / 2 + 2.0 ** -24) * np.abs(want) + HALF_SUBNORMAL[dtype]).all()
        if pad or offset:  # what lies between the rows is as it was
            base = out._base
            mask = torch.zeros_like(base, dtype=torch.bool)
            mask[offset:].view(count, dim + pad)[:, :dim] = True
            assert torch.equal(base[~mask].view(torch.uint8), before[~mask].view(torch.uint8))


def test_lookup_of_infinities_and_empty_calls(B):
    table = torch.tensor([[float("inf"), float("nan"), -1.0, 2.0]], device="cuda")
    ids = torch.tensor([0, 1, -1], dtype=torch.int32, device="cuda")
    out = B.gnnpre_embedding_lookup(table, ids, scale=3.0)
    assert torch.isinf(out[0, 0]) and torch.isnan(out[0, 1]) and out[0, 2:].tolist() == [-3.0, 6.0]
    assert (out[1:] == 0).all()  # padding reads as zeros whatever the table holds
    assert B.gnnpre_embedding_lookup(table, ids[:0]).shape == (0, 4)


GRADS = [
    # rows, dim, count, ids
    (1, 1, 1, "uniform"), (3, 5, 2, "one"), (9, 8, 33, "mixed"), (300, 64, 255, "mixed"), (4096, 64, 4096, "uniform"),
    (50, 100, 8192, "mixed"), (50, 100, 8193, "mixed"), (70000, 24, 20000, "mixed"), (2048, 16, 20001, "descending"),
    (300, 36, 131073, "mixed"), (70000, 12, 150000, "uniform"), (5, 33, 140000, "one"), (2, 130, 9000, "one"),
    (1000, 602, 3001, "mixed"), (40, 7, 5000, "padding"), (4200000, 4, 9001, "uniform"), (600, 1100, 700, "mixed")]


@pytest.mark.parametrize("rows,dim,count,how", GRADS)
def test_grad_exact_on_integers(B, rows, dim, count, how):
    d_out = matrix(count, dim, F32, 3, integers=True)
    ids, ids_np = draw_ids(count, rows, how, count + 1, torch.int32 if count % 2 else torch.int64)
    out = B.gnnpre_embedding_grad(d_out, ids, rows, scale=2.0)
    assert out.dtype is F32 and out.shape == (rows, dim)
    want = orc.embedding_grad(wide(d_out), ids_np, rows, 2.0)
    assert np.array_equal(wide(out), want)
    # added to what is there: only the rows asked for, and bit for bit the same again
    old = matrix(rows, dim, F32, 4, integers=True)
    out = B.gnnpre_embedding_grad(d_out, ids, rows, scale=2.0, out=old.clone(), accumulate=True)
    assert np.array_equal(wide(out), want + wide(old))


@pytest.mark.parametrize("dtype,to", [(F32, F32), (BF16, F32), (BF16, BF16), (F16, F32), (F16, F16)])
@pytest.mark.parametrize("rows,dim,count,how,pad,offset", [
    (300, 64, 255, "mixed", 0, 0), (50, 100, 9000, "mixed", 0, 0), (777, 17, 5000, "mixed", 0, 0), (777, 18, 5000, "mixed", 2, 2),
    (64, 602, 3000, "mixed", 6, 0), (5, 33, 70000, "mixed", 3, 1), (64, 602, 300, "uniform", 0, 0)])
def test_grad_within_the_bound_of_the_types(B, dtype, to, rows, dim, count, how, pad, offset):
    d_out = matrix(count, dim, dtype, 5, pad, offset)
    ids, ids_np = draw_ids(count, rows, how, count, torch.int64)
    old = matrix(rows, dim, to, 6, pad, offset)
    base = old._base
    before = base.clone()
    for accumulate in (False, True):
        base.copy_(before)
        start = wide(old)
        B.gnnpre_embedding_grad(d_out, ids, rows, scale=0.7, out=old, accumulate=accumulate)
        want, size, terms = orc.embedding_grad(wide(d_out), ids_np, rows, float(np.float32(0.7)), want_abs=True)
        if accumulate:
            want, size = want + start, size + np.abs(start)
        bound = (terms[:, None] + 3) * 2.0 ** -24 * size + (torch.finfo(to).eps / 2) * np.abs(want) * (1 + 2.0 ** -10) + HALF_SUBNORMAL[to]
        err = np.abs(wide(old) - want)
        assert (err <= bound).all(), float((err / np.maximum(bound, 1e-300)).max())
        if accumulate:  # untouched rows keep their bits
            untouched = torch.from_numpy(np.flatnonzero(terms == 0)).cuda()
            then = before[offset:].view(rows, dim + pad)[:, :dim]
            assert torch.equal(old[untouched], then[untouched])
        if pad or offset:
            mask = torch.zeros_like(base, dtype=torch.bool)
            mask[offset:].view(rows, dim + pad)[:, :dim] = True
            assert torch.equal(base[~mask].view(torch.uint8), before[~mask].view(torch.uint8))


def test_grad_ignores_what_padding_holds(B):
    d_out = torch.ones((100, 12), device="cuda")
    ids = torch.arange(100, device="cuda") % 10
    d_out[7::10], ids[7::10] = float("nan"), -1
    d_out[3::10], ids[3::10] = float("inf"), 10
    out = B.gnnpre_embedding_grad(d_out, ids, 10)
    want = torch.full((10, 12), 10.0)
    want[7], want[3] = 0, 0
    assert torch.equal(out.cpu(), want)


def test_grad_without_ids_and_of_one_row(B):
    none = torch.empty((0, 6), device="cuda")
    ids = torch.empty(0, dtype=torch.int32, device="cuda")
    assert (B.gnnpre_embedding_grad(none, ids, 11) == 0).all()
    kept = torch.full((11, 6), 3.0, device="cuda")
    assert (B.gnnpre_embedding_grad(none, ids, 11, out=kept, accumulate=True) == 3).all()


def test_grad_is_reproducible_and_is_the_difference_quotient(B):
    ids, ids_np = draw_ids(30000, 500, "mixed", 1, torch.int32)
    d_out = matrix(30000, 40, F32, 2)
    first = B.gnnpre_embedding_grad(d_out, ids, 500, scale=1.5)
    for _ in range(3):
        assert torch.equal(B.gnnpre_embedding_grad(d_out, ids, 500, scale=1.5).view(torch.int32), first.view(torch.int32))
    # the lookup is linear: <d_out, lookup(E + D) - lookup(E)> = <d_table, D>, here with integers so that both are exact
    E, D = matrix(500, 40, F32, 3, integers=True), matrix(500, 40, F32, 4, integers=True)
    g = matrix(30000, 40, F32, 5, integers=True)
    change = B.gnnpre_embedding_lookup(E + D, ids, scale=2.0) - B.gnnpre_embedding_lookup(E, ids, scale=2.0)
    grad = B.gnnpre_embedding_grad(g, ids, 500, scale=2.0)
    assert float((change.double() * g.double()).sum()) == float((grad.double() * D.double()).sum())


def test_embedding_in_a_graph_and_on_another_stream(B):
    rows, dim, count = 900, 72, 12000
    table, d_out = matrix(rows, dim, F32, 1, integers=True), matrix(count, dim, F32, 2, integers=True)
    ids, ids_np = draw_ids(count, rows, "mixed", 3, torch.int32)
    out, grad = torch.empty((count, dim), device="cuda"), torch.empty((rows, dim), device="cuda")
    room = torch.empty(B.gnnpre_embedding_grad_workspace(rows, dim, count), dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.gnnpre_embedding_lookup(table, ids, scale=2.0, out=out, stream=side)
    B.gnnpre_embedding_grad(d_out, ids, rows, scale=2.0, out=grad, stream=side)
    side.synchronize()
    assert np.array_equal(wide(out), orc.embedding_lookup(wide(table), ids_np, 2.0))
    assert np.array_equal(wide(grad), orc.embedding_grad(wide(d_out), ids_np, rows, 2.0))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.gnnpre_embedding_lookup(table, ids, scale=2.0, out=out)
        B.gnnpre_embedding_grad(d_out, ids, rows, scale=2.0, out=grad, workspace=room)
    for seed in (7, 8):
        new, ids_np = draw_ids(count, rows, "mixed", seed, torch.int32)
        ids.copy_(new)
        d_out.copy_(matrix(count, dim, F32, seed, integers=True))
        out.fill_(9.0), grad.fill_(9.0), room.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(wide(out), orc.embedding_lookup(wide(table), ids_np, 2.0))
        assert np.array_equal(wide(grad), orc.embedding_grad(wide(d_out), ids_np, rows, 2.0))


def test_rows_of_a_table_beyond_32_bit_offsets(B):
    """The last rows of a table of more than 4 G elements (8.6 GB of bf16), and their gradient."""
    rows, dim = 33_600_000, 128
    table = torch.zeros((rows, dim), dtype=BF16, device="cuda")
    ids = torch.tensor([rows - 1, 0, rows - 2, rows], dtype=torch.int32, device="cuda")
    values = torch.randint(-4, 5, (4, dim), device="cuda").to(BF16)
    table[rows - 1], table[0], table[rows - 2] = values[0], values[1], values[2]
    out = B.gnnpre_embedding_lookup(table, ids)
    assert torch.equal(out[:3], values[:3]) and (out[3] == 0).all()
    table.fill_(1.0)
    B.gnnpre_embedding_grad(values, ids, rows, out=table)
    assert torch.equal(table[rows - 1], values[0]) and torch.equal(table[0], values[1]) and torch.equal(table[rows - 2], values[2])
    assert int(torch.count_nonzero(table[1:rows - 2])) == 0


@pytest.mark.parametrize("dtype,to", [(F32, F32), (BF16, BF16)])
@pytest.mark.parametrize("rows,dim,count,how", [
    (3000, 8, 262_145, "mixed"), (3000, 20, 524_289, "mixed"), (100, 12, 606_208, "uniform"), (100, 12, 606_209, "uniform"),
    (70_000, 16, 700_001, "mixed"), (5_000_000, 4, 1_000_003, "mixed"), (2, 33, 800_000, "one"), (40, 6, 650_000, "padding"),
    (1000, 8, 2_100_000, "descending"), (300, 130, 620_000, "mixed")])
def test_grad_of_long_lists_is_exact_on_integers(B, rows, dim, count, how, dtype, to):
    """Segments of 64 and 128 entries, and blocks of 4,096 keys in the sort (from 606,209 ids on), in one to three passes.  In 16 bits the
    d_out of all but a few positions of a row are zero, so that its sum is still a small integer."""
    d_out = matrix(count, dim, dtype, 3, integers=True)
    if to is not F32:
        d_out[torch.rand(count, generator=torch.Generator().manual_seed(1)).cuda() < 1 - 20 * min(rows, 1000) / count] = 0
        d_out.clamp_(-1, 1)
    ids, ids_np = draw_ids(count, rows, how, count + 1, torch.int32 if count % 2 else torch.int64)
    known = (ids >= 0) & (ids < rows)
    want = torch.zeros((rows, dim), dtype=torch.float64, device="cuda").index_add_(0, ids[known].long(), d_out[known].double())
    if to is not F32 and float(want.abs().max()) > 256:
        d_out[:] = 0  # (one row takes everything: 200 positions of it)
        d_out[::count // 200] = 1
        want = torch.zeros((rows, dim), dtype=torch.float64, device="cuda").index_add_(0, ids[known].long(), d_out[known].double())
    out = B.gnnpre_embedding_grad(d_out, ids, rows, scale=2.0, out=torch.full((rows, dim), float("nan"), dtype=to, device="cuda"))
    assert torch.equal(out.double(), 2 * want)
    old = matrix(rows, dim, to, 4, integers=True)
    again = B.gnnpre_embedding_grad(d_out, ids, rows, scale=-2.0, out=old.clone(), accumulate=True)
    assert torch.equal(again.double(), (old.double() - 2 * want).to(to).double())


@pytest.mark.parametrize("dim", (602, 100, 7))
def test_the_hops_take_what_a_lookup_makes(B, dim):
    """The default result is X_0 of a graph as it is, whatever the table's width; 16-bit rows start on 16-byte boundaries too."""
    n = 60
    rowptr, colidx = torch.arange(n + 1, dtype=torch.int64, device="cuda"), ((torch.arange(n, device="cuda") + 1) % n).to(torch.int32)
    table = matrix(20, dim, F32, 1, integers=True)
    ids = torch.arange(n, device="cuda") % 20
    X = B.gnnpre_embedding_lookup(table, ids)
    assert X.shape == (n, dim) and torch.equal(X, table[ids])
    plan = B.gnnpre_build_plan(rowptr, colidx, B.GNNPRE_OP_SAGE_MEAN, dim)
    hops, _ = B.gnnpre_propagate(plan, X, 1)  # every node has one neighbour: the next one
    assert torch.equal(hops[0], torch.roll(X, -1, 0))
    Wt = matrix(16, dim, F32, 2, pad=-dim % 4, integers=True)
    want = (X.double() @ Wt.double().T).float()
    assert torch.equal(B.gnnpre_lc_first_layer([X], None, Wt, precision=B.GNNPRE_LC_TF32X3)[0], want)
    for dtype in (BF16, F16):
        rows = B.gnnpre_embedding_lookup(table.to(dtype), ids)
        assert rows.stride(0) % 8 == 0 and torch.equal(rows.float(), X)
    plan.close()
