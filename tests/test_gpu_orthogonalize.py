"""gnnpre_orthogonalize against the oracle.

Two kinds of comparison:
  * matrices with one nonzero per row and column: every product has one term, so nothing is summed and each singular value goes
    through the polynomial by itself.  A step computes A (three roundings of 2^-22: two operands, the stored sum), A A, the sum
    a + b t + c t^2 and its product with X.  A rounding moves a term by 2^-22 of itself, of which up to eight meet in a term, so
    with S(t) = a + |b| t + |c| t^2 the new value is off by at most 8 * 2^-22 * s S(s^2), and what s was off by before enters
    with the slope of p, |p'| <= a + 3 |b| t + 5 |c| t^2.  (Where several steps are multiplied together the same bound holds for
    each factor.)  The recurrence of that bound is computed beside the values.  Layouts, padding and transposes show up here.
  * dense matrices: in the Frobenius norm, each step adds at most (8 * 2^-22 + K * 2^-24) S ||X||_F (K terms summed in fp32) to an
    error that the step before carries over with at most the slope above; and, because that bound is a worst case, an error of
    at most eight times that of the same recurrence in plain fp32, whose operands carry 24 bits where these carry 22.
Then one rounding to the output's type: eps / 2 relative, half a subnormal at least.
"""
import numpy as np
import pytest
import torch

import oracle as orc

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
HALF_SUBNORMAL = {F32: 2.0 ** -150, BF16: 2.0 ** -134, F16: 2.0 ** -25}
QUINTIC, CUBIC, SLOW = (3.4445, -4.7750, 2.0315), (1.5, -0.5, 0.0), (1.875, -1.25, 0.375)


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2207_12000_b200 import binding
    return binding


def wide(t):
    return t.detach().cpu().double().numpy()


def f32(c):
    return tuple(float(np.float32(x)) for x in c)


def slope(t, c):
    return c[0] + 3 * abs(c[1]) * t + 5 * abs(c[2]) * t * t


def size(t, c):
    return abs(c[0]) + abs(c[1]) * t + abs(c[2]) * t * t


SHAPES = [(1, 1), (1, 7), (9, 1), (16, 16), (100, 37), (128, 128), (129, 130), (256, 128), (65, 1000), (602, 256), (256, 602), (640, 200),
          (500, 2000), (1000, 777), (1300, 1290), (2048, 384)]


LARGE = [(1750, 2800), (2800, 1750), (2040, 2048)]  # products whose tiles fill the machine at twice the width


@pytest.mark.parametrize("coeffs,steps", [(QUINTIC, 5), (QUINTIC, 4), (QUINTIC, 1), (CUBIC, 7), (SLOW, 2)])
@pytest.mark.parametrize("rows,cols", SHAPES + LARGE)
def test_one_value_per_row_and_column(B, rows, cols, coeffs, steps):
    rng = np.random.default_rng(rows * 7 + cols)
    r = min(rows, cols)
    i, j = rng.permutation(rows)[:r], rng.permutation(cols)[:r]
    values = rng.uniform(0.3, 1.0, r) * rng.choice([-1, 1], r)
    G = np.zeros((rows, cols), dtype=np.float32)
    G[i, j] = values
    got = wide(B.gnnpre_orthogonalize(torch.from_numpy(G).cuda(), steps=steps, coeffs=coeffs, scale=1.25))
    c = f32(coeffs)
    s = np.abs(G[i, j].astype(np.float64))
    s = s / (np.sqrt((s ** 2).sum()) + float(np.float32(1e-7)))
    err = 2.0 ** -22 * s
    for _ in range(steps):
        t = s * s
        err = slope(t, c) * err + 8 * 2.0 ** -22 * s * size(t, c)
        s = s * (c[0] + c[1] * t + c[2] * t * t)
    want = np.zeros((rows, cols))
    want[i, j] = 1.25 * s * np.sign(G[i, j])
    bound = np.zeros((rows, cols))
    bound[i, j] = 1.25 * err + 2.0 ** -23 * np.abs(want[i, j])
    assert (np.abs(got - want) <= bound).all(), float(np.max(np.abs(got - want)[i, j] / bound[i, j]))
    assert np.count_nonzero(got) <= r


def dense(shape, seed, scale=1e-3):
    """A few strong directions above a floor of noise, as a weight's gradient has."""
    rng = np.random.default_rng(seed)
    *batch, m, n = shape
    k = min(m, n, 5)
    U, V = rng.standard_normal((*batch, m, k)), rng.standard_normal((*batch, k, n))
    return (scale * (rng.standard_normal(shape) + (U * 4.0 ** -np.arange(k) * 8) @ V)).astype(np.float32)


def plain_f32(G, steps, coeffs, eps, scale):
    a, b, c = coeffs
    X = G.float()
    X = X / (X.double().square().sum((-2, -1), keepdim=True).sqrt() + eps).float()
    for _ in range(steps):
        A = X @ X.mT
        X = a * X + (b * A + c * (A @ A)) @ X
    return X * scale


@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("shape", SHAPES[3:])
def test_dense(B, dtype, shape):
    assert not torch.backends.cuda.matmul.allow_tf32
    steps, scale, c = 5, 0.8, f32(QUINTIC)
    G = torch.from_numpy(dense(shape, sum(shape))).cuda().to(dtype)
    out = B.gnnpre_orthogonalize(G, steps=steps, coeffs=QUINTIC, scale=scale)
    assert out.dtype is dtype and out.shape == G.shape
    want = orc.orthogonalize(wide(G), steps, c, float(np.float32(1e-7)), float(np.float32(scale)))
    X = wide(G)
    X = X / np.sqrt((X ** 2).sum())
    s = np.linalg.svd(X, compute_uv=False)
    K, off = max(shape), 2.0 ** -22
    for _ in range(steps):
        top = (s * s).max()
        off = slope(top, c) * off + (8 * 2.0 ** -22 + K * 2.0 ** -24) * size(top, c) * np.sqrt((s ** 2).sum())
        s = s * (c[0] + c[1] * s ** 2 + c[2] * s ** 4)
    rounding = torch.finfo(dtype).eps / 2 * np.linalg.norm(want) + HALF_SUBNORMAL[dtype] * np.sqrt(want.size)
    err = np.linalg.norm(wide(out) - want)
    assert err <= scale * off + rounding, (err, scale * off, rounding)
    tall = G.shape[0] > G.shape[1]
    plain = plain_f32(G.mT if tall else G, steps, c, 1e-7, scale)
    plain = wide(plain.mT if tall else plain)
    assert err <= 8 * np.linalg.norm(plain - want) + rounding + 2.0 ** -20 * np.linalg.norm(want), (err, np.linalg.norm(plain - want))


@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("shape", LARGE)
def test_large_dense(B, shape, dtype):
    """The same comparison with plain fp32 as above, both against the recurrence in 64 bits on the device; steps that 16-bit outputs
    multiply together are off by no more than in test_steps_that_are_multiplied_together."""
    G = torch.from_numpy(dense(shape, 8)).cuda().to(dtype)
    c = f32(QUINTIC)
    X = G.double() / (G.double().square().sum().sqrt() + float(np.float32(1e-7)))
    tall = shape[0] > shape[1]
    X = X.mT if tall else X
    for _ in range(5):
        A = X @ X.mT
        X = c[0] * X + (c[1] * A + c[2] * (A @ A)) @ X
    want = X.mT if tall else X
    plain = plain_f32(G.mT if tall else G, 5, c, 1e-7, 1.0)
    plain = plain.mT if tall else plain
    got = B.gnnpre_orthogonalize(G)
    carried = {F32: 0.0, BF16: 2 * 2.0 ** -11, F16: 3 * 2.0 ** -14}[dtype]
    bound = 8 * (plain.double() - want).norm() + (2.0 ** -20 + carried + torch.finfo(dtype).eps / 2) * want.norm()
    assert float((got.double() - want).norm()) <= float(bound)


@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("steps", (1, 2, 3, 4, 6, 8))
def test_steps_that_are_multiplied_together(B, steps, dtype):
    """A long matrix, where the polynomials of up to three (bf16) or two (fp16) steps meet before X does.  A is then carried from step
    to step: its error, 8 * 2^-22 in the first, grows by a^2 < 12 per step and enters P with |b| / a < 1.4 of itself relative to P:
    12^2 * 8 * 2^-22 * 1.4 < 2^-11 for three steps, 12 * 8 * 2^-22 * 1.4 < 2^-14 for two, once per segment."""
    G = torch.from_numpy(dense((300, 4000), 3)).cuda().to(dtype)
    got = wide(B.gnnpre_orthogonalize(G, steps=steps))
    want = orc.orthogonalize(wide(G), steps, f32(QUINTIC), 1e-7, 1.0)
    plain = wide(plain_f32(G, steps, f32(QUINTIC), 1e-7, 1.0))
    carried = {F32: 0.0, BF16: -(-steps // 3) * 2.0 ** -11, F16: -(-steps // 2) * 2.0 ** -14}[dtype]
    bound = 8 * np.linalg.norm(plain - want) + (2.0 ** -20 + carried + torch.finfo(dtype).eps / 2) * np.linalg.norm(want)
    assert np.linalg.norm(got - want) <= bound


@pytest.mark.parametrize("dtype", (F32, F16))
@pytest.mark.parametrize("shape,pad", [((3, 256, 100), 0), ((5, 40, 130), 3), ((2, 520, 300), 1), ((130, 17, 5), 2)])
def test_batches_strides_and_in_place(B, dtype, shape, pad):
    n, m, k = shape
    room = torch.full((n, m + pad, k + pad), float("nan"), dtype=dtype, device="cuda")
    G = room[:, :m, :k]
    G.copy_(torch.from_numpy(dense(shape, 11)).cuda())
    # each matrix by itself, and all at once: the same bits
    alone = [B.gnnpre_orthogonalize(G[i], steps=5) for i in range(n)]
    together = B.gnnpre_orthogonalize(G, steps=5)
    for i in range(n):
        want = orc.orthogonalize(wide(G[i]), 5, f32(QUINTIC), 1e-7, 1.0)
        assert np.linalg.norm(wide(together[i]) - want) <= (2.0 ** -10 + torch.finfo(dtype).eps) * np.linalg.norm(want)
        assert np.linalg.norm(wide(together[i]) - wide(alone[i])) <= (2.0 ** -10 + torch.finfo(dtype).eps) * np.linalg.norm(want)
    again = B.gnnpre_orthogonalize(G, steps=5, out=G)  # out is G
    assert again is G and torch.equal(G, together)
    rest = torch.ones_like(room, dtype=torch.bool)
    rest[:, :m, :k] = False
    assert torch.isnan(room[rest]).all()


def test_side_by_side_in_one_buffer(B):
    """G and out as column views of one buffer, and as matrices that alternate in one."""
    room = torch.zeros((3, 40, 120), device="cuda")
    room[:, :, :60] = torch.from_numpy(dense((3, 40, 60), 1)).cuda()
    want = B.gnnpre_orthogonalize(room[:, :, :60].clone())
    assert torch.equal(B.gnnpre_orthogonalize(room[:, :, :60], out=room[:, :, 60:]), want)
    turns = torch.zeros((6, 40, 60), device="cuda")
    turns[::2] = room[:, :, :60]
    assert torch.equal(B.gnnpre_orthogonalize(turns[::2], out=turns[1::2]), want)


def test_zeros_tiny_huge_and_not_finite(B):
    assert (B.gnnpre_orthogonalize(torch.zeros((130, 60), device="cuda")) == 0).all()
    assert torch.isnan(B.gnnpre_orthogonalize(torch.zeros((130, 60), device="cuda"), eps=0.0)).all()
    G = torch.from_numpy(dense((130, 60), 5, 1.0)).cuda()
    want = wide(B.gnnpre_orthogonalize(G, eps=0.0))
    for factor in (2.0 ** -100, 2.0 ** 100):  # the squares leave the range of fp32; the result does not change
        assert np.array_equal(wide(B.gnnpre_orthogonalize(G * factor, eps=0.0)), want)
    both = torch.stack([G, G, G])
    both[1, 7, 9] = float("nan")
    both[2, 100, 3] = float("inf")
    out = B.gnnpre_orthogonalize(both, eps=0.0)
    assert np.array_equal(wide(out[0]), want) and torch.isnan(out[1]).all() and torch.isnan(out[2]).all()


def test_result_is_near_orthogonal_and_reproducible(B):
    G = torch.randn((256, 512), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    out = B.gnnpre_orthogonalize(G, steps=25, coeffs=SLOW)  # coefficients that converge to 1
    gram = wide(out) @ wide(out).T
    assert np.abs(gram - np.eye(256)).max() <= 2.0 ** -14
    first = B.gnnpre_orthogonalize(G)
    for _ in range(3):
        assert torch.equal(B.gnnpre_orthogonalize(G), first)


def test_in_a_graph_on_a_stream_and_with_a_kept_workspace(B):
    shape, steps = (300, 700), 5
    G, out = torch.zeros(shape, device="cuda"), torch.empty(shape, device="cuda")
    room = torch.empty(B.gnnpre_orthogonalize_workspace(1, *shape, steps), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    B.gnnpre_orthogonalize(G, steps=steps, out=out, workspace=room)
    with torch.cuda.graph(graph):
        B.gnnpre_orthogonalize(G, steps=steps, out=out, workspace=room, check=False)
    side = torch.cuda.Stream()
    for seed in (1, 2):
        G.copy_(torch.from_numpy(dense(shape, seed)).cuda())
        room.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        eager = B.gnnpre_orthogonalize(G, steps=steps, stream=side)
        assert torch.equal(out, eager)
        want = orc.orthogonalize(wide(G), steps, f32(QUINTIC), 1e-7, 1.0)
        assert np.linalg.norm(wide(out) - want) <= 2.0 ** -10 * np.linalg.norm(want)


def test_waits_that_run_out_are_reported_and_leave_the_device_usable(B):
    for shape in ((100, 60), (300, 200), (1500, 1500)):
        G = torch.from_numpy(dense(shape, 1)).cuda()
        assert B.gnnpre_orthogonalize_selftest_wait_timeout(G, polls=50) == -8
        got = wide(B.gnnpre_orthogonalize(G))
        want = orc.orthogonalize(wide(G), 5, f32(QUINTIC), 1e-7, 1.0)
        assert np.linalg.norm(got - want) <= 2.0 ** -10 * np.linalg.norm(want)


@pytest.mark.parametrize("shape", [(128, 256), (60, 130), (130, 60), (100, 1500), (300, 500), (500, 300), (1500, 1500)])
def test_the_largest_numbers_are_finite(B, shape):
    """Entries up to the largest that fp32 holds: the result is that of the same matrix scaled down by a power of two."""
    G = dense(shape, 4, 1.0)
    G[3, 5] = -np.abs(G).max() * 2
    top = np.abs(G).max()
    G = G / top
    big = torch.from_numpy((G * np.finfo(np.float32).max).astype(np.float32)).cuda()
    assert float(big[3, 5]) == -float(np.finfo(np.float32).max)
    got = B.gnnpre_orthogonalize(big)
    assert torch.equal(got, B.gnnpre_orthogonalize(big * 2.0 ** -100, eps=0.0)) and float(got.abs().max()) > 0


@pytest.mark.parametrize("shape", [(128, 256), (256, 128), (100, 2000), (300, 500), (1500, 1600)])
def test_the_norm_is_summed_in_64_bits(B, shape):
    """A few ones along the longer side, before and among entries whose squares, 2^-24 each, fp32 drops beside a one: with them the
    norm is larger by 2^-19 of itself.  With P = I the result is G / ||G||, off by the operands' rounding (2^-22 for X, its scale and
    factor 2^-23, the result 2^-24)."""
    G = np.full(sorted(shape), 2.0 ** -12, dtype=np.float32)
    for first in (0, 8, 16, 24):
        G[:, first::256] = 1.0
    if shape[0] > shape[1]:
        G = np.ascontiguousarray(G.T)
    got = wide(B.gnnpre_orthogonalize(torch.from_numpy(G).cuda(), steps=1, coeffs=(1.0, 0.0, 0.0), eps=0.0))
    want = G.astype(np.float64) / np.sqrt((G.astype(np.float64) ** 2).sum())
    ones = G == 1.0
    assert (np.abs(got - want)[ones] <= 2.0 ** -21 * want[ones]).all(), float((np.abs(got - want)[ones] / want[ones]).max() * 2.0 ** 21)


SMALL = [(128, 256), (256, 100), (60, 1500), (300, 500), (500, 300), (1500, 1600), (1600, 1500)]


def near(got, G, steps, coeffs, eps, scale, dtype, carried=0.0):
    """Whether `got` is as near the oracle as plain fp32 is (eight times its error, as in test_dense), and rounded once."""
    want = orc.orthogonalize(wide(G), steps, f32(coeffs), float(np.float32(eps)), float(np.float32(scale)))
    plain = wide(plain_f32(G, steps, f32(coeffs), float(np.float32(eps)), scale))
    size = np.linalg.norm(want)
    rounding = torch.finfo(dtype).eps / 2 * size + HALF_SUBNORMAL[dtype] * np.sqrt(want.size)
    err = np.linalg.norm(wide(got) - want)
    assert err <= 8 * np.linalg.norm(plain - want) + (2.0 ** -20 + carried) * size + rounding, (err / size, np.linalg.norm(plain - want) / size)


@pytest.mark.parametrize("ratio", (0.3, 2.0 ** -6, 1e-4, 1e-6, 1e-9, 1e-20))
@pytest.mark.parametrize("shape", SMALL)
def test_an_update_far_below_eps(B, shape, ratio):
    """||G|| = ratio * eps: X_0 is that small, and the steps enlarge it by up to a each.  Nothing of its 22 bits may be lost."""
    G = torch.from_numpy(dense(shape, 6, 1.0)).cuda()
    eps = float(np.float32(float(G.double().norm()) / ratio))
    for steps in (1, 5):
        near(B.gnnpre_orthogonalize(G, steps=steps, eps=eps, scale=0.7), G, steps, QUINTIC, eps, 0.7, F32)
    if ratio <= 1e-4:  # steps enough to bring it to one
        steps = 5 + int(np.log(1 / ratio) / np.log(3.4445))
        near(B.gnnpre_orthogonalize(G, steps=steps, eps=eps), G, steps, QUINTIC, eps, 1.0, F32)


@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("ratio", (1e-2, 1e-6))
def test_an_update_far_below_eps_whose_steps_are_multiplied_together(B, dtype, ratio):
    G = torch.from_numpy(dense((300, 4000), 7, 1.0)).cuda().to(dtype)
    eps = float(np.float32(float(G.double().norm()) / ratio))
    for steps in (2, 3, 5, 12):
        scale = 1.0 if steps > 5 else 1.0 / ratio  # (so that fp16 holds the result)
        carried = -(-steps // 3) * 2.0 ** -11 if dtype is BF16 else -(-steps // 2) * 2.0 ** -14
        near(B.gnnpre_orthogonalize(G, steps=steps, eps=eps, scale=scale), G, steps, QUINTIC, eps, scale, dtype, carried)


@pytest.mark.parametrize("shape", [(100, 60), (300, 500), (1500, 1600)])
def test_matrices_of_a_batch_lie_at_their_own_distance_from_eps(B, shape):
    G = torch.from_numpy(dense((4, *shape), 8, 1.0)).cuda() * torch.tensor([1.0, 1e-3, 1e-7, 0.0], device="cuda")[:, None, None]
    eps = float(np.float32(1e-2 * float(G[0].double().norm())))
    out = B.gnnpre_orthogonalize(G, eps=eps)
    for i in range(3):
        near(out[i], G[i], 5, QUINTIC, eps, 1.0, F32)
        assert torch.equal(out[i], B.gnnpre_orthogonalize(G[i], eps=eps)) or shape == (1500, 1600)  # (there tiles go by the batch)
    assert (out[3] == 0).all()


@pytest.mark.parametrize("coeffs,steps", [((0.01, 0.0, 0.0), 5), ((0.1, -0.05, 0.01), 8), ((0.0, 0.5, 0.0), 3), ((0.3, 0.0, 0.1), 6), ((0.0, 0.0, 0.0), 2)])
@pytest.mark.parametrize("shape", SMALL)
def test_coefficients_that_shrink_the_update(B, shape, coeffs, steps):
    """Within the recurrence of the worst case that test_dense computes (X' = A X / 2 three times is a 27th power: it enlarges what X_0 is
    off by as many times, which plain fp32 shows as well as these operands' 22 bits do)."""
    G = torch.from_numpy(dense(shape, 9, 1.0)).cuda()
    c = f32(coeffs)
    want = orc.orthogonalize(wide(G), steps, c, float(np.float32(1e-7)), 1.0)
    X = wide(G)
    s = np.linalg.svd(X / np.sqrt((X ** 2).sum()), compute_uv=False)
    off = 2.0 ** -22
    for _ in range(steps):
        top = (s * s).max()
        off = slope(top, c) * off + (8 * 2.0 ** -22 + max(shape) * 2.0 ** -24) * size(top, c) * np.sqrt((s ** 2).sum())
        s = s * np.abs(c[0] + c[1] * s ** 2 + c[2] * s ** 4)
    assert np.linalg.norm(wide(B.gnnpre_orthogonalize(G, steps=steps, coeffs=coeffs)) - want) <= off + 2.0 ** -24 * np.linalg.norm(want)


@pytest.mark.parametrize("dtype", (F32, BF16, F16))
@pytest.mark.parametrize("shape", [
    (3, 1000, 777), (2, 600, 2500), (4, 2500, 300), (2, 1500, 1600), (7, 256, 602), (9, 602, 256), (7, 384, 1024), (8, 1024, 384),
    (2, 128, 2048), (2, 2048, 128), (3, 100, 1100), (3, 600, 100), (40, 60, 257), (6, 384, 1024), (2, 20, 40000), (1, 3000, 70)])
def test_batches_of_every_form(B, shape, dtype):
    """Several matrices at once, by a launch per product (steps by themselves and multiplied together), by clusters of 8 and of 16 CTAs with
    up to all the tiles they hold, on the chip by one to eight CTAs: each matrix as near the oracle as plain fp32 is."""
    G = torch.from_numpy(dense(shape, sum(shape))).cuda().to(dtype)
    out = B.gnnpre_orthogonalize(G, scale=0.9)
    r, n = sorted(shape[1:])
    alone = r > 128 or n > 2048
    carried = {F32: 0.0, BF16: 2 * 2.0 ** -11, F16: 3 * 2.0 ** -14}[dtype] if alone else 0.0
    for i in range(0, shape[0], max(1, shape[0] // 4)):
        near(out[i], G[i], 5, QUINTIC, 1e-7, 0.9, dtype, carried)
    if not alone:  # on the chip nothing depends on how many there are
        assert torch.equal(out[-1], B.gnnpre_orthogonalize(G[-1], scale=0.9))
    assert torch.equal(B.gnnpre_orthogonalize(G, scale=0.9), out)


@pytest.mark.parametrize("shape", [(64, 128), (300, 500), (1300, 1290)])
def test_weak_values_beside_strong_ones(B, shape):
    """One value per row and column, from 1 to 2^-36 of the largest: below some 2^-16 an operand's entry is off by 2^-39 of the bound (two,
    here) instead of 2^-22 of itself, in every X that is held; the rest as in test_one_value_per_row_and_column."""
    rng = np.random.default_rng(4)
    r = min(shape)
    i, j = rng.permutation(shape[0])[:r], rng.permutation(shape[1])[:r]
    G = np.zeros(shape, dtype=np.float32)
    G[i, j] = 2.0 ** -(36 * np.arange(r) / r) * rng.choice([-1, 1], r)
    got = wide(B.gnnpre_orthogonalize(torch.from_numpy(G).cuda()))
    c = f32(QUINTIC)
    s = np.abs(G[i, j].astype(np.float64))
    s = s / (np.sqrt((s ** 2).sum()) + float(np.float32(1e-7)))
    err = 2.0 ** -22 * s + 2.0 ** -38
    for _ in range(5):
        t = s * s
        err = slope(t, c) * err + 8 * 2.0 ** -22 * s * size(t, c) + 2.0 ** -38
        s = s * (c[0] + c[1] * t + c[2] * t * t)
    want = s * np.sign(G[i, j])
    assert (np.abs(got[i, j] - want) <= err + 2.0 ** -24 * np.abs(want)).all()


@pytest.mark.parametrize("shape", [(100, 60), (100, 900), (300, 700), (1500, 1600)])
def test_replayed_and_after_waits_that_ran_out_it_is_as_exact_as_ever(B, shape):
    G, out = torch.zeros(shape, device="cuda"), torch.empty(shape, device="cuda")
    room = torch.empty(B.gnnpre_orthogonalize_workspace(1, *shape, 5), dtype=torch.uint8, device="cuda")
    graph = torch.cuda.CUDAGraph()
    B.gnnpre_orthogonalize(G, out=out, workspace=room)
    with torch.cuda.graph(graph):
        B.gnnpre_orthogonalize(G, out=out, workspace=room, check=False)
    for seed in (1, 2):
        G.copy_(torch.from_numpy(dense(shape, seed)).cuda())
        room.fill_(255)
        graph.replay()
        torch.cuda.synchronize()
        near(out, G, 5, QUINTIC, 1e-7, 1.0, F32)
    assert B.gnnpre_orthogonalize_selftest_wait_timeout(G, polls=50) == -8
    assert torch.equal(B.gnnpre_orthogonalize(G), out)


@pytest.mark.parametrize("dtype", (F32, BF16))
@pytest.mark.parametrize("shape", [(7, 256, 1000), (8, 256, 1000), (14, 200, 384), (15, 200, 384), (12, 384, 130), (16, 130, 130), (1, 257, 257), (3, 256, 1030)])
def test_both_sides_of_where_clusters_end(B, shape, dtype):
    """Clusters of 16 CTAs up to seven matrices, of 8 up to fourteen, for a smaller side of at most 256 and 32 tiles; a launch per product
    beyond."""
    G = torch.from_numpy(dense(shape, 2)).cuda().to(dtype)
    out = B.gnnpre_orthogonalize(G)
    carried = 0.0 if dtype is F32 else 2 * 2.0 ** -11
    for i in {0, shape[0] // 2, shape[0] - 1}:
        near(out[i], G[i], 5, QUINTIC, 1e-7, 1.0, dtype, carried)


@pytest.mark.parametrize("shape", [(14, 1100, 40), (15, 40, 1100), (15, 1024, 100), (100, 30, 70)])
def test_many_small_matrices(B, shape):
    """Up to fourteen by eight CTAs each on the chip, more of them by a launch per product; any number by up to four CTAs."""
    G = torch.from_numpy(dense(shape, 3)).cuda()
    out = B.gnnpre_orthogonalize(G)
    for i in (0, shape[0] // 2, shape[0] - 1):
        near(out[i], G[i], 5, QUINTIC, 1e-7, 1.0, F32)
