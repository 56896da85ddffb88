"""Refusals of the operators of the training step, as the C entry points give them before they touch a device, and what their
workspaces are asked to be.  No GPU: the addresses are never followed."""
import pytest

from paper_2207_12000_b200 import build as libbuild

INVALID_ARG, ALIGN = -1, -3


@pytest.fixture(scope="module")
def lib():
    libbuild.build()
    from paper_2207_12000_b200 import binding
    return binding._lib


def call(fn, base, **changes):
    args = dict(base)
    for k, v in changes.items():
        assert k in args
        args[k] = v
    return fn(*args.values())


LOOKUP = dict(table=0x100000, n=1000, dim=64, ldt=64, dtype=0, ids=0x900000, ids_type=0, count=100, scale=1.0, out=0xa00000, ldo=64,
              stream=None)


@pytest.mark.parametrize("changes,status", [
    (dict(table=None), INVALID_ARG), (dict(ids=None), INVALID_ARG), (dict(out=None), INVALID_ARG), (dict(n=0), INVALID_ARG),
    (dict(n=1 << 31), INVALID_ARG), (dict(dim=0, ldt=0, ldo=0), INVALID_ARG), (dict(dim=(1 << 20) + 1, ldt=1 << 21, ldo=1 << 21), INVALID_ARG),
    (dict(ldt=63), INVALID_ARG), (dict(ldo=63), INVALID_ARG), (dict(dtype=3), INVALID_ARG), (dict(dtype=-1), INVALID_ARG),
    (dict(ids_type=2), INVALID_ARG), (dict(count=-1), INVALID_ARG), (dict(count=1 << 31), INVALID_ARG),
    (dict(table=0x100002), ALIGN), (dict(out=0xa00001, dtype=1), ALIGN), (dict(ids=0x900004, ids_type=1), ALIGN),
    (dict(out=0x100000), INVALID_ARG), (dict(out=0x100000 + 4 * 64 * 999), INVALID_ARG), (dict(out=0x900000), INVALID_ARG),
    (dict(out=0x100000 + 4 * 32, ldt=128, ldo=128), INVALID_ARG)])
def test_lookup_refuses(lib, changes, status):
    assert call(lib.gnnpre_embedding_lookup, LOOKUP, **changes) == status


GRAD = dict(d_out=0x100000, ldd=64, dtype=0, ids=0x900000, ids_type=0, count=100, n=1000, dim=64, scale=1.0, accumulate=0,
            d_table=0xa00000, ldt=64, table_dtype=0, workspace=0x4000000, workspace_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("changes,status", [
    (dict(d_out=None), INVALID_ARG), (dict(ids=None), INVALID_ARG), (dict(d_table=None), INVALID_ARG), (dict(workspace=None), INVALID_ARG),
    (dict(n=0), INVALID_ARG), (dict(n=1 << 31), INVALID_ARG), (dict(dim=0), INVALID_ARG), (dict(count=-1), INVALID_ARG),
    (dict(ldd=63), INVALID_ARG), (dict(ldt=63), INVALID_ARG), (dict(dtype=7), INVALID_ARG), (dict(table_dtype=1), INVALID_ARG),
    (dict(dtype=1, table_dtype=2), INVALID_ARG), (dict(ids_type=-1), INVALID_ARG), (dict(workspace_bytes=1000), INVALID_ARG),
    (dict(workspace=0x4000010), ALIGN), (dict(d_out=0x100001), ALIGN), (dict(d_table=0xa00002), ALIGN), (dict(ids=0x900002), ALIGN),
    (dict(d_table=0x100000), INVALID_ARG), (dict(d_table=0x900000 - 4 * 64 * 999), INVALID_ARG), (dict(workspace=0xa00000), INVALID_ARG),
    (dict(workspace=0x100000), INVALID_ARG), (dict(workspace=0x900000), INVALID_ARG)])
def test_embedding_grad_refuses(lib, changes, status):
    assert call(lib.gnnpre_embedding_grad, GRAD, **changes) == status


def test_embedding_grad_workspace(lib):
    size = lib.gnnpre_embedding_grad_workspace
    assert size(1000, 64, 0) == 0
    for n, dim, count in ((0, 64, 1), (1 << 31, 64, 1), (10, 0, 1), (10, (1 << 20) + 1, 1), (10, 64, -1), (10, 64, 1 << 31)):
        assert size(n, dim, count) == INVALID_ARG
    # two pairs of arrays, and at most a row of parts for every four entries
    for n, dim, count in ((1, 1, 1), (1000, 64, 100), (169343, 128, 65553), ((1 << 31) - 1, 602, 2449029), (65536, 100, (1 << 31) - 1)):
        rows = (dim + 3) // 4 * 4
        assert 16 * count <= size(n, dim, count) <= 16 * count + rows * count + 8 * rows * 4 + count // 64 + (1 << 22) + (count // 4096 + 1) * 8192


def coefficients(a=3.4445, b=-4.7750, c=2.0315):
    import ctypes
    return (ctypes.c_float * 3)(a, b, c)


ORTH = dict(G=0x100000, rows=100, cols=60, ldg=60, g_stride=6000, batch=2, dtype=0, steps=5, coeffs=coefficients(), eps=1e-7, scale=1.0,
            out=0x400000, ldo=60, o_stride=6000, workspace=0x4000000, workspace_bytes=1 << 30, error_flag=None, stream=None)


@pytest.mark.parametrize("changes,status", [
    (dict(G=None), INVALID_ARG), (dict(out=None), INVALID_ARG), (dict(workspace=None), INVALID_ARG), (dict(coeffs=None), INVALID_ARG),
    (dict(rows=0), INVALID_ARG), (dict(cols=0), INVALID_ARG), (dict(rows=65537), INVALID_ARG), (dict(cols=65537, ldg=70000, ldo=70000), INVALID_ARG),
    (dict(batch=-1), INVALID_ARG), (dict(batch=16385), INVALID_ARG), (dict(ldg=59), INVALID_ARG), (dict(ldo=59), INVALID_ARG),
    (dict(g_stride=-1), INVALID_ARG), (dict(o_stride=5999), INVALID_ARG), (dict(dtype=3), INVALID_ARG), (dict(steps=0), INVALID_ARG),
    (dict(steps=65), INVALID_ARG), (dict(eps=-1.0), INVALID_ARG), (dict(eps=float("nan")), INVALID_ARG), (dict(eps=float("inf")), INVALID_ARG),
    (dict(coeffs=coefficients(a=float("nan"))), INVALID_ARG), (dict(coeffs=coefficients(b=float("inf"))), INVALID_ARG),
    (dict(coeffs=coefficients(3.0, 3.0, 3.0)), INVALID_ARG), (dict(coeffs=coefficients(20.0, 0.0, 0.0)), INVALID_ARG),
    (dict(workspace_bytes=1000), INVALID_ARG), (dict(workspace=0x4000080), ALIGN), (dict(G=0x100002), ALIGN), (dict(out=0x400001, dtype=1), ALIGN),
    (dict(workspace=0x100000), INVALID_ARG), (dict(workspace=0x400000), INVALID_ARG), (dict(batch=0), 0),
    # out on G, but not matrix for matrix: the next matrix, a row further, another pitch, another distance, a part of it
    (dict(out=0x100000 + 4 * 6000), INVALID_ARG), (dict(out=0x100000 + 4 * 60), INVALID_ARG), (dict(out=0x100000, ldo=64, o_stride=6400), INVALID_ARG),
    (dict(out=0x100000, o_stride=7000), INVALID_ARG), (dict(out=0x100000 + 4 * 30, batch=1), INVALID_ARG),
    (dict(ldg=120, ldo=120, g_stride=12000, o_stride=12000, out=0x100000 + 4 * 59), INVALID_ARG)])
def test_orthogonalize_refuses(lib, changes, status):
    assert call(lib.gnnpre_orthogonalize, ORTH, **changes) == status


def test_orthogonalize_workspace(lib):
    size = lib.gnnpre_orthogonalize_workspace
    assert size(0, 10, 10, 5) == 0
    for args in ((-1, 10, 10, 5), (16385, 10, 10, 5), (1, 0, 10, 5), (1, 10, 0, 5), (1, 65537, 10, 5), (1, 10, 65537, 5), (1, 10, 10, 0), (1, 10, 10, 65)):
        assert size(*args) == INVALID_ARG
    assert size(3, 256, 602, 5) == size(3, 602, 256, 5)  # the smaller side counts, not which it is
    for batch, rows, cols in ((1, 1, 1), (3, 256, 602), (1, 2048, 4096)):
        r, n = (-(-x // 128) * 128 for x in sorted((rows, cols)))
        assert 0 < size(batch, rows, cols, 5) <= batch * (4 * (3 * r * n + 6 * r * r) + 512) + 16384


def pointers(*p):
    import ctypes
    return (ctypes.c_void_p * len(p))(*p)


LC_GRAD = dict(hops=pointers(0x100000, 0x200000), num_hops=2, n=1000, feat_dim=60, ldh=64, batch=0x900000, batch_size=100, dY=0x910000, lddy=32,
               dy_hop_stride=3200, Y=0x920000, ldy=32, y_hop_stride=3200, relu_mask=2, hidden=32, accumulate=0, dWt=0x930000, ldw=60,
               workspace=0x4000000, workspace_bytes=1 << 30, error_flag=None, stream=None)


@pytest.mark.parametrize("changes,status", [
    (dict(hops=None), INVALID_ARG), (dict(hops=pointers(0x100000, None)), INVALID_ARG), (dict(hops=pointers(0x100000, 0x200008)), ALIGN),
    (dict(num_hops=0), INVALID_ARG), (dict(num_hops=65), INVALID_ARG), (dict(n=0), INVALID_ARG), (dict(n=1 << 31), INVALID_ARG),
    (dict(feat_dim=0), INVALID_ARG), (dict(feat_dim=(1 << 20) + 4, ldh=1 << 21, ldw=1 << 21), INVALID_ARG), (dict(ldh=56), INVALID_ARG),
    (dict(ldh=62), ALIGN), (dict(ldw=59), INVALID_ARG), (dict(lddy=31), INVALID_ARG), (dict(ldy=31), INVALID_ARG), (dict(dy_hop_stride=-4), INVALID_ARG),
    (dict(y_hop_stride=-4), INVALID_ARG), (dict(batch_size=-1), INVALID_ARG), (dict(batch_size=1 << 31), INVALID_ARG),
    (dict(batch=None, batch_size=1001), INVALID_ARG), (dict(dY=None), INVALID_ARG), (dict(Y=None), INVALID_ARG), (dict(dWt=None), INVALID_ARG),
    (dict(workspace=None), INVALID_ARG), (dict(workspace_bytes=100), INVALID_ARG), (dict(workspace=0x4000040), ALIGN), (dict(hidden=8), INVALID_ARG),
    (dict(hidden=24), INVALID_ARG), (dict(hidden=272, lddy=272, ldy=272), INVALID_ARG), (dict(dY=0x910002), ALIGN), (dict(Y=0x920001), ALIGN),
    (dict(dWt=0x930002), ALIGN), (dict(batch=0x900002), ALIGN), (dict(dWt=0x910000), INVALID_ARG), (dict(dWt=0x920000), INVALID_ARG),
    (dict(dWt=0x900000), INVALID_ARG), (dict(dWt=0x200000), INVALID_ARG), (dict(dWt=0x4000000), INVALID_ARG)])
def test_lc_grad_refuses(lib, changes, status):
    assert call(lib.gnnpre_lc_first_layer_grad, LC_GRAD, **changes) == status


def test_lc_grad_workspace(lib):
    size = lib.gnnpre_lc_first_layer_grad_workspace
    assert size(3, 0, 100, 256) == 0
    for args in ((0, 1, 1, 16), (65, 1, 1, 16), (1, -1, 1, 16), (1, 1 << 31, 1, 16), (1, 1, 0, 16), (1, 1, (1 << 20) + 1, 16), (1, 1, 1, 0),
                 (1, 1, 1, 20), (1, 1, 1, 272)):
        assert size(*args) == INVALID_ARG
    for K, rows, F, H in ((1, 1, 1, 16), (3, 4096, 128, 256), (2, 20011, 602, 192), (3, 2449029, 100, 256)):
        tiles = -(-H // 128) * -(-F // 128)
        assert 0 < size(K, rows, F, H) <= 4 * max(1, 192 // tiles) * H * (F + 16 * -(-F // 128))


@pytest.mark.parametrize("where", ("dY", "Y", "batch", "hop"))
def test_lc_grad_refuses_a_workspace_on_its_inputs(lib, where):
    at = dict(dY=0x4000000, Y=0x4000000 + 0x100, batch=0x4000000 + 0x200)
    changes = dict(hops=pointers(0x100000, 0x4000000 - 4 * 64 * 999)) if where == "hop" else {where: at[where]}
    assert call(lib.gnnpre_lc_first_layer_grad, LC_GRAD, **changes) == INVALID_ARG


def test_lc_grad_looks_at_no_more_of_its_workspace_than_it_asks_for(lib):
    """An input behind the part that the call needs is none of its business: the call gets as far as asking for a device."""
    need = lib.gnnpre_lc_first_layer_grad_workspace(2, 100, 60, 32)
    assert call(lib.gnnpre_lc_first_layer_grad, LC_GRAD, dY=0x4000000 + need) not in (INVALID_ARG, ALIGN)


@pytest.mark.parametrize("rows,cols", [(64, 64), (100, 1100), (130, 130), (256, 1024), (256, 1030), (200, 300), (300, 500), (1500, 1600)])
def test_orthogonalize_workspace_grows_with_the_batch(lib, rows, cols):
    """One that is kept for so many matrices serves fewer, whichever form those take; and more steps ask for no less."""
    size = lib.gnnpre_orthogonalize_workspace
    for steps in (1, 2, 3, 5, 9):
        sizes = [size(batch, rows, cols, steps) for batch in range(1, 40)]
        assert all(0 < a <= b for a, b in zip(sizes, sizes[1:]))
        assert sizes[-1] <= size(39, rows, cols, steps + 1)
