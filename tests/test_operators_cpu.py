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
