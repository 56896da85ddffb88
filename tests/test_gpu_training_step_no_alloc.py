"""The training step's calls allocate nothing where the caller brings results and workspaces: neither through torch nor from the device."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    from paper_2207_12000_b200 import binding
    return binding


def room(size):
    return torch.empty(size, dtype=torch.uint8, device="cuda")


def lookup(B):
    table, ids, out = torch.ones((500, 64), device="cuda"), torch.arange(5000, device="cuda") % 500, torch.empty((5000, 64), device="cuda")
    return lambda: B.gnnpre_embedding_lookup(table, ids, out=out)


def table_grad(B, count):
    d_out, ids, out = torch.ones((count, 16), device="cuda"), torch.arange(count, device="cuda") % 500, torch.empty((500, 16), device="cuda")
    w = room(B.gnnpre_embedding_grad_workspace(500, 16, count))
    return lambda: B.gnnpre_embedding_grad(d_out, ids, 500, out=out, workspace=w)


def weight_grad(B, hops):
    X, dY, out = torch.ones((3000, 100), device="cuda"), torch.ones((hops, 3000, 64), device="cuda"), torch.empty((64, 100), device="cuda")
    w = room(B.gnnpre_lc_first_layer_grad_workspace(hops, 3000, 100, 64))
    return lambda: B.gnnpre_lc_first_layer_grad([X] * hops, None, dY, out=out, workspace=w, check=False)


def update(B, *shape):
    G, out = torch.ones(shape, device="cuda"), torch.empty(shape, device="cuda")
    w = room(B.gnnpre_orthogonalize_workspace(shape[0], *shape[1:], 5))
    return lambda: B.gnnpre_orthogonalize(G, out=out, workspace=w, check=False)


CALLS = {"lookup": lookup, "short list": lambda B: table_grad(B, 5000), "list": lambda B: table_grad(B, 50_000), "long list": lambda B: table_grad(B, 700_000),
         "weight, 2 hops": lambda B: weight_grad(B, 2), "weight, 9 hops": lambda B: weight_grad(B, 9), "update, chip": lambda B: update(B, 2, 100, 900),
         "update, cluster": lambda B: update(B, 2, 300, 500), "update, launches": lambda B: update(B, 2, 1500, 1600)}


@pytest.mark.parametrize("name", CALLS)
def test_no_allocation(B, name):
    call = CALLS[name](B)
    call()  # the first call on a device sets its kernels up
    torch.cuda.synchronize()
    free, made = torch.cuda.mem_get_info()[0], torch.cuda.memory_stats()["allocation.all.allocated"]
    for _ in range(3):
        call()
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == free and torch.cuda.memory_stats()["allocation.all.allocated"] == made
