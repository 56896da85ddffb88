"""The operators with which the first dense stage of a model over precomputed hops learns, as cases that can be timed and compared.

Each case is one call of an entry point of ``paper_2207_12000_b200.binding`` or, where ``own`` is false, the same operator in
elementary torch operations.  Sizes are those of this repository's workloads (``gnnpre_inputs.configs``), or generic.

Kinds of case:

  lookup   rows of a learned table, scaled:  out[i] = scale * table[ids[i]]; ids outside the table are padding and give zeros
  grad     the table's gradient:  d_table[v] = scale * sum of the rows of d_out whose id is v
  lc_grad  the weight gradient of act(X_k[batch] W^T) over the hops X_k:  sum_k (d_Y_k where Y_k > 0)^T X_k[batch]
  orth     an update orthogonalised by Newton-Schulz products:  X <- (a I + b A + c A^2) X,  A = X X^T
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
COEFFS = (3.4445, -4.7750, 2.0315)
EPS = 1e-7


def listed():
    return [
        # A handful of nodes looked up while a model answers: latency alone.  A width that is no multiple of the vector loads.
        {"name": "lookup_few_f16_d602", "kind": "lookup", "V": 232965, "D": 602, "N": 37, "type": "f16", "ids": "uniform", "wide": True},
        # Node embeddings of a training mini-batch of 4096 distinct nodes.
        {"name": "lookup_batch_f32_d128", "kind": "lookup", "V": 169343, "D": 128, "N": 4096, "type": "f32", "ids": "distinct", "wide": False},
        # The feature matrix of all nodes of a large graph from their categories, the frequent ones far more often, some unknown.
        {"name": "lookup_all_bf16_d256", "kind": "lookup", "V": 65536, "D": 256, "N": 2449029, "type": "bf16", "ids": "zipf", "wide": True},
        # The gradient of a small graph's table, every node once on average.
        {"name": "grad_batch_f32_d64", "kind": "grad", "V": 4096, "D": 64, "N": 4096, "type": "f32", "to": "f32", "ids": "uniform", "wide": False},
        # Tokens of a batch of text attributes into a larger table; 16-bit rows, the table's gradient in 32 bits.
        {"name": "grad_tokens_bf16_d128", "kind": "grad", "V": 169343, "D": 128, "N": 65553, "type": "bf16", "to": "f32", "ids": "zipf", "wide": True},
        # All nodes of a large graph at once: one category has 6 % of them.
        {"name": "grad_all_f32_d100", "kind": "grad", "V": 65536, "D": 100, "N": 2449029, "type": "f32", "to": "f32", "ids": "zipf", "wide": False},
        # The weight gradient of a mini-batch of 4096 nodes over three hops, hidden width 256.
        {"name": "lcgrad_batch_f128_h256", "kind": "lc_grad", "n": 169343, "rows": 4096, "F": 128, "K": 3, "H": 256},
        # Wide rows, an odd number of them, two hops.
        {"name": "lcgrad_wide_f602_h192", "kind": "lc_grad", "n": 232965, "rows": 20011, "F": 602, "K": 2, "H": 192},
        # A full-batch step: every node of the co-purchase graph, three hops.
        {"name": "lcgrad_epoch_f100_h256", "kind": "lc_grad", "n": 2449029, "rows": 2449029, "F": 100, "K": 3, "H": 256},
        # The update of that stage's weight, hidden 256 on 128 features.
        {"name": "orth_w1_f32", "kind": "orth", "batch": 1, "rows": 256, "cols": 128, "steps": 5, "type": "f32"},
        # One weight per hop on wide features, 16-bit updates.
        {"name": "orth_hops_bf16", "kind": "orth", "batch": 3, "rows": 256, "cols": 602, "steps": 5, "type": "bf16"},
        # A large layer's update.
        {"name": "orth_large_f32", "kind": "orth", "batch": 1, "rows": 2048, "cols": 4096, "steps": 5, "type": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    kind = rng.choice(["lookup", "grad", "lc_grad", "orth"])
    if kind in ("lookup", "grad"):
        D = _log(rng, 16, 602)
        kind_of = rng.choice(sorted(TYPES))
        size = 4 if kind_of == "f32" else 2
        c = {"kind": kind, "V": _log(rng, 500, min(2449029, 9e8 / (4 * D))), "D": D, "N": _log(rng, 1, min(2449029, 1e9 / (size * D))),
             "type": kind_of, "ids": rng.choice(["uniform", "zipf"]), "wide": rng.random() < 0.5}
        return c if kind == "lookup" else {**c, "to": rng.choice(["f32", kind_of])}
    if kind == "lc_grad":
        F, K, H = _log(rng, 16, 602), rng.randint(1, 3), 16 * rng.randint(1, 16)
        n = _log(rng, 10000, min(2449029, 1.5e9 / (K * F)))
        return {"kind": kind, "n": n, "rows": _log(rng, 100, min(n, 2.5e9 / (K * (F + 2 * H)))), "F": F, "K": K, "H": H}
    rows, cols = _log(rng, 16, 2048), _log(rng, 16, 4096)
    batch = min(rng.randint(1, 8), max(1, int(8e6 / (rows * cols))))
    return {"kind": kind, "batch": batch, "rows": rows, "cols": cols, "steps": rng.choice([3, 5, 5, 6]), "type": rng.choice(sorted(TYPES))}


def _matrix(n, F, gen, dtype=torch.float32):
    """Standard-normal rows that start on 16-byte boundaries, as the library wants them."""
    per = 16 // torch.empty(0, dtype=dtype).element_size()
    buf = torch.zeros((n, (F + per - 1) // per * per), device="cuda", dtype=dtype)
    buf[:, :F].normal_(generator=gen)
    return buf[:, :F]


def _ids(case, gen):
    V, N = case["V"], case["N"]
    if case["ids"] == "distinct":
        ids = torch.randperm(V, generator=gen, device="cuda")[:N]
    elif case["ids"] == "uniform":
        ids = torch.randint(V, (N,), generator=gen, device="cuda")
    else:  # the share of the r-th most frequent id falls as 1 / r; one in fifty is padding
        u = torch.rand(N, generator=gen, device="cuda", dtype=torch.float64)
        ids = ((u * math.log(V + 1)).exp().long() - 1).clamp_(0, V - 1)
        ids[torch.rand(N, generator=gen, device="cuda") < 0.02] = -1
    return ids.to(torch.int64 if case["wide"] else torch.int32).contiguous()


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind = case["kind"]
    s = {"case": case}
    if kind == "lookup":
        t = TYPES[case["type"]]
        s["table"] = _matrix(case["V"], case["D"], gen, t)
        s["ids"] = _ids(case, gen)
        s["scale"] = math.sqrt(case["D"])
        s["out"] = _matrix(case["N"], case["D"], gen, t)
    elif kind == "grad":
        s["d_out"] = _matrix(case["N"], case["D"], gen, TYPES[case["type"]])
        s["ids"] = _ids(case, gen)
        s["scale"] = math.sqrt(case["D"])
        s["d_table"] = _matrix(case["V"], case["D"], gen, TYPES[case["to"]])
    elif kind == "lc_grad":
        K, n, rows, F, H = (case[k] for k in ("K", "n", "rows", "F", "H"))
        s["hops"] = [_matrix(n, F, gen) for _ in range(K)]
        s["batch"] = torch.randperm(n, generator=gen, device="cuda", dtype=torch.int32)[:rows].contiguous()
        s["Y"] = torch.empty((K, rows, H), device="cuda").normal_(generator=gen).relu_()
        s["dY"] = torch.empty((K, rows, H), device="cuda").normal_(generator=gen).mul_(1.0 / rows)  # of a mean over the batch
        s["relu_mask"] = (1 << K) - 2  # every term but the first has another layer after it
        s["linear"] = torch.arange(K, device="cuda").view(K, 1, 1) == 0
        s["dWt"] = _matrix(H, F, gen)
    else:
        # an update: a few strong directions above a floor of noise
        b, m, n, t = case["batch"], case["rows"], case["cols"], TYPES[case["type"]]
        G = torch.empty((b, m, n), device="cuda").normal_(generator=gen)
        strong = 8 * 0.5 ** torch.arange(6, device="cuda", dtype=torch.float32)
        U = torch.empty((b, m, 6), device="cuda").normal_(generator=gen) * strong
        G += U @ torch.empty((b, 6, n), device="cuda").normal_(generator=gen)
        per = 16 // torch.empty(0, dtype=t).element_size()
        room = [torch.zeros((b, m, (n + per - 1) // per * per), device="cuda", dtype=t)[:, :, :n] for _ in range(2)]
        s["G"], s["out"] = room[0].copy_(G * 1e-3), room[1]
        s["scale"] = math.sqrt(max(1.0, m / n))
    return s


def _plain_lookup(s):
    table, ids = s["table"], s["ids"]
    known = (ids >= 0) & (ids < table.shape[0])
    rows = table[torch.where(known, ids, 0)].float() * s["scale"]
    return torch.where(known[:, None], rows, 0.0).to(table.dtype)


def _plain_grad(s):
    d_out, ids, (V, D) = s["d_out"], s["ids"], s["d_table"].shape
    known = (ids >= 0) & (ids < V)
    sums = torch.zeros((V + 1, D), device=ids.device)  # the last row takes the padding
    sums.index_add_(0, torch.where(known, ids, V), d_out.float() * s["scale"])
    return sums[:V].to(s["d_table"].dtype)


BLOCK = 4096  # rows of one product: partial sums in 32 bits, added up in 64


def _plain_lc_grad(s):
    X = torch.stack([h[s["batch"]] for h in s["hops"]])
    dZ = torch.where((s["Y"] > 0) | s["linear"], s["dY"], 0.0)
    whole = X.shape[1] // BLOCK * BLOCK
    parts = dZ[:, :whole].unflatten(1, (-1, BLOCK)).transpose(-1, -2) @ X[:, :whole].unflatten(1, (-1, BLOCK))
    rest = dZ[:, whole:].transpose(-1, -2) @ X[:, whole:]
    return (parts.sum((0, 1), dtype=torch.float64) + rest.sum(0, dtype=torch.float64)).float()


def _plain_orth(s):
    a, b, c = COEFFS
    X = s["G"].float()
    X = X / (X.square().sum((1, 2), keepdim=True, dtype=torch.float64).sqrt() + EPS).float()
    tall = X.shape[1] > X.shape[2]
    X = X.transpose(1, 2) if tall else X
    for _ in range(s["case"]["steps"]):
        A = X @ X.transpose(1, 2)
        X = a * X + (b * A + c * (A @ A)) @ X
    X = X.transpose(1, 2) if tall else X
    return (X * s["scale"]).to(s["G"].dtype)


def run(s):
    kind = s["case"]["kind"]
    if not own:
        return {"lookup": _plain_lookup, "grad": _plain_grad, "lc_grad": _plain_lc_grad, "orth": _plain_orth}[kind](s)
    from paper_2207_12000_b200 import binding as B
    if kind == "lookup":
        return B.gnnpre_embedding_lookup(s["table"], s["ids"], scale=s["scale"], out=s["out"])
    if kind == "grad":
        return B.gnnpre_embedding_grad(s["d_out"], s["ids"], s["case"]["V"], scale=s["scale"], out=s["d_table"])
    if kind == "lc_grad":
        return B.gnnpre_lc_first_layer_grad(s["hops"], s["batch"], s["dY"], Y=s["Y"], relu_mask=s["relu_mask"], out=s["dWt"],
                                            check=False)
    return B.gnnpre_orthogonalize(s["G"], steps=s["case"]["steps"], coeffs=COEFFS, eps=EPS, scale=s["scale"], out=s["out"],
                                  check=False)


def work(case):
    """Every input read once, every output written once; of a table no more rows than are asked for."""
    size = {"f32": 4, "bf16": 2, "f16": 2}
    kind = case["kind"]
    if kind == "lookup":
        N, D, es = case["N"], case["D"], size[case["type"]]
        return {"bytes": N * (8 if case["wide"] else 4) + (min(N, case["V"]) + N) * D * es, "flops": N * D}
    if kind == "grad":
        N, D = case["N"], case["D"]
        return {"bytes": N * (8 if case["wide"] else 4) + N * D * size[case["type"]] + case["V"] * D * size[case["to"]], "flops": 2 * N * D}
    if kind == "lc_grad":
        K, rows, F, H = case["K"], case["rows"], case["F"], case["H"]
        return {"bytes": 4 * (rows + K * rows * (F + H) + (K - 1) * rows * H + H * F), "flops": 2 * K * rows * F * H}
    r, n, steps = min(case["rows"], case["cols"]), max(case["rows"], case["cols"]), case["steps"]
    # the products as they stand, half of each symmetric one; or all polynomials of A multiplied together before X
    each = min(steps * (r * r * n + r ** 3 + 2 * r * r * n), 3 * r * r * n + steps * 4 * r ** 3)
    return {"bytes": 2 * case["batch"] * r * n * size[case["type"]], "flops": case["batch"] * each}


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "lookup":
        wide = torch.cat([s["table"].double() * s["scale"], torch.zeros((1, case["D"]), device="cuda", dtype=torch.float64)])
        ids = s["ids"].long()
        ids[(ids < 0) | (ids >= case["V"])] = case["V"]
        return wide.index_select(0, ids)
    if kind == "grad":
        ids = s["ids"].long()
        at = torch.nonzero((ids >= 0) & (ids < case["V"])).flatten()
        sums = torch.zeros((case["V"], case["D"]), device="cuda", dtype=torch.float64)
        return sums.index_put_((ids[at],), s["d_out"][at].double(), accumulate=True) * s["scale"]
    if kind == "lc_grad":
        total = torch.zeros((case["H"], case["F"]), device="cuda", dtype=torch.float64)
        for k, hop in enumerate(s["hops"]):
            for lo in range(0, case["rows"], 262144):
                dz = s["dY"][k, lo:lo + 262144].double()
                if s["relu_mask"] >> k & 1:
                    dz = dz * (s["Y"][k, lo:lo + 262144] > 0)
                total += torch.einsum("bh,bf->hf", dz, hop.index_select(0, s["batch"][lo:lo + 262144]).double())
        return total
    a, b, c = COEFFS
    G = s["G"].double()
    X = G / (torch.linalg.vector_norm(G, dim=(1, 2), keepdim=True) + EPS)
    for _ in range(case["steps"]):
        step = torch.baddbmm(X, torch.bmm(X, X.mT), X, beta=b, alpha=c) if X.shape[1] <= X.shape[2] else torch.baddbmm(X, X, torch.bmm(X.mT, X), beta=b, alpha=c)
        X = torch.baddbmm(X, torch.bmm(X, X.mT), step, beta=a) if X.shape[1] <= X.shape[2] else torch.baddbmm(X, step, torch.bmm(X.mT, X), beta=a)
    return X * s["scale"]
