"""Products whose shape a language model gives them: ragged groups of rows
against a stack of weights with both gradients, a shared projection with the
low-rank adapters of many requests, and the orthogonalisation of an update by
Newton-Schulz products.

A case names the operator and its sizes.  ``run`` with ``own`` false computes
it from elementary torch operations in 32 bits, rounded once at the end; with
``own`` true it calls the library.  ``exact`` computes it in 64 bits.

    fwd    Y[r] = X[r] W_g^T                     rows, groups, n, k
    bwd    dX[r] = dY[r] W_g, dW_g = dY_g^T X_g  rows, groups, n, k; dW in `grad`
    adapt  Y[t] = X[t] W^T + s_a (X[t] A_a^T) B_a^T, a = ids[t] (-1: none)
                                                 rows, n, k, adapters, rank, requests
    orth   Newton-Schulz steps on a stack        count, m, n
``pad`` adds columns to the row pitch of the activations (a slice of a wider
matrix).
"""
import math

import numpy as np
import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
STEPS, COEFFICIENTS, EPS = 5, (3.4445, -4.7750, 2.0315), 1e-7


def _grouped(op, rows, groups, n, k, dtype, grad="f32", pad=0):
    c = {"op": op, "rows": rows, "groups": groups, "n": n, "k": k, "dtype": dtype, "pad": pad}
    return dict(c, grad=grad) if op == "bwd" else c


def _adapt(rows, requests, adapters, rank, n, k, dtype, pad=0):
    return {"op": "adapt", "rows": rows, "requests": requests, "adapters": adapters, "rank": rank, "n": n, "k": k,
            "dtype": dtype, "pad": pad}


def _orth(count, m, n, dtype):
    return {"op": "orth", "count": count, "m": m, "n": n, "dtype": dtype}


def listed():
    return [
        # one generated token routed to two of eight experts: what a call costs
        dict(_grouped("fwd", 2, 8, 2048, 1024, "bf16"), name="token_2of8"),
        # a decode step of 64 requests, four experts each: the weights are read once
        dict(_grouped("fwd", 256, 64, 1024, 2048, "bf16"), name="decode_256_64"),
        # a prompt batch through the experts' up projection
        dict(_grouped("fwd", 16384, 16, 4096, 2048, "bf16"), name="prompt_16384"),
        # both gradients, every size odd, a slice of a wider activation, an fp16 gradient
        dict(_grouped("bwd", 4999, 7, 1031, 777, "f16", "f16", pad=3), name="grads_odd"),
        # both gradients of a training batch, weight gradients kept in 32 bits
        dict(_grouped("bwd", 32768, 32, 2048, 4096, "bf16", "f32"), name="grads_32768"),
        # one token of one request beside a shared projection
        dict(_adapt(1, 1, 8, 16, 4096, 4096, "bf16"), name="adapter_token"),
        # a decode step: 64 requests, each with an adapter of its own choice
        dict(_adapt(64, 64, 64, 16, 4096, 4096, "bf16"), name="adapter_decode_64"),
        # a few short prompts, odd sizes, some without an adapter
        dict(_adapt(333, 9, 5, 24, 1000, 1111, "f16", pad=1), name="adapter_odd"),
        # prompts of eight requests in one batch
        dict(_adapt(4100, 8, 32, 64, 4096, 4096, "bf16"), name="adapter_prompts"),
        # a stack of small square blocks (one per head)
        dict(_orth(32, 128, 128, "bf16"), name="orth_heads"),
        # ragged tall updates kept in 32 bits
        dict(_orth(3, 1537, 515, "f32"), name="orth_tall_odd"),
        # the large weights of a layer
        dict(_orth(2, 4096, 4096, "bf16"), name="orth_4096"),
    ]


def _size(rng, lo, hi):
    """A size spread over the logarithm of [lo, hi]; half of them multiples of
    64 (as a model's widths are), the others as they come."""
    v = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 1 / 2 and v >= 64:
        v = v // 64 * 64
    return max(lo, min(hi, v))


def draw(rng):
    dtype = rng.choice(["bf16", "bf16", "f16"])
    pad = rng.choice([0, 0, 0, 8, 3])
    kind = rng.choice(["decode", "fwd", "bwd", "serve", "prompts", "orth", "orth"])
    if kind == "decode":
        return _grouped("fwd", _size(rng, 1, 512), _size(rng, 2, 64), _size(rng, 256, 4096), _size(rng, 256, 4096), dtype, pad=pad)
    if kind in ("fwd", "bwd"):
        return _grouped(kind, _size(rng, 512, 32768), _size(rng, 2, 32), _size(rng, 256, 4096), _size(rng, 256, 2048),
                        dtype, rng.choice(["f32", dtype]), pad)
    if kind == "serve":
        rows = _size(rng, 1, 256)
        return _adapt(rows, rows, _size(rng, 1, 64), rng.choice([8, 16, 24, 32, 64]), _size(rng, 512, 4096), _size(rng, 512, 4096), dtype, pad)
    if kind == "prompts":
        return _adapt(_size(rng, 257, 8192), _size(rng, 1, 32), _size(rng, 1, 32), rng.choice([8, 16, 24, 32, 64]),
                      _size(rng, 512, 4096), _size(rng, 512, 4096), dtype, pad)
    m, n = _size(rng, 64, 2048), _size(rng, 64, 2048)
    return _orth(max(1, min(32, int(_size(rng, 1 << 20, 1 << 24) // (m * n)))), m, n, rng.choice(["bf16", "f32", "f16"]))


def _normal(gen, shape, dtype, scale=1.0, pad=0):
    full = torch.empty((*shape[:-1], shape[-1] + pad), dtype=dtype, device="cuda")
    full.normal_(0.0, scale, generator=gen)
    return full[..., :shape[-1]]


def _group_sizes(case, seed):
    """Rows per group as a router gives them: some groups sought after, some
    not, and with four or more groups one that nothing chose."""
    rng = np.random.default_rng(seed)
    p = np.exp(rng.normal(0.0, 0.5, case["groups"]))
    if case["groups"] >= 4:
        p[rng.integers(case["groups"])] = 0.0
    return rng.multinomial(case["rows"], p / p.sum())


def _requests(case, seed):
    """The adapter of each row: rows of one request are neighbours, one request
    in eight has no adapter."""
    rng = np.random.default_rng(seed)
    rows, requests = case["rows"], min(case["requests"], case["rows"])
    cuts = np.sort(rng.choice(np.arange(1, rows), requests - 1, replace=False)) if requests > 1 else np.empty(0, np.int64)
    which = rng.integers(0, case["adapters"], requests)
    which[rng.random(requests) < 1 / 8] = -1
    if requests == 1:
        which[:] = seed % case["adapters"]
    return np.repeat(which, np.diff(np.concatenate([[0], cuts, [rows]]).astype(np.int64)))


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = TYPES[case["dtype"]]
    st = {"case": case}
    if case["op"] == "orth":
        # a momentum buffer: correlated rows, so the singular values spread
        count, m, n = case["count"], case["m"], case["n"]
        mix = _normal(gen, (count, m, 1), torch.float32) * _normal(gen, (count, 1, n), torch.float32)
        st["G"] = ((_normal(gen, (count, m, n), torch.float32) + 0.5 * mix) * 1e-3).to(dt)
        return st
    rows, n, k, pad = case["rows"], case["n"], case["k"], case["pad"]
    st["X"] = _normal(gen, (rows, k), dt, 1.0, pad)
    if case["op"] == "adapt":
        ids = _requests(case, seed)
        st["ids"] = torch.from_numpy(ids.astype(np.int32)).cuda()
        st["W"] = _normal(gen, (n, k), dt, k ** -0.5)
        st["A"] = _normal(gen, (case["adapters"], case["rank"], k), dt, k ** -0.5)
        st["B"] = _normal(gen, (case["adapters"], n, case["rank"]), dt, 0.25)
        st["scales"] = torch.rand((case["adapters"],), device="cuda", generator=gen) + 0.5
        return st
    sizes = _group_sizes(case, seed)
    st["largest"] = int(sizes.max())
    st["ends"] = torch.from_numpy(np.cumsum(sizes).astype(np.int32)).cuda()
    st["W"] = _normal(gen, (case["groups"], n, k), dt, k ** -0.5)
    if case["op"] == "bwd":
        st["dY"] = _normal(gen, (rows, n), dt, 1.0, pad)
    return st


def _places(ends, rows):
    """The group of each row and its place in it."""
    r = torch.arange(rows, device=ends.device)
    g = torch.searchsorted(ends.long(), r, right=True)
    starts = torch.cat([ends.new_zeros(1), ends[:-1]]).long()
    return g, r - starts[g]


def _padded(t, g, p, groups, largest):
    out = torch.zeros((groups, largest, t.shape[1]), dtype=torch.float32, device=t.device)
    out[g, p] = t.float()
    return out


def _plain(st):
    case = st["case"]
    if case["op"] == "orth":
        a, b, c = COEFFICIENTS
        X = st["G"].float()
        tall = case["m"] > case["n"]
        X = X.transpose(1, 2).contiguous() if tall else X
        X = X / (X.square().sum((1, 2), keepdim=True).sqrt() + EPS)
        for _ in range(STEPS):
            S = torch.bmm(X, X.transpose(1, 2).contiguous())
            X = a * X + torch.bmm(b * S + c * torch.bmm(S, S), X)
        return (X.transpose(1, 2) if tall else X).to(torch.bfloat16).contiguous()
    dt = TYPES[case["dtype"]]
    if case["op"] == "adapt":
        X, ids = st["X"].float(), st["ids"].long()
        L, r = case["adapters"], case["rank"]
        H = torch.matmul(X, st["A"].float().reshape(L * r, -1).t()).reshape(-1, L, r)
        named = ids[:, None] == torch.arange(L, device=ids.device)
        H = torch.where(named[:, :, None], H * st["scales"][:, None], 0.0).reshape(-1, L * r)
        Y = torch.matmul(X, st["W"].float().t())
        return (Y + torch.matmul(H, st["B"].float().transpose(1, 2).reshape(L * r, -1))).to(dt)
    g, p = _places(st["ends"], case["rows"])
    W = st["W"].float()
    if case["op"] == "fwd":
        return torch.bmm(_padded(st["X"], g, p, case["groups"], st["largest"]), W.transpose(1, 2))[g, p].to(dt)
    X = _padded(st["X"], g, p, case["groups"], st["largest"])
    dY = _padded(st["dY"], g, p, case["groups"], st["largest"])
    return {"dX": torch.bmm(dY, W)[g, p].to(dt), "dW": torch.bmm(dY.transpose(1, 2), X).to(TYPES[case["grad"]])}


def run(st):
    if not own:
        return _plain(st)
    import paper_2609_09095_amd as oz
    case = st["case"]
    if case["op"] == "orth":
        G = st["G"]
        room = torch.empty((oz.ozaki25_orthogonalise_workspace_size(*G.shape),), dtype=torch.uint8, device=G.device)
        return oz.ozaki25_orthogonalise(G, steps=STEPS, coefficients=COEFFICIENTS, eps=EPS, workspace=room)
    if case["op"] == "adapt":
        X, W, A = st["X"], st["W"], st["A"]
        room = torch.empty((oz.ozaki25_adapter_matmul_workspace_size(X.shape[0], W.shape[0], X.shape[1], A.shape[0], A.shape[1]),),
                           dtype=torch.uint8, device=X.device)
        return oz.ozaki25_adapter_matmul(X, W, st["ids"], A, st["B"], st["scales"], workspace=room)
    if case["op"] == "fwd":
        return oz.ozaki25_grouped_matmul(st["X"], st["W"], st["ends"])
    return {"dX": oz.ozaki25_grouped_matmul_dx(st["dY"], st["W"], st["ends"]),
            "dW": oz.ozaki25_grouped_matmul_dw(st["dY"], st["X"], st["ends"], out_dtype=TYPES[case["grad"]])}


def work(case):
    """Each input read and each output written once; of the weights and
    adapters those that rows reach.  The steps' symmetric products count as
    half."""
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "orth":
        s, l = sorted((case["m"], case["n"]))
        return {"bytes": case["count"] * s * l * (e + 2),
                "flops": case["count"] * STEPS * (s * (s + 1) * l + s * s * (s + 1) + 2 * s * s * l)}
    rows, n, k = case["rows"], case["n"], case["k"]
    if case["op"] == "adapt":
        r, reached = case["rank"], min(case["adapters"], case["requests"], rows)
        return {"bytes": e * (rows * (n + k) + n * k + reached * r * (n + k)), "flops": 2 * rows * (n * k + r * (n + k))}
    reached = case["groups"] * (1.0 - (1.0 - 1.0 / case["groups"]) ** rows)
    if case["op"] == "fwd":
        return {"bytes": e * (rows * (n + k) + reached * n * k), "flops": 2 * rows * n * k}
    g = 4 if case["grad"] == "f32" else 2
    return {"bytes": e * (rows * (n + 2 * k) + reached * n * k) + g * case["groups"] * n * k, "flops": 4 * rows * n * k}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "orth":
        # one matrix after another on the side of its rows or columns, whichever is shorter,
        # the polynomial by Horner's rule: a X + S (b X + c S X)
        a, b, c = COEFFICIENTS
        out = []
        for G in st["G"].double():
            X = G / (torch.linalg.vector_norm(G) + EPS)
            for _ in range(STEPS):
                if case["m"] <= case["n"]:
                    S = X @ X.t()
                    X = a * X + S @ (b * X + c * (S @ X))
                else:
                    S = X.t() @ X
                    X = a * X + (b * X + c * (X @ S)) @ S
            out.append(X)
        return torch.stack(out)
    X, W = st["X"].double(), st["W"]
    if case["op"] == "adapt":
        Y = X @ W.double().t()
        for a in range(case["adapters"]):
            at = torch.nonzero(st["ids"] == a).flatten()
            if len(at):
                Y[at] += st["scales"][a].double() * ((X[at] @ st["A"][a].double().t()) @ st["B"][a].double().t())
        return Y
    cuts = [0] + st["ends"].tolist()
    parts = list(zip(cuts[:-1], cuts[1:]))
    if case["op"] == "fwd":
        return torch.cat([X[i:j] @ W[g].double().t() for g, (i, j) in enumerate(parts)])
    dY = st["dY"].double()
    return {"dX": torch.cat([dY[i:j] @ W[g].double() for g, (i, j) in enumerate(parts)]),
            "dW": torch.stack([dY[i:j].t() @ X[i:j] for i, j in parts])}
