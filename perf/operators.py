"""Operators on rows that belong to groups (one weight matrix per expert of a mixture, per type of vertex), and on gradients.

What a pass does (`op`):

  group    rows brought into the order of their groups: offsets of the groups and the rows, the first of a group first;
           what belongs to no group comes last
  product  out = X W_g on the rows of every group g
  input    grad_X = grad_out W_g^T on the rows of every group
  weight   grad_W[g] = X^T grad_out, summed over the rows of every group
  clip     norm of all gradients together, and the gradients scaled so that it is at most max_norm

A case gives m entries, dealt to `groups` groups of uneven sizes, some of them empty (how many rows a group has depends on the
seed, as routing does).  `n`: rows of the matrices where the entries name rows through an index list, as the active
vertices of a graph do (0: the entries are the rows, one after another); `shared`: entries to a row of the input,
as a token that goes to two experts has.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
LARGEST_PRODUCT = 2 * 32_768 * 4_096 * 2_048  # operations of the largest listed case
LARGEST_CLIP = 260_000_000                    # elements


def _case(op, m, groups, f_in, f_out, dtype, n=0, shared=1):
    return {"op": op, "m": m, "groups": groups, "f_in": f_in, "f_out": f_out, "dtype": dtype, "n": n, "shared": shared}


def _clip(matrices, rows, cols, vectors, length, dtype, max_norm):
    """`matrices` gradients of rows x cols in `dtype`, `vectors` of `length` floats."""
    return {"op": "clip", "matrices": matrices, "rows": rows, "cols": cols, "vectors": vectors, "length": length,
            "dtype": dtype, "max_norm": max_norm}


def listed():
    return [
        # one decoding step's routing: 64 tokens, two of 16 experts each
        {"name": "group tokens"} | _case("group", 128, 16, 0, 0, "float32"),
        # a co-purchase graph's active vertices sorted by their type, once for every training set
        {"name": "group vertices"} | _case("group", 1_000_003, 8, 0, 0, "float32", n=2_449_029),
        # a single token served: two of eight experts, nothing but their weights to read
        {"name": "product token"} | _case("product", 2, 8, 2_048, 4_096, "bfloat16", shared=2),
        # a decoding batch: 128 tokens, two of 64 experts each, a handful of rows to an expert
        {"name": "product decode"} | _case("product", 256, 64, 2_048, 1_024, "float16", shared=2),
        # the largest: a training batch of 16,384 tokens through the experts' first matrices
        {"name": "product experts"} | _case("product", 32_768, 32, 4_096, 2_048, "bfloat16", shared=2),
        # typed vertices of a dense social graph, a class count for a width, products on the active rows
        {"name": "product vertices"} | _case("product", 153_757, 4, 16, 41, "float32", n=232_965),
        # back through the experts' matrices
        {"name": "input gradient experts"} | _case("input", 16_384, 16, 2_048, 4_096, "bfloat16"),
        # odd widths, a few uneven groups
        {"name": "input gradient odd"} | _case("input", 5_003, 7, 777, 1_001, "float16"),
        # the experts' weight gradients in 32 bits, as they are accumulated
        {"name": "weight gradient experts"} | _case("weight", 32_768, 16, 2_048, 2_048, "bfloat16", shared=2),
        # typed vertices of a social network, all their rows contracted onto small matrices
        {"name": "weight gradient vertices"} | _case("weight", 1_134_890, 5, 64, 47, "float32", n=1_134_890),
        # the gradients of a three-layer graph network: latency
        {"name": "clip small"} | _clip(3, 128, 128, 3, 128, "float32", 1.0),
        # the gradients of a mixture's experts, and vectors beside them
        {"name": "clip experts"} | _clip(30, 4_096, 2_048, 30, 2_047, "bfloat16", 1.0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi))))))


def _width(rng, lo, hi):
    w = _log(rng, lo, hi)
    return w if rng.random() < 0.3 else max(lo, w // 16 * 16) if w >= 16 else w


def draw(rng):
    op = rng.choice(("group", "product", "product", "input", "input", "weight", "weight", "clip"))
    if op == "group":
        m = _log(rng, 1, 1_000_000)
        return _case(op, m, _log(rng, 2, 256), 0, 0, "float32", n=rng.choice((0, m + _log(rng, 1, 1_000_000))))
    if op == "clip":
        rows, cols = _log(rng, 16, 4_096), _log(rng, 16, 4_096)
        most = max(1, min(40, LARGEST_CLIP // (rows * cols)))
        return _clip(rng.randint(1, most), rows, cols, rng.randint(0, 20), _log(rng, 1, 10_000), rng.choice(list(DTYPES)),
                     rng.choice((0.5, 1.0, 1e6)))
    kind = rng.choice(("vertices", "few", "many"))
    if kind == "vertices":
        m = _log(rng, 1_000, 1_000_000)
        return _case(op, m, rng.randint(1, 12), _width(rng, 3, 160), _width(rng, 3, 160), "float32", n=m + _log(rng, 1, 500_000))
    dtype = rng.choice(("bfloat16", "bfloat16", "float16", "float32"))
    shared = rng.choice((1, 2, 4))
    if kind == "few":
        return _case(op, shared * _log(rng, 1, 128), _log(rng, 4, 64), _width(rng, 500, 4_096), _width(rng, 500, 4_096), dtype, shared=shared)
    f_in, f_out = _width(rng, 256, 4_096), _width(rng, 256, 4_096)
    most = LARGEST_PRODUCT // (2 * f_in * f_out * (8 if dtype == "float32" else 1))
    return _case(op, shared * (_log(rng, 512, max(512, min(32_768, most))) // shared), _log(rng, 2, 64), f_in, f_out, dtype, shared=shared)


def _sizes(case, rng):
    """Rows of each group: uneven as routers and types are, about one group in eight without a row."""
    g = case["groups"]
    share = rng.exponential(size=g) + 0.3
    share[rng.random(g) < 0.125] = 0.0
    if not share.any():
        share[int(rng.integers(g))] = 1.0
    return rng.multinomial(case["m"], share / share.sum())


def prepare(case, seed):
    dev = torch.device("cuda", torch.cuda.current_device())
    rng = np.random.Generator(np.random.PCG64([seed & 0x7FFFFFFF, 77]))
    gen = torch.Generator(dev).manual_seed(seed & 0x7FFFFFFF)
    dtype = DTYPES[case["dtype"]]
    randn = lambda *shape: torch.randn(*shape, device=dev, generator=gen)  # noqa: E731
    s = {"op": case["op"]}
    if case["op"] == "clip":
        grads = [(randn(case["rows"], case["cols"]) * 1e-2).to(dtype) for _ in range(case["matrices"])]
        grads += [randn(case["length"]) * 1e-2 for _ in range(case["vectors"])]
        s |= {"grads": grads, "max_norm": case["max_norm"], "out": [torch.empty_like(g) for g in grads], "norm": torch.empty(1, device=dev)}
        if own:
            import paper_2204_02662_amd as epp
            s["workspace"] = torch.empty(epp.epp_gradient_norm_workspace(len(grads)), dtype=torch.uint8, device=dev)
        return s
    m, n, G = case["m"], case["n"], case["groups"]
    sizes = _sizes(case, rng)
    group = torch.from_numpy(np.repeat(np.arange(G, dtype=np.int32), sizes)).to(dev)[torch.randperm(m, device=dev, generator=gen)]
    # the entries' rows: the active vertices, ascending
    rows = torch.randperm(n, device=dev, generator=gen)[:m].sort().values.int() if n else None
    if case["op"] == "group":
        # (one entry in a hundred belongs to no group)
        group = torch.where(torch.rand(m, device=dev, generator=gen) < 0.01, -1, group).int()
        if n:
            every = torch.full((n,), -1, dtype=torch.int32, device=dev)
            every[rows.long()] = group
            group = every
        s |= {"group_of": group, "rows": rows, "groups": G, "offsets": torch.empty(G + 1, dtype=torch.int32, device=dev),
              "order": torch.empty(m, dtype=torch.int32, device=dev)}
        if own:
            import paper_2204_02662_amd as epp
            s["workspace"] = torch.empty(epp.epp_group_rows_workspace(m, G), dtype=torch.uint8, device=dev)
        return s
    order = torch.sort(group, stable=True).indices.int()
    offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int32)).to(dev)
    if n:          # matrices of all vertices, the groups' rows in both of them
        first = second = rows[order.long()]
        n_first = n_second = n
    else:          # tokens of the input, gathered; the other matrix in the groups' order
        first, second = ((order // case["shared"]).int() if case["shared"] > 1 else None), None
        n_first, n_second = (m // case["shared"] if case["shared"] > 1 else m), m
    f_in, f_out = case["f_in"], case["f_out"]
    s |= {"offsets": offsets, "sizes": sizes.tolist(), "first": first, "second": second}
    if case["op"] == "weight":
        s |= {"X": randn(n_first, f_in).to(dtype), "grad_out": (randn(n_second, f_out) * 1e-2).to(dtype),
              "grad_W": torch.empty(G, f_in, f_out, device=dev)}
        if own:
            import paper_2204_02662_amd as epp
            s["workspace"] = torch.empty(epp.epp_grouped_weight_gradient_workspace(m, G, f_in, f_out), dtype=torch.uint8, device=dev)
        return s
    s["W"] = (randn(G, f_in, f_out) / math.sqrt(f_in)).to(dtype)
    if case["op"] == "product":
        return s | {"X": randn(n_first, f_in).to(dtype), "out": torch.zeros(n_second, f_out, dtype=dtype, device=dev)}
    return s | {"X": (randn(n_first, f_out) * 1e-2).to(dtype), "out": torch.zeros(n_second, f_in, dtype=dtype, device=dev)}


def _gathered(x, rows):
    return x.float() if rows is None else x[rows.long()].float()


def _plain_group(s):
    group, rows, G = s["group_of"], s["rows"], s["groups"]
    mine = group if rows is None else group[rows.long()]
    key, at = torch.sort(torch.where((mine < 0) | (mine >= G), G, mine), stable=True)
    s["order"].copy_(at if rows is None else rows[at])
    s["offsets"].copy_(torch.searchsorted(key, torch.arange(G + 1, device=key.device, dtype=key.dtype)))
    return {"offsets": s["offsets"], "order": s["order"]}


def _plain_rows(s, transposed):
    parts = zip(_gathered(s["X"], s["first"]).split(s["sizes"]), s["W"], s["sizes"])
    y = torch.cat([x @ (w.float().T if transposed else w.float()) for x, w, size in parts if size])
    if s["second"] is None:
        s["out"].copy_(y)
    else:
        s["out"][s["second"].long()] = y
    return s["out"]


def _plain_weight(s):
    x, y = _gathered(s["X"], s["first"]).split(s["sizes"]), _gathered(s["grad_out"], s["second"]).split(s["sizes"])
    return torch.stack([a.T @ b for a, b in zip(x, y)], out=s["grad_W"])


def _plain_clip(s):
    # (a sum of squares over hundreds of millions of elements, and a bound that the norm may lie next to: 64 bits)
    norm = torch.stack([g.double().square().sum() for g in s["grads"]]).sum().sqrt()
    scale = torch.where(norm <= s["max_norm"], 1.0, s["max_norm"] / norm).float()
    return {"norm": norm.float().reshape(1), "grads": [(g.float() * scale).to(g.dtype) for g in s["grads"]]}


def _own(s):
    import paper_2204_02662_amd as epp
    if s["op"] == "group":
        epp.epp_group_rows(s["group_of"], s["groups"], s["offsets"], s["order"], s["workspace"], rows=s["rows"])
        return {"offsets": s["offsets"], "order": s["order"]}
    if s["op"] == "product":
        epp.epp_grouped_product(s["X"], s["W"], s["offsets"], s["out"], in_rows=s["first"], out_rows=s["second"])
        return s["out"]
    if s["op"] == "input":
        epp.epp_grouped_input_gradient(s["X"], s["W"], s["offsets"], s["out"], in_rows=s["first"], out_rows=s["second"])
        return s["out"]
    if s["op"] == "weight":
        epp.epp_grouped_weight_gradient(s["X"], s["grad_out"], s["offsets"], s["grad_W"], s["workspace"], x_rows=s["first"],
                                        grad_rows=s["second"])
        return s["grad_W"]
    epp.epp_clip_gradients(s["grads"], s["max_norm"], s["norm"], s["workspace"], out=s["out"])
    return {"norm": s["norm"], "grads": s["out"]}


def run(state):
    if own:
        return _own(state)
    if state["op"] == "group":
        return _plain_group(state)
    if state["op"] == "weight":
        return _plain_weight(state)
    if state["op"] == "clip":
        return _plain_clip(state)
    return _plain_rows(state, state["op"] == "input")


def work(case):
    size = 4 if case["dtype"] == "float32" else 2
    if case["op"] == "clip":
        elements, floats = case["matrices"] * case["rows"] * case["cols"], case["vectors"] * case["length"]
        return {"bytes": 2 * (elements * size + floats * 4) + 4, "flops": 3 * (elements + floats)}
    m, n, G, f_in, f_out = (case[k] for k in ("m", "n", "groups", "f_in", "f_out"))
    if case["op"] == "group":
        return {"bytes": (8 if n else 4) * m + 4 * m + 4 * (G + 1), "flops": 0}
    index = (8 * m if n else 4 * m if case["shared"] > 1 else 0) + 4 * (G + 1)
    # (an eighth of the groups has no rows, and m rows reach m groups at most; with many groups and few rows, this many)
    reached = max(1, G * 7 / 8 * (1 - math.exp(-m / (G * 7 / 8))))
    first = m // (1 if n else case["shared"])
    a, b = (f_out, f_in) if case["op"] == "input" else (f_in, f_out)
    rows = (first * a + m * b) * size
    matrices = G * f_in * f_out * 4 if case["op"] == "weight" else int(reached * f_in * f_out) * size
    return {"bytes": rows + matrices + index, "flops": 2 * m * f_in * f_out}


def exact(case, seed):
    s = prepare(case, seed)
    if s["op"] == "clip":
        total = math.fsum(float((g.double() ** 2).sum()) for g in s["grads"])
        factor = 1.0 if math.sqrt(total) <= s["max_norm"] else s["max_norm"] / math.sqrt(total)
        return {"norm": torch.tensor([math.sqrt(total)], dtype=torch.float64), "grads": [g.double() * factor for g in s["grads"]]}
    if s["op"] == "group":
        group = s["group_of"].cpu().numpy()
        rows = np.arange(group.size) if s["rows"] is None else s["rows"].cpu().numpy()
        of = [np.flatnonzero(group[rows] == g) for g in range(s["groups"])]
        rest = np.flatnonzero((group[rows] < 0) | (group[rows] >= s["groups"]))
        return {"offsets": np.cumsum([0] + [len(a) for a in of]).astype(np.int32), "order": rows[np.concatenate(of + [rest])].astype(np.int32)}
    ends = np.cumsum(s["sizes"])
    first = torch.arange(case["m"], device=s["X"].device) if s["first"] is None else s["first"].long()
    second = torch.arange(case["m"], device=s["X"].device) if s["second"] is None else s["second"].long()
    spans = [(g, int(e - c), int(e)) for g, (e, c) in enumerate(zip(ends, s["sizes"])) if c]
    if s["op"] == "weight":
        w = torch.zeros(s["grad_W"].shape, dtype=torch.float64, device=s["X"].device)
        for g, a, b in spans:
            w[g] = torch.mm(s["X"][first[a:b]].double().t().contiguous(), s["grad_out"][second[a:b]].double())
        return w
    y = torch.zeros(s["out"].shape, dtype=torch.float64, device=s["X"].device)
    for g, a, b in spans:
        w = s["W"][g].double()
        y[second[a:b]] = torch.mm(s["X"][first[a:b]].double(), w.t().contiguous() if s["op"] == "input" else w)
    return y
