"""The operators on groups and on gradients as a training step uses them: a graph network whose vertices have types, eagerly and from a HIP
graph; experts with two choices to a token; two streams at once; what the calls allocate."""
import numpy as np
import pytest
import torch

import graphgen
import paper_2204_02662_amd as epp
from _grouped import TYPES, assert_sums, offsets_of, product, randn, weight_gradient
from _util import dev, gpu_prepare

pytestmark = pytest.mark.gpu


class TypedLayers:
    """Backward pass of L layers with a weight matrix per type of vertex: Y' = X' W[type]^T and W'[type] on the active rows, aggregation,
    and the weights' gradients clipped.  Everything that a step needs is there before it."""

    def __init__(self, G=3, widths=(24, 41, 16)):
        self.g = graphgen.random_graph("rmat", 3_000, seed=5, raw_draws=30_000)
        train = graphgen.training_set(self.g.n, 150, 6)
        self.L, self.G, n = len(widths) - 1, G, self.g.n
        self.paths = gpu_prepare(self.g, train, self.L)
        self.types = torch.from_numpy(np.random.default_rng(7).integers(0, G, size=n).astype(np.int32)).to(dev())
        self.layers, self.norm = [], torch.zeros(1, device=dev())
        for l in range(self.L):
            rows = self.paths.active_set(self.L - l - 1)
            Fi, Fo, m = widths[l], widths[l + 1], rows.numel()
            self.paths.path(l).prepare_width(Fi)
            self.layers.append(dict(
                rows=rows, W=torch.empty(G, Fi, Fo, device=dev()), Y=torch.empty(n, Fi, device=dev()), grad_Y=torch.zeros(n, Fi, device=dev()),
                grad_X=torch.zeros(n, Fi, device=dev()), grad_W=torch.empty(G, Fi, Fo, device=dev()), clipped=torch.empty(G, Fi, Fo, device=dev()),
                offsets=torch.empty(G + 1, dtype=torch.int32, device=dev()), order=torch.empty(m, dtype=torch.int32, device=dev()),
                ws1=torch.empty(epp.epp_group_rows_workspace(m, G), dtype=torch.uint8, device=dev()),
                ws2=torch.empty(epp.epp_grouped_weight_gradient_workspace(m, G, Fi, Fo), dtype=torch.uint8, device=dev())))
        self.X = torch.zeros(n, widths[-1], device=dev())
        self.ws = torch.empty(epp.epp_gradient_norm_workspace(self.L), dtype=torch.uint8, device=dev())

    def fill(self, seed):
        for l, a in enumerate(self.layers):
            a["W"].copy_(randn(*a["W"].shape, seed=seed + l))
            a["Y"].copy_(randn(*a["Y"].shape, seed=seed + 10 + l))
        rows = self.layers[-1]["rows"].long()
        self.X[rows] = randn(rows.numel(), self.X.shape[1], seed=seed + 20)
        self.types.copy_(torch.from_numpy(np.random.default_rng(seed).integers(0, self.G, size=self.g.n).astype(np.int32)))

    def step(self):
        for l in range(self.L - 1, -1, -1):
            a, grad = self.layers[l], self.layers[l + 1]["grad_X"] if l + 1 < self.L else self.X
            epp.epp_group_rows(self.types, self.G, a["offsets"], a["order"], a["ws1"], rows=a["rows"])
            epp.epp_grouped_weight_gradient(a["Y"], grad, a["offsets"], a["grad_W"], a["ws2"], x_rows=a["order"], grad_rows=a["order"])
            epp.epp_grouped_input_gradient(grad, a["W"], a["offsets"], a["grad_Y"], in_rows=a["order"], out_rows=a["order"])
            epp.epp_backward_aggregate(self.paths.path(l), a["grad_Y"], a["grad_X"])
        epp.epp_clip_gradients([a["grad_W"] for a in self.layers], 0.5, self.norm, self.ws, out=[a["clipped"] for a in self.layers])

    def check(self):
        M = torch.zeros(self.g.n, self.g.n, dtype=torch.float64)
        row = np.repeat(np.arange(self.g.n), np.diff(self.g.rowptr))
        M[torch.from_numpy(row), torch.from_numpy(self.g.col).long()] = torch.from_numpy(self.g.val).double()
        grad, types, total = self.X.double().cpu(), self.types.long().cpu(), 0.0
        wants = []
        for l in range(self.L - 1, -1, -1):
            a = self.layers[l]
            rows = a["rows"].long().cpu()
            Y, W, want_W = a["Y"].double().cpu(), a["W"].double().cpu(), torch.zeros(a["W"].shape, dtype=torch.float64)
            grad_Y = torch.zeros(self.g.n, W.shape[1], dtype=torch.float64)
            for g in range(self.G):
                r = rows[types[rows] == g]
                want_W[g] = Y[r].T @ grad[r]
                grad_Y[r] = grad[r] @ W[g].T
            wants.append((a, want_W))
            total += want_W.square().sum().item()
            grad = M @ grad_Y
            keep = torch.zeros(self.g.n, dtype=torch.bool)
            keep[self.paths.path(l).export()[0].long().cpu()] = True
            grad[~keep] = 0.0
        norm = total ** 0.5
        assert abs(self.norm.item() - norm) <= 1e-5 * norm
        for a, want in wants:
            size = want.abs().max().item()
            # (sums of up to 3,000 products of sums over two layers: 1e-5 of the largest, as the aggregation's own tests allow)
            assert (a["grad_W"].double().cpu() - want).abs().max().item() <= 1e-5 * size
            assert (a["clipped"].double().cpu() - want * min(1.0, 0.5 / norm)).abs().max().item() <= 2e-5 * size * min(1.0, 0.5 / norm)
        first = self.layers[0]["grad_X"].double().cpu()
        assert (first - grad).abs().max().item() <= 1e-5 * grad.abs().max().item()


def test_typed_layers_eager_and_captured():
    t = TypedLayers()
    t.fill(100)
    t.step()
    torch.cuda.synchronize()
    t.check()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        t.step()
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t.step()
    for seed in (200, 300, 400):
        t.fill(seed)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for a in t.layers for x in (a["grad_W"], a["clipped"], a["grad_X"], a["order"], a["offsets"])] + [t.norm.clone()]
        t.check()
        t.step()  # eager work in between, and bit for bit the same
        torch.cuda.synchronize()
        for x, y in zip(got, [x for a in t.layers for x in (a["grad_W"], a["clipped"], a["grad_X"], a["order"], a["offsets"])] + [t.norm]):
            assert torch.equal(x, y)


@pytest.mark.parametrize("dtype", TYPES)
def test_experts_with_two_choices(dtype):
    """Tokens to two experts each, one of them to none: gather, product, product back to the slots, and the gradients."""
    tokens, choices, G, F, H = 50, 2, 6, 40, 72
    m = tokens * choices
    chosen = torch.stack([torch.randperm(G, generator=torch.Generator().manual_seed(i))[:choices] for i in range(tokens)]).int()
    chosen[7, 1] = -1
    chosen = chosen.reshape(-1).to(dev())
    offsets, order = torch.empty(G + 1, dtype=torch.int32, device=dev()), torch.empty(m, dtype=torch.int32, device=dev())
    epp.epp_group_rows(chosen, G, offsets, order, torch.empty(epp.epp_group_rows_workspace(m, G), dtype=torch.uint8, device=dev()))
    assert offsets[G].item() == m - 1 and order[-1].item() == 15
    token = order // choices
    x, W1, W2 = randn(tokens, F, seed=1, dtype=dtype), randn(G, F, H, seed=2, dtype=dtype), randn(G, H, F, seed=3, dtype=dtype)
    hidden, slots = torch.zeros(m, H, dtype=dtype, device=dev()), torch.zeros(m, F, dtype=dtype, device=dev())
    epp.epp_grouped_product(x, W1, offsets, hidden, in_rows=token)
    want, size, terms = product(x, W1, offsets, m, token)
    assert_sums(hidden[:m - 1], want[:m - 1], size[:m - 1], terms)
    epp.epp_grouped_product(hidden, W2, offsets, slots, out_rows=order)
    want, size, terms = product(hidden, W2, offsets, m)
    assert_sums(slots[order[:m - 1].long()], want[:m - 1], size[:m - 1], terms)
    assert (slots[15] == 0).all() and (hidden[m - 1] == 0).all()
    d = randn(m, F, seed=4, dtype=dtype)  # gradient of the slots
    grad_hidden, grad_W2 = torch.zeros_like(hidden), torch.empty(G, H, F, device=dev())
    epp.epp_grouped_input_gradient(d, W2, offsets, grad_hidden, in_rows=order)
    want, size, terms = product(d, W2, offsets, m, order, transposed=True)
    assert_sums(grad_hidden[:m - 1], want[:m - 1], size[:m - 1], terms)
    ws = torch.empty(epp.epp_grouped_weight_gradient_workspace(m, G, H, F), dtype=torch.uint8, device=dev())
    epp.epp_grouped_weight_gradient(hidden, d, offsets, grad_W2, ws, grad_rows=order)
    want, size, terms = weight_gradient(hidden, d, offsets, m, None, order)
    assert_sums(grad_W2, want, size, terms + 8)


def test_two_streams_at_once():
    """Calls on two streams, each with memory of its own."""
    def make(seed):
        sizes = [700, 0, 900, 400]
        m, offsets = sum(sizes), offsets_of(sizes)
        x, W, d = randn(m, 264, seed=seed, dtype=torch.bfloat16), randn(4, 264, 136, seed=seed + 1, dtype=torch.bfloat16), randn(m, 136, seed=seed + 2, dtype=torch.bfloat16)
        return dict(x=x, W=W, d=d, offsets=offsets, y=torch.empty_like(d), dx=torch.empty_like(x), dW=torch.empty(4, 264, 136, device=dev()),
                    out=torch.empty(4, 264, 136, device=dev()), norm=torch.empty(1, device=dev()),
                    ws=torch.empty(epp.epp_grouped_weight_gradient_workspace(m, 4, 264, 136), dtype=torch.uint8, device=dev()),
                    ws2=torch.empty(epp.epp_gradient_norm_workspace(1), dtype=torch.uint8, device=dev()))

    def run(s):
        epp.epp_grouped_product(s["x"], s["W"], s["offsets"], s["y"])
        epp.epp_grouped_input_gradient(s["d"], s["W"], s["offsets"], s["dx"])
        epp.epp_grouped_weight_gradient(s["x"], s["d"], s["offsets"], s["dW"], s["ws"])
        epp.epp_clip_gradients([s["dW"]], 1.0, s["norm"], s["ws2"], out=[s["out"]])
    both = [make(31), make(41)]
    alone = []
    for s in both:
        run(s)
        torch.cuda.synchronize()
        alone.append([s[k].clone() for k in ("y", "dx", "dW", "out", "norm")])
        for k in ("y", "dx", "dW", "out", "norm"):
            s[k].zero_()
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in both]
    for _ in range(5):
        for s, stream in zip(both, streams):
            with torch.cuda.stream(stream):
                run(s)
    torch.cuda.synchronize()
    for s, want in zip(both, alone):
        for k, w in zip(("y", "dx", "dW", "out", "norm"), want):
            assert torch.equal(s[k], w), k


def test_nothing_is_allocated():
    t = TypedLayers()
    t.fill(1)
    t.step()
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated(), torch.cuda.mem_get_info()[0], epp.alloc_stats["allocs"]
    t.step()
    torch.cuda.synchronize()
    assert (torch.cuda.memory_allocated(), torch.cuda.mem_get_info()[0], epp.alloc_stats["allocs"]) == before
