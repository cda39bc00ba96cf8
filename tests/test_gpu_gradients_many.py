"""The clipping of more gradients than one launch takes."""
import pytest
import torch

import paper_2204_02662_amd as epp
from _util import dev
from test_gpu_gradients import assert_norm, assert_scaled

pytestmark = pytest.mark.gpu


def slices(count, each, seed):
    held = torch.randn(count * each, device=dev(), generator=torch.Generator(dev()).manual_seed(seed), dtype=torch.bfloat16)
    return held, list(held.split(each))


def replayed(call):
    """Milliseconds of a captured call, which the host does not hold up: the best of three."""
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    best = float("inf")
    for _ in range(4):
        begin, end = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        begin.record()
        graph.replay()
        end.record()
        torch.cuda.synchronize()
        best = min(best, begin.elapsed_time(end))
    return best


def test_the_time_of_many_gradients():
    """12,288 gradients, 128 launches of 2,016 sums each.  Clipping reads everything twice and writes it once, the norm reads it once: three times
    the traffic, and launches as long as the norm's twice.  Were all sums added again for every launch, by each of its workgroups, those
    would be 128 x 2,016 reads of 2 MB, 0.5 TB beside 13 GB of gradients."""
    n, each = 128 * 96, 21 * 8192 - 5
    held, grads = slices(n, each, 1)
    written, out = slices(n, each, 2)
    ws, norm = torch.empty(epp.epp_gradient_norm_workspace(n), dtype=torch.uint8, device=dev()), torch.empty(1, device=dev())
    norms = replayed(lambda: epp.epp_gradient_norm(grads, norm, ws))
    want = norm.clone()
    clips = replayed(lambda: epp.epp_clip_gradients(grads, 1.0, norm, ws, out=out))
    assert torch.equal(norm, want)
    total = sum(part.double().square().sum() for part in held.split(1 << 27)).sqrt().item()
    assert_norm(norm, total)
    for part, got in zip(held.split(1 << 27), written.split(1 << 27)):
        assert_scaled(got, part, total, 1.0)
    assert clips <= 8 * norms, (clips, norms)
