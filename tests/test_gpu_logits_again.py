"""Calls of the operators behind the classifier that overwrite what they read, and graphs that run them again."""
import numpy as np
import pytest
import torch

from paper_1805_12549_amd import binding as B

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.int8), b.contiguous().view(torch.int8))


def inputs(rows, classes, top, dtype):
    rng = np.random.default_rng(rows + classes)
    z = torch.from_numpy((2.5 * rng.standard_normal((rows, classes))).astype(np.float32)).cuda().to(TYPES[dtype])
    ids = rng.integers(0, classes, (rows, top))
    ids[rng.random((rows, top)) < 0.2] = -1
    if top > 1:
        ids[:, 1] = ids[:, 0]
    t = rng.standard_normal((rows, top)).astype(np.float32)
    labels = rng.integers(-1, classes, rows)
    return z, [torch.from_numpy(a).cuda() for a in (ids, t, labels)], torch.from_numpy(rng.standard_normal(rows).astype(np.float32)).cuda()


@pytest.mark.parametrize("temperature", [1.0, 2.0])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("rows,classes,top", [(1, 1, 1), (5, 1000, 17), (70, 4099, 128), (600, 777, 16), (3, 50003, 128), (1, 200003, 64), (300, 70001, 33),
                                              (512, 40000, 20)])
def test_backward_in_place_of_the_logits(rows, classes, top, dtype, temperature):
    """A row's parts overwrite their logits while others still ask for the teacher's classes: each uses those of its own part only."""
    z, teacher, up = inputs(rows, classes, top, dtype)
    kw = dict(teacher_weight=0.5, label_weight=0.5, temperature=temperature)
    _, stats, _ = B.distill(z, *teacher, **kw)
    want = B.distill_backward(z, stats, *teacher, grad_loss=up, **kw)
    for _ in range(3):
        again = z.clone()
        assert B.distill_backward(again, stats, *teacher, grad_loss=up, grad=again, **kw) is again
        assert same_bits(again, want)


@pytest.mark.parametrize("rows,classes", [(3, 1000), (4, 90001), (600, 5000)])
def test_replays_rewrite_every_output(rows, classes):
    """Two graphs, each on a stream of its own that waits for what overwrote its outputs; eager work of the same inputs between the replays."""
    z, (ids, t, labels), up = inputs(rows, classes, 20, "bf16")
    kw = dict(teacher_weight=0.5, label_weight=0.5, temperature=2.0)

    def all_of_them():
        first = B.logprobs(z, labels, top=20)
        second = B.distill(z, ids, t, labels, grad=True, grad_loss=up, **kw)
        return [*first, *second, B.distill_backward(z, second[1], ids, t, labels, grad_loss=up, **kw)]

    def same(got, want):
        return all(same_bits(g, w) for g, w in zip(got, want))

    want = all_of_them()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            all_of_them()
            torch.cuda.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                out = all_of_them()
        torch.cuda.synchronize()
        graphs.append((side, graph, out))
    for again in range(3):
        for side, graph, out in graphs:
            for o in out:
                o.view(torch.int8).fill_(again)
        for side, graph, out in graphs:        # (both on their way at once)
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                graph.replay()
        eager = all_of_them()
        torch.cuda.synchronize()
        assert same(eager, want) and all(same(out, want) for _, _, out in graphs)
