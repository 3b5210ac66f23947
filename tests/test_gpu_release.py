"""Requests of a paged cache that end, on the GPU: recorded releases among forks; every cached row compared bit for bit after each step."""
import pytest
import torch

from test_gpu_sampled_decoding import D, HKV, LAYERS, Server, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("request_of", [lambda: 0, lambda: slice(0, 1), lambda: torch.tensor([True, False, False, False], device="cuda")])
def test_a_release_recorded_before_the_first_fork(request_of):
    """Replayed when requests share pages, with the program's own steps between the replays."""
    s = Server(6, 4, 100, 16, 512)
    s.new_tokens([40, 0, 20, 33])
    first = request_of()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.cache.release(first)
    for sources in ([0, 0, 2, 3], [1, 1, 2, 2], [3, 1, 1, 3]):
        s.fork(sources)
        s.check()
        graph.replay()
        torch.cuda.synchronize()
        s.rows[0] = []
        s.check()
        s.new_tokens([20, 0, 1, 0])
        s.check()
        s.new_tokens([70, 5, 0, 1])
        s.check()


@pytest.mark.parametrize("when", ["before the rows are written", "between the layers", "after them", "recorded"])
def test_a_release_in_a_planned_step(when):
    """The others' rows, in pages that the plan gave them, are kept; the request's are not, and its pages are free but for what others share."""
    s = Server(7, 4, 60, 16, 512)
    c = s.cache
    s.new_tokens([100, 37, 20, 16])
    s.fork([0, 0, 2, 3])
    release, graph = (lambda: c.release(1)), torch.cuda.CUDAGraph()
    if when == "recorded":
        torch.cuda.synchronize()
        with torch.cuda.graph(graph):
            c.release(1)
        release = graph.replay
    for _ in range(3):
        news = [40, 30, 0, 9]
        t = sum(news)
        c.plan(ints(news), t)
        q, k, v = s.values(t, 4, D), s.values(t, HKV, D), s.values(t, HKV, D)
        for layer in range(LAYERS):
            if layer == {"before the rows are written": 0, "between the layers": 1}.get(when):
                release()
            c.write(layer, q, k, v, s.cos_sin, torch.empty_like(q))
        if when in ("after them", "recorded"):
            release()
        out, lse = torch.empty_like(q), torch.empty((t, 4), device="cuda")
        c.attend(0, q, out, lse, 40, 300)
        assert (out[40:70] == 0).all() and (lse[40:70] == -torch.inf).all() and lse[:40].isfinite().all() and lse[70:].isfinite().all()
        c.keep_new()
        assert c.err.tolist() == [0, 1, 0, 0]
        s.rows[1] = []
        for b, at in ((0, 0), (3, 70)):
            s.rows[b] = s.rows[b] + [(k[at + i].clone(), v[at + i].clone()) for i in range(news[b])]
        s.check()
        assert c.pages_held[1].item() == 0
        s.fork([0, 2, 2, 3])
        s.check()
