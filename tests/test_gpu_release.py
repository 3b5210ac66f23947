"""Requests of a paged cache that end, on the GPU: recorded releases among forks; every cached row compared bit for bit after each step."""
import pytest
import torch

from test_gpu_sampled_decoding import Server

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
