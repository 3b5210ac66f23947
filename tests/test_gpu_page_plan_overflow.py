"""More tokens than the arrays of slots and positions have room for."""
import numpy as np
import pytest
import torch

from paper_2502_17421_amd import binding as ls
from test_gpu_page_plan import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("repeat", [1, 100])
def test_requests_without_tokens_are_not_concerned(repeat):
    """Behind a request whose tokens do not fit, a request that has ended gives its pages back, one that is idle keeps its state, one
    that holds more than it needs gives back the rest; one with tokens is refused, as is one whose lengths are impossible."""
    kv = np.array([4, 0, 20, 9, 3, 0, 90], np.int32)
    new = np.array([8, 0, 0, 0, 1, 0, 0], np.int32)
    held = np.array([1, 2, 2, 3, 1, 0, 5], np.int32)
    kv, new, held = (np.tile(x, repeat) for x in (kv, new, held))
    n, page_size, width = len(kv), 16, 6
    table = np.full((n, width), -1, np.int32)
    order = np.random.default_rng(1).permutation(held.sum() + 4).astype(np.int32)
    at = 0
    for b in range(n):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    free = np.full(len(order), -1, np.int32)
    free[:4] = order[at:]
    args = [dev(x) for x in (kv, new, held, table, free, [4])]
    outs = [torch.full((m,), -99, dtype=torch.int32, device="cuda") for m in (n, 1, n + 1, n, 5, 5, n)]
    ls.ls_page_plan(ls.make_page_desc(args[3], 5, page_size, len(order)), *args, *outs)
    new_held, free_count, cu, total, slots, positions, err = (x.cpu().numpy() for x in outs)
    np.testing.assert_array_equal(err, np.tile([2, 0, 0, 0, 2, 0, 2], repeat))
    np.testing.assert_array_equal(new_held, np.tile([1, 0, 2, 1, 1, 0, 5], repeat))
    np.testing.assert_array_equal(total, np.tile([0, 0, 20, 9, 0, 0, 0], repeat))
    np.testing.assert_array_equal(cu, np.concatenate([[0], np.cumsum(new)]))
    back = np.concatenate([table[b, new_held[b]:held[b]] for b in range(n)])  # request after request, in order of the table
    assert free_count[0] == 4 + 4 * repeat
    np.testing.assert_array_equal(args[4].cpu().numpy()[:free_count[0]], np.concatenate([order[at:], back]))
    np.testing.assert_array_equal(args[3].cpu().numpy(), table)
    assert slots.tolist() == [-1] * 5 and positions.tolist() == [4, 5, 6, 7, 8]
