"""Tensors of sampled decoding that are not on the device of the others: refused before anything is launched."""
import pytest
import torch

from paper_2502_17421_amd import binding as ls
from test_gpu_tree_sample import Case

pytestmark = pytest.mark.gpu


def test_acceptance_refuses_tensors_of_the_host():
    c = Case(1, 3, 5, 501)
    c.run()
    for at in [i for i, x in enumerate(c.args[:-1]) if isinstance(x, torch.Tensor)]:
        args = list(c.args)
        args[at] = args[at].cpu()
        with pytest.raises(ValueError):
            ls.ls_tree_accept_sampled(*args)
    c.run()
    c.check()
