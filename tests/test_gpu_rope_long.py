"""Rotary positions of more tokens than one launch takes."""
import numpy as np
import pytest
import torch

from paper_2502_17421_amd import binding as ls
from test_gpu_rope import close, expected, table

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("d", [64, 128])
def test_tokens_of_three_launches(d):
    """One query head, in place; all rows turned, and those around the ends of the launches and of the tokens as they have to be."""
    t = (1 << 24) + 5
    q = torch.randn((64, 1, d), generator=torch.Generator().manual_seed(7)).bfloat16()
    rows = q.cuda().repeat(-(-t // 64), 1, 1)[:t]
    cos_sin = table(50, d // 2)
    cs, pos = torch.from_numpy(cos_sin).cuda(), (torch.arange(t, dtype=torch.int32, device="cuda") * 7 % 49 + 1)[None]
    ls.ls_rope(ls.make_rope_desc(rows, None, None, rows, None, None, None, pos, cs), rows, None, pos, cs, rows, None)
    places = np.concatenate([np.arange(a - 70, a + 70) for a in (1 << 22, 1 << 23, 1 << 24)] + [np.arange(70), np.arange(t - 70, t)])
    at = torch.from_numpy(places[places < t])
    want = expected(q[at % 64], pos[:, at].cpu().numpy(), cos_sin, [d // 2], False, "bf16")
    close(rows[at.cuda()], *want, "q")
    turned = 0
    for part, start in zip(rows.split(1 << 21), range(0, t, 1 << 21)):  # (64 is a divisor of a part)
        was = q.cuda().repeat(-(-part.shape[0] // 64), 1, 1)[:part.shape[0]]
        turned += int((part != was).any(2).sum())
    assert turned == t
