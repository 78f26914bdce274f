"""The attention cache in 8 bits at the ends of its range."""
import numpy as np
import pytest

from tests.test_gpu_kv import Pair, starts_of

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


@pytest.mark.parametrize("fill", [float("inf"), 3e38, float("nan"), 0.0])
@pytest.mark.parametrize("n,max_new", [(130, 130), (65, 64)])
def test_a_page_that_is_not_there_reaches_only_who_sees_it(n, max_new, fill):
    """As a prompt and as rows that are split (65 tokens of which 64 are asked for): rows before the page that is not there share a tile with rows that see it,
    and page 0, which nothing has been written to, holds anything."""
    torch = _torch()
    for dtype in ("bf16", "f32"):
        p = Pair(1, 1, 64, 5, dtype, seed=n)
        p.kv.page_table.copy_(torch.tensor([[5, 3, 7, 1, 2]], dtype=torch.int32))
        p.append([127])
        p.append([n])
        scales = p.kv.scales.view(p.kv.n_pages, 1, 2)
        scales[0] = fill
        p.kv.page_table[0, 2] = -1                          # tokens 128..191
        k, v, _ = p.ref[0].pages[2]
        p.ref[0].pages[2] = (k, v, np.ones(1, bool))
        q = p.rand(n, 1)
        out, lse = torch.full((n, 1, 64), 7.0, dtype=p.dt, device="cuda"), torch.full((n, 1), 7.0, device="cuda")
        ws = p.b.alloc_kv_workspace(p.kv, 1, n, max_new, 127 + n)
        p.b.slicer_kv_attend(p.kv, q.cuda(), starts_of([n]), max_new, 127 + n, 0.125, out, ws, lse=lse)
        torch.cuda.synchronize()
        seen = torch.isnan(out).view(n, 64)
        assert not seen[0].any() and seen[1:max_new].all()  # the first query's own token is the last one before the page
        p.check([n], q, 0.125, torch.cat([out[:max_new].cpu(), torch.full((n - max_new, 1, 64), float("nan"), dtype=p.dt)]),
                torch.cat([lse[:max_new].cpu(), torch.full((n - max_new, 1), float("nan"))]))
