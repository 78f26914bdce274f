"""The attention cache in 8 bits at the padded head sizes 160, 192 and 224, each as steps, drafts and prompts, whose kernels are instantiations of their own."""
import numpy as np
import pytest

from tests.kv_ref import PAGE
from tests.test_gpu_kv import Pair, starts_of

pytestmark = pytest.mark.gpu

DIMS = [136, 160, 168, 176, 192, 200, 224]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", DIMS)
def test_append_then_read(dim, dtype):
    import torch
    p = Pair(3, 2, dim, 5, dtype, seed=dim)
    for counts in ([1, 0, 63], [62, 65, 1], [1, 130, 64], [70, 3, 1]):
        p.append(counts)
    lens = [len(r) for r in p.ref]
    for dt in (torch.float32, torch.bfloat16):
        k = torch.full((sum(lens) + 3, 2, dim), 7.0, dtype=dt, device="cuda")
        v = torch.full_like(k, 7.0)
        p.b.slicer_kv_read(p.kv, starts_of(lens), max(lens), k, v)
        for which, got in ((0, k), (1, v)):
            assert torch.equal(got[: sum(lens)].cpu(), torch.tensor(np.concatenate([r.values()[which] for r in p.ref])).float().to(dt))
            assert (got[sum(lens):] == 7.0).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("past,new", [([300, 130, 64], [1, 3, 1]),             # steps: up to 12 rows
                                      ([500, 31], [9, 16]),                    # up to 64 rows
                                      ([0, 200, 700], [150, 210, 1]),          # prompts, several pages and a tail, and a single token
                                      ([640, 64], [130, 192])])                # prompts, whole pages
@pytest.mark.parametrize("dim", DIMS)
def test_attend(dim, past, new, dtype):
    import torch
    p = Pair(len(past), 2, dim, max(-(-(a + n) // PAGE) for a, n in zip(past, new)) + 1, dtype, seed=dim + len(past))
    p.append(past)
    p.append(new)
    q = p.rand(sum(new), 8)
    # the cache shared out over workgroups where there are few tiles, and not; all tokens and those up to the query's own
    for max_len, causal in ((None, True), (0, True), (0, False)):
        mass = torch.rand(len(past), 2, p.kv.max_pages, device="cuda")
        old = mass.clone()
        out, lse = p.attend(new, q.cuda(), dim ** -0.5, causal, mass, decay=0.5, max_len=max_len)
        p.check(new, q, dim ** -0.5, out, lse, causal, mass, old, 0.5)
