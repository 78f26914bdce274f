"""Lengths of the attention cache that are taken back, as after drafted tokens that were refused: within the open page, to whole pages, and over a page's end
with a copy of the tail.  What the cache then holds is compared bit for bit with a sequence that never had the other tokens."""
import numpy as np
import pytest

from tests.kv_ref import PAGE
from tests.test_gpu_kv import Pair, starts_of

pytestmark = pytest.mark.gpu


def shorten(p, i, length):
    """Sequence i, in the definition, back to `length` tokens."""
    r = p.ref[i]
    pages = length // PAGE
    if pages < len(r.pages):
        assert length % PAGE == 0
        r.open = []
    r.pages, r.open = r.pages[:pages], r.open[: length - pages * PAGE]
    assert len(r) == length
    p.sync_lens()


def check_held(p):
    import torch
    lens = [len(r) for r in p.ref]
    k = torch.empty(sum(lens), p.kv.kv_heads, p.kv.head_dim, device="cuda")
    v = torch.empty_like(k)
    p.b.slicer_kv_read(p.kv, starts_of(lens), max(lens), k, v)
    for which, got in ((0, k), (1, v)):
        assert torch.equal(got.cpu(), torch.tensor(np.concatenate([r.values()[which] for r in p.ref])).float())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("before,drafts,length", [(10, 4, 11), (10, 4, 10), (64, 5, 64), (64, 5, 66), (100, 27, 101), (130, 0, 128), (130, 3, 64), (200, 1, 0), (62, 4, 64), (62, 4, 65)])
def test_within_the_open_page_and_to_whole_pages(before, drafts, length, dtype):
    p = Pair(2, 2, 72, 5, dtype, seed=before + drafts)
    p.append([before, 33])
    p.append([drafts, 1])
    shorten(p, 0, length)
    check_held(p)
    for new in ([1, 2], [70, 40]):
        p.append(new)
        check_held(p)
        q = p.rand(sum(new), 4)
        out, lse = p.attend(new, q.cuda(), 0.125)
        p.check(new, q, 0.125, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("before", [61, 62, 63, 127])
@pytest.mark.parametrize("stay", [0, 1, 2, 3, 4])
def test_over_a_pages_end_with_a_copy_of_the_tail(stay, before, dtype):
    p = Pair(2, 2, 40, 5, dtype, seed=before)
    p.append([5, before])
    saved = [(list(r.pages), list(r.open)) for r in p.ref]
    tail = p.kv.tails.view(2, -1)[1].clone()
    k, v = p.rand(6, 2), p.rand(6, 2)                       # two tokens of the first sequence, four drafted ones of the second
    p.append([2, 4], k, v)
    q = p.rand(6, 4)
    out, lse = p.attend([2, 4], q.cuda(), 0.2)
    p.check([2, 4], q, 0.2, out, lse)
    p.kv.tails.view(2, -1)[1] = tail
    p.ref[1].pages, p.ref[1].open = saved[1]
    p.append([0, stay], k[2: 2 + stay], v[2: 2 + stay])
    check_held(p)
    for new in ([1, 1], [3, 66]):
        p.append(new)
        check_held(p)
