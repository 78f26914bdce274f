"""slicer_kv_*, calls that need no GPU: refusals of scales that fp32 does not hold, workspace sizes of calls made at the same time."""
import ctypes as C

import pytest
import torch

from tests.test_kv_cpu import attend, handle, lib  # noqa: F401 (a fixture)


@pytest.mark.parametrize("scale", [3e38, -3e38, 1e39, 1e300, -1e300])
def test_scales_beyond_fp32_are_refused(lib, scale):  # noqa: F811
    """3e38 is finite in fp32, and times log2(e) it is not."""
    assert attend(lib, handle(), scale=scale) == -1


class Turn(int):
    """A number that hands the turn to another thread's call while it is compared."""
    other = None

    def __eq__(self, x):
        if Turn.other:
            call, Turn.other = Turn.other, None
            call()
        return int(self) == int(x)

    def __ne__(self, x):
        return not self == x

    __hash__ = int.__hash__


def test_workspace_sizes_of_two_calls_at_once(lib):  # noqa: F811
    """The size that a call checks its workspace against is that of its own shape, whatever another call on the same cache does between its steps."""
    from paper_2511_11608_amd import binding
    kv, c = binding.alloc_kv(2, 4, 64, 16, 8, device="cpu"), handle()
    small, large = (8, 2, 1, 100, 0), (8, 4000, 2000, 512, 1)
    want = [binding.KvCache.workspace_bytes(binding.alloc_kv(2, 4, 64, 16, 8, device="cpu"), c, *shape) for shape in (small, large)]
    assert 0 < want[0] < want[1]
    for mine, others, size in ((large, small, want[1]), (small, large, want[0])):
        shape = tuple(Turn(x) for x in mine)
        assert kv.workspace_bytes(c, *shape) == size
        Turn.other = lambda: kv.workspace_bytes(c, *others)
        assert kv.workspace_bytes(c, *(Turn(x) for x in mine)) == size
        assert Turn.other is None
    # and of another handle of the same cache
    assert kv.workspace_bytes(handle(seqs=200), *large) > want[1] and kv.workspace_bytes(c, *large) == want[1]


def test_caches_of_more_bytes_than_a_size_holds_are_refused(lib):  # noqa: F811
    n = C.c_size_t(7)
    for kw in (dict(n_pages=(1 << 31) - 1, seqs=1, kv_heads=1 << 20, head_dim=256), dict(n_pages=1 << 30, seqs=1, kv_heads=1 << 21, head_dim=128)):
        kv = handle(**kw)
        assert lib.slicer_kv_sizes(C.byref(kv), C.byref(n), None, None) == -1 and n.value == 7
        assert attend(lib, kv, heads=kv.kv_heads) == -1
    kv = handle(n_pages=1 << 30, seqs=1, kv_heads=1 << 16, head_dim=128)
    assert lib.slicer_kv_sizes(C.byref(kv), C.byref(n), None, None) == 0 and n.value == 1 << 60


def test_a_workspace_of_no_bytes_may_be_null(lib):  # noqa: F811
    """Prompts of the same length without weights, more than the chip has places for, need none; whether they can be launched is another matter here."""
    kv, n = handle(seqs=64, kv_heads=8, max_pages=32), C.c_size_t(7)
    assert lib.slicer_kv_attend_sizes(C.byref(kv), 32, 64 * 512, 512, 512, 0, C.byref(n)) == 0 and n.value == 0
    assert lib.slicer_kv_attend_sizes(C.byref(kv), 32, 64 * 512, 512, 512, 1, C.byref(n)) == 0 and n.value > 0
    call = dict(heads=32, tokens=64 * 512, max_new=512, max_len=512, ws=None)
    assert attend(lib, kv, mass=256, **call) == -1
    if not torch.cuda.is_available():                       # (the handle's pointers lead nowhere)
        assert attend(lib, kv, **call) == -3
