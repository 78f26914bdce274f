"""slicer_kv_*: what needs no GPU -- sizes in closed form, refusals before anything is launched, the binding's checks, and the
definition in tests/kv_ref.py against hand-worked numbers."""
import ctypes as C
import os

import numpy as np
import pytest

from tests import kv_ref


@pytest.fixture(scope="module")
def lib():
    from paper_2511_11608_amd import binding
    if not os.path.exists(binding.LIB_PATH):
        from paper_2511_11608_amd import build
        build.build()
    return binding.load()


def handle(**kw):
    from paper_2511_11608_amd import binding
    a = dict(pages=256, scales=256, tails=256, page_table=256, lens=256, seqs=2, kv_heads=4, head_dim=64, max_pages=8, n_pages=16)   # never followed
    a.update(kw)
    return binding.SlicerKv(**a)


def attend(lib, kv, q=256, dt=1, heads=8, tokens=2, starts=256, max_new=1, max_len=100, scale=0.1, out=256, mass=None, decay=0.0, ws=256):
    return lib.slicer_kv_attend(C.byref(kv) if kv else None, q, dt, heads, tokens, starts, max_new, max_len, 8 * 64, 64, scale, 1, out, None, mass, decay, ws, None)


def append(lib, kv, k=256, v=256, dt=1, tokens=2, starts=256, max_new=1):
    return lib.slicer_kv_append(C.byref(kv) if kv else None, k, v, dt, tokens, starts, max_new, 256, 64, 256, 64, None)


def read(lib, kv, k=256, v=256, dt=1, tokens=2, starts=256, max_new=1):
    return lib.slicer_kv_read(C.byref(kv) if kv else None, k, v, dt, tokens, starts, max_new, None)


def evict(lib, kv, mass=256, keep=4, sink=1, recent=1, outs=(256, 256, 256, 256, 256), ws=256):
    return lib.slicer_kv_evict(C.byref(kv) if kv else None, mass, keep, sink, recent, *outs, ws, None)


def test_sizes_in_closed_form(lib):
    from paper_2511_11608_amd import binding
    for seqs, heads, dim, n_pages, dp in ((1, 1, 8, 1, 32), (2, 8, 80, 10, 96), (256, 8, 128, 8192, 128), (3, 5, 256, 7, 256), (1, 2, 200, 3, 224)):
        assert binding.slicer_kv_sizes(seqs, heads, dim, n_pages, 4) == (n_pages * heads * 128 * dp, n_pages * heads * 8, seqs * heads * 256 * dp)


def test_shapes_that_are_refused(lib):
    for kw in (dict(seqs=0), dict(seqs=-1), dict(kv_heads=0), dict(head_dim=0), dict(head_dim=4), dict(head_dim=36), dict(head_dim=264), dict(max_pages=0),
               dict(max_pages=(1 << 24) + 1), dict(n_pages=0), dict(n_pages=1 << 31), dict(seqs=1 << 20, kv_heads=4)):
        kv = handle(**kw)
        assert lib.slicer_kv_sizes(C.byref(kv), None, None, None) == -1, kw
        for call in (append, attend, read, evict):
            assert call(lib, kv) == -1, (kw, call)
        assert lib.slicer_kv_attend_sizes(C.byref(kv), 8, 2, 1, 100, 1, None) == -1
    assert lib.slicer_kv_sizes(None, None, None, None) == -1
    for call in (append, attend, read, evict):
        assert call(lib, None) == -1


def test_null_pointers_types_and_counts_are_refused(lib):
    kv = handle()
    for name in ("pages", "scales", "tails", "page_table", "lens"):
        for call in (append, attend, read):
            assert call(lib, handle(**{name: None})) == -1, name
    assert evict(lib, handle(page_table=None)) == -1 and evict(lib, handle(lens=None)) == -1
    for call in (append, attend, read):
        assert call(lib, kv, dt=2) == -2 and call(lib, kv, dt=-1) == -2
        assert call(lib, kv, tokens=-1) == -1 and call(lib, kv, tokens=1 << 31) == -1
        assert call(lib, kv, max_new=0) == -1 and call(lib, kv, starts=None) == -1
        assert call(lib, kv, tokens=0, starts=None, max_new=0) == 0                       # nothing to do
    for name in ("pages", "scales", "tails"):
        for call in (append, attend, read):
            assert call(lib, handle(**{name: 264})) == -1, name                           # 16-byte loads
    assert attend(lib, kv, out=264) == -1 and attend(lib, kv, ws=264) == -1 and evict(lib, kv, ws=264) == -1
    assert append(lib, kv, k=None) == -1 and append(lib, kv, v=None) == -1 and read(lib, kv, k=None) == -1 and read(lib, kv, v=None) == -1
    assert attend(lib, kv, q=None) == -1 and attend(lib, kv, out=None) == -1 and attend(lib, kv, ws=None) == -1
    assert attend(lib, kv, heads=0) == -1 and attend(lib, kv, heads=6) == -1 and attend(lib, kv, max_len=-1) == -1
    for scale in (float("nan"), float("inf")):
        assert attend(lib, kv, scale=scale) == -1
    # more workgroups than a launch can have
    assert attend(lib, handle(seqs=1 << 12, kv_heads=512), heads=512 * 512, tokens=1 << 20, max_new=1 << 10) == -1
    assert evict(lib, handle(seqs=1 << 20, kv_heads=1, max_pages=1 << 16)) == -1
    for decay in (-0.1, 1.1, float("nan")):
        assert attend(lib, kv, decay=decay) == -1
    assert evict(lib, kv, mass=None) == -1 and evict(lib, kv, ws=None) == -1
    for i in range(5):
        assert evict(lib, kv, outs=tuple(None if j == i else 256 for j in range(5))) == -1
    assert evict(lib, kv, keep=-1, sink=0, recent=0) == -1 and evict(lib, kv, sink=-1) == -1 and evict(lib, kv, recent=-1) == -1
    assert evict(lib, kv, keep=2, sink=2, recent=1) == -1 and evict(lib, kv, keep=2 ** 31 - 1, sink=2 ** 31 - 1, recent=2 ** 31 - 1) == -1
    assert lib.slicer_kv_attend_sizes(C.byref(kv), 6, 2, 1, 100, 1, None) == -1 and lib.slicer_kv_attend_sizes(C.byref(kv), 8, 2, 0, 100, 1, None) == -1
    assert lib.slicer_kv_attend_sizes(C.byref(kv), 8, 2, 1, -1, 1, None) == -1


def test_workspace_covers_every_split(lib):
    """Partial sums for up to 64 rows a head, weights of every page of the table, and the rows' sums of longer queries."""
    w = C.c_size_t(0)
    for seqs, G, D, P, H, tokens, max_new, max_len in ((1, 8, 128, 4096, 32, 1, 1, 262144), (256, 8, 128, 32, 64, 256, 1, 2048), (3, 2, 80, 40, 10, 900, 400, 2000),
                                                       (1, 1, 8, 1, 1, 1, 1, 0)):
        kv = handle(seqs=seqs, kv_heads=G, head_dim=D, max_pages=P)
        assert lib.slicer_kv_attend_sizes(C.byref(kv), H, tokens, max_new, max_len, 1, C.byref(w)) == 0
        rows, with_mass = min(64, min(tokens, max_new) * (H // G)), w.value
        assert with_mass >= seqs * G * rows * 8 * (P + 1)
        tiles = -(-max_new * (H // G) // 128) if max_new * (H // G) > 64 else 0
        assert with_mass >= min(seqs * G * tiles, 256) * P * 1024 + seqs * G * tiles * P * 4
        assert with_mass < 1 << 31
        assert lib.slicer_kv_attend_sizes(C.byref(kv), H, tokens, max_new, max_len, 0, C.byref(w)) == 0
        assert seqs * G * rows * 8 <= w.value < with_mass
    assert lib.slicer_kv_attend_sizes(C.byref(kv), 1, 0, 0, 0, 1, C.byref(w)) == 0 and w.value == 0


def test_the_binding_refuses_what_is_not_on_the_gpu(lib):
    import torch
    from paper_2511_11608_amd import binding
    kv = binding.alloc_kv(2, 2, 64, 4, 4, device="cpu")
    x, starts = torch.zeros(2, 2, 64), torch.zeros(3, dtype=torch.int32)
    with pytest.raises(ValueError):
        binding.slicer_kv_append(kv, x, x, starts, 1)
    with pytest.raises(ValueError):
        binding.slicer_kv_read(kv, starts, 1, x, x)
    with pytest.raises(ValueError):
        binding.slicer_kv_attend(kv, x, starts, 1, 1, 1.0, x, torch.zeros(1))
    with pytest.raises(ValueError):
        binding.slicer_kv_evict(kv, torch.zeros(2, 2, 4), 1, 0, 0, binding.alloc_kv_evict(kv))
    with pytest.raises(binding.SlicerError):
        binding.alloc_kv(2, 2, 60, 4, 4, device="cpu")


def test_definition_of_a_page_by_hand():
    """amax 2: scale = 2 / 127 and inv = 63.5, an exact quotient, so that 1/127-steps of 2 come back; 0.0078125 * 63.5 = 0.49609375 -> 0, 3 * 2^-7 * 63.5 = 1.488 -> 1,
    and 5 * 2^-7 ... * 63.5 = 2.48 -> 2; a quotient of exactly 0.5 (1/127) cannot be written in bf16, one of 31.75 (0.5) goes to 32."""
    x = np.zeros((64, 4))
    x[0] = [2.0, -0.5, 2.0 ** -7, 3 * 2.0 ** -7]
    x[1] = [-2.0, 0.25, 5 * 2.0 ** -7, -1.0]
    codes, scale = kv_ref.hold(x)
    assert scale == float(np.float32(2.0) / np.float32(127.0))
    assert codes[0].tolist() == [127, -32, 0, 1] and codes[1].tolist() == [-127, 16, 2, -64]          # 63.5 is a tie: the even 64
    assert kv_ref.hold(np.full((64, 4), 2.0 ** -120)) [1] == 0.0
    assert kv_ref.hold(np.full((64, 4), 2.0 ** -119))[1] > 0.0


def test_definition_of_attention_and_eviction_by_hand():
    import torch
    s = kv_ref.Sequence(1, 2)
    s.append(torch.tensor([[[0.0, 0.0]], [[1.0, 0.0]]]), torch.tensor([[[1.0, 2.0]], [[3.0, -2.0]]]))
    out, lse, mass, absv, size, allv = s.attend(torch.tensor([[[9.0, 9.0]], [[np.log(3.0), 5.0]]], dtype=torch.float64), 1.0)
    assert np.allclose(out[0, 0], [1, 2]) and np.allclose(lse[0, 0], 0)                                # the first query sees the first token
    assert np.allclose(out[1, 0], [0.25 * 1 + 0.75 * 3, 0.25 * 2 - 0.75 * 2]) and np.allclose(lse[1, 0], np.log(4.0))
    assert np.allclose(mass, 2.0) and np.allclose(absv[1, 0], [2.5, 2.0]) and np.allclose(allv[1, 0], [4, 4])
    w = np.array([[5.0, 1.0, 3.0, 3.0, 2.0, 0.0]])
    assert kv_ref.evict(w, 6, 4, 1, 1) == [0, 2, 3, 5] and kv_ref.evict(w, 6, 3, 1, 1) == [0, 2, 5]    # ties: the lower place
    assert kv_ref.evict(w, 5, 5, 0, 0) == [0, 1, 2, 3, 4] and kv_ref.evict(w, 6, 0, 0, 0) == []
    w[0, 1] = np.nan
    assert kv_ref.evict(w, 6, 3, 1, 1) == [0, 1, 5]
