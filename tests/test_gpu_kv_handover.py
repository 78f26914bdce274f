"""The cache's rows handed over: what slicer_kv_read gives goes through slicer_encode and slicer_decode as any feature does, byte for byte as the oracle says."""
import numpy as np
import pytest

from tests.test_gpu_kv import Pair, starts_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_read_from_the_cache_are_encoded(oracle, dtype):
    import torch
    from paper_2511_11608_amd import binding
    from paper_2511_11608_amd.devmem import to_host
    p = Pair(2, 4, 64, 4, dtype, seed=3)
    p.append([150, 70])
    p.append([1, 5])
    lens = [len(r) for r in p.ref]
    k, v = (torch.empty(sum(lens), 4, 64, dtype=p.dt, device="cuda") for _ in range(2))
    p.b.slicer_kv_read(p.kv, starts_of(lens), max(lens), k, v)
    for x in (k.view(sum(lens), 256), v.view(sum(lens), 256)):
        sb, meta, ws = binding.alloc_buffers(x, 0.5, 8, 0x1FC)
        binding.slicer_encode(x, 0.5, 8, 0x1FC, 1e-3, sb, meta, ws)
        y = torch.empty_like(x)
        binding.slicer_decode(sb, meta, y)
        words = binding.slicer_stream_words(meta)
        torch.cuda.synchronize()
        s_ref, m_ref = oracle.encode(to_host(x), dtype, 0.5, 8, 0x1FC, 1e-3)
        assert np.array_equal(meta.cpu().numpy(), m_ref) and np.array_equal(sb[:words].cpu().numpy().view(np.uint32), s_ref)
        y_ref = oracle.decode(s_ref, m_ref)
        assert np.array_equal(to_host(y), y_ref)
