"""A prompt's chunk with its weights and an eviction, captured once: replays with other tokens in the buffers, ordinary and steep scores in turn, eager work between
them, every one equal to the eager calls bit for bit."""
import pytest

from tests.test_gpu_kv import starts_of

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("max_len", [0, 700])
def test_chunks_and_eviction(max_len, dtype):
    import torch
    from paper_2511_11608_amd import binding
    dt = torch.float32 if dtype == "f32" else torch.bfloat16
    gen = torch.Generator().manual_seed(max_len)
    counts, G, H, D, P = [150, 80, 3], 2, 8, 64, 12
    starts, total = starts_of(counts), sum(counts)

    def rand(n, heads, scale=1.0):
        return (torch.randn(n, heads, D, generator=gen) * scale).to(dt).cuda()

    def cache():
        kv = binding.alloc_kv(3, G, D, 3 * P, P)
        kv.page_table.copy_(torch.arange(3 * P, dtype=torch.int32).flip(0).view(3, P))
        return kv

    past = [400, 64, 130]
    old_k, old_v = rand(sum(past), G), rand(sum(past), G)

    def fill(kv):
        kv.lens.copy_(torch.tensor(past, dtype=torch.int32))
        binding.slicer_kv_append(kv, old_k, old_v, starts_of(past), max(past))
        kv.lens.copy_(torch.tensor([a + b for a, b in zip(past, counts)], dtype=torch.int32))

    def buffers(kv):
        return {"q": rand(total, H), "k": rand(total, G), "v": rand(total, G), "out": torch.empty(total, H, D, dtype=dt, device="cuda"),
                "lse": torch.empty(total, H, device="cuda"), "mass": torch.zeros(3, G, P, device="cuda"), "ev": binding.alloc_kv_evict(kv),
                "ws": binding.alloc_kv_workspace(kv, H, total, 150, max_len)}

    def step(kv, b):
        binding.slicer_kv_append(kv, b["k"], b["v"], starts, 150)
        binding.slicer_kv_attend(kv, b["q"], starts, 150, max_len, 0.125, b["out"], b["ws"], lse=b["lse"], mass=b["mass"], mass_decay=0.5)
        binding.slicer_kv_evict(kv, b["mass"], 3, 1, 1, b["ev"])

    kvs = [cache(), cache()]
    bufs = [buffers(kv) for kv in kvs]
    fill(kvs[0])
    step(kvs[0], bufs[0])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step(kvs[0], bufs[0])
    for i in range(5):
        x = {"q": rand(total, H, 2.0 ** 20 if i % 2 else 1.0), "k": rand(total, G), "v": rand(total, G)}
        for kv, b in zip(kvs, bufs):
            fill(kv)
            for name, t in x.items():
                b[name].copy_(t)
            b["out"].fill_(3.0)
            b["ws"].fill_(0x5A)
            b["mass"].fill_(0.25)
        torch.cuda.synchronize()
        g.replay()
        step(kvs[1], bufs[1])
        torch.cuda.synchronize()
        a, b = bufs
        assert torch.isfinite(a["out"].float()).all()
        assert all(torch.equal(a[n], b[n]) for n in ("out", "lse", "mass"))
        assert all(torch.equal(getattr(a["ev"], n), getattr(b["ev"], n)) for n in ("page_table", "lens", "mass", "freed", "n_freed"))
        assert a["ev"].n_freed.tolist() == [5, 0, 0]
