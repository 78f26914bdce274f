"""The attention cache in 8 bits on the GPU (slicer_kv_*), against its definition in 64 bits (tests/kv_ref.py).

Tolerances.  What the cache holds is compared bit for bit.  An output is off by
  half a step of its type (which below the smallest normal number is that number's),
  the rounding of the probabilities: fp16, half a step 2^-11 of each (bf16 outputs); two fp16 numbers for fp32 outputs, 2^-22 of each and
  less than that again where the second is below fp16's smallest normal number,
  the scores' error delta: D products summed in fp32, and scale, maximum and exponential after it, (D + 16) 2^-24 of sum |q k| scale, plus 2^-22 from
    the exponential (twice: numerator and sum),
  sums over the tokens in fp32: length * 2^-24,
the last three times sum p |v|; and 2^-32 of sum |v|: a probability is held times 2^13 and times the ratio of two scales, at least 2^-6, in fp16, whose
steps do not get smaller than 2^-24: half a step is 2^-25 / 2^13 * 2^6.
"""
import numpy as np
import pytest

from tests import kv_ref
from tests.kv_ref import PAGE

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def starts_of(counts):
    torch = _torch()
    return torch.tensor(np.concatenate([[0], np.cumsum(counts)]), dtype=torch.int32, device="cuda")


class Pair:
    """A cache on the GPU and its definition, fed with the same tokens."""

    def __init__(self, seqs, kv_heads, dim, max_pages, dtype="bf16", seed=0, spare=3):
        torch = _torch()
        from paper_2511_11608_amd import binding
        self.b, self.torch = binding, torch
        self.dt = torch.float32 if dtype == "f32" else torch.bfloat16
        self.gen = torch.Generator().manual_seed(seed)
        n_pages = seqs * max_pages + spare
        self.kv = binding.alloc_kv(seqs, kv_heads, dim, n_pages, max_pages)
        self.kv.pages.fill_(0xFF)                       # nothing may rest on what the buffers held
        self.kv.scales.fill_(float("nan"))
        self.kv.tails.fill_(float("nan"))
        table = torch.randperm(n_pages, generator=self.gen)[: seqs * max_pages].view(seqs, max_pages)
        self.kv.page_table.copy_(table.int())
        self.ref = [kv_ref.Sequence(kv_heads, dim) for _ in range(seqs)]

    def rand(self, n, heads, scale=1.0):
        torch = self.torch
        x = torch.randn(n, heads, self.kv.head_dim, generator=self.gen)
        x[:, :, ::7] *= 3.0
        return (x * scale).to(self.dt)

    def sync_lens(self):
        self.kv.lens.copy_(self.torch.tensor([len(r) for r in self.ref], dtype=self.torch.int32))

    def append(self, counts, k=None, v=None, max_new=None):
        total = sum(counts)
        k = self.rand(total, self.kv.kv_heads) if k is None else k
        v = self.rand(total, self.kv.kv_heads) if v is None else v
        at = 0
        for r, n in zip(self.ref, counts):
            r.append(k[at: at + n], v[at: at + n])
            at += n
        self.sync_lens()
        self.b.slicer_kv_append(self.kv, k.cuda(), v.cuda(), starts_of(counts), max_new or max(max(counts), 1))

    def attend(self, counts, q, scale, causal=True, mass=None, decay=0.0, max_len=None, lse=True):
        torch = self.torch
        total, H = q.shape[0], q.shape[1]
        out = torch.full((total, H, self.kv.head_dim), 7.0, dtype=q.dtype, device="cuda")
        lse_t = torch.full((total, H), 7.0, dtype=torch.float32, device="cuda") if lse else None
        max_new, max_len = max(max(counts), 1), max(len(r) for r in self.ref) if max_len is None else max_len
        ws = self.b.alloc_kv_workspace(self.kv, H, total, max_new, max_len)
        ws.fill_(0xA5)
        self.b.slicer_kv_attend(self.kv, q, starts_of(counts), max_new, max_len, scale, out, ws, lse=lse_t, mass=mass, mass_decay=decay, causal=causal)
        torch.cuda.synchronize()
        return out, lse_t

    def check(self, counts, q, scale, out, lse, causal=True, mass=None, old=None, decay=0.0):
        torch = self.torch
        D = self.kv.head_dim
        at = 0
        for i, (r, n) in enumerate(zip(self.ref, counts)):
            o, l, w, absv, size, allv = r.attend(q[at: at + n], scale, causal)
            got, got_l = out[at: at + n].double().cpu().numpy(), lse[at: at + n].double().cpu().numpy() if lse is not None else None
            at += n
            delta = (D + 16) * 2.0 ** -24 * size + 2.0 ** -22
            p_bits = 2.0 ** -11 if q.dtype == torch.bfloat16 else 2.0 ** -21
            fi = torch.finfo(q.dtype)
            tol = fi.eps / 2 * (1 + 2.0 ** -7) * np.abs(o) + fi.eps / 2 * fi.smallest_normal + (p_bits + 2 * delta + (len(r) + 64) * 2.0 ** -24)[..., None] * absv + 2.0 ** -32 * allv
            assert np.array_equal(np.isnan(o), np.isnan(got)), i
            fine = ~np.isnan(o)
            assert (np.abs(got - o)[fine] <= tol[fine]).all(), (i, np.abs(got - o)[fine].max(), (np.abs(got - o)[fine] / np.maximum(tol[fine], 1e-300)).max())
            if got_l is not None:
                assert np.array_equal(np.isnan(l), np.isnan(got_l)) and np.array_equal(np.isneginf(l), np.isneginf(got_l)), i
                fl = np.isfinite(l)
                assert (np.abs(got_l[fl] - l[fl]) <= (delta + (len(r) + 64) * 2.0 ** -24 + 2.0 ** -22 * np.abs(l))[fl]).all(), i
            if mass is not None:
                g = mass[i].double().cpu().numpy()
                was = old[i].double().cpu().numpy()
                want = was.copy()
                pages = w.shape[1]
                if n:
                    want[:, :pages] = (decay * was[:, :pages] if decay else 0.0) + w
                fine = ~np.isnan(want)
                assert np.array_equal(np.isnan(g), ~fine), i
                worst = 2 * delta.max() + (len(r) + n * q.shape[1] + 64) * 2.0 ** -24 if n else 0.0
                assert (np.abs(g - want)[fine] <= worst * np.abs(want)[fine] + 1e-30).all(), (i, np.abs(g - want)[fine].max())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,dim", [(1, 8), (2, 32), (3, 80), (2, 128), (1, 256), (5, 200)])
def test_append_then_read_is_the_definition(dtype, heads, dim):
    torch = _torch()
    p = Pair(4, heads, dim, 5, dtype, seed=dim)
    for counts in ([1, 0, 63, 64], [62, 65, 1, 0], [1, 1, 64, 130], [70, 0, 3, 1]):
        p.append(counts)
    lens = [len(r) for r in p.ref]
    want = [r.values() for r in p.ref]
    for dt in (torch.float32, torch.bfloat16):
        k = torch.full((sum(lens) + 3, heads, dim), 7.0, dtype=dt, device="cuda")
        v = torch.full_like(k, 7.0)
        p.b.slicer_kv_read(p.kv, starts_of(lens), max(lens), k, v)
        torch.cuda.synchronize()
        for which, got in ((0, k), (1, v)):
            ref = torch.tensor(np.concatenate([w[which] for w in want])).float().to(dt)      # code * scale is a product of fp32 numbers
            assert torch.equal(got[: sum(lens)].cpu(), ref)
            assert (got[sum(lens):] == 7.0).all()                                            # rows behind the last sequence


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_the_cache_does_not_depend_on_how_tokens_arrive(dtype):
    torch = _torch()
    k, v = None, None
    reads = []
    for pieces in ([200], [1] * 200, [63, 2, 135], [64, 64, 72], [10, 190]):
        p = Pair(1, 2, 96, 4, dtype, seed=5)
        if k is None:
            k, v = p.rand(200, 2), p.rand(200, 2)
        at = 0
        for n in pieces:
            p.append([n], k[at: at + n], v[at: at + n])
            at += n
        ko, vo = torch.empty(200, 2, 96, dtype=p.dt, device="cuda"), torch.empty(200, 2, 96, dtype=p.dt, device="cuda")
        p.b.slicer_kv_read(p.kv, starts_of([200]), 200, ko, vo)
        reads.append(torch.stack([ko, vo]).cpu())
    assert all(torch.equal(reads[0], r) for r in reads[1:])


@pytest.mark.parametrize("kind", ["zeros", "ties", "tiny", "huge", "one"])
def test_pages_of_unusual_values(kind):
    torch = _torch()
    p = Pair(1, 1, 64, 2, "f32", seed=9)
    g = torch.Generator().manual_seed(4)
    x = torch.randn(2, 128, 1, 64, generator=g)
    if kind == "zeros":
        x[:, :64] = 0.0
    elif kind == "ties":
        x = torch.randint(-254, 255, x.shape, generator=g).float() / 2                        # quotients that lie between two codes
    elif kind == "tiny":
        x *= 2.0 ** -118
        x[:, :64] *= 2.0 ** -6
    elif kind == "huge":
        x = (x * 2.0 ** 100).clamp(-2.0 ** 100, 2.0 ** 100)
    else:
        x = torch.where(torch.arange(64) == 3, x, torch.zeros(()))
    p.append([128], x[0], x[1])
    k, v = torch.empty(128, 1, 64, device="cuda"), torch.empty(128, 1, 64, device="cuda")
    p.b.slicer_kv_read(p.kv, starts_of([128]), 128, k, v)
    wk, wv, _ = p.ref[0].values()
    assert torch.equal(k.cpu(), torch.tensor(wk).float()) and torch.equal(v.cpu(), torch.tensor(wv).float())
    for n in (1, 90):                                     # as split rows and as a prompt's
        q = p.rand(n, 1, 2.0 ** -100 if kind == "huge" else 1.0)
        out, lse = p.attend([n], q.cuda(), 0.125)
        p.check([n], q, 0.125, out, lse)


SHAPES = [
    # lens before, new, heads, kv_heads, dim
    ([0], [1], 1, 1, 8),
    ([76], [1], 12, 12, 64),
    ([63, 64, 65, 0, 127, 300], [1, 1, 1, 1, 0, 1], 8, 2, 128),
    ([700, 0, 129, 64], [1, 2, 1, 0], 7, 1, 80),
    ([500, 31], [4, 5], 16, 4, 96),                                   # two row tiles
    ([333, 1, 0], [16, 16, 2], 4, 1, 32),                             # 64 rows: the most that are split
    ([200, 5], [3, 1], 6, 3, 256),
    ([90, 64], [1, 1], 32, 1, 160),                                   # 32 query heads of one cache head
    ([0, 64, 200, 10], [65, 100, 17, 1], 4, 1, 64),                   # split and not split in one call
    ([0, 100, 640], [300, 33, 129], 4, 2, 128),
    ([0], [257], 3, 3, 80),
    ([120, 0], [70, 127], 2, 1, 256),
    ([64], [130], 5, 1, 224),
    ([3], [200], 1, 1, 40),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("shape", range(len(SHAPES)))
def test_attend(shape, causal, dtype):
    torch = _torch()
    past, new, H, G, D = SHAPES[shape]
    p = Pair(len(past), G, D, max(-(-(a + n) // PAGE) for a, n in zip(past, new)) + 1, dtype, seed=shape)
    if sum(past):
        p.append(past)
    p.append(new)
    q = p.rand(sum(new), H)
    scale = D ** -0.5
    mass = torch.rand(len(past), G, p.kv.max_pages, device="cuda")
    old = mass.clone()
    out, lse = p.attend(new, q.cuda(), scale, causal, mass, decay=0.5)
    p.check(new, q, scale, out, lse, causal, mass, old, 0.5)
    again, lse2 = p.attend(new, q.cuda(), scale, causal)
    assert torch.equal(out, again) and torch.equal(lse, lse2)                                # with weights or without, today or tomorrow


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("max_len", [0, 64, 3000, 10 ** 6])
def test_any_split_of_a_long_cache(max_len, dtype):
    torch = _torch()
    p = Pair(2, 2, 64, 48, dtype, seed=3)
    p.append([2900, 700])
    p.append([1, 3])
    q = p.rand(4, 8)
    mass = torch.full((2, 2, 48), float("nan"), device="cuda")                               # decay 0: old contents are not read
    old = torch.zeros_like(mass)
    old[:] = float("nan")
    out, lse = p.attend([1, 3], q.cuda(), 0.2, mass=mass, max_len=max_len)
    p.check([1, 3], q, 0.2, out, lse, mass=mass, old=old)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("past,new,heads,kv_heads,dim", [([1100], [70], 2, 1, 64), ([1985], [40], 16, 2, 96), ([3000, 130], [90, 33], 4, 1, 128), ([2040], [200], 1, 1, 32), ([1600, 900], [80, 80], 8, 4, 256)])
def test_long_cache_before_few_rows(past, new, heads, kv_heads, dim, dtype):
    """Row tiles that do not fill the chip: their pages are shared out, the rows and weights put together behind it."""
    torch = _torch()
    p = Pair(len(past), kv_heads, dim, max(-(-(a + n) // PAGE) for a, n in zip(past, new)) + 2, dtype, seed=sum(past))
    p.append(past)
    p.append(new)
    q = p.rand(sum(new), heads)
    for causal in (True, False):
        mass = torch.rand(len(past), kv_heads, p.kv.max_pages, device="cuda")
        old = mass.clone()
        out, lse = p.attend(new, q.cuda(), dim ** -0.5, causal, mass, decay=1.0)
        p.check(new, q, dim ** -0.5, out, lse, causal, mass, old, 1.0)


@pytest.mark.parametrize("seqs,heads,kv_heads,dim,new", [(33, 8, 4, 16, 1), (66, 8, 4, 24, 1), (43, 12, 3, 8, 5), (17, 16, 4, 16, 2), (130, 3, 1, 16, 1)])
def test_steps_of_many_sequences_with_a_long_one(seqs, heads, kv_heads, dim, new):
    """More row tiles than half of the chip, full and hardly full last rounds: shares of a long sequence, and ones that are empty in the others."""
    torch = _torch()
    past = [(37 * i) % 300 for i in range(seqs)]
    past[seqs // 2], past[-1] = 6300, 6143
    p = Pair(seqs, kv_heads, dim, 100, "bf16", seed=seqs)
    p.append(past)
    counts = [new if i % 5 else 0 for i in range(seqs)]
    counts[seqs // 2] = counts[-1] = new
    p.append(counts)
    q = p.rand(sum(counts), heads)
    mass = torch.rand(seqs, kv_heads, 100, device="cuda")
    old = mass.clone()
    out, lse = p.attend(counts, q.cuda(), dim ** -0.5, mass=mass, decay=0.5)
    p.check(counts, q, dim ** -0.5, out, lse, mass=mass, old=old, decay=0.5)


def test_many_tiles_give_the_same_bits_every_time():
    """Hundreds of workgroups whose wavefronts share operands in LDS: any order of theirs gives the same result."""
    torch = _torch()
    p = Pair(6, 4, 128, 20, "bf16", seed=40)
    p.append([0, 100, 64, 500, 3, 630])
    new = [600, 511, 512, 400, 640, 577]
    p.append(new)
    q = p.rand(sum(new), 16).cuda()
    first = None
    for _ in range(12):
        mass = torch.zeros(6, 4, 20, device="cuda")
        out, lse = p.attend(new, q, 0.1, mass=mass)
        got = (out.clone(), lse.clone(), mass)
        first = first or got
        assert all(torch.equal(a, b) for a, b in zip(first, got))
    rows = list(range(0, 40)) + list(range(590, 600))
    o, l, _, absv, size, allv = p.ref[0].attend(q[:600], 0.1)
    tol = 2.0 ** -8 * np.abs(o) + (2.0 ** -11 + 2 * (144 * 2.0 ** -24 * size + 2.0 ** -22) + 700 * 2.0 ** -24)[..., None] * absv + 2.0 ** -32 * allv
    assert (np.abs(first[0][:600].double().cpu().numpy() - o) <= tol * (1 + 2.0 ** -7))[rows].all()


@pytest.mark.parametrize("new", [[2, 1], [40, 30]])
def test_scores_far_below_and_above_zero(new):
    """Weights that vanish and weights that stand alone: the maximum of a part of the cache is far from the whole row's."""
    torch = _torch()
    p = Pair(2, 1, 64, 12, "bf16", seed=8)
    p.append([600, 100])
    p.append(new)
    for scale in (-3.0, 5.0, 30.0):
        q = p.rand(sum(new), 2)
        out, lse = p.attend(new, q.cuda(), scale)
        p.check(new, q, scale, out, lse)
    # all scores far below zero: nothing may be added under a maximum of zero
    k = torch.full((p.kv.kv_heads, 64), 4.0, dtype=torch.bfloat16)
    p2 = Pair(1, 1, 64, 12, "bf16", seed=2)
    p2.append([600], -k.expand(600, 1, 64).contiguous() + 0.25 * p2.rand(600, 1), None)
    q = torch.full((3, 2, 64), 4.0, dtype=torch.bfloat16)
    out, lse = p2.attend([3], q.cuda(), 1.0)
    p2.check([3], q, 1.0, out, lse)


def test_value_scales_far_apart():
    torch = _torch()
    for new in ([1], [100]):
        p = Pair(1, 1, 64, 9, "f32", seed=6)
        v = p.rand(512, 1)
        for i, e in enumerate((0, -40, -20, 20, 60, -60, 3, 0)):
            v[i * 64: i * 64 + 64] *= 2.0 ** e
        p.append([512 - new[0]], None, v[: 512 - new[0]])
        p.append(new, None, v[512 - new[0]:])
        q = p.rand(new[0], 1)
        out, lse = p.attend(new, q.cuda(), 0.1)
        p.check(new, q, 0.1, out, lse)


def test_queries_that_see_nothing_and_empty_sequences():
    torch = _torch()
    p = Pair(3, 2, 64, 3, "bf16", seed=1)
    p.append([5, 0, 70])
    # more queries than tokens: the first ones stand before the first token
    counts = [9, 4, 100]
    q = p.rand(sum(counts) + 2, 4)
    out, lse = p.attend(counts, q.cuda(), 0.3)
    p.check(counts, q[: sum(counts)], 0.3, out[: sum(counts)], lse[: sum(counts)])
    assert (out[:4] == 0).all() and torch.isneginf(lse[:4]).all() and (out[9:13] == 0).all()
    assert (out[sum(counts):] == 7.0).all() and (lse[sum(counts):] == 7.0).all()             # rows of no sequence
    mass = torch.ones(3, 2, 3, device="cuda")
    out, _ = p.attend([0, 0, 2], p.rand(2, 4).cuda(), 0.3, mass=mass)
    assert (mass[:2] == 1.0).all()                                                           # sequences without queries keep theirs
    assert p.attend([0, 0, 0], torch.empty(0, 4, 64, dtype=torch.bfloat16, device="cuda"), 0.3)[0].numel() == 0


@pytest.mark.parametrize("where", ["tail", "page"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_values_that_are_not_finite_reach_only_who_sees_them(where, bad):
    torch = _torch()
    past, new = ([64, 70], [40, 1]) if where == "tail" else ([20, 70], [100, 1])
    p = Pair(2, 2, 64, 4, "bf16", seed=12)
    p.append(past)
    k, v = p.rand(sum(new), 2), p.rand(sum(new), 2)
    k[7, 0, 3] = bad                                     # head 0 by a key, head 1 by a value, a later token
    v[30, 1, 60] = bad
    p.append(new, k, v)
    q = p.rand(sum(new), 4)
    mass = torch.zeros(2, 2, 4, device="cuda")
    out, lse = p.attend(new, q.cuda(), 0.125, mass=mass)
    p.check(new, q, 0.125, out, lse, mass=mass, old=torch.zeros_like(mass))
    assert torch.isfinite(out[new[0]:]).all()            # the other sequence
    q1 = p.rand(2, 4)
    out, lse = p.attend([1, 1], q1.cuda(), 0.125)
    p.check([1, 1], q1, 0.125, out, lse)


@pytest.mark.parametrize("new", [1, 90])
def test_pages_that_are_not_there(new):
    """Entries outside the cache are not written and read as NaN; the cache's own pages stay as they were."""
    torch = _torch()
    p = Pair(2, 1, 64, 8, "bf16", seed=4)
    p.append([200, 200])
    before = p.kv.pages.clone()
    good = p.kv.page_table.clone()
    for id_ in (-1, -2 ** 31, p.kv.n_pages, 2 ** 31 - 1):
        p.kv.page_table.copy_(good)
        p.kv.page_table[0, 1] = id_
        q = p.rand(new + 1, 2)
        out, lse = p.attend([new, 1], q.cuda(), 0.125)
        assert torch.isnan(out[0]).all() if new == 1 else torch.isnan(out[-2]).all()
        assert torch.isfinite(out[-1]).all()
        kv = torch.zeros(200, 1, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(200, 1, 64, dtype=torch.bfloat16, device="cuda")
        p.b.slicer_kv_read(p.kv, starts_of([200, 0]), 200, *kv)
        assert torch.isnan(kv[0][64:128]).all() and torch.isfinite(kv[0][128:]).all() and torch.isfinite(kv[1][:64]).all()
        p.kv.page_table[0, 3] = id_
        p.kv.lens.copy_(torch.tensor([256, 200], dtype=torch.int32))
        p.b.slicer_kv_append(p.kv, p.rand(56, 1).cuda(), p.rand(56, 1).cuda(), starts_of([56, 0]), 56)
        assert torch.equal(p.kv.pages, before)
        p.kv.lens.copy_(torch.tensor([200, 200], dtype=torch.int32))


def test_lengths_and_starts_outside_their_range_stay_in_the_buffers():
    torch = _torch()
    p = Pair(2, 1, 64, 3, "bf16", seed=4)
    p.append([100, 150])
    q = p.rand(3, 2).cuda()
    ok, _ = p.attend([1, 2], q, 0.125)
    ws = p.b.alloc_kv_workspace(p.kv, 2, 3, 2, 192)
    for lens, starts in (([-5, 150], [0, 1, 3]), ([2 ** 31 - 1, 150], [0, 1, 3]), ([100, 150], [-7, 1, 2 ** 30]), ([100, 150], [5, 1, 3])):
        p.kv.lens.copy_(torch.tensor(lens, dtype=torch.int32))
        out = torch.full_like(ok, 7.0)
        p.b.slicer_kv_attend(p.kv, q, torch.tensor(starts, dtype=torch.int32, device="cuda"), 2, 192, 0.125, out, ws)
        torch.cuda.synchronize()
        assert torch.equal(out[1:], ok[1:])              # the sequence whose numbers are right


def test_strides_and_unaligned_rows():
    torch = _torch()
    for dtype in ("bf16", "f32"):
        for off in (0, 1):
            p = Pair(2, 2, 72, 4, dtype, seed=21)
            p.append([30, 90])
            new = [50, 40]
            # one fused tensor of queries, keys and values, heads apart by more than their size
            fused = p.rand(sum(new), 8)
            store = torch.zeros(sum(new) * 8 * 81 + 8, dtype=p.dt, device="cuda")
            base = store[off:].as_strided((sum(new), 8, 72), (8 * (80 + off), 80 + off, 1))
            base.copy_(fused)
            q, k, v = base[:, :4], base[:, 4:6], base[:, 6:8]
            at = 0
            for r, n in zip(p.ref, new):
                r.append(fused[at: at + n, 4:6], fused[at: at + n, 6:8])
                at += n
            p.sync_lens()
            p.b.slicer_kv_append(p.kv, k, v, starts_of(new), max(new))
            out, lse = p.attend(new, q, 0.2)
            p.check(new, q, 0.2, out, lse)
            # queries of one token for every sequence, the same for all of them
            one = q[:1].expand(2, 4, 72)
            out, lse = p.attend([1, 1], one, 0.2)
            p.check([1, 1], one, 0.2, out, lse)


def test_sequences_share_full_pages():
    torch = _torch()
    p = Pair(2, 2, 64, 4, "bf16", seed=31)
    p.append([128, 0])
    p.kv.page_table[1, :2] = p.kv.page_table[0, :2]
    p.ref[1].pages = list(p.ref[0].pages)
    p.append([3, 70])
    q = p.rand(2, 4)
    out, lse = p.attend([1, 1], q.cuda(), 0.125)
    p.check([1, 1], q, 0.125, out, lse)


def ref_evict(table, lens, mass, keep, sink, recent):
    seqs, P = table.shape
    t2, l2, m2, freed, n = np.full_like(table, -1), lens.copy(), np.zeros_like(mass), np.full_like(table, -1), np.zeros_like(lens)
    for b in range(seqs):
        full = lens[b] // PAGE
        stay = kv_ref.evict(mass[b], full, keep, sink, recent)
        rest = stay + list(range(full, P))
        gone = sorted(set(range(full)) - set(stay))
        t2[b, : len(rest)], m2[b][:, : len(rest)] = table[b][rest], mass[b][:, rest]
        freed[b, : len(gone)], n[b] = table[b][gone], len(gone)
        l2[b] -= PAGE * len(gone)
    return t2, l2, m2, freed, n


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("seqs,heads,pages,keep,sink,recent,kind", [
    (1, 1, 1, 0, 0, 0, "plain"), (3, 2, 9, 4, 1, 1, "plain"), (2, 8, 70, 70, 1, 4, "plain"), (5, 3, 65, 20, 0, 0, "ties"),
    (2, 4, 1500, 700, 4, 64, "ties"), (1, 8, 5000, 17, 0, 1, "plain"), (2, 2, 40, 10, 5, 5, "plain"), (2, 2, 64, 13, 2, 3, "nan"),
    (2, 1, 300, 100, 0, 0, "equal"), (3, 12, 33, 5, 0, 2, "tiny"),
    (2, 3, 256, 100, 1, 1, "ties"), (2, 2, 1024, 1000, 0, 0, "ties"), (2, 2, 1025, 3, 1, 2, "plain"), (1, 2, 40000, 30000, 4, 4, "ties"), (2, 1, 17000, 16500, 0, 0, "equal"),
    (2, 2, 2000, 30, 5, 5, "nan"), (1, 3, 3000, 0, 0, 0, "plain"), (2, 12, 1500, 700, 0, 2, "tiny")])
def test_evict(seqs, heads, pages, keep, sink, recent, kind, in_place):
    torch = _torch()
    from paper_2511_11608_amd import binding
    rng = np.random.default_rng(pages + keep)
    kv = binding.alloc_kv(seqs, heads, 8, seqs * pages, pages)
    table = rng.permutation(seqs * pages).reshape(seqs, pages).astype(np.int32)
    lens = np.array([pages * PAGE - (0 if i == 0 else int(rng.integers(0, pages * PAGE))) for i in range(seqs)], dtype=np.int32)
    mass = rng.random((seqs, heads, pages)).astype(np.float32) ** 8
    if kind == "ties":
        mass = np.round(mass * 16).astype(np.float32) / 16
    elif kind == "equal":
        mass[:] = 0.25
    elif kind == "nan":
        mass[0, 1, 7] = np.nan
        mass[1, 0, 11] = np.inf
    elif kind == "tiny":                                 # sums that only more than 32 bits can tell apart
        mass = (1.0 + rng.integers(0, 3, mass.shape) * 2.0 ** -23).astype(np.float32)
    kv.page_table.copy_(torch.tensor(table))
    kv.lens.copy_(torch.tensor(lens))
    m = torch.tensor(mass, device="cuda")
    out = binding.alloc_kv_evict(kv)
    if in_place:
        out.page_table, out.lens, out.mass = kv.page_table, kv.lens, m
    out.workspace.fill_(0xA5)
    binding.slicer_kv_evict(kv, m, keep, sink, recent, out)
    torch.cuda.synchronize()
    t2, l2, m2, freed, n = ref_evict(table, lens, mass, keep, sink, recent)
    assert np.array_equal(out.n_freed.cpu().numpy(), n) and np.array_equal(out.lens.cpu().numpy(), l2)
    assert np.array_equal(out.page_table.cpu().numpy(), t2) and np.array_equal(out.freed.cpu().numpy(), freed)
    assert np.array_equal(out.mass.cpu().numpy(), m2, equal_nan=True)


def test_a_budgeted_dialogue():
    """Prompts, tokens one by one, weights kept, pages dropped and handed out again: the calls together, as a program makes them."""
    torch = _torch()
    from paper_2511_11608_amd import binding
    G, H, D, seqs, P, budget = 2, 8, 64, 2, 8, 3
    p = Pair(seqs, G, D, P, "bf16", seed=77, spare=0)
    free = [[], []]
    mass = torch.zeros(seqs, G, P, device="cuda")
    want = np.zeros((seqs, G, P))
    out_e = binding.alloc_kv_evict(p.kv)
    out_e.page_table, out_e.lens, out_e.mass = p.kv.page_table, p.kv.lens, mass
    for step, new in enumerate([[150, 200]] + [[1, 1]] * 30 + [[60, 3]] + [[1, 0]] * 20 + [[100, 190]]):
        p.append(new)
        q = p.rand(sum(new), H)
        old = mass.clone()
        out, lse = p.attend(new, q.cuda(), 0.2, mass=mass, decay=1.0)
        p.check(new, q, 0.2, out, lse, mass=mass, old=old, decay=1.0)
        host = mass.cpu().numpy()
        lens = [len(r) for r in p.ref]
        binding.slicer_kv_evict(p.kv, mass, budget, 1, 1, out_e)
        n = out_e.n_freed.tolist()
        for b in range(seqs):
            full = lens[b] // PAGE
            stay = kv_ref.evict(host[b], full, budget, 1, 1)
            assert n[b] == full - len(stay)
            p.ref[b].pages = [p.ref[b].pages[i] for i in stay]
            # the freed pages go to the places that are open again
            p.kv.page_table[b, P - n[b]:] = out_e.freed[b, : n[b]]
        assert p.kv.lens.tolist() == [len(r) for r in p.ref]
        assert sorted(p.kv.page_table.flatten().tolist()) == list(range(seqs * P))


def test_graph_replays():
    """A decoding step captured once: replays with other tokens, lengths and weights in the buffers, eager work between them."""
    torch = _torch()
    from paper_2511_11608_amd import binding
    p = Pair(3, 2, 128, 6, "bf16", seed=50)
    p.append([100, 63, 250])
    H, counts = 8, [1, 1, 1]
    q, k, v = (torch.zeros(3, h, 128, dtype=torch.bfloat16, device="cuda") for h in (H, 2, 2))
    out, lse, mass = torch.empty_like(q), torch.empty(3, H, device="cuda"), torch.zeros(3, 2, 6, device="cuda")
    starts = starts_of(counts)
    ws = binding.alloc_kv_workspace(p.kv, H, 3, 1, 384)

    def step():
        p.kv.lens.add_(1)
        binding.slicer_kv_append(p.kv, k, v, starts, 1)
        binding.slicer_kv_attend(p.kv, q, starts, 1, 384, 0.1, out, ws, lse=lse, mass=mass, mass_decay=0.5)

    def feed():
        kk, vv, qq = p.rand(3, 2), p.rand(3, 2), p.rand(3, H)
        k.copy_(kk), v.copy_(vv), q.copy_(qq)
        for i, r in enumerate(p.ref):
            r.append(kk[i: i + 1], vv[i: i + 1])
        return qq

    qq = feed()
    old = mass.clone()
    step()
    torch.cuda.synchronize()
    p.check(counts, qq, 0.1, out, lse, mass=mass, old=old, decay=0.5)
    lens = p.kv.lens.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    p.kv.lens.copy_(lens)
    for _ in range(5):
        qq = feed()
        old = mass.clone()
        out.fill_(3.0)
        ws.fill_(0x5A)
        torch.cuda.synchronize()
        g.replay()
        torch.cuda.synchronize()
        p.check(counts, qq, 0.1, out, lse, mass=mass, old=old, decay=0.5)


def test_calls_on_streams_of_their_own():
    torch = _torch()
    pairs = [Pair(2, 2, 64, 20, "bf16", seed=i) for i in range(2)]
    for p in pairs:
        p.append([1000, 300])
    qs = [p.rand(90, 4) for p in pairs]
    outs, streams = [], [torch.cuda.Stream() for _ in pairs]
    qd = [q.cuda() for q in qs]
    torch.cuda.synchronize()
    for i, p in enumerate(pairs):
        with torch.cuda.stream(streams[i]):
            outs.append(p.attend([70, 20], qd[i], 0.1))
    torch.cuda.synchronize()
    for p, q, (o, l) in zip(pairs, qs, outs):
        p.check([70, 20], q, 0.1, o, l)


def test_a_cache_beyond_four_gigabytes():
    """Pages and query rows whose places do not fit 32 bits."""
    torch = _torch()
    from paper_2511_11608_amd import binding
    G, D = 8, 128
    n_pages = (5 << 30) // (G * 128 * D)
    p = Pair(2, G, D, 5, "bf16", seed=60)
    big = binding.alloc_kv(2, G, D, n_pages, 5)          # (260 tokens: five pages)
    big.page_table.copy_(n_pages - 1 - p.kv.page_table)
    p.kv = big
    p.append([130, 200])
    new = [1, 60]
    wide = 1 << 26                                       # elements from token to token
    store = torch.empty(61 * wide, dtype=torch.bfloat16, device="cuda")
    q = store.as_strided((61, 16, D), (wide, D, 1))
    q.copy_(p.rand(61, 16))
    k = store[4096:].as_strided((61, G, D), (wide, D, 1))
    v = store[8192:].as_strided((61, G, D), (wide, D, 1))
    k.copy_(p.rand(61, G))
    v.copy_(p.rand(61, G))
    at = 0
    for r, n in zip(p.ref, new):
        r.append(k[at: at + n], v[at: at + n])
        at += n
    p.sync_lens()
    p.b.slicer_kv_append(p.kv, k, v, starts_of(new), max(new))
    out, lse = p.attend(new, q, 0.08)
    p.check(new, q, 0.08, out, lse)
