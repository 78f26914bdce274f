"""The attention cache in 8 bits at the ends of its range: pages that are not there, scores and values far from one, lengths that are taken back.

Scores here are exact: keys are whole numbers (a page's largest magnitude is 127, its scale 1) and a query is a power of two in one element, so that equal
scores are equal in 32 bits too and others are so far apart that their weights are 0.  What is left of a tolerance is half a step of the output's
type, the probabilities' rounding (fp16 2^-11; two fp16 numbers 2^-21) and fp32 sums over the tokens, length * 2^-24, the last two times sum p |v|: a weight of
0 allows nothing, however large its value.
"""
import numpy as np
import pytest

from tests.kv_ref import PAGE
from tests.test_gpu_kv import Pair, starts_of

pytestmark = pytest.mark.gpu


def _torch():
    import torch
    return torch


def check_exact_scores(p, counts, q, scale, out, lse, mass=None):
    torch = _torch()
    fi, at = torch.finfo(q.dtype), 0
    p_bits = 2.0 ** -11 if q.dtype == torch.bfloat16 else 2.0 ** -21
    for i, (r, n) in enumerate(zip(p.ref, counts)):
        o, l, w, absv, _, _ = r.attend(q[at: at + n], scale)
        got, got_l = out[at: at + n].double().cpu().numpy(), lse[at: at + n].double().cpu().numpy()
        at += n
        tol = fi.eps / 2 * (1 + 2.0 ** -7) * np.abs(o) + fi.eps / 2 * fi.smallest_normal + (p_bits + (len(r) + 64) * 2.0 ** -24) * absv
        assert np.array_equal(np.isnan(o), np.isnan(got)), (i, np.argwhere(np.isnan(o) != np.isnan(got))[:4])
        wrong = ~np.isnan(o) & ~(np.abs(got - o) <= tol)
        assert not wrong.any(), (i, np.argwhere(wrong)[:4], got[wrong][:4], o[wrong][:4])
        # scale times log2(e), its product with a score, and the way back: six roundings of 2^-24
        assert np.array_equal(np.isnan(l), np.isnan(got_l)), i
        fine = ~np.isnan(l)
        assert (np.abs(got_l - l)[fine] <= 6 * 2.0 ** -24 * np.abs(l)[fine] + 2.0 ** -20).all(), (i, np.abs(got_l - l)[fine].max())
        if mass is not None and n:
            g = mass[i].double().cpu().numpy()[:, : w.shape[1]]
            assert (np.abs(g - w) <= ((len(r) + n * q.shape[1] + 64) * 2.0 ** -24 + 2.0 ** -21) * w + 2.0 ** -126).all(), (i, g, w)      # (a weight below fp32's range is 0)


def whole_keys(codes, dim, dtype):
    """Keys whose element 0 is the token's code and whose element 1 is 127."""
    torch = _torch()
    k = torch.zeros(len(codes), 1, dim)
    k[:, 0, 0] = torch.as_tensor(codes, dtype=torch.float32)
    k[:, 0, 1] = 127.0
    return k.to(dtype)


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


ROWS = [(1, 400), (4, 400), (16, 700), (70, 400), (130, 0), (300, 900)]        # new tokens before 2 heads, tokens before them


def large_scores(rows, exponent, dtype, rising):
    torch = _torch()
    n, past = rows
    p = Pair(1, 1, 40, -(-(n + past) // PAGE), dtype, seed=n + exponent)
    rng = np.random.default_rng(exponent + n)
    total = n + past
    # a narrow range of codes that moves on with the tokens: the maximum changes from page to page
    codes = np.linspace(-100, 100, total).astype(int) * (1 if rising else -1) + rng.integers(-20, 21, total)
    k, v = whole_keys(codes, 40, p.dt), p.rand(total, 1)
    if past:
        p.append([past], k[:past], v[:past])
    p.append([n], k[past:], v[past:])
    q = torch.zeros(n, 2, 40)
    q[:, 0, 0], q[:, 1, 0] = 2.0 ** exponent, -2.0 ** exponent
    q = q.to(p.dt)
    mass = torch.zeros(1, 1, p.kv.max_pages, device="cuda")
    out, lse = p.attend([n], q.cuda(), 0.125, mass=mass)
    check_exact_scores(p, [n], q, 0.125, out, lse, mass)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("exponent", [14, 20, 23, 24, 26, 30, 60, 100])
@pytest.mark.parametrize("rows", [r for r in ROWS if r[0] <= 32])
def test_large_scores_of_split_rows(rows, exponent, dtype):
    for rising in (True, False):
        large_scores(rows, exponent, dtype, rising)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("exponent", [14, 20, 23, 24, 26, 30, 60, 100])
@pytest.mark.parametrize("rows", [r for r in ROWS if r[0] > 32])
def test_large_scores_of_prompts(rows, exponent, dtype):
    for rising in (True, False):
        large_scores(rows, exponent, dtype, rising)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [3, 100, 200])
@pytest.mark.parametrize("order", ["LSTZ", "SLTZ", "STLZ", "TSZL", "ZTLS", "LTEZ", "TLZE"])
def test_values_of_any_scale(order, n, dtype):
    """Pages whose values are far apart: L large (2^90) under a score between the others', S (2^-7) and T (2^-95) under the scores that queries look for,
    Z zeros, E as large as L with S's score, zeros in one element: every row is made of the pages that it has weight on, in every element."""
    torch = _torch()
    p = Pair(1, 1, 32, 4 + -(-n // PAGE), dtype, seed=n)
    codes = {"L": 0, "S": 50, "T": -50, "Z": 3, "E": 50}
    size = {"L": 2.0 ** 90, "S": 2.0 ** -7, "T": 2.0 ** -95, "Z": 0.0, "E": 2.0 ** 90}
    k = whole_keys(np.concatenate([np.full(PAGE, codes[c]) for c in order] + [np.zeros(n)]), 32, p.dt)
    v = p.rand(4 * PAGE + n, 1).float().clamp(-4.0, 4.0)
    for i, c in enumerate(order):
        v[i * PAGE: i * PAGE + PAGE] *= size[c]
        if c == "E":
            v[i * PAGE: i * PAGE + PAGE, 0, 5] = 0.0
    if "E" in order:                                        # (its partner is S's place in the tokens that follow)
        k[4 * PAGE:, 0, 0] = 50.0
    v = v.to(p.dt)
    p.append([4 * PAGE], k[: 4 * PAGE], v[: 4 * PAGE])
    p.append([n], k[4 * PAGE:], v[4 * PAGE:])
    q = torch.zeros(n, 2, 32)
    q[:, 0, 0], q[:, 1, 0] = 32.0, -32.0                   # 200 between L and what is looked for
    q = q.to(p.dt)
    mass = torch.zeros(1, 1, p.kv.max_pages, device="cuda")
    out, lse = p.attend([n], q.cuda(), 0.125, mass=mass)
    check_exact_scores(p, [n], q, 0.125, out, lse, mass)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n", [1, 70])
@pytest.mark.parametrize("max_len", [0, 70000])
def test_the_largest_values_of_a_long_cache(max_len, n, dtype):
    """Sums of 70000 values of 2^95, before they are divided by the weights' sum: a value times the tokens is below 2^112; the first page's scores are 4 below the others', too little for a new maximum
    of a prompt's rows."""
    torch = _torch()
    p = Pair(1, 1, 8, -(-70000 // PAGE), dtype, seed=n)
    v = torch.full((70000, 1, 8), 2.0 ** 95).to(p.dt)
    k, q = torch.zeros(70000, 1, 8), torch.zeros(n, 2, 8)
    k[PAGE:, 0, 0], q[:, :, 0] = 16.0, 1.0
    k, q = k.to(p.dt), q.to(p.dt)
    for first, count in ((0, 70000 - n), (70000 - n, n)):
        p.kv.lens.fill_(first + count)
        p.b.slicer_kv_append(p.kv, k[first: first + count].cuda(), v[first: first + count].cuda(), starts_of([count]), count)
    p.ref[0].open = [None] * 70000                          # (only their number)
    for causal in (True, False):
        out, _ = p.attend([n], q.cuda(), 0.25, causal, max_len=max_len)
        # half a step, the probabilities' rounding, and sums in fp32, of the values and of the weights
        off = torch.finfo(p.dt).eps / 2 + (2.0 ** -11 if dtype == "bf16" else 2.0 ** -21) + 2 * 70064 * 2.0 ** -24
        assert (np.abs(out.double().cpu().numpy() / 2.0 ** 95 - 1.0) <= off).all()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [8, 32, 64, 96, 128, 160, 192, 224, 256])
def test_prompts_outside_the_pipeline_at_every_head_size(dim, dtype):
    """Steep scores and value scales far apart at once, whole pages and a tail, pages shared out and not."""
    torch = _torch()
    p = Pair(1, 1, dim, 8, dtype, seed=dim)
    total = 7 * PAGE + 9
    rng = np.random.default_rng(dim)
    k = whole_keys(rng.integers(-120, 121, total), dim, p.dt)
    v = p.rand(total, 1).float().clamp(-4.0, 4.0)
    for i, e in enumerate((0, 70, -70, 3, 0, 40, 0)):
        v[i * PAGE: i * PAGE + PAGE] *= 2.0 ** e
    v = v.to(p.dt)
    n = 100
    p.append([total - n], k[: total - n], v[: total - n])
    p.append([n], k[total - n:], v[total - n:])
    q = torch.zeros(n, 2, dim)
    q[:, 0, 0], q[:, 1, 0] = 2.0 ** 24, -(2.0 ** 16)
    q = q.to(p.dt)
    for max_len in (None, 0):
        mass = torch.zeros(1, 1, 8, device="cuda")
        out, lse = p.attend([n], q.cuda(), 0.125, mass=mass, max_len=max_len)
        check_exact_scores(p, [n], q, 0.125, out, lse, mass)


def test_steep_tiles_leave_the_others_as_they_are():
    """More row tiles than workgroups that keep weights: a workgroup goes from steep tiles to ordinary ones.  Sequences of ordinary scores have the same bits whatever
    the others' scores are, and steep ones are right."""
    torch = _torch()
    seqs, G, R, D, n = 44, 3, 2, 16, 260
    got = []
    for steep in (False, True):
        p = Pair(seqs, G, D, 6, "bf16", seed=2)
        k, v, q = p.rand(seqs * n, G), p.rand(seqs * n, G), p.rand(seqs * n, G * R)
        codes = np.random.default_rng(1).integers(-120, 121, n)
        for b in range(0, seqs, 3):                         # one sequence of three
            if steep:
                k[b * n: b * n + n] = whole_keys(codes, D, p.dt)
                q[b * n: b * n + n] = 0.0
                q[b * n: b * n + n, :, 0] = 2.0 ** 26
        p.append([n] * seqs, k, v)
        mass = torch.zeros(seqs, G, 6, device="cuda")
        out, lse = p.attend([n] * seqs, q.cuda(), 0.125, mass=mass)
        got.append((out.view(seqs, n, G * R, D), lse.view(seqs, n, G * R), mass))
        if steep:
            for b in (0, 21, 42):
                one, refs = slice(b * n, b * n + n), p.ref
                p.ref = [refs[b]]
                check_exact_scores(p, [n], q[one], 0.125, out[one], lse[one], mass[b: b + 1])
                p.ref = refs
    ordinary = [b for b in range(seqs) if b % 3]
    assert all(torch.equal(a[ordinary], c[ordinary]) for a, c in zip(*got))
    assert not torch.equal(got[0][0][0], got[1][0][0])
