"""Softmax weights of attention over the paged cache where they span a wide range: a first key that takes nearly all the weight, scores far from
zero, scales at the ends of fp32.  Against the formula in fp64 over what the cache holds (reading it back is exact).

Tolerances, derived.  Weights are rounded to fp16, relative to 2^-11 of the largest one seen so far at the least: half a unit, 2^-11 of the weight, or half
the smallest fp16, 2^-25 * 2^-11 = 2^-36 of the largest weight, where that is more.  The output is rounded once to bf16 (2^-8), and 1e-4 of the weights is left for scores and
powers (fp32).  Per element: |error| <= 2^-8 |out| + (2^-11 + 1e-4) sum_j w_j |v_j| + 2^-36 max_j w_j sum_j |v_j|; lse to 1e-5 (1 + |lse|)."""
import numpy as np
import pytest
import torch

from paper_2607_02461_b200 import binding as B

pytestmark = pytest.mark.gpu

TOP = {"fp8": 57344.0, "fp4": 49152.0}


class Cache:
    """One sequence whose keys and values [n, kv_heads, d] are written into pages in falling order; width: positions of the table's row."""

    def __init__(self, k, v, kind, width=0, page=64):
        n, heads, self.d = k.shape
        held = -(-n // page)
        self.kind, self.pages = kind, B.oq_cache_alloc(held, page, heads, self.d, kind)
        table = list(range(held))[::-1] + [-1] * (max(width // page, held) - held)
        self.table, self.lens = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([table], [n]))
        B.oq_cache_write(self.pages, k, v, self.table, self.lens, kind=kind)
        self.k, self.v = (x.double() for x in B.oq_cache_read(self.pages, self.d, self.table, self.lens, None, n, kind=kind, out_dtype=torch.float32))

    def attend(self, q, **kw):
        out = B.oq_cache_attention(q, self.pages, self.table, self.lens, kind=self.kind, want_lse=True, **kw)
        torch.cuda.synchronize()
        assert B.oq_device_status() == 0
        return out

    def plain(self, q, left=-1, right=0, sinks=0, scale=0.0):
        """(out [T, H, D], lse [H, T], sum of weights times |v|, largest weight times the sum of |v|) in fp64."""
        n, heads, d = q.shape
        nk, kv_heads = self.k.shape[:2]
        group = heads // kv_heads
        k, v = (x.repeat_interleave(group, 1) for x in (self.k, self.v))
        z = (scale or d ** -0.5) * torch.einsum("ihd,jhd->hij", q.double(), k)
        at, j = torch.arange(n, device="cuda")[:, None] + nk - n, torch.arange(nk, device="cuda")[None]
        seen = (j <= at + right) if right >= 0 else torch.ones_like(j <= at)
        if left >= 0:
            seen &= (j >= at - left) | (j < sinks)
        z = z.masked_fill(~seen, -np.inf)
        lse = torch.logsumexp(z, 2)
        w = torch.softmax(z, 2)
        a = v.abs()
        ends = torch.einsum("hij,jhd->ihd", w, v), lse, torch.einsum("hij,jhd->ihd", w, a)
        return *ends, w.amax(2).T[..., None] * torch.einsum("ij,jhd->ihd", seen.double(), a)


def _verify(got, ref):
    out, lse, size, floor = ref
    assert bool(torch.isfinite(got[0]).all())
    err = (got[0].double() - out).abs()
    bound = 2.0 ** -8 * out.abs() + (2.0 ** -11 + 1e-4) * size + 2.0 ** -36 * floor + 1e-30
    worst = (err / bound).amax((0, 2))
    assert bool((err <= bound).all()), f"error over bound of each head: {worst.tolist()}"
    far = (got[1].double() - lse).abs() / (1 + lse.abs())
    assert bool((far <= 1e-5).all()), f"lse of each head: {far.amax(1).tolist()}"


# nk, positions of the table (up to 512 items are whole, beyond that they are cut along the keys)
LENGTHS = [(300, 320), (500, 40000), (32760, 32768), (131072, 131072)]


@pytest.mark.parametrize("where", ["first", "middle", "last"])
@pytest.mark.parametrize("nq", [1, 40])                       # both kernels
@pytest.mark.parametrize("kind,d", [("fp8", 64), ("fp4", 128)])
@pytest.mark.parametrize("nk,width", LENGTHS)
def test_a_key_that_takes_nearly_all_the_weight(nk, width, kind, d, nq, where):
    """One key is 2^gap times as heavy as each of the others and has a value of nothing, or a hundredth of theirs: the others make the result."""
    gaps = [4.0, 12.0, 16.0, 20.0, 22.0, 24.0, 25.0, 26.0, 28.0, 32.0]
    g = torch.Generator(device="cuda").manual_seed(nk + nq)
    at = {"first": 0, "middle": nk // 2, "last": nk - nq}[where]
    k = torch.randn((nk, 2, d), generator=g, device="cuda")
    k[:, :, 0] = 0.0
    k[at] = 0.0
    k[at, :, 0] = 1.0
    v = 1 + 0.25 * torch.randn((nk, 2, d), generator=g, device="cuda")
    v[at, 0] = 0.0
    v[at, 1] *= 0.01
    cache = Cache(k, v, kind, width)
    q = 0.3 * d ** -0.5 * torch.randn((nq, 2, len(gaps), d), generator=g, device="cuda")       # the others' scores: 0.3 in standard deviation
    q[..., 0] = torch.tensor(gaps, device="cuda") * np.log(2.0)
    q = q.flatten(1, 2).bfloat16()
    got, ref = cache.attend(q, scale=1.0), cache.plain(q, scale=1.0)
    _verify(got, ref)
    near = (torch.tensor(gaps * 2, device="cuda") <= 25).nonzero()[:, 0]
    diff = (got[0].double() - ref[0])[:, near]
    assert float(diff.norm() / ref[0][:, near].norm()) <= 2.4e-3


@pytest.mark.parametrize("nk,width", [(450, 512), (450, 40000), (6000, 6016), (40000, 40000)])
@pytest.mark.parametrize("nq", [1, 3, 60])
@pytest.mark.parametrize("kind", ["fp8", "fp4"])
def test_scores_far_from_zero(kind, nq, nk, width):
    """Scores up to 2^48 whose differences fp32 holds exactly, so the weights are known: the largest among the first keys, in the middle or among the last, hugely
    negative ones before and behind ordinary ones, and slowly rising ones far from zero (by whole numbers, all of them small beside their common part)."""
    big, third = TOP[kind], nk // 3
    steps = torch.tensor([0.0, 1.0, 2.0, 3.0, 4.0, 6.0])
    j = torch.arange(nk)
    k = torch.zeros((nk, 1, 64))
    first, middle, last = j < third, (j >= third) & (j < nk - third), j >= nk - third
    k[:, 0, 0] = big * (first.float() - last.float())
    k[:, 0, 33] = -big * (~middle).float()
    k[middle, 0, 1] = -steps[j[middle] % 6]
    ramp = torch.zeros((nk, 1, 64))
    ramp[:, 0, 0] = 2048.0
    ramp[:, 0, 33] = steps[(j * 6 // nk).long()]               # rising with the place ...
    ramp[:, 0, 34] = steps[(5 - j * 6 // nk).long()]           # ... and falling
    v = torch.randn((nk, 2, 64), generator=torch.Generator().manual_seed(nk))
    cache = Cache(torch.cat((k, ramp), 1).cuda(), v.cuda(), kind, width)
    # a row: coordinates of the query.  (scale 1/8: a query of 8 makes a key's number the score)
    rows = [{0: 2.0 ** 20, 1: 8}, {0: -2.0 ** 20, 1: 8}, {33: 2.0 ** 20, 1: 8}, {33: -2.0 ** 20, 1: 8}, {33: 2.0 ** 36, 1: 8}, {33: 2.0 ** 10, 1: 8}, {33: 2.0 ** 14, 1: 24},
            {0: 2.0 ** 30, 33: 2.0 ** 30}]
    slow = [{0: 2.0 ** 4, 33: 8}, {0: -2.0 ** 4, 33: 24}, {0: 2.0 ** 10, 33: 8}, {0: 2.0 ** 10, 33: 24}, {0: -2.0 ** 10, 34: 24}, {0: 2.0 ** 14, 33: 8}, {0: -2.0 ** 14, 34: 8},
            {0: 2.0 ** 20, 33: 128}]
    q = torch.zeros((nq, 16, 64))
    for h, row in enumerate(rows + slow):
        for c, x in row.items():
            q[:, h, c] = x
    q = q.bfloat16().cuda()
    for mask in (dict(right=-1), dict()):
        got, ref = cache.attend(q, **mask), cache.plain(q, **mask)
        _verify(got, ref)


@pytest.mark.parametrize("nk,width", [(200, 256), (3000, 3008)])
@pytest.mark.parametrize("nq", [2, 40])
def test_scales_at_the_ends_of_fp32(nq, nk, width):
    """Queries of zero, tiny and huge ones, with scales from 1e-38 to 9e29: uniform weights where the scores are all alike, however small or large the factor is."""
    g = torch.Generator().manual_seed(nk)
    k, v = torch.randn((nk, 1, 64), generator=g), torch.randn((nk, 1, 64), generator=g)
    cache, flat = Cache(k.cuda(), v.cuda(), "fp8", width), Cache(0 * k.cuda(), v.cuda(), "fp8", width)
    q = torch.randn((nq, 4, 64), generator=g)
    q[:, 0] = 0.0
    q[:, 1] *= 1e-36
    q[:, 2] *= 1e-12
    mask = dict(left=nk // 2, sinks=3)
    for scale in (1e-38, 1e-13, 1e-11):
        x = q.bfloat16().cuda()
        _verify(cache.attend(x, scale=scale, **mask), cache.plain(x, scale=scale, **mask))
    q[:, 3] *= 1e30
    x = q.bfloat16().cuda()
    for scale in (1.0, 9e29):                                  # keys of zero: all scores are 0
        _verify(flat.attend(x, scale=scale, **mask), flat.plain(x, scale=scale, **mask))
