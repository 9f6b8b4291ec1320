"""GPU parity of the paged cache of quantized keys and values (write, read, attention over it) against the fp64 form, and its refusals.

Tolerances, derived.  Writes and reads are exact: a power of two times a float is exact, so an element has one rounding, and every cached
value is an exact bf16.  Attention: scores are fp32 sums of exact products (relative 2^-24 an addition, 128 of them and the scaling: below
2^-16 of sum |q k| <= 40 at the worst, 1e-6 typically), so the powers are right to 6e-4 at the worst and 1e-5 typically; the softmax weights
are rounded once to fp16 (half a unit: 2^-11), the output once to bf16 (2^-8).  Per element: |error| <= 2^-8 |out| + (2^-11 + 1e-4) sum_j w_j |v_j|, and lse to
1e-5 * (1 + |lse|).  Over a whole tensor the error of the output's rounding is at most 2^-8 / sqrt(3) in root mean square, that of the weights below a
tenth of it: the relative Frobenius error stays below 2.4e-3."""
import numpy as np
import pytest

from oracle import cache as oc
from paper_2607_02461_b200 import binding as B

pytestmark = pytest.mark.gpu

FRO = 2.4e-3
LSE = 1e-5


def _i32(x):
    import torch
    return torch.tensor(np.asarray(x), dtype=torch.int32, device="cuda")


def _starts(lens):
    return _i32(np.concatenate([[0], np.cumsum(lens)]))


class Pool:
    """Pages of some sequences, scattered over a pool in random order, as numpy arrays and on the device.  What is in no page of a sequence, and what
    lies behind its end, is random bytes or (nan=True) bytes that decode to NaN."""

    def __init__(self, lens, page, heads, d, kind, seed=0, spare=3, nan=False):
        g = np.random.default_rng(seed)
        held = [-(-n // page) for n in lens]
        order = g.permutation(sum(held) + spare)
        self.table = np.full((len(lens), max(held + [0]) + 1), -1, np.int64)
        at = 0
        for s, n in enumerate(held):
            self.table[s, :n] = order[at:at + n]
            at += n
        self.lens, self.kind, self.d, self.heads, self.page = list(lens), kind, d, heads, page
        shape = (sum(held) + spare, heads, oc.block_bytes(page, d, kind))
        self.pages = np.full(shape, 255, np.uint8) if nan else g.integers(0, 256, shape, dtype=np.uint8)

    def fill(self, seed=0):
        """Random keys and values for all tokens of all sequences, by the oracle."""
        g = np.random.default_rng(seed)
        n = sum(self.lens)
        k, v = g.standard_normal((2, n, self.heads, self.d))
        oc.write(self.pages, k, v * np.exp(g.standard_normal((n, self.heads, 1))), self.table, self.lens, self.lens, self.d, self.kind)
        return self

    def device(self):
        import torch
        return torch.from_numpy(self.pages.copy()).cuda(), _i32(self.table), _i32(self.lens)


def _bf16(shape, seed, spread=0.5):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * torch.exp(spread * torch.randn(*shape[:-1], 1, generator=g))).bfloat16()


def _f64(t):
    return t.double().cpu().numpy()


# ---------------------------------------------------------------------------------------------------- writing and reading

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind,d,page,heads", [("fp8", 128, 64, 5), ("fp8", 64, 16, 3), ("fp4", 128, 32, 1), ("fp4", 64, 256, 9), ("fp8", 128, 128, 40)])
@pytest.mark.parametrize("new,lens", [([1], [1]), ([37], [300]), ([5, 0, 70, 1], [5, 17, 200, 64]), ([33, 16], [40, 16])])
def test_write_and_read(new, lens, kind, d, page, heads, dtype):
    """Every byte of the pages, and both types of what is read back."""
    import torch
    pool = Pool(lens, page, heads, d, kind, seed=sum(new))
    pages, table, at = pool.device()
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    kv = _bf16((sum(new), 2 * heads, d), 3).to(t)
    if t == torch.float32:
        kv = kv * 1.01                                       # no bf16 any more
    kv = kv.cuda()
    B.oq_cache_write(pages, kv[:, :heads], kv[:, heads:], table, at, _starts(new), kind=kind)
    oc.write(pool.pages, _f64(kv[:, :heads]), _f64(kv[:, heads:]), pool.table, lens, new, d, kind)
    assert np.array_equal(pages.cpu().numpy(), pool.pages)
    k, v, _ = oc.read(pool.pages, pool.table, lens, new, d, kind)
    for out in (torch.bfloat16, torch.float32):
        got = B.oq_cache_read(pages, d, table, at, _starts(new), sum(new), kind=kind, out_dtype=out)
        assert np.array_equal(_f64(got[0]), k) and np.array_equal(_f64(got[1]), v)
    assert np.array_equal(pages.cpu().numpy(), pool.pages)


def _groups(kind):
    """Rows of 64 whose groups are at the borders of the scale, at ties, zero, tiny, and beyond the range."""
    g = np.random.default_rng(5)
    top, most = (448.0, 7) if kind == "fp8" else (6.0, 13)
    rows = []
    for e in (-16, -15, -14, -13, -1, 0, most - 1, most, most + 1):
        for x in (top * 2.0 ** e, np.nextafter(np.float32(top * 2.0 ** e), np.float32(np.inf)), np.nextafter(np.float32(top * 2.0 ** e), np.float32(0))):
            rows.append(np.float32(x) * g.uniform(-1, 1, 64).astype(np.float32))
            rows[-1][[7, 40]] = x, -x
    v = oc.values(kind)
    v = v[np.isfinite(v) & (v >= 0)]
    ties = np.resize((v[1:] + v[:-1]) / 2, 62)                # halfway between neighbours, the scale held by the largest value
    for sign in (1, -1):
        rows.append(np.concatenate([[top], sign * ties[:31], [top], sign * ties[31:]]).astype(np.float32))
    rows += [np.zeros(64, np.float32), -np.zeros(64, np.float32), np.full(64, 1e-40, np.float32), np.full(64, -3e38, np.float32),
             np.resize(np.float32([1e-45, -1e-38, 2.0 ** -24, 2.0 ** -23, 0.75 * 2.0 ** -23]), 64)]
    return np.stack(rows)


@pytest.mark.parametrize("kind", ["fp8", "fp4"])
def test_borders_of_the_formats(kind):
    import torch
    x = _groups(kind)
    pool = Pool([len(x)], 32, 1, 64, kind)
    pages, table, at = pool.device()
    k = torch.from_numpy(x)[:, None].cuda()
    v = torch.from_numpy(x[::-1].copy())[:, None].cuda()
    B.oq_cache_write(pages, k, v, table, at, kind=kind)
    oc.write(pool.pages, _f64(k), _f64(v), pool.table, pool.lens, pool.lens, 64, kind)
    assert np.array_equal(pages.cpu().numpy(), pool.pages)
    for a, b in zip(B.oq_cache_read(pages, 64, table, at, None, len(x), kind=kind, out_dtype=torch.bfloat16), oc.read(pool.pages, pool.table, pool.lens, pool.lens, 64, kind)):
        assert np.array_equal(_f64(a), b)                    # (bf16 holds them all)


@pytest.mark.parametrize("kind", ["fp8", "fp4"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_tokens_that_are_not_finite(kind, bad):
    """One such value in a key or a value marks that token of that head, and no other."""
    import torch
    pool = Pool([40], 16, 3, 128, kind)
    pages, table, at = pool.device()
    k, v = _bf16((40, 3, 128), 1).cuda(), _bf16((40, 3, 128), 2).cuda()
    k[7, 1, 100], v[20, 0, 0], v[39, 2, 127] = bad, bad, bad
    B.oq_cache_write(pages, k, v, table, at, kind=kind)
    oc.write(pool.pages, _f64(k), _f64(v), pool.table, [40], [40], 128, kind)
    assert np.array_equal(pages.cpu().numpy(), pool.pages)
    for got in B.oq_cache_read(pages, 128, table, at, None, 40, kind=kind):
        broken = torch.isnan(got).all(2).cpu().numpy()
        assert np.argwhere(broken).tolist() == [[7, 1], [20, 0], [39, 2]] and int(torch.isnan(got).sum()) == 3 * 128


@pytest.mark.parametrize("kind", ["fp8", "fp4"])
def test_tokens_without_a_place(kind):
    """More new tokens than the sequence is long, pages that are not there, lengths that the table cannot hold, tokens of no sequence: nothing else is
    touched, and what is read for them is 0 (left as it was where no sequence owns the row)."""
    import torch
    lens, new = [20, 100, -5, 70], [30, 100, 4, 40]
    pool = Pool([20, 100, 0, 70], 16, 2, 64, kind)
    pool.lens = lens
    pool.table[1, 2], pool.table[1, 3], pool.table[3, 4] = -1, len(pool.pages), 1 << 30
    pool.table = pool.table[:, :6].copy()                     # sequence 1 reaches behind its row: positions 0 .. 95
    pages, table, at = pool.device()
    start = _starts([3] + new)[1:].contiguous()               # rows 0 .. 2 belong to none, nor do the last four
    total = 3 + sum(new) + 4
    k, v = _bf16((total, 2, 64), 1).cuda(), _bf16((total, 2, 64), 2).cuda()
    B.oq_cache_write(pages, k, v, table, at, start, kind=kind)
    oc.write(pool.pages, _f64(k), _f64(v), pool.table, lens, new, 64, kind, first=3)
    assert np.array_equal(pages.cpu().numpy(), pool.pages)
    out = [torch.full((total, 2, 64), 7.0, device="cuda") for _ in range(2)]
    B.oq_cache_read(pages, 64, table, at, start, kind=kind, out_k=out[0], out_v=out[1])
    for got, ref in zip(out, oc.read(pool.pages, pool.table, lens, new, 64, kind)):
        assert bool((got[:3] == 7).all()) and bool((got[-4:] == 7).all())
        assert np.array_equal(_f64(got[3:-4]), ref)


def test_strides_and_single_outputs():
    """Broadcast heads, rows taken apart, outputs inside a larger tensor, only one of the two."""
    import torch
    pool = Pool([50], 16, 4, 64, "fp8")
    pages, table, at = pool.device()
    one, wide = _bf16((50, 1, 64), 1).cuda().expand(50, 4, 64), _bf16((100, 6, 80), 2).cuda()[::2, 1:5, 8:72]
    B.oq_cache_write(pages, one, wide, table[:, :5], at)
    oc.write(pool.pages, _f64(one), _f64(wide), pool.table, [50], [50], 64, "fp8")
    assert np.array_equal(pages.cpu().numpy(), pool.pages)
    k, v, _ = oc.read(pool.pages, pool.table, [50], [50], 64, "fp8")
    big = torch.full((50, 4, 2, 64), 3.0, device="cuda", dtype=torch.bfloat16)
    assert B.oq_cache_read(pages, 64, table, at, out_v=big[:, :, 1])[0] is None
    assert np.array_equal(_f64(big[:, :, 1]), v) and bool((big[:, :, 0] == 3).all())
    B.oq_cache_read(pages, 64, table, at, out_k=big[:, :, 0])
    assert np.array_equal(_f64(big[:, :, 0]), k) and np.array_equal(_f64(big[:, :, 1]), v)
    token = wide[:1].contiguous().expand(50, 4, 64)              # token stride 0
    B.oq_cache_write(pages, token, token, table, at)
    oc.write(pool.pages, _f64(token), _f64(token), pool.table, [50], [50], 64, "fp8")
    assert np.array_equal(pages.cpu().numpy(), pool.pages)


def test_pages_behind_four_gigabytes():
    """The last pages of a pool of 5 GB."""
    import torch
    size = oc.block_bytes(256, 128, "fp8") * 8
    n = 5 * (1 << 30) // size
    pages = torch.zeros((n, 8, size // 8), dtype=torch.uint8, device="cuda")
    table, lens = _i32([[n - 1, 3, n - 2]]), _i32([600])
    k, v = _bf16((600, 8, 128), 1).cuda(), _bf16((600, 8, 128), 2).cuda()
    B.oq_cache_write(pages, k, v, table, lens)
    small = np.zeros((4, 8, size // 8), np.uint8)
    oc.write(small, _f64(k[:, :1]).repeat(8, 1) * 0 + _f64(k), _f64(v), np.array([[0, 3, 1]]), [600], [600], 128, "fp8")
    for at, page in ((n - 1, 0), (3, 3), (n - 2, 1)):
        assert np.array_equal(pages[at].cpu().numpy(), small[page])
    ref = [torch.from_numpy(x).cuda() for x in oc.read(small, np.array([[0, 3, 1]]), [600], [600], 128, "fp8")[:2]]
    for got, want in zip(B.oq_cache_read(pages, 128, table, lens, None, 600), ref):
        assert torch.equal(got.double(), want)
    for tokens in (2, 100):                                   # both kernels
        q = _bf16((tokens, 8, 128), 3, 0.1).cuda()
        out = B.oq_cache_attention(q, pages, table, lens)
        here = torch.from_numpy(small).cuda()
        assert torch.equal(out, B.oq_cache_attention(q, here, _i32([[0, 3, 1]]), lens))
    del pages
    torch.cuda.empty_cache()


# ------------------------------------------------------------------------------------------------------------ attention

def _verify(q, pool, new, out, lse, **mask):
    ref, ref_lse, size = oc.attention(_f64(q), pool.pages, pool.table, pool.lens, new, pool.kind, **mask)
    got, got_lse = _f64(out), _f64(lse)
    assert np.array_equal(np.isnan(ref), np.isnan(got)) and np.array_equal(np.isnan(ref_lse), np.isnan(got_lse))
    none, nan = np.isneginf(ref_lse), np.isnan(ref_lse)
    assert np.array_equal(none, np.isneginf(got_lse))
    fine = ~none & ~nan
    assert np.all(np.abs(got_lse[fine] - ref_lse[fine]) <= LSE * (1 + np.abs(ref_lse[fine])))
    assert np.all(got[none.T] == 0)
    ref, got, size = (x[~nan.T] for x in (ref, got, size))
    err = np.abs(got - ref)
    assert np.all(err <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 1e-4) * size + 1e-30), err.max()
    if ref.size and np.linalg.norm(ref):
        assert np.linalg.norm(got - ref) <= FRO * np.linalg.norm(ref)


def _run(q, pool, new, **mask):
    import torch
    pages, table, lens = pool.device()
    out, lse = B.oq_cache_attention(q, pages, table, lens, _starts(new), kind=pool.kind, want_lse=True, **mask)
    torch.cuda.synchronize()
    assert B.oq_device_status() == 0
    return out, lse


MASKS = [dict(), dict(right=-1), dict(left=40), dict(left=100, right=30, sinks=5), dict(left=0, sinks=3), dict(left=150, right=-1, sinks=200),
         dict(left=3, right=129, sinks=1)]
SIZES = [(1, 1), (1, 129), (5, 3), (16, 16), (24, 130), (25, 130), (128, 128), (127, 257), (129, 128), (300, 411), (8, 700)]


@pytest.mark.parametrize("mask", MASKS, ids=str)
@pytest.mark.parametrize("kind,d,page", [("fp8", 128, 64), ("fp8", 64, 16), ("fp4", 128, 16), ("fp4", 64, 128)])
@pytest.mark.parametrize("nq,nk", SIZES)
def test_one_sequence(nq, nk, kind, d, page, mask):
    import torch
    pool = Pool([nk], page, 1, d, kind, seed=nq, nan=True).fill(nk)
    q = _bf16((nq, 2, d), nq + nk, 0.1).cuda()
    out, lse = _run(q, pool, [nq], **mask)
    _verify(q, pool, [nq], out, lse, **mask)
    pages, table, lens = pool.device()
    assert torch.equal(B.oq_cache_attention(q, pages, table, lens, kind=kind, **mask), out)     # without a table of starts: one sequence


@pytest.mark.parametrize("mask", [dict(), dict(left=60, right=0, sinks=20), dict(right=-1)], ids=str)
@pytest.mark.parametrize("kind,heads,kv_heads,page", [("fp8", 6, 2, 16), ("fp4", 3, 3, 32), ("fp8", 8, 1, 256)])
def test_packed_sequences(kind, heads, kv_heads, page, mask):
    """Sequences for both kernels in one call: long chunks, single tokens, none, more queries than keys, no keys."""
    new = [70, 0, 1, 300, 3, 9, 0, 33, 1, 5]
    lens = [70, 5, 400, 300, 0, 4, 0, 290, 17, 1000]
    pool = Pool(lens, page, kv_heads, 64, kind, seed=3, nan=True).fill(1)
    q = _bf16((sum(new), heads, 64), 7, 0.1).cuda()
    out, lse = _run(q, pool, new, **mask)
    _verify(q, pool, new, out, lse, **mask)
    for max_q in (300, 1):                                   # the hint, and one that is not true
        again, lse2 = _run(q, pool, new, max_q=max_q, **mask)
        _verify(q, pool, new, again, lse2, **mask)


@pytest.mark.parametrize("n_seqs", [33, 256])
@pytest.mark.parametrize("most", [1, 12])
def test_many_sequences(n_seqs, most):
    g = np.random.default_rng(n_seqs)
    new = g.integers(0, most + 1, n_seqs).tolist()
    lens = [n + int(k) for n, k in zip(new, g.integers(0, 300, n_seqs))]
    new[-1] += 40                                             # and one for the other kernel
    lens[-1] += 40
    pool = Pool(lens, 16, 1, 64, "fp8", nan=True).fill(2)
    q = _bf16((sum(new), 4, 64), 5, 0.1).cuda()
    out, lse = _run(q, pool, new)
    _verify(q, pool, new, out, lse)


@pytest.mark.parametrize("nq", [1, 3, 60])
@pytest.mark.parametrize("kind,heads,kv_heads,d", [("fp8", 2, 2, 128), ("fp4", 8, 2, 128), ("fp8", 3, 1, 64)])
def test_long_cache_is_cut_and_joined(nq, kind, heads, kv_heads, d):
    pool = Pool([9001], 64, kv_heads, d, kind, nan=True).fill(4)
    q = _bf16((nq, heads, d), 5, 0.1).cuda()
    for mask in (dict(), dict(left=3000, sinks=200)):
        out, lse = _run(q, pool, [nq], **mask)
        _verify(q, pool, [nq], out, lse, **mask)


@pytest.mark.parametrize("most", [384, 512, 528])
def test_tables_at_the_length_from_which_items_are_cut(most):
    """Up to 512 positions a row of the table, items are whole and no workspace is wanted; more than that, they are cut.  Many items a CTA and few."""
    for new, kv_heads in (([1, 2, 40], 1), ([1] * 20 + [30] * 12, 12)):
        lens = [most - 3 * i for i in range(len(new))]
        pool = Pool(lens, 16, kv_heads, 64, "fp8", nan=True).fill(most)
        pool.table = np.concatenate([pool.table, np.full((len(new), 40), -1)], 1)[:, :most // 16]
        q = _bf16((sum(new), 2 * kv_heads, 64), 5, 0.1).cuda()
        out, lse = _run(q, pool, new)
        _verify(q, pool, new, out, lse)


def test_more_blocks_than_threads_of_a_plan():
    """Blocks of queries that do not fit one round of the division of the work (chunks: 512 blocks of 256 rows; few rows: 256 blocks of 8)."""
    import torch
    pool = Pool([40], 16, 1, 64, "fp8", nan=True).fill(4)
    pages, table, lens = pool.device()
    q = _bf16((1, 8, 64), 5, 0.1).cuda().expand(20000, 8, 64)     # all queries alike, 160000 rows
    mask = dict(right=-1)
    for max_q in (0, 1):
        out, lse = B.oq_cache_attention(q, pages, table, lens, want_lse=True, max_q=max_q, **mask)
        first, first_lse = B.oq_cache_attention(q[:1], pages, table, lens, want_lse=True, **mask)
        assert float((out.float() - first.float()).abs().max()) <= 2.0 ** -7 * float(first.abs().max())
        assert float((lse - first_lse).abs().max()) <= 2 * LSE * (1 + float(first_lse.abs().max()))
        assert torch.equal(out, out[:1].expand_as(out)) or max_q == 0


@pytest.mark.parametrize("nq", [2, 50])
@pytest.mark.parametrize("kind", ["fp8", "fp4"])
def test_pages_that_are_not_there(nq, kind):
    """Holes inside what a query sees, given-back pages in front of it, all of it missing."""
    pool = Pool([500, 300, 200], 16, 2, 128, kind, nan=True).fill(1)
    pool.table[0, [3, 4, 17]] = -1, len(pool.pages), -7
    pool.table[1, :15] = -1
    pool.table[2] = -1
    new = [nq, nq, nq]
    q = _bf16((3 * nq, 4, 128), 5, 0.1).cuda()
    for mask in (dict(), dict(left=20, sinks=4)):
        out, lse = _run(q, pool, new, **mask)
        _verify(q, pool, new, out, lse, **mask)
        assert bool((out[2 * nq:] == 0).all()) and bool((lse[:, 2 * nq:] == -np.inf).all())


@pytest.mark.parametrize("nq", [4, 200])
def test_tokens_and_queries_that_are_not_finite(nq):
    """They reach what sees them and nothing else."""
    import torch
    pool = Pool([nq + 300], 16, 2, 64, "fp8", nan=True)
    pages, table, lens = pool.device()
    k, v = _bf16((nq + 300, 2, 64), 1, 0.1).cuda(), _bf16((nq + 300, 2, 64), 2).cuda()
    k[301, 0, 3], v[302, 1, 60] = float("nan"), float("inf")     # seen by queries from place 301 (302) on
    v[10, 0, 0] = float("nan")                                   # outside the window
    B.oq_cache_write(pages, k, v, table, lens)
    pool.pages = pages.cpu().numpy()
    q = _bf16((nq, 2, 64), 3, 0.1).cuda()
    q[3, 0, 5] = float("inf")
    mask = dict(left=100, right=0)
    out, lse = B.oq_cache_attention(q, pages, table, lens, want_lse=True, **mask)
    _verify(q, pool, [nq], out, lse, **mask)
    assert bool(torch.isfinite(out[0]).all()) and not bool(torch.isfinite(out[3, 0]).any())


@pytest.mark.parametrize("nq", [3, 40])
@pytest.mark.parametrize("size", [1e-30, 1e-3, 300.0, 1e6, 1e30])
def test_queries_of_any_size(nq, size):
    """Scores from nothing to 1e31: uniform weights at one end, the largest score's alone at the other."""
    pool = Pool([400], 64, 1, 64, "fp8", nan=True).fill(3)
    q = (_bf16((nq, 2, 64), 3, 0.1).double() * size).bfloat16().cuda()
    q[1] *= 1e-6                                                 # beside a row of another size
    out, lse = _run(q, pool, [nq])
    ref, ref_lse, weight = oc.attention(_f64(q), pool.pages, pool.table, pool.lens, [nq], "fp8")
    got, got_lse = _f64(out), _f64(lse)
    assert np.isfinite(got).all()
    # relative to the scores themselves, as an fp32 score is no more exact (2^-16 of sum |q k|): weights by as much in the exponent
    z = np.abs(_f64(q)).sum(-1).T * 40
    assert np.all(np.abs(got_lse - ref_lse) <= LSE + 2.0 ** -16 * z + LSE * np.abs(ref_lse))
    slack = np.minimum(2.0, np.expm1(np.minimum(2.0 ** -16 * z, 1.0)) * 2).T[..., None]
    top = np.abs(oc.read(pool.pages, pool.table, [400], [400], 64, "fp8")[1]).max()
    assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 1e-4) * weight + slack * top)


def test_rows_of_no_sequence_stay():
    import torch
    pool = Pool([60, 0, 200], 32, 1, 128, "fp8", nan=True).fill(3)
    pages, table, lens = pool.device()
    new, front, behind = [2, 1, 50], 3, 5
    q = _bf16((front + 53 + behind, 2, 128), 3, 0.1).cuda()
    out = torch.full_like(q, 9.0)
    start = _starts([front] + new)[1:].contiguous()
    got, lse = B.oq_cache_attention(q, pages, table, lens, start, out=out, want_lse=True)
    assert got is out and bool((out[:front] == 9).all()) and bool((out[-behind:] == 9).all())
    _verify(q[front:-behind], pool, new, out[front:-behind], lse[:, front:-behind])


@pytest.mark.parametrize("nq", [2, 90])
def test_strides_of_queries_and_results(nq):
    import torch
    pool = Pool([300], 64, 2, 64, "fp4", nan=True).fill(3)
    pages, table, lens = pool.device()
    q = _bf16((nq, 4, 64), 3, 0.1).cuda()
    ref = B.oq_cache_attention(q, pages, table, lens, kind="fp4")
    wide = torch.zeros((2 * nq, 5, 88), dtype=torch.bfloat16, device="cuda")
    wide[::2, 1:, 8:72] = q
    out = torch.zeros((nq, 4, 72), dtype=torch.bfloat16, device="cuda")[..., :64]
    assert torch.equal(B.oq_cache_attention(wide[::2, 1:, 8:72], pages, table, lens, kind="fp4", out=out), ref)
    one = q[:, :1].expand(nq, 4, 64)
    assert torch.equal(B.oq_cache_attention(one, pages, table, lens, kind="fp4"), B.oq_cache_attention(one.contiguous(), pages, table, lens, kind="fp4"))
    padded = torch.full((1, table.shape[1] + 3), 5, dtype=torch.int32, device="cuda")
    padded[:, :-3] = table
    assert torch.equal(B.oq_cache_attention(q, pages, padded[:, :-3], lens, kind="fp4"), ref)


def test_repeats_streams_and_workspaces():
    import torch
    pool = Pool([3000, 17, 900], 64, 2, 128, "fp8", nan=True).fill(3)
    pages, table, lens = pool.device()
    new = [1, 2, 200]
    q, start = _bf16((203, 4, 128), 3, 0.1).cuda(), _starts(new)
    ref, lse = B.oq_cache_attention(q, pages, table, lens, start, want_lse=True)
    _verify(q, pool, new, ref, lse)
    for _ in range(3):
        again = B.oq_cache_attention(q, pages, table, lens, start, want_lse=True)
        assert torch.equal(again[0], ref) and torch.equal(again[1], lse)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    outs = []
    for s in streams:                                            # two calls at once, a workspace each
        with torch.cuda.stream(s):
            outs.append([B.oq_cache_attention(q, pages, table, lens, start) for _ in range(4)])
    torch.cuda.synchronize()
    assert all(torch.equal(o, ref) for each in outs for o in each)
    space = torch.full((64 << 20,), 255, dtype=torch.uint8, device="cuda")       # whatever it holds; not on 32 bytes
    assert torch.equal(B.oq_cache_attention(q, pages, table, lens, start, workspace=space[16:]), ref)
    with pytest.raises(B.OqError) as e:
        B.oq_cache_attention(q, pages, table, lens, start, workspace=space[:4096])
    assert e.value.code == 6


def test_a_step_in_a_graph():
    """Write, attention and read captured once and replayed while the sequences grow."""
    import torch
    page, heads, kv_heads, d = 16, 4, 2, 64
    pool = Pool([100, 40], page, kv_heads, d, "fp8", spare=12, nan=True).fill(3)
    pool.table = np.concatenate([pool.table, np.full((2, 3), -1)], 1)
    used = set(pool.table[pool.table >= 0].tolist())
    free = iter([p for p in range(len(pool.pages)) if p not in used])
    pages, table, lens = pool.device()
    new = [1, 30]
    start = _starts(new)
    qkv = torch.zeros((31, heads + 2 * kv_heads, d), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros((31, heads, d), dtype=torch.bfloat16, device="cuda")
    read = [torch.zeros((31, kv_heads, d), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    def step():
        q, k, v = qkv.split([heads, kv_heads, kv_heads], 1)
        B.oq_cache_write(pages, k, v, table, lens, start)
        _, lse = B.oq_cache_attention(q, pages, table, lens, start, out=out, want_lse=True)
        B.oq_cache_read(pages, d, table, lens, start, out_k=read[0], out_v=read[1])
        return lse
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        lse = step()
    for turn in range(3):
        qkv.copy_(_bf16(qkv.shape, 10 + turn, 0.1))
        for s, n in enumerate(new):
            pool.lens[s] += n
            for x in range(-(-pool.lens[s] // page)):
                if pool.table[s, x] < 0:
                    pool.table[s, x] = next(free)
        table.copy_(_i32(pool.table))
        lens.copy_(_i32(pool.lens))
        pool.pages = pages.cpu().numpy()
        graph.replay()
        torch.cuda.synchronize()
        q, k, v = qkv.split([heads, kv_heads, kv_heads], 1)
        oc.write(pool.pages, _f64(k), _f64(v), pool.table, pool.lens, new, d, "fp8")
        assert np.array_equal(pages.cpu().numpy(), pool.pages)
        _verify(q, pool, new, out, lse)
        for got, want in zip(read, oc.read(pool.pages, pool.table, pool.lens, new, d, "fp8")):
            assert np.array_equal(_f64(got), want)


def test_refusals():
    import torch
    pool = Pool([50], 16, 2, 64, "fp8")
    pages, table, lens = pool.device()
    k = torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda")
    q, start = torch.zeros((4, 4, 64), dtype=torch.bfloat16, device="cuda"), _starts([4])
    def code(fn, *a, **kw):
        with pytest.raises(B.OqError) as e:
            fn(*a, **kw)
        return e.value.code
    w, r, at = B.oq_cache_write, B.oq_cache_read, B.oq_cache_attention
    assert code(w, pages, k, k[:3], table, lens) == 1
    assert code(w, pages, k, k.float(), table, lens) == 1
    assert code(w, pages, k.half(), k.half(), table, lens) == 1
    assert code(w, pages, k[:, :1], k[:, :1], table, lens) == 1
    assert code(w, pages, k.transpose(1, 2).contiguous().transpose(1, 2), k, table, lens) == 3
    assert code(w, pages, k, k, table, lens, kind="fp6") == 1
    assert code(w, pages, k, k, table.long(), lens) == 1
    assert code(w, pages, k, k, table, lens.long()) == 1
    assert code(w, pages, k, k, table[0], lens) == 1
    assert code(w, pages, k, k, table, _i32([50, 50])) == 1
    assert code(w, pages, k, k, table, lens, _starts([2, 2])) == 1
    assert code(w, pages, k, k, table, lens, start.cpu()) == 1
    assert code(w, pages.cpu(), k, k, table, lens) == 1
    assert code(w, pages[:, :, :-16], k, k, table, lens) == 1
    assert code(w, pages.transpose(0, 1), k, k, table, lens) == 1
    assert code(w, pages, k, k, torch.zeros((1, 10), dtype=torch.int32, device="cuda")[:, ::2], lens) == 3
    assert code(w, pages[:, :, :132 * 12].contiguous(), k, k, table, lens) == 2       # 12 tokens a page
    assert code(r, pages, 64, table, lens) == 1
    assert code(r, pages, 96, table, lens, None, 4) == 2
    assert code(r, pages, 64, table, lens, None, 4, out_dtype=torch.float16) == 1
    assert code(r, pages, 64, table, lens, None, 5, out_k=k) == 1
    assert code(r, pages, 64, table, lens, out_k=k, out_v=k.float()) == 1
    assert code(r, pages, 64, table, lens, out_k=k[:, :1].expand(4, 2, 64)) == 1
    assert code(at, q.float(), pages, table, lens) == 1
    assert code(at, q[:, :3].contiguous(), pages, table, lens) == 1
    assert code(at, q, pages, table, lens, sinks=-1) == 1
    assert code(at, q, pages, table, lens, left=1 << 40) == 1
    assert code(at, q, pages, table, lens, max_q=-1) == 1
    assert code(at, q, pages, table, lens, out=q.float()) == 1
    assert code(at, q, pages, table, lens, workspace=torch.empty(16, dtype=torch.int32, device="cuda")) == 1
    assert code(at, torch.zeros((4, 4, 64 * 2), dtype=torch.bfloat16, device="cuda")[..., ::2], pages, table, lens) == 3
    empty = at(q[:0], pages, table, lens, want_lse=True)
    assert empty[0].shape == (0, 4, 64) and empty[1].shape == (4, 0)
    w(pages, k[:0], k[:0], table, lens)
    assert r(pages, 64, table, lens, None, 0)[0].shape == (0, 2, 64)


@pytest.mark.parametrize("kind", ["fp8", "fp4"])
def test_a_page_size_that_the_pages_do_not_have_is_refused(kind):
    """Pages of 16 tokens of head_dim 128 are as long as pages of 32 of head_dim 64: who says what they hold is told."""
    import torch
    pages = B.oq_cache_alloc(4, 16, 2, 128, kind)
    table, lens = _i32([[0, 1, 2, 3]]), _i32([20])
    k = torch.zeros((20, 2, 64), dtype=torch.bfloat16, device="cuda")
    for call in (lambda **kw: B.oq_cache_write(pages, k, k, table, lens, kind=kind, **kw), lambda **kw: B.oq_cache_read(pages, 64, table, lens, None, 20, kind=kind, **kw),
                 lambda **kw: B.oq_cache_attention(k, pages, table, lens, kind=kind, **kw)):
        with pytest.raises(B.OqError) as e:
            call(page_size=16)
        assert e.value.code == 1
        call(page_size=32)
        call()


@pytest.mark.parametrize("n_seqs", [33, 256])
@pytest.mark.parametrize("most", [1, 12])
def test_many_sequences_in_long_tables(n_seqs, most):
    """More sequences than lanes where items are cut along their keys: short ones, some of thousands of keys, and one for the other kernel."""
    g = np.random.default_rng(n_seqs + most)
    new = g.integers(0, most + 1, n_seqs).tolist()
    lens = [n + int(k) for n, k in zip(new, g.integers(0, 200, n_seqs))]
    for s in (0, n_seqs // 2, n_seqs - 2):
        lens[s] += 2500
    new[-1] += 40
    lens[-1] += 900
    pool = Pool(lens, 16, 1, 64, "fp8", nan=True).fill(2)
    q = _bf16((sum(new), 4, 64), 5, 0.1).cuda()
    out, lse = _run(q, pool, new)
    _verify(q, pool, new, out, lse)


@pytest.mark.parametrize("mask", [dict(), dict(left=700, right=5, sinks=150)], ids=str)
def test_more_blocks_of_chunks_than_lanes(mask):
    """56 blocks of 256 rows of three sequences, cut along their keys, beside a single token."""
    new, lens = [1100, 1, 500, 150], [1500, 2000, 1300, 150]
    pool = Pool(lens, 64, 1, 64, "fp4", nan=True).fill(2)
    q = _bf16((sum(new), 8, 64), 5, 0.1).cuda()
    out, lse = _run(q, pool, new, **mask)
    _verify(q, pool, new, out, lse, **mask)


@pytest.mark.parametrize("max_q", [0, 1])
def test_more_blocks_than_threads_of_a_plan_that_cuts(max_q):
    """625 blocks of 256 rows (20000 of 8) over 2000 positions, cut along their keys."""
    pool = Pool([2000], 64, 1, 64, "fp8", nan=True).fill(4)
    pages, table, lens = pool.device()
    q = _bf16((1, 8, 64), 5, 0.1).cuda()
    many = q.expand(20000, 8, 64)                                # all queries alike
    out, lse = B.oq_cache_attention(many, pages, table, lens, want_lse=True, max_q=max_q, right=-1)
    _verify(many[:1], pool, [1], out[:1], lse[:, :1], right=-1)
    # (rows differ by where a cut falls alone: twice what one of them may be off by)
    ref, ref_lse, size = oc.attention(_f64(q), pool.pages, pool.table, pool.lens, [1], "fp8", right=-1)
    err = (out.double() - out[:1].double()).abs().amax(0).cpu().numpy()
    assert np.all(err <= 2 * (2.0 ** -8 * np.abs(ref[0]) + (2.0 ** -11 + 1e-4) * size[0]))
    assert np.all(np.abs(_f64(lse) - ref_lse) <= LSE * (1 + np.abs(ref_lse)))


@pytest.mark.parametrize("byte", [0x7F, 0xFF])
@pytest.mark.parametrize("kind,d", [("fp8", 64), ("fp4", 128)])
@pytest.mark.parametrize("nq", [1, 5, 60, 300])
@pytest.mark.parametrize("nk", [500, 1000])                      # items whole and cut
def test_places_that_nothing_was_written_to_outside_the_window(nk, nq, kind, d, byte):
    """A request taken over with its window alone: what lies before that, in pages that are there, may be any bytes, such as elements or scales that decode to NaN."""
    left, sinks = nk // 5 + 7, 20
    pool = Pool([nk], 32, 2, d, kind).fill(3)
    for p in range(sinks, nk - nq - left):
        for part in [x for block in pool.pages[pool.table[0, p // 32]] for x in oc._parts(block, 32, d, kind)]:
            part[p % 32] = byte
    q = _bf16((nq, 4, d), 5, 0.1).cuda()
    pool.table = pool.table[:, :-(-nk // 32)].copy()
    for mask in (dict(left=left, sinks=sinks), dict(left=left, right=-1, sinks=sinks)):
        out, lse = _run(q, pool, [nq], **mask)
        _verify(q, pool, [nq], out, lse, **mask)


@pytest.mark.parametrize("kind", ["fp8", "fp4"])
def test_a_shared_beginning_written_by_all_of_its_sequences(kind):
    """The same tokens to the same places from several sequences of one call, and further ones to pages of their own."""
    import torch
    lens = [100, 130, 64]
    pool = Pool(lens, 32, 2, 64, kind)
    pool.table[1, :2], pool.table[2, :2] = pool.table[0, :2], pool.table[0, :2]
    pages, table, at = pool.device()
    k, v = _bf16((64, 2, 64), 1), _bf16((64, 2, 64), 2)
    k, v = (torch.cat([x for n in lens for x in (own, _bf16((n - 64, 2, 64), 3 + n))]).cuda() for own in (k, v))
    for _ in range(3):
        B.oq_cache_write(pages, k, v, table, at, _starts(lens), kind=kind)
    oc.write(pool.pages, _f64(k), _f64(v), pool.table, lens, lens, 64, kind)
    assert np.array_equal(pages.cpu().numpy(), pool.pages)
