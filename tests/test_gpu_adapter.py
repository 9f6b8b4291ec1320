"""GPU parity of the low-rank adapters against the fp64 form, through the C ABI, and their refusals.

Tolerances, derived: the update is two fp32 accumulations of products that are exact in fp32 (at most 8192 + 128 terms,
added by the tensor cores in blocks: below 2^-18 of the sums of absolute products), and A x is carried in 16 bits (bf16
output, 2^-16) or 24 (fp32).  With S = |scale| sum |B| (sum |A| |x|): |error| <= 2^-17 S + 2^-23 |Y| for fp32, and for
bf16 (2^-16 + 2^-17) S before the one rounding of the output (2^-8 |Y|)."""
import numpy as np
import pytest

from oracle import attention as oat
from paper_2607_02461_b200 import binding as B

pytestmark = pytest.mark.gpu


def _inputs(n, d, m, rank, adapters, dtype, seed, pad=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, d + pad, generator=g).bfloat16().cuda()[:, :d]
    a = (torch.randn(adapters, rank, d, generator=g) / np.sqrt(d)).bfloat16().cuda()
    b = (0.3 * torch.randn(adapters, m, rank, generator=g)).bfloat16().cuda()
    scale = (0.5 + torch.rand(adapters, generator=g)).cuda()
    base = torch.randn(n, m + pad, generator=g).to(dtype).cuda()[:, :m]
    return x, a, b, scale, base


def _tables(lens, ids):
    import torch
    return (torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda"),
            torch.tensor(ids, dtype=torch.int32, device="cuda"))


def _verify(out, x, a, b, scale, base, lens, ids):
    import torch
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    ref = oat.adapter_add(f(x), f(a), f(b), f(scale), lens, ids, f(base))
    size = oat.adapter_add(np.abs(f(x)), np.abs(f(a)), np.abs(f(b)), f(scale), lens, ids, np.zeros(base.shape))
    err = np.abs(f(out) - ref)
    tol = 2.0 ** -17 * size + 2.0 ** -23 * np.abs(ref) if out.dtype == torch.float32 else \
        (2.0 ** -16 + 2.0 ** -17) * size + 2.0 ** -8 * np.abs(ref) * 1.01
    assert np.all(err <= tol + 1e-30), (err / (tol + 1e-30)).max()
    at = 0
    for n, i in zip(lens, ids):                                  # rows without an adapter are the base, bit for bit
        if not 0 <= i < a.shape[0]:
            assert torch.equal(out[at:at + n], base[at:at + n])
        at += n


CASES = [
    # lengths, adapters of the segments, adapters, rank, d, m
    ([1], [0], 1, 8, 8, 8),
    ([1, 1, 1], [2, 0, 1], 3, 16, 200, 136),
    ([130], [0], 1, 32, 64, 72),
    ([5, 0, 300, 1, 127, 128], [1, 0, -1, 0, 1, 7], 2, 24, 1000, 520),
    ([129, 257], [1, 0], 2, 64, 3072, 328),
    ([64, 200], [0, 1], 2, 128, 1024, 264),
    ([40], [0], 1, 72, 328, 64),
    ([2, 3], [0, 1], 2, 40, 2048, 9216),
    ([700], [1], 2, 16, 16, 2048),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens,ids,adapters,rank,d,m", CASES)
def test_matches_fp64(lens, ids, adapters, rank, d, m, dtype):
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    x, a, b, scale, base = _inputs(sum(lens), d, m, rank, adapters, t, rank + d, pad=16)
    start, seg = _tables(lens, ids)
    out = B.oq_adapter_add(x, a, b, scale, start, seg, base)
    torch.cuda.synchronize()
    assert B.oq_device_status() == 0
    _verify(out, x, a, b, scale, base, lens, ids)
    # in place, into a wider buffer; a second call gives the same bits
    wide = torch.full((sum(lens), m + 24), 7.0, dtype=t, device="cuda")
    B.oq_adapter_add(x, a, b, scale, start, seg, base, out=wide[:, :m])
    assert torch.equal(wide[:, :m], out) and torch.all(wide[:, m:] == 7.0)
    held = base.clone()
    B.oq_adapter_add(x, a, b, scale, start, seg, held, out=held)
    assert torch.equal(held, out)


def test_many_small_segments_and_streams():
    import torch
    rng = np.random.default_rng(3)
    lens, ids = rng.integers(0, 4, 300).tolist(), rng.integers(-1, 5, 300).tolist()
    x, a, b, scale, base = _inputs(sum(lens), 256, 384, 16, 5, torch.bfloat16, 9)
    start, seg = _tables(lens, ids)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out = B.oq_adapter_add(x, a, b, scale, start, seg, base)
    side.synchronize()
    _verify(out, x, a, b, scale, base, lens, ids)


def test_tokens_in_no_segment_are_left_alone():
    import torch
    x, a, b, scale, base = _inputs(300, 128, 192, 16, 2, torch.float32, 4)
    start = torch.tensor([10, 60, 200], dtype=torch.int32, device="cuda")
    out = torch.full_like(base, 7.0)
    B.oq_adapter_add(x, a, b, scale, start, torch.tensor([1, 0], dtype=torch.int32, device="cuda"), base, out=out)
    assert torch.all(out[:10] == 7.0) and torch.all(out[200:] == 7.0)
    _verify(out[10:200], x[10:200], a, b, scale, base[10:200], [50, 140], [1, 0])


def test_segments_that_leave_most_tokens_out():
    """Few tiles where the sizes alone promise many: the products of a tile are cut into more parts."""
    import torch
    n, d, m = 20000, 4096, 192
    x, a, b, scale, base = _inputs(n, d, m, 16, 2, torch.bfloat16, 5)
    start = torch.tensor([700, 760, 960], dtype=torch.int32, device="cuda")
    held = base.clone()
    B.oq_adapter_add(x, a, b, scale, start, torch.tensor([1, 0], dtype=torch.int32, device="cuda"), held, out=held)
    assert torch.equal(held[:700], base[:700]) and torch.equal(held[960:], base[960:])
    _verify(held[700:960], x[700:960], a, b, scale, base[700:960], [60, 200], [1, 0])


def test_other_segments_values_do_not_leak():
    """NaN and infinities in a neighbouring segment's tokens or base stay there, although its rows share a tile's loads."""
    import torch
    lens, ids = [70, 20, 60], [0, 1, 0]
    x, a, b, scale, base = _inputs(150, 256, 320, 32, 2, torch.bfloat16, 6)
    start, seg = _tables(lens, ids)
    want = B.oq_adapter_add(x, a, b, scale, start, seg, base)
    x2, base2 = x.clone(), base.clone()
    x2[75], base2[80], x2[85] = float("nan"), float("inf"), float("inf")
    got = B.oq_adapter_add(x2, a, b, scale, start, seg, base2)
    assert torch.equal(got[:70], want[:70]) and torch.equal(got[90:], want[90:]) and torch.equal(got[70:75], want[70:75])
    assert torch.all(torch.isnan(got[75]))


def test_empty_and_refusals():
    import torch
    x, a, b, scale, base = _inputs(4, 64, 64, 16, 2, torch.bfloat16, 1)
    start, seg = _tables([4], [0])
    assert B.oq_adapter_add(x[:0], a, b, scale, start, seg, base[:0]).shape == (0, 64)

    def code(*args, **kw):
        with pytest.raises(B.OqError) as e:
            B.oq_adapter_add(*args, **kw)
        return e.value.code

    assert code(x, a[:, :12].contiguous(), b[:, :, :12].contiguous(), scale, start, seg, base) == 2           # rank 12
    big = _inputs(4, 64, 64, 136, 1, torch.bfloat16, 1)
    assert code(big[0], big[1], big[2], big[3], start, seg, big[4]) == 2                                      # rank 136
    assert code(x[:, :60], a[:, :, :60].contiguous(), b, scale, start, seg, base) == 2                        # d 60
    assert code(x, a, b, scale, start, seg, base[:, :32]) == 1
    assert code(x.float(), a, b, scale, start, seg, base) == 1
    assert code(x, a, b, scale.double(), start, seg, base) == 1
    assert code(x, a, b, scale, start.long(), seg, base) == 1
    assert code(x, a, b, scale, start, seg, base.half()) == 1
    assert code(x, a, b, scale, start, seg, base, out=base.float()) == 1
    wide = torch.zeros(4, 72, dtype=torch.bfloat16, device="cuda")
    assert code(wide[:, 4:68], a, b, scale, start, seg, base) == 3
    many = _inputs(300, 64, 64, 16, 2, torch.bfloat16, 1)
    small = torch.zeros(64, dtype=torch.uint8, device="cuda")
    assert code(*many[:4], *_tables([300], [0]), many[4], workspace=small) == 6
    odd = torch.zeros(4, 68, dtype=torch.bfloat16, device="cuda")
    assert code(x, a, b, scale, start, seg, odd[:, :64]) == 3


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n,segs,rank", [(1024, 64, 32), (5000, 300, 128), (24, 64, 16)])
def test_a_table_that_is_not_ascending_stays_inside_the_buffers(n, segs, rank, dtype):
    """Segments that name the same tokens again and again make more tiles than the workspace has places for."""
    import ctypes
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    d, m = 192, 136
    x, a, b, scale, base = _inputs(n + 70, d, m, rank, 2, t, 8)
    start = torch.tensor([0, n] * (segs // 2) + [0], dtype=torch.int32, device="cuda")
    seg = torch.arange(segs, dtype=torch.int32, device="cuda") % 2
    need = ctypes.c_size_t()
    assert B.lib().oq_adapter_workspace_bytes(n + 70, segs, d, rank, ctypes.byref(need)) == 0
    space = torch.full((need.value + (1 << 24),), 77, dtype=torch.uint8, device="cuda")
    out = torch.full((n + 70, m), 7.0, dtype=t, device="cuda")
    B.oq_adapter_add(x, a, b, scale, start, seg, base, out=out, workspace=space[:max(need.value, 16)])
    torch.cuda.synchronize()
    assert B.oq_device_status() == 0
    assert torch.all(space[max(need.value, 16):] == 77) and torch.all(out[n:] == 7.0)
    lens = [n]                                             # a sound call right after it
    _verify(B.oq_adapter_add(x[:n], a, b, scale, *_tables(lens, [1]), base[:n]), x[:n], a, b, scale, base[:n], lens, [1])


def test_tensors_off_the_device_and_odd_tables_are_refused():
    import torch
    x, a, b, scale, base = _inputs(300, 64, 64, 16, 2, torch.bfloat16, 1)
    start, seg = _tables([300], [0])
    args = dict(X=x, A=a, Bm=b, scale=scale, seg_start=start, seg_adapter=seg, base=base, out=torch.empty_like(base),
                workspace=torch.empty(1 << 24, dtype=torch.uint8, device="cuda"))
    B.oq_adapter_add(**args)
    bad = [{name: t.cpu()} for name, t in args.items()]
    bad += [dict(workspace=torch.empty(1 << 22, device="cuda")), dict(workspace=args["workspace"][:1].expand(1 << 24)),
            dict(seg_adapter=torch.zeros(1, 0, dtype=torch.int32, device="cuda"))]
    for change in bad:
        with pytest.raises(B.OqError) as e:
            B.oq_adapter_add(**{**args, **change})
        assert e.value.code == 1, change.keys()


def test_rows_too_far_apart_are_refused():
    """A leading dimension that 32 bits cannot hold is an error and not another leading dimension."""
    import torch
    x, a, b, scale, base = _inputs(2, 64, 64, 16, 2, torch.bfloat16, 1)
    far = torch.empty(2 ** 32 + 256, dtype=torch.bfloat16, device="cuda").as_strided((2, 64), (2 ** 32 + 64, 1))
    far.copy_(x)
    for args in ((far, base, None), (x, far, None), (x, base, far)):
        with pytest.raises(B.OqError) as e:
            B.oq_adapter_add(args[0], a, b, scale, *_tables([2], [0]), args[1], out=args[2])
        assert e.value.code == 2


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rank", [8, 24, 72, 128])
def test_infinities_come_out_the_same_on_every_path(rank, dtype):
    """An infinite token: A x is infinite with A's signs, and so is the output where B's signs agree, NaN where they do not; the other
    tokens of the tile do not notice.  As one segment (tensor cores) and as segments of one token (ordinary cores)."""
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    n, d, m = 40, 200, 136
    x, a, b, scale, base = _inputs(n, d, m, rank, 1, t, 77)
    a, b = a.abs() + 0.01, b.clone()
    b[:, :100] = b[:, :100].abs() + 0.01
    b[:, :30] *= -1                                        # columns of minus infinity, plus infinity, and both
    x = x.clone()
    x[3, 17], x[21, 199], x[30, 5], x[35, 0] = float("inf"), -float("inf"), float("nan"), float("inf")
    f = lambda v: v.double().cpu().numpy()  # noqa: E731
    with np.errstate(invalid="ignore"):
        ref = oat.adapter_add(f(x), f(a), f(b), f(scale), [n], [0], f(base))
    whole = B.oq_adapter_add(x, a, b, scale, *_tables([n], [0]), base)
    singles = B.oq_adapter_add(x, a, b, scale, *_tables([1] * n + [0] * 64 * n, [0] * (65 * n)), base)
    for got in (f(whole), f(singles)):
        assert np.array_equal(np.isnan(got), np.isnan(ref))
        assert np.array_equal(np.isposinf(got), np.isposinf(ref)) and np.array_equal(np.isneginf(got), np.isneginf(ref))
    rows = [i for i in range(n) if i not in (3, 21, 30, 35)]
    clean = _inputs(n, d, m, rank, 1, t, 77)[0].clone()
    want = B.oq_adapter_add(clean, a, b, scale, *_tables([n], [0]), base)
    assert torch.equal(whole[rows], want[rows])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("lens", [[250] + [0] * 63, [0] * 40 + [1, 9, 8, 17, 0, 100, 2] + [0] * 20, [3] * 60 + [0] * 9])
def test_long_segments_among_empty_ones(lens, dtype):
    """Few tokens a segment on average, all of them in a few: tiles of 8 tokens in clusters of their own."""
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    n, ids = sum(lens), [i % 4 - 1 for i in range(len(lens))]
    ids[0] = 2
    x, a, b, scale, base = _inputs(n, 520, 1096, 16, 3, t, 19, pad=16)
    start, seg = _tables(lens, ids)
    out = B.oq_adapter_add(x, a, b, scale, start, seg, base)
    torch.cuda.synchronize()
    assert B.oq_device_status() == 0
    _verify(out, x, a, b, scale, base, lens, ids)
    held = base.clone()
    B.oq_adapter_add(x, a, b, scale, start, seg, held, out=held)
    assert torch.equal(held, out)
