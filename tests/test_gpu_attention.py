"""GPU parity of windowed attention against the fp64 form, through the C ABI, and its refusals.

Tolerances, derived: the scores are fp32 sums of exact products of bf16 numbers (relative 2^-24 per addition, 128 of
them: below 2^-17 of sum |q k| <= 40 in these inputs, so the powers are right to 4e-4 at the worst and 1e-6 typically);
the softmax weights are rounded once to bf16 (unit roundoff 2^-8) and so is the output.  Per element:
|error| <= 2^-8 |out| + (2^-8 + 1e-3) sum_j w_j |v_j|, and lse to 1e-5 * (1 + |lse|).
Over a whole tensor both roundings are independent and of root mean square 2^-8 / (2 sqrt(3)) * (1.0 .. 1.4): the
relative Frobenius error stays below 4e-3."""
import numpy as np
import pytest

from oracle import attention as oat
from paper_2607_02461_b200 import binding as B

pytestmark = pytest.mark.gpu

FRO = 4e-3
LSE = 1e-5


def _inputs(tq, tk, h, hk, d, seed):
    import torch
    g = torch.Generator().manual_seed(seed)
    q = torch.randn(tq, h, d, generator=g) * (0.6 + torch.rand(1, h, 1, generator=g))
    k = torch.randn(tk, hk, d, generator=g)
    v = torch.randn(tk, hk, d, generator=g)
    return [t.bfloat16().cuda() for t in (q, k, v)]


def _starts(lens):
    import torch
    return torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")


def _verify(q, k, v, ql, kl, out, lse, **mask):
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    ref, ref_lse = oat.attention(f(q), f(k), f(v), ql, kl, **mask)
    size, _ = oat.attention(f(q), f(k), np.abs(f(v)), ql, kl, **mask)
    got, got_lse = f(out), f(lse)
    none = np.isneginf(ref_lse)
    assert np.array_equal(none, np.isneginf(got_lse))
    assert np.all(np.abs(got_lse[~none] - ref_lse[~none]) <= LSE * (1 + np.abs(ref_lse[~none])))
    assert np.all(got[none.T] == 0)
    err = np.abs(got - ref)
    assert np.all(err <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 1e-3) * size + 1e-30), (err.max(), np.unravel_index(err.argmax(), err.shape))
    if ref.size and np.linalg.norm(ref):
        assert np.linalg.norm(got - ref) <= FRO * np.linalg.norm(ref)


def _run(q, k, v, ql, kl, **mask):
    import torch
    out, lse = B.oq_attention(q, k, v, _starts(ql), _starts(kl), want_lse=True, **mask)
    torch.cuda.synchronize()
    assert B.oq_device_status() == 0
    return out, lse


MASKS = [dict(), dict(right=0), dict(left=40, right=0), dict(left=100, right=30, sinks=5), dict(left=0, right=0, sinks=3),
         dict(left=150, sinks=200), dict(left=3, right=129, sinks=1)]


@pytest.mark.parametrize("mask", MASKS, ids=str)
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("nq,nk", [(1, 1), (1, 129), (5, 3), (128, 128), (127, 257), (129, 128), (300, 411), (513, 40)])
def test_one_sequence(nq, nk, d, mask):
    import torch
    q, k, v = _inputs(nq, nk, 2, 1, d, nq + nk)
    out, lse = _run(q, k, v, [nq], [nk], **mask)
    _verify(q, k, v, [nq], [nk], out, lse, **mask)
    again = B.oq_attention(q, k, v, **mask)              # without tables: one sequence
    assert torch.equal(again, out)


@pytest.mark.parametrize("mask", MASKS[:5], ids=str)
def test_packed_sequences(mask):
    ql, kl = [70, 0, 1, 300, 128, 9, 0, 33], [70, 5, 400, 300, 0, 4, 0, 290]
    q, k, v = _inputs(sum(ql), sum(kl), 3, 3, 128, 7)
    out, lse = _run(q, k, v, ql, kl, **mask)
    _verify(q, k, v, ql, kl, out, lse, **mask)


@pytest.mark.parametrize("mask", [dict(), dict(right=0), dict(left=700, right=0, sinks=4), dict(left=20, right=0)], ids=str)
@pytest.mark.parametrize("ql,kl,h,hk,d", [([1], [5000], 8, 8, 128), ([3], [3001], 6, 2, 64), ([1, 4, 2], [4000, 17, 2500], 4, 1, 128),
                                          ([200], [6000], 2, 2, 128)])
def test_few_queries_are_split_and_joined(ql, kl, h, hk, d, mask):
    q, k, v = _inputs(sum(ql), sum(kl), h, hk, d, 11)
    out, lse = _run(q, k, v, ql, kl, **mask)
    _verify(q, k, v, ql, kl, out, lse, **mask)


def test_many_sequences_and_heads():
    rng = np.random.default_rng(5)
    ql = rng.integers(0, 20, 256).tolist()
    kl = [int(a + rng.integers(0, 30)) for a in ql]
    q, k, v = _inputs(sum(ql), sum(kl), 4, 2, 64, 13)
    out, lse = _run(q, k, v, ql, kl, right=0)
    _verify(q, k, v, ql, kl, out, lse, right=0)


def test_scores_that_grow_rescale_the_sums():
    """Keys ordered by score, so that the running maximum moves in every tile, up and down by hundreds."""
    import torch
    nq, nk, d = 150, 1100, 128
    q, k, v = _inputs(nq, nk, 2, 2, d, 3)
    for order in (1, -1):
        ramp = torch.linspace(-1, 1, nk, device="cuda")[:, None, None] * order
        kk = (k.float() * 0.1 + ramp * 3 * torch.sign(q[0].float())[None]).bfloat16()
        qq = (q.float().abs() * torch.sign(q[0].float())[None]).bfloat16()
        for mask in (dict(), dict(left=300, right=100, sinks=50)):
            out, lse = _run(qq, kk, v, [nq], [nk], scale=0.5, **mask)
            # scores reach sum |q k| ~ 300 * 0.5, so the fp32 sums and the fp32 product with log2(e) are off by up to 2^-16
            # of that in the exponent
            f = lambda t: t.double().cpu().numpy()  # noqa: E731
            ref, ref_lse = oat.attention(f(qq), f(kk), f(v), [nq], [nk], scale=0.5, **mask)
            size, _ = oat.attention(f(qq), f(kk), np.abs(f(v)), [nq], [nk], scale=0.5, **mask)
            assert np.all(np.abs(f(lse) - ref_lse) <= 1e-5 * (1 + np.abs(ref_lse)))
            assert np.all(np.abs(f(out) - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 6e-3) * size)


@pytest.mark.parametrize("nq,nk", [(200, 200), (2, 3000)])
def test_nothing_unseen_reaches_a_row(nq, nk):
    """NaN, infinities and the type's lowest value in keys and values that a row does not see change nothing."""
    import torch
    mask = dict(left=60, right=0, sinks=3)
    q, k, v = _inputs(nq, nk, 2, 2, 128, 21)
    clean, clean_lse = _run(q, k, v, [nq], [nk], **mask)
    at = nk - 20                                    # seen by the last rows of the sequence alone (causal)
    lowest = torch.finfo(torch.bfloat16).min
    for what in (float("nan"), float("inf"), -float("inf"), lowest):
        kk, vv = k.clone(), v.clone()
        kk[at], vv[at] = what, what
        out, lse = _run(q, kk, vv, [nq], [nk], **mask)
        sees = oat.visible(nq, nk, **mask)[:, at]
        keep = torch.from_numpy(~sees).cuda()
        err = (out[keep].float() - clean[keep].float()).abs()
        assert torch.all(torch.isfinite(out[keep]))
        assert torch.all(err <= 2.0 ** -7 * (clean[keep].float().abs() + 1)) and torch.allclose(lse[:, keep], clean_lse[:, keep], rtol=1e-5, atol=1e-5)
        if what != what:
            assert torch.all(torch.isnan(out[~keep]))
    # the same beyond a sequence's end: its neighbour's keys, and rows of the buffer past the last sequence
    big_k, big_v = torch.full((nk + 300, 2, 128), float("nan"), dtype=torch.bfloat16, device="cuda"), torch.full((nk + 300, 2, 128), float("nan"), dtype=torch.bfloat16, device="cuda")
    big_k[150:150 + nk], big_v[150:150 + nk] = k, v
    qs = torch.tensor([0, 0, nq, nq], dtype=torch.int32, device="cuda")
    ks = torch.tensor([0, 150, 150 + nk, 300 + nk], dtype=torch.int32, device="cuda")
    out, lse = B.oq_attention(q, big_k, big_v, qs, ks, want_lse=True, **mask)
    assert torch.all(torch.isfinite(out))
    err = (out.float() - clean.float()).abs()
    assert torch.all(err <= 2.0 ** -7 * (clean.float().abs() + 1)) and torch.allclose(lse, clean_lse, rtol=1e-5, atol=1e-5)


def test_strides_heads_first_and_streams():
    import torch
    nq, nk, h, hk, d = 260, 300, 4, 2, 128
    q, k, v = _inputs(nq, nk, h, hk, d, 31)
    want, want_lse = _run(q, k, v, [nq], [nk], right=0)
    # side by side in one projection output
    fused = torch.zeros(nk, (h + 2 * hk) * d + 64, dtype=torch.bfloat16, device="cuda")
    fused[:nq, :h * d] = q.flatten(1)
    fused[:, h * d:(h + hk) * d], fused[:, (h + hk) * d:(h + 2 * hk) * d] = k.flatten(1), v.flatten(1)
    views = (fused[:nq, :h * d].view(nq, h, d), fused[:, h * d:(h + hk) * d].view(nk, hk, d), fused[:, (h + hk) * d:(h + 2 * hk) * d].view(nk, hk, d))
    assert torch.equal(B.oq_attention(*views, right=0), want)
    # heads first, output into a wider buffer, on another stream
    first = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in (q, k, v)]
    wide = torch.full((nq, h, d + 64), 7.0, dtype=torch.bfloat16, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        out, lse = B.oq_attention(*first, right=0, out=wide[:, :, :d], want_lse=True)
    side.synchronize()
    assert torch.equal(wide[:, :, :d], want) and torch.equal(lse, want_lse) and torch.all(wide[:, :, d:] == 7.0)


@pytest.mark.parametrize("ql,kl", [([3, 2], [5000, 4000]), ([300, 200], [300, 200])])
def test_queries_outside_the_sequences_are_left_alone(ql, kl):
    import torch
    q, k, v = _inputs(sum(ql) + 9, sum(kl), 2, 2, 128, 61)
    out = torch.full_like(q, 7.0)
    starts = (_starts(ql) + 4).to(torch.int32)
    B.oq_attention(q, k, v, starts, _starts(kl), right=0, out=out)
    want = B.oq_attention(q[4:4 + sum(ql)], k, v, _starts(ql), _starts(kl), right=0)
    assert torch.equal(out[4:4 + sum(ql)], want)
    assert torch.all(out[:4] == 7.0) and torch.all(out[4 + sum(ql):] == 7.0)


def test_repeated_calls_are_bit_identical():
    import torch
    for ql, kl in [([700], [700]), ([2], [9000])]:
        q, k, v = _inputs(sum(ql), sum(kl), 8, 8, 128, 41)
        a = _run(q, k, v, ql, kl)
        for _ in range(3):
            b = _run(q, k, v, ql, kl)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_large_joint_sequence_against_fp32():
    import torch
    n, h, d = 4608, 3, 128
    q, k, v = _inputs(n, n, h, h, d, 51)
    out, lse = _run(q, k, v, [n], [n])
    z = torch.einsum("ihd,jhd->hij", q.double(), k.double()) / np.sqrt(d)
    ref_lse = torch.logsumexp(z, 2)
    ref = torch.einsum("hij,jhd->ihd", torch.exp(z - ref_lse[..., None]), v.double())
    assert (lse - ref_lse).abs().max() <= 1e-5 * (1 + ref_lse.abs().max())
    assert (out.double() - ref).norm() <= FRO * ref.norm()


def test_empty_and_refusals():
    import torch
    q, k, v = _inputs(4, 6, 2, 2, 128, 1)
    assert B.oq_attention(q[:0], k, v).shape == (0, 2, 128)
    out, lse = B.oq_attention(q, k[:0], v[:0], want_lse=True)
    assert torch.all(out == 0) and torch.all(torch.isneginf(lse))

    def code(*a, **kw):
        with pytest.raises(B.OqError) as e:
            B.oq_attention(*a, **kw)
        return e.value.code

    assert code(q[:, :, :96], k[:, :, :96], v[:, :, :96]) == 2
    assert code(q, k.float(), v) == 1 and code(q, k[:5], v) == 1
    assert code(torch.cat([q, q[:, :1]], 1), k, v) == 1                                   # 3 heads on 2
    assert code(q, k, v, sinks=-1) == 1 and code(q, k, v, scale=-1.0) == 1 and code(q, k, v, scale=float("nan")) == 1
    assert code(q, k, v, _starts([4])) == 1                                              # one table without the other
    assert code(q, k, v, _starts([4]), _starts([3, 3])) == 1
    assert code(q, k, v, _starts([4]).long(), _starts([6]).long()) == 1
    many = torch.zeros(258, dtype=torch.int32, device="cuda")
    assert code(q, k, v, many, many) == 2
    wide = torch.zeros(6, 2, 136, dtype=torch.bfloat16, device="cuda")
    assert code(q, wide[:, :, 4:132], v) == 3
    small = torch.zeros(16, dtype=torch.uint8, device="cuda")
    long = _inputs(1, 9000, 2, 2, 128, 2)
    assert code(*long, workspace=small) == 6


@pytest.mark.parametrize("which", ["q", "k", "v", "kv", "qkv"])
@pytest.mark.parametrize("nq,nk,d", [(130, 270, 128), (2, 3000, 128), (40, 77, 64)])
def test_one_head_expanded_over_all(which, nq, nk, d):
    """A head stride of 0 reads the one head that is there, on every path: single part, joined parts, rows made again."""
    import torch
    h = 8
    mask = dict(left=nk // 2, right=0, sinks=2)
    full = dict(zip("qkv", _inputs(nq, nk, h, h, d, 71)))
    for name in which:
        full[name] = full[name][:, :1].expand(-1, h, -1)
    full["v"] = full["v"].clone() if "v" not in which else full["v"][:, :1].clone().expand(-1, h, -1)
    full["v"][nk - 1, 0] = float("nan")                    # seen by the last query alone
    out, lse = B.oq_attention(*full.values(), want_lse=True, **mask)
    copies = [t.contiguous() for t in full.values()]
    want, want_lse = B.oq_attention(*copies, want_lse=True, **mask)
    torch.cuda.synchronize()
    assert B.oq_device_status() == 0
    assert torch.equal(lse, want_lse) and torch.equal(torch.isnan(out), torch.isnan(want))
    assert torch.equal(torch.nan_to_num(out), torch.nan_to_num(want))
    _verify(*[t[:nq - 1] for t in copies[:1]], copies[1][:nk - 1], copies[2][:nk - 1], [nq - 1], [nk - 1], out[:nq - 1], lse[:, :nq - 1], **mask)


def test_strides_that_cannot_be_served_are_refused():
    import torch
    q, k, v = _inputs(4, 6, 2, 2, 128, 1)
    for args in ((q[:1].expand(4, -1, -1), k, v), (q, k[:1].expand(6, -1, -1), v), (q, k, v[:1].expand(6, -1, -1)),
                 (q, k.as_strided((6, 2, 128), (64, 768, 1)), v), (q, k, v.as_strided((6, 2, 128), (256, 64, 1)))):
        with pytest.raises(B.OqError) as e:
            B.oq_attention(*args)
        assert e.value.code == 1
    for out in (q[:, :1].clone().expand(-1, 2, -1), q[:1].clone().expand(4, -1, -1)):
        with pytest.raises(B.OqError) as e:
            B.oq_attention(q, k, v, out=out)
        assert e.value.code == 1


def test_tensors_off_the_device_and_odd_workspaces_are_refused():
    import torch
    q, k, v = _inputs(4, 6, 2, 2, 128, 1)
    args = dict(Q=q, K=k, V=v, q_start=_starts([4]), k_start=_starts([6]), out=torch.empty_like(q),
                workspace=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
    B.oq_attention(**args)
    bad = [{name: t.cpu()} for name, t in args.items()]
    bad += [dict(workspace=torch.empty(1 << 18, device="cuda")), dict(workspace=args["workspace"][:1].expand(1 << 20))]
    for change in bad:
        with pytest.raises(B.OqError) as e:
            B.oq_attention(**{**args, **change})
        assert e.value.code == 1, change.keys()


def test_window_numbers_that_do_not_fit_are_refused():
    q, k, v = _inputs(4, 6, 2, 2, 128, 1)
    for kw in (dict(left=2 ** 40), dict(right=-2 ** 40), dict(sinks=2 ** 31), dict(scale=1e60)):
        with pytest.raises(B.OqError) as e:
            B.oq_attention(q, k, v, **kw)
        assert e.value.code == 1


@pytest.mark.parametrize("size", [1e5, 3e7, 1e11, 1e20, 1e30])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("nq,nk", [(5, 1), (150, 300), (2, 5000)])
def test_scores_of_any_finite_size(nq, nk, sign, size):
    """The largest score's key gets its weight however large the scores are.  The scores are fp32 sums of exact products, off by at
    most 2^-17 of sum |q k|: rows whose best two keys lie closer than twice that and 40 exponents are left out, and in
    the others one key has weight 1, so that out is its value (one rounding of a weight, one of the output)."""
    d, h, hk = 128, 2, 1
    q, k, v = _inputs(nq, nk, h, hk, d, 81)
    q, k = (q.abs() * sign * size ** 0.5).bfloat16(), (k.abs() * size ** 0.5).bfloat16()
    out, lse = _run(q, k, v, [nq], [nk])
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    z = np.einsum("ihd,jd->hij", f(q), f(k)[:, 0]) / np.sqrt(d)           # (all products have one sign: sum |q k| = |z|)
    best = z.argmax(2)
    top = z.max(2)
    rest = np.where(np.arange(nk) == best[..., None], -np.inf, z).max(2)
    clear = top - rest > 2 * 2.0 ** -17 * np.abs(z).max(2) + 40
    assert clear.mean() > 0.5 or size < 1e6
    want = f(v)[best, 0].transpose(1, 0, 2)
    err = np.abs(f(out) - want)
    assert np.all((err <= 2.0 ** -7 * np.abs(want))[clear.T])
    assert np.all(np.isfinite(f(lse))) and np.all(np.abs(f(lse) - top)[clear] <= 2.0 ** -16 * np.abs(top)[clear])


@pytest.mark.parametrize("score", [700.0, -9e4, 6e10, -1.7e11, 2e20])
@pytest.mark.parametrize("nq,nk", [(130, 257), (1, 5003)])
def test_equal_scores_share_their_weight_at_any_size(nq, nk, score):
    """Equal keys have equal scores bit for bit, so out is the mean of the values, also across parts of unequal length.  The weights
    and l are equal powers and their sum: fp32 sums (2^-20 here) and the one rounding of the output."""
    import torch
    _, _, v = _inputs(1, nk, 1, 1, 128, 82)
    half = abs(score) ** 0.5
    q = torch.full((nq, 1, 128), half if score > 0 else -half, dtype=torch.bfloat16, device="cuda")
    k = torch.full((nk, 1, 128), half, dtype=torch.bfloat16, device="cuda")
    out, lse = _run(q, k, v, [nq], [nk], scale=1 / 128)
    mean = v.double().mean(0)
    assert torch.all((out.double() - mean).abs() <= 2.0 ** -8 * mean.abs() + 2.0 ** -8 * v.double().abs().mean(0) + 1e-30)
    z = q[0, 0, 0].double() * k[0, 0, 0].double()
    assert torch.all((lse.double() - z - np.log(nk)).abs() <= 1e-5 * (1 + z.abs()))


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("mask", [dict(right=0), dict(left=60, right=0, sinks=3), dict(left=30, right=20), dict()], ids=str)
@pytest.mark.parametrize("nq,nk", [(200, 200), (300, 555), (2, 3000), (129, 2900)])
def test_values_that_are_not_finite_reach_exactly_the_rows_that_see_them(nq, nk, mask, d):
    """NaN and both infinities strewn over V (several columns, some of them met twice in a column) and one key: every element is the
    definition's, finite, infinite or NaN."""
    import torch
    h = 2
    q, k, v = _inputs(nq, nk, h, 1, d, 91)
    g = np.random.default_rng(nq + nk)
    for what in (float("nan"), float("inf"), -float("inf"), float("nan"), float("inf")):
        for at in (int(g.integers(nk)), nk - 1 - int(g.integers(min(nk, 120)))):
            v[at, 0, int(g.integers(d))] = what
    v[nk - 7, 0, 5], v[nk - 40, 0, 5], v[nk - 60, 0, 9] = float("inf"), float("nan"), -float("inf")
    k[nk - 3, 0, 1] = float("nan")
    out, lse = _run(q, k, v, [nq], [nk], **mask)
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    with np.errstate(invalid="ignore"):
        ref, ref_lse = oat.attention(f(q), f(k), f(v), [nq], [nk], **mask)
    got, got_lse = f(out), f(lse)
    assert np.array_equal(np.isnan(got), np.isnan(ref)) and np.array_equal(np.isnan(got_lse), np.isnan(ref_lse))
    assert np.array_equal(np.isposinf(got), np.isposinf(ref)) and np.array_equal(np.isneginf(got), np.isneginf(ref))
    ok = np.isfinite(ref)
    size, _ = oat.attention(f(q), f(torch.nan_to_num(k, 0.0)), np.abs(f(torch.nan_to_num(v, 0.0, 0.0, 0.0))), [nq], [nk], **mask)
    assert np.all(np.abs(got - ref)[ok] <= (2.0 ** -8 * np.abs(ref) + (2.0 ** -8 + 1e-3) * size)[ok] + 1e-30)
    ok = np.isfinite(ref_lse)
    assert np.all(np.abs(got_lse - ref_lse)[ok] <= LSE * (1 + np.abs(ref_lse[ok])))


@pytest.mark.parametrize("nq,nk", [(200, 300), (1, 4100)])
def test_sums_that_leave_the_range_on_the_way_do_not_show(nq, nk):
    """Values near the type's largest: a sum of weights above 1 times such a value is infinite, the weighted mean is not."""
    import torch
    q, k, v = _inputs(nq, nk, 1, 1, 128, 92)
    q[:], k[:] = 0, 0
    q[..., 0], k[nk - 60, 0, 0] = 1.0, 5.25 * 128 ** 0.5      # the last tile's best key: weight 2^7.6 against the others'
    k[nk - 55, 0, 0] = 40 * 128 ** 0.5
    v[:] = 1e37
    out, lse = _run(q, k, v, [nq], [nk])
    assert torch.all((out.double() - v[0, 0, 0].double()).abs() <= 2.0 ** -7 * 1e37) and torch.all(torch.isfinite(lse))


def test_one_nan_that_many_rows_see_does_not_change_the_pace():
    """A NaN in a value that thousands of rows see is their result: they are not made again one by one.  (Key by key the rows would take
    over a hundred times as long.)"""
    import torch
    n, h = 8192, 4
    q, k, v = _inputs(n, n, h, h, 128, 93)

    def pace(values):
        times = []
        for _ in range(5):
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
            out = B.oq_attention(q, k, values, right=0)
            e1.record()
            torch.cuda.synchronize()
            times.append(e0.elapsed_time(e1))
        return min(times), out

    clean, want = pace(v)
    bad = v.clone()
    bad[300, :, 3] = float("nan")
    slow, got = pace(bad)
    print("clean %.3f ms, one NaN %.3f ms" % (clean, slow))
    assert torch.all(torch.isnan(got[300:, :, 3])) and torch.equal(got[300:, :, 4:], want[300:, :, 4:])
    assert torch.equal(got[:256], want[:256]) and torch.all(torch.isfinite(got[256:300]))         # (the latter share the NaN's tile and are made again)
    assert slow <= 10 * clean


def test_a_buffer_that_nothing_was_written_to_does_not_change_the_pace():
    """Keys and values in a larger buffer whose rest is NaN: nothing is made again, so the call takes what it takes beside zeros."""
    import torch
    nq, nk, h = 1000, 4001, 8
    q, k, v = _inputs(nq, nk, h, h, 128, 94)
    want, want_lse = _run(q, k, v, [nq], [nk])
    times = {}
    for rest in (0.0, float("nan")):
        big_k, big_v = (torch.full((2 * nk, h, 128), rest, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        big_k[:nk], big_v[:nk] = k, v
        for _ in range(5):
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
            out, lse = B.oq_attention(q, big_k, big_v, _starts([nq]), _starts([nk]), want_lse=True)
            e1.record()
            torch.cuda.synchronize()
            times[rest != 0] = min(times.get(rest != 0, 1e9), e0.elapsed_time(e1))
        # (the plan goes by the buffer's length, so the keys may be cut elsewhere: two roundings of the output and of the weights)
        assert torch.all(torch.isfinite(out)) and (lse - want_lse).abs().max() <= 1e-5 * (1 + want_lse.abs().max())
        assert (out.double() - want.double()).norm() <= 2 * FRO * want.double().norm()
    print("beside zeros %.3f ms, beside NaN %.3f ms" % (times[False], times[True]))
    assert times[True] <= 3 * times[False]
