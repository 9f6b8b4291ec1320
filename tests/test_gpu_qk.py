"""GPU parity of the q/k norms with rotation by position against the fp64 form, through the C ABI, and its refusals."""
import numpy as np
import pytest

from oracle import attention as oat
from paper_2607_02461_b200 import binding as B

pytestmark = pytest.mark.gpu

# fp32 arithmetic: a mean over at most 32768 squares added in a tree (<= 64 roundings), rsqrt, two products, one
# rotation of table values rounded once: below 96 units of 2^-24 of the two coordinates of a pair
F32_EPS = 96 * 2.0 ** -24
# bf16 outputs have no tolerance: they are the fp32 outputs rounded once


def _inputs(n, hq, hk, d, seed, dtype, extra=0):
    """q and k as strided views of one fused projection output."""
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, (hq + hk) * d + extra, generator=g) * torch.exp(torch.randn(n, 1, generator=g))
    x[:, ::37] *= 20
    x = x.to(dtype).cuda()
    return x, x[:, :hq * d].view(n, hq, d), x[:, hq * d:(hq + hk) * d].view(n, hk, d)


def _check(got, x, w, norm, pos, rope, eps=1e-6):
    x64 = x.double().cpu().numpy()
    w64 = None if w is None else w.double().cpu().numpy()
    kw = {} if rope is None else dict(pos=pos.cpu().numpy(), axis_dims=rope.axis_dims, theta=rope.theta, layout=rope.layout)
    ref = oat.norm_rope(x64, w64, norm, eps, **kw)
    # the size of a coordinate's pair bounds the rounding of its rotation
    size = np.sqrt((oat.norm_rope(x64, w64, norm, eps) ** 2).max(axis=2, keepdims=True)) * 1.5
    err = np.abs(got.double().cpu().numpy() - ref)
    tol = F32_EPS * size + 1e-30
    assert np.all(err <= tol), (err / tol).max()


CASES = [
    # tokens, q heads, k heads, head_dim, axes, positions, norm, layout
    (1, 40, 40, 128, (44, 42, 42), (21, 30, 52), "row", "pairs"),
    (7, 24, 24, 128, (16, 56, 56), (1, 64, 64), "head", "pairs"),
    (33, 5, 1, 128, (96,), (70000,), "head", "pairs"),
    (130, 3, 3, 64, (16, 24, 24), (9, 9, 9), "row", "pairs"),
    (19, 16, 4, 64, (64,), (300,), "head", "halves"),
    (12, 6, 2, 128, (32, 48, 48), (8, 9, 10), "row", "halves"),
    (5, 2, 2, 256, (64, 32, 32, 64), (3, 4, 5, 6), "head", "halves"),
    (9, 7, 3, 32, (32,), (64,), "head", "pairs"),
    (4, 256, 1, 128, (6, 2), (5, 5), "row", "pairs"),
]


@pytest.mark.parametrize("dtypes", ["bf16-bf16", "f32-f32", "bf16-f32", "f32-bf16"])
@pytest.mark.parametrize("n,hq,hk,d,axes,tops,norm,layout", CASES)
def test_matches_fp64(n, hq, hk, d, axes, tops, norm, layout, dtypes):
    import torch
    tin, tout = [torch.bfloat16 if t == "bf16" else torch.float32 for t in dtypes.split("-")]
    _, q, k = _inputs(n, hq, hk, d, 10 * n + d, tin, extra=64)
    g = torch.Generator().manual_seed(3)
    pos = torch.stack([torch.randint(0, t, (n,), generator=g) for t in tops], 1).to(torch.int32).cuda()
    pos[0] = torch.tensor([t - 1 for t in tops])                       # the last position that the table has
    wq = (1 + 0.3 * torch.randn(d if norm == "head" else hq * d, generator=g)).bfloat16().cuda()
    wk = (1 + 0.3 * torch.randn(d if norm == "head" else hk * d, generator=g)).bfloat16().cuda()
    rope = B.oq_make_rope(axes, tops, 10000.0, layout)
    yq, yk = B.oq_qk_norm_rope(q, k, rope, pos, wq, wk, norm=norm, out_dtype=torch.float32)
    if tout == torch.bfloat16:
        rq, rk = B.oq_qk_norm_rope(q, k, rope, pos, wq, wk, norm=norm, out_dtype=tout)
        assert torch.equal(rq, yq.bfloat16()) and torch.equal(rk, yk.bfloat16())
    _check(yq, q, wq, norm, pos, rope)
    _check(yk, k, wk, norm, pos, rope)


def test_parts_can_be_left_out():
    import torch
    _, q, k = _inputs(21, 4, 2, 128, 1, torch.bfloat16)
    rope = B.oq_make_rope([44, 42, 42], [8, 8, 8], 10000.0)
    pos = torch.randint(0, 8, (21, 3), dtype=torch.int32, device="cuda")
    w = torch.full((128,), 1.25, dtype=torch.bfloat16, device="cuda")
    for norm, ww, rp in [("none", None, rope), ("head", None, rope), ("head", w, None), ("row", None, None), ("none", None, None)]:
        yq, yk = B.oq_qk_norm_rope(q, k, rp, pos if rp else None, ww, ww, norm=norm, out_dtype=torch.float32)
        _check(yq, q, ww, norm, pos, rp)
        _check(yk, k, ww, norm, pos, rp)
    alone, none = B.oq_qk_norm_rope(q, None, rope, pos, w, None)
    both, _ = B.oq_qk_norm_rope(q, k, rope, pos, w, w)
    assert none is None and torch.equal(alone, both)


@pytest.mark.parametrize("norm,layout,axes", [("head", "pairs", [44, 42, 42]), ("row", "halves", [32, 48, 48])])
def test_in_place_strides_and_streams(norm, layout, axes):
    import torch
    n, hq, hk, d = 200, 6, 6, 128
    x, q, k = _inputs(n, hq, hk, d, 5, torch.bfloat16, extra=256)
    rope = B.oq_make_rope(axes, [50, 50, 50], 256.0, layout)
    pos = torch.randint(0, 50, (n, 3), dtype=torch.int32, device="cuda")
    want_q, want_k = B.oq_qk_norm_rope(q, k, rope, pos, norm=norm)
    # head-major tensors, positions with a stride of their own, another stream
    wide = torch.zeros(n, 5, dtype=torch.int32, device="cuda")
    wide[:, :3] = pos
    qt, kt = q.transpose(0, 1).contiguous().transpose(0, 1), k.transpose(0, 1).contiguous().transpose(0, 1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        gq, gk = B.oq_qk_norm_rope(qt, kt, rope, wide[:, :3], norm=norm)
    side.synchronize()
    assert torch.equal(gq, want_q) and torch.equal(gk, want_k)
    # in place in the fused projection's output; what lies beside the heads stays
    rest = x[:, (hq + hk) * d:].clone()
    B.oq_qk_norm_rope(q, k, rope, pos, norm=norm, out_q=q, out_k=k)
    assert torch.equal(q, want_q) and torch.equal(k, want_k) and torch.equal(x[:, (hq + hk) * d:], rest)


def test_edge_values():
    import torch
    n, h, d = 6, 3, 128
    x = torch.randn(n, h, d, device="cuda")
    x[1] = 0                                       # a zero token: 0 / sqrt(eps)
    x[2] *= 1e15                                   # squares near the top of fp32
    x[3, 1, 5] = float("inf")
    x[4, 2, 7] = float("nan")
    rope = B.oq_make_rope([16, 56, 56], [4, 4, 4], 10000.0)
    pos = torch.ones(n, 3, dtype=torch.int32, device="cuda")
    pos[5, 1] = 4                                  # outside the table: NaN on that axis alone
    y, _ = B.oq_qk_norm_rope(x, None, rope, pos)
    assert torch.all(y[1] == 0) and torch.all(torch.isfinite(y[2]))
    assert torch.all(torch.isfinite(y[3, 0])) and torch.all(torch.isfinite(y[4, :2])) and torch.all(torch.isnan(y[4, 2]))
    assert torch.all(torch.isnan(y[5, :, 16:72])) and torch.all(torch.isfinite(y[5, :, :16])) and torch.all(torch.isfinite(y[5, :, 72:]))
    pos[5, 1] = -1
    y, _ = B.oq_qk_norm_rope(x, None, rope, pos)
    assert torch.all(torch.isnan(y[5, :, 16:72]))
    e = torch.empty(0, h, d, device="cuda")
    assert B.oq_qk_norm_rope(e, e, rope, pos[:0])[0].shape == (0, h, d)


def test_refusals():
    import torch
    rope = B.oq_make_rope([16, 56, 56], [4, 4, 4], 10000.0)
    pos = torch.zeros(3, 3, dtype=torch.int32, device="cuda")
    x = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda")
    wide = torch.zeros(3, 2 * 128 + 8, dtype=torch.bfloat16, device="cuda")

    def code(*a, **k):
        with pytest.raises(B.OqError) as e:
            B.oq_qk_norm_rope(*a, **k)
        return e.value.code

    assert code(x[:, :, :96], None, None) == 2                                           # head_dim
    assert code(x[:, :, :64], None, rope, pos) == 1                                      # rotation wider than a head
    assert code(x, None, rope, None) == 1 and code(x, None, rope, pos[:2]) == 1 and code(x, None, rope, pos.long()) == 1
    assert code(x, None, rope, pos, norm="both") == 1
    assert code(x, None, rope, pos, x[0, 0], norm="none") == 1
    assert code(x, None, rope, pos, torch.ones(64, dtype=torch.bfloat16, device="cuda")) == 1
    assert code(x, None, rope, pos, torch.ones(128, device="cuda")) == 1
    assert code(wide[:, 4:260].view(3, 2, 128), None, rope, pos) == 3                    # base of a row not 16-byte aligned
    assert code(x.half(), None, rope, pos) == 1
    assert code(x, x.float(), rope, pos) == 1
    assert code(x, None, rope, pos, eps=-1.0) == 1


def test_tensors_off_the_device_are_refused():
    import torch
    x = torch.zeros(3, 2, 128, dtype=torch.bfloat16, device="cuda")
    w = torch.ones(128, dtype=torch.bfloat16, device="cuda")
    args = dict(Q=x, K=x.clone(), rope=B.oq_make_rope([16, 56, 56], [4, 4, 4], 10000.0), pos=torch.zeros(3, 3, dtype=torch.int32, device="cuda"),
                wq=w, wk=w.clone(), out_q=x.clone(), out_k=x.clone())
    B.oq_qk_norm_rope(**args)
    for name in ("Q", "K", "pos", "wq", "wk", "out_q", "out_k"):
        with pytest.raises(B.OqError) as e:
            B.oq_qk_norm_rope(**{**args, name: args[name].cpu()})
        assert e.value.code == 1, name


def test_positions_too_far_apart_are_refused():
    import torch
    x = torch.zeros(2, 2, 128, dtype=torch.bfloat16, device="cuda")
    far = torch.empty(2 ** 32 + 16, dtype=torch.int32, device="cuda").as_strided((2, 3), (2 ** 32 + 3, 1))
    far.zero_()
    with pytest.raises(B.OqError) as e:
        B.oq_qk_norm_rope(x, None, B.oq_make_rope([16, 56, 56], [4, 4, 4], 10000.0), far)
    assert e.value.code == 2


def test_first_use_of_a_table_on_a_side_stream():
    """A table of 27 MB whose upload the kernel on a stream of its own must not overtake."""
    import torch
    _, q, k = _inputs(300, 4, 2, 128, 11, torch.bfloat16)
    pos = torch.arange(70000 - 300, 70000, dtype=torch.int32, device="cuda")[:, None].contiguous()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for theta in (10000.0, 500.0, 77.0):
        rope = B.oq_make_rope([96], [70000], theta)
        with torch.cuda.stream(side):
            y, _ = B.oq_qk_norm_rope(q, None, rope, pos, out_dtype=torch.float32)
        side.synchronize()
        _check(y, q, None, "head", pos, rope)


def test_first_use_of_a_table_while_a_stream_is_captured():
    import torch
    _, q, k = _inputs(50, 4, 2, 128, 12, torch.bfloat16)
    pos = torch.randint(0, 40, (50, 3), dtype=torch.int32, device="cuda")
    rope, again = (B.oq_make_rope([44, 42, 42], [40, 40, 40], 10000.0) for _ in range(2))
    B.oq_qk_norm_rope(q, k)                          # (the kernel itself is loaded)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        yq, yk = B.oq_qk_norm_rope(q, k, rope, pos)
    for _ in range(2):
        yq.zero_()
        graph.replay()
        torch.cuda.synchronize()
        want_q, want_k = B.oq_qk_norm_rope(q, k, again, pos)
        assert torch.equal(yq, want_q) and torch.equal(yk, want_k)


def test_expanded_inputs_are_read_and_expanded_outputs_refused():
    import torch
    x = torch.randn(70, 1, 128, device="cuda").bfloat16()
    rope = B.oq_make_rope([16, 56, 56], [9, 9, 9], 10000.0)
    pos = torch.randint(0, 9, (70, 3), dtype=torch.int32, device="cuda")
    for norm in ("head", "row"):
        for view in (x.expand(70, 5, 128), x[:1].expand(70, 5, 128)):
            got, _ = B.oq_qk_norm_rope(view, None, rope, pos, norm=norm)
            want, _ = B.oq_qk_norm_rope(view.contiguous(), None, rope, pos, norm=norm)
            assert torch.equal(got, want)
            with pytest.raises(B.OqError) as e:
                B.oq_qk_norm_rope(view.contiguous(), None, rope, pos, norm=norm, out_q=x.clone().expand(70, 5, 128))
            assert e.value.code == 1
