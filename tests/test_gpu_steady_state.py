"""The operators around the projections at sizes where every CTA goes around its rings and over several items: stages refilled many times,
accumulators handed back, sums carried over runs, query tiles reused, rows requested ahead.  Against the fp64 forms, with
the tolerances that test_gpu_adapter, test_gpu_qk and test_gpu_attention derive."""
import numpy as np
import pytest

from oracle import attention as oat
from paper_2607_02461_b200 import binding as B

pytestmark = pytest.mark.gpu


def _f(t):
    return t.double().cpu().numpy()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rank", [32, 128])
def test_adapters(rank, dtype):
    """19 tiles of tokens x 144 (fp32: 288) column tiles over 148 SMs: 18 (37) of them an SM in rings of 5 to 8 stages; before that 128 steps of
    the first product for each tile, 16 an SM in rings of 6 or 9, in fp32 in runs of 4."""
    import torch
    t = torch.bfloat16 if dtype == "bf16" else torch.float32
    d, m, lens, ids = 8192, 9216, [700, 1, 129, 333, 0, 256, 581], [0, 1, -1, 1, 0, 2, 0]
    n = sum(lens)
    g = torch.Generator(device="cuda").manual_seed(rank)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    x, a, b = rnd(n, d).bfloat16(), (rnd(3, rank, d) / d ** 0.5).bfloat16(), (0.3 * rnd(3, m, rank)).bfloat16()
    scale, base = 0.5 + torch.rand(3, device="cuda", generator=g), rnd(n, m).to(t)
    start = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    seg = torch.tensor(ids, dtype=torch.int32, device="cuda")
    out = B.oq_adapter_add(x, a, b, scale, start, seg, base)
    torch.cuda.synchronize()
    assert B.oq_device_status() == 0
    ref = oat.adapter_add(_f(x), _f(a), _f(b), _f(scale), lens, ids, _f(base))
    size = oat.adapter_add(np.abs(_f(x)), np.abs(_f(a)), np.abs(_f(b)), _f(scale), lens, ids, np.zeros((n, m)))
    tol = 2.0 ** -17 * size + 2.0 ** -23 * np.abs(ref) if t == torch.float32 else (2.0 ** -16 + 2.0 ** -17) * size + 2.0 ** -8 * np.abs(ref) * 1.01
    assert np.all(np.abs(_f(out) - ref) <= tol + 1e-30)
    assert torch.equal(out[701:830], base[701:830])
    held = base.clone()
    B.oq_adapter_add(x, a, b, scale, start, seg, held, out=held)
    assert torch.equal(held, out)


@pytest.mark.parametrize("dtypes", ["bf16-bf16", "f32-f32"])
@pytest.mark.parametrize("norm", ["head", "row"])
@pytest.mark.parametrize("layout", ["pairs", "halves"])
@pytest.mark.parametrize("heads,d,axes", [(24, 128, (16, 48, 64)), (10, 64, (16, 16, 32))])
def test_norms_with_rotation(heads, d, axes, layout, norm, dtypes):
    """3001 tokens: a warp (or CTA) walks over several of them, with rows, table entries and positions requested ahead."""
    import torch
    t = torch.bfloat16 if dtypes == "bf16-bf16" else torch.float32
    n, tops = 3001, (7, 64, 64)
    g = torch.Generator(device="cuda").manual_seed(d)
    fused = (torch.randn(n, 2 * heads * d + 64, device="cuda", generator=g) * torch.exp(torch.randn(n, 1, device="cuda", generator=g))).to(t)
    q, k = fused[:, :heads * d].view(n, heads, d), fused[:, heads * d:2 * heads * d].view(n, heads, d)
    pos = torch.stack([torch.randint(0, top, (n,), device="cuda", generator=g) for top in tops], 1).to(torch.int32)
    w = [(1 + 0.3 * torch.randn(d if norm == "head" else heads * d, device="cuda", generator=g)).bfloat16() for _ in range(2)]
    rope = B.oq_make_rope(axes, tops, 10000.0, layout)
    outs = B.oq_qk_norm_rope(q, k, rope, pos, *w, norm=norm, out_dtype=torch.float32)
    for x, ww, got in zip((q, k), w, outs):
        kw = dict(pos=pos.cpu().numpy(), axis_dims=rope.axis_dims, theta=rope.theta, layout=layout)
        ref = oat.norm_rope(_f(x), _f(ww), norm, 1e-6, **kw)
        size = np.sqrt((oat.norm_rope(_f(x), _f(ww), norm, 1e-6) ** 2).max(axis=2, keepdims=True)) * 1.5
        assert np.all(np.abs(_f(got) - ref) <= 96 * 2.0 ** -24 * size + 1e-30)
    B.oq_qk_norm_rope(q, k, rope, pos, *w, norm=norm, out_q=q, out_k=k)                    # in place
    assert torch.equal(q, outs[0].to(t)) and torch.equal(k, outs[1].to(t))


@pytest.mark.parametrize("mask", [dict(), dict(left=1500, right=0, sinks=70)], ids=str)
@pytest.mark.parametrize("ql,kl,h,hk,d", [
    ([1, 3, 128, 2, 77, 1, 5, 200], [2500, 2819, 2689, 3001, 2947, 2561, 2600, 2700], 40, 8, 128),      # few queries: 360 items, both tiles on one block
    ([1, 2, 130], [2500, 2819, 2689], 80, 80, 64),
    ([600, 1, 257, 300, 513, 40, 255, 256, 90, 400], [600, 77, 300, 300, 513, 900, 255, 256, 90, 700], 20, 5, 128),   # 340 items of 1 to 8 key tiles
])
def test_attention_items(ql, kl, h, hk, d, mask):
    import torch
    g = torch.Generator(device="cuda").manual_seed(d)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g).bfloat16()  # noqa: E731
    q, k, v = rnd(sum(ql), h, d), rnd(sum(kl), hk, d), rnd(sum(kl), hk, d)
    starts = [torch.tensor(np.concatenate([[0], np.cumsum(x)]), dtype=torch.int32, device="cuda") for x in (ql, kl)]
    out, lse = B.oq_attention(q, k, v, *starts, want_lse=True, **mask)
    torch.cuda.synchronize()
    assert B.oq_device_status() == 0
    q0 = k0 = 0
    for nq, nk in zip(ql, kl):
        qq, kk, vv = q[q0:q0 + nq].double(), k[k0:k0 + nk].double().repeat_interleave(h // hk, 1), v[k0:k0 + nk].double().repeat_interleave(h // hk, 1)
        z = torch.einsum("ihd,jhd->hij", qq, kk) / d ** 0.5
        z = z.masked_fill(~torch.from_numpy(oat.visible(nq, nk, mask.get("left", -1), mask.get("right", -1), mask.get("sinks", 0))).cuda(), -np.inf)
        ref_lse = torch.logsumexp(z, 2)
        w = torch.exp(z - ref_lse[..., None]).nan_to_num(0.0)
        ref, size = torch.einsum("hij,jhd->ihd", w, vv), torch.einsum("hij,jhd->ihd", w, vv.abs())
        got, got_lse = out[q0:q0 + nq].double(), lse[:, q0:q0 + nq].double()
        assert torch.equal(torch.isneginf(got_lse), torch.isneginf(ref_lse))
        some = ~torch.isneginf(ref_lse)
        assert torch.all((got_lse - ref_lse)[some].abs() <= 1e-5 * (1 + ref_lse[some].abs()))
        assert torch.all((got - ref).abs() <= 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 1e-3) * size + 1e-30)
        assert (got - ref).norm() <= 4e-3 * ref.norm()
        q0, k0 = q0 + nq, k0 + nk
