"""A whole attention layer on quantized projections: every step of it against the fp64 forms, from what the step before
produced, and the layer's command."""
import json
import subprocess
import sys

import numpy as np
import pytest

from oracle import attention as oat
from oracle import bf16 as obf
from oracle import codebook as ocb
from oracle import qlinear as oql
from oracle import quantize as oq
from oracle import rpbh as orp
from paper_2607_02461_b200 import attention_layer as L
from paper_2607_02461_b200 import binding as B

pytestmark = pytest.mark.gpu

# relative Frobenius errors: one bf16 rounding of the output (root mean square 2^-8 / (2 sqrt 3) = 1.13e-3 at the start of a
# binade, less above) plus that of the softmax weights for attention; the projections as in their own tests
STEP, ATTENTION, PROJECTION = 2.5e-3, 4e-3, 3e-3


def _f(t):
    return t.double().cpu().numpy()


def _rel(got, ref):
    return np.linalg.norm(_f(got) - ref) / np.linalg.norm(ref)


def _projection(p, x):
    """fp64 product of the operands the quantizers choose (the oracle quantizes the tokens itself)."""
    import torch
    bits = x.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
    perm, signs = orp.make_rpbh(p.dim, 128, 0)
    o = ocb.lloyd_max(p.dim, 4)
    qa = oq.quantize_rows(bits, 128, perm, signs, o.boundaries)
    idx = B.oq_unpack_indices(p.wq, p.wq.shape[0], p.dim, 4).cpu().numpy()
    wr = obf.bf16_bits_to_f64(p.wr.view(torch.int16).cpu().numpy().view(np.uint16))
    return oql.qlinear(qa["idx"], qa["norm"].astype(np.float32), o.centroids_decoded, idx, wr, o.centroids_decoded)


@pytest.mark.parametrize("mask", [dict(), dict(left=90, right=0, sinks=4)], ids=str)
def test_every_step_matches_fp64(mask):
    import torch
    layer, x, pos, starts, adapters = L.make_layer("small")
    keep = {}
    y = layer(x, pos, starts, adapters=adapters, keep=keep, **mask)
    torch.cuda.synchronize()
    assert B.oq_device_status() == 0
    lens, ids = np.diff(starts.cpu().numpy()).tolist(), adapters[2].cpu().numpy().tolist()
    assert _rel(keep["qkv_shared"], _projection(layer.qkv, x)) <= PROJECTION
    a = adapters[0]
    ref = oat.adapter_add(_f(x), _f(a.a), _f(a.b), _f(a.scale), lens, ids, _f(keep["qkv_shared"]))
    assert _rel(keep["qkv"], ref) <= STEP
    h, d = layer.heads, layer.head_dim
    kw = dict(pos=pos.cpu().numpy(), axis_dims=layer.rope.axis_dims, theta=layer.rope.theta)
    for name, at, w in (("q", 0, layer.wq), ("k", h * d, layer.wk)):
        part = _f(keep["qkv"])[:, at:at + h * d].reshape(-1, h, d)
        assert _rel(keep[name], oat.norm_rope(part, _f(w), layer.norm, 1e-6, **kw)) <= STEP
    assert torch.equal(keep["v"].flatten(1), keep["qkv"][:, 2 * h * d:])
    ref, _ = oat.attention(_f(keep["q"]), _f(keep["k"]), _f(keep["v"]), lens, lens, **mask)
    assert _rel(keep["o"], ref.reshape(len(ref), -1)) <= ATTENTION
    assert _rel(keep["y_shared"], _projection(layer.proj, keep["o"])) <= PROJECTION
    a = adapters[1]
    ref = oat.adapter_add(_f(keep["o"]), _f(a.a), _f(a.b), _f(a.scale), lens, ids, _f(keep["y_shared"]))
    assert _rel(y, ref) <= STEP
    assert torch.equal(layer(x, pos, starts, adapters=adapters, **mask), y)
    with pytest.raises(B.OqError):
        layer(x, pos, adapters=adapters, **mask)             # adapters go by request
    plain = layer(x, pos, starts, **mask)
    assert not torch.equal(plain, y)


def test_command():
    out = subprocess.run([sys.executable, "-m", "paper_2607_02461_b200.attention_layer", "--shape", "small", "--iters", "3"],
                         capture_output=True, text=True, timeout=300)
    assert out.returncode == 0, out.stderr[-2000:]
    line = json.loads(out.stdout.strip().splitlines()[-1])
    assert line["tokens"] == 512 and line["ms"] > 0 and line["ms_attention"] > 0 and line["ms_adapter_qkv"] > 0
