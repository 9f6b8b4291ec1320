"""One self-attention layer of a diffusion transformer on quantized projections, from the library's calls:

    x -> rotate+quantize -> QKV projection -> + low-rank adapters -> q/k norms and rotation by position (in place)
      -> attention -> rotate+quantize -> output projection -> + low-rank adapters

    python -m paper_2607_02461_b200.attention_layer [--shape flux|wan|small] [--adapters 2] [--window 0]

runs a layer of the named shape on synthetic data and prints one JSON line with the time of each step.
"""
import argparse
import json

import torch

from . import binding as B


class Adapters:
    """Low-rank updates of one projection for several requests: A [n, rank, d], B [n, m, rank] (bf16), scale [n] (fp32)."""

    def __init__(self, a, b, scale):
        self.a, self.b, self.scale = a, b, scale

    def add(self, x, y, seg_start, seg_adapter):
        return B.oq_adapter_add(x, self.a, self.b, self.scale, seg_start, seg_adapter, y, out=y)


class _Projection:
    def __init__(self, w, bits_a, bits_w, block, seed):
        d = w.shape[1]
        self.dim, self.rot = d, B.oq_make_rpbh(d, block, seed)
        self.cb_a, self.cb_w = B.oq_build_codebook(d, bits_a), B.oq_build_codebook(d, bits_w)
        self.wq, self.wr = B.oq_quantize_weights(w, self.rot, self.cb_w)

    def __call__(self, x):
        xq, xs = B.oq_rotate_quantize_act(x, self.rot, self.cb_a)
        return B.oq_qlinear(xq, xs, self.cb_a, self.wq, self.wr, self.cb_w, self.dim)


class AttentionLayer:
    """w_qkv: CUDA bf16 [(heads + 2 kv_heads) * head_dim, d], w_proj: [d, heads * head_dim]; both are quantized here.
    rope: Rope handle or None.  wq, wk: bf16 norm weights, norm: "head", "row" or "none" (see oq_qk_norm_rope)."""

    def __init__(self, w_qkv, w_proj, heads, kv_heads, head_dim, rope=None, wq=None, wk=None, norm="head", bits_a=4, bits_w=4,
                 block=128, seed=0):
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.rope, self.wq, self.wk, self.norm = rope, wq, wk, norm
        self.qkv, self.proj = _Projection(w_qkv, bits_a, bits_w, block, seed), _Projection(w_proj, bits_a, bits_w, block, seed)

    def __call__(self, x, pos=None, starts=None, left=-1, right=-1, sinks=0, adapters=None, keep=None):
        """x: CUDA bf16 [T, d], the tokens of one or several requests one after the other; pos: int32 [T, axes];
        starts: int32 [requests + 1] or None (one request); left, right, sinks: the attention window of oq_attention.
        adapters: None or (Adapters of the QKV projection or None, Adapters of the output projection or None, seg_adapter
        int32 [requests]), which needs starts.  keep: a dict that receives what passes between the steps."""
        if adapters is not None and starts is None:
            raise B.OqError(1, "AttentionLayer: adapters go by request, so they need starts")
        t, (h, hk, d) = x.shape[0], (self.heads, self.kv_heads, self.head_dim)
        if keep is not None:
            keep["x"] = x
        qkv = self.qkv(x)
        if keep is not None:
            keep["qkv_shared"] = qkv.clone()
        if adapters is not None and adapters[0] is not None:
            adapters[0].add(x, qkv, starts, adapters[2])
        if keep is not None:
            keep["qkv"] = qkv.clone()
        q, k, v = (qkv[:, a * d:b * d].view(t, -1, d) for a, b in ((0, h), (h, h + hk), (h + hk, h + 2 * hk)))
        B.oq_qk_norm_rope(q, k, self.rope, pos, self.wq, self.wk, norm=self.norm, out_q=q, out_k=k)
        o = B.oq_attention(q, k, v, q_start=starts, k_start=starts, left=left, right=right, sinks=sinks).flatten(1)
        y = self.proj(o)
        if keep is not None:
            keep.update(q=q, k=k, v=v, o=o, y_shared=y.clone())
        if adapters is not None and adapters[1] is not None:
            adapters[1].add(o, y, starts, adapters[2])
        return y


SHAPES = {  # tokens per request, d, heads, head_dim, axes, positions, norm
    "small": ([300, 212], 512, 4, 128, (16, 56, 56), (1, 32, 32), "head"),
    "flux": ([4608], 3072, 24, 128, (16, 56, 56), (1, 64, 64), "head"),
    "wan": ([32760], 5120, 40, 128, (44, 42, 42), (21, 30, 52), "row"),
}


def make_layer(shape, n_adapters=2, rank=16, seed=0):
    """A layer of SHAPES[shape] with random weights and adapters, and (x, pos, starts, adapters) for it."""
    lens, d, heads, hd, axes, tops, norm = SHAPES[shape]
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(s, device="cuda", generator=g)  # noqa: E731
    width = hd * heads if norm == "row" else hd
    layer = AttentionLayer((0.02 * rnd(3 * heads * hd, d)).bfloat16(), (0.02 * rnd(d, heads * hd)).bfloat16(), heads, heads, hd,
                           B.oq_make_rope(axes, tops), (1 + 0.1 * rnd(width)).bfloat16(), (1 + 0.1 * rnd(width)).bfloat16(), norm)
    x = rnd(sum(lens), d)
    x[:, :: 97] *= 20
    pos = torch.stack([torch.randint(0, t, (sum(lens),), device="cuda", generator=g) for t in tops], 1).to(torch.int32)
    starts = torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)
    adapters = None
    if n_adapters:
        make = lambda n, k: Adapters((rnd(n_adapters, rank, k) / k ** 0.5).bfloat16(), (0.1 * rnd(n_adapters, n, rank)).bfloat16(),  # noqa: E731
                                     torch.ones(n_adapters, device="cuda"))
        adapters = (make(3 * heads * hd, d), make(d, heads * hd),
                    torch.arange(len(lens), device="cuda", dtype=torch.int32) % n_adapters)
    return layer, x.bfloat16(), pos, starts, adapters


def main():
    from . import build as oqbuild
    oqbuild.build()
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--shape", choices=sorted(SHAPES), default="flux")
    ap.add_argument("--adapters", type=int, default=2)
    ap.add_argument("--window", type=int, default=0, help="keys seen to the left of a query (0: all)")
    ap.add_argument("--iters", type=int, default=10)
    a = ap.parse_args()
    layer, x, pos, starts, adapters = make_layer(a.shape, a.adapters)
    left = a.window if a.window > 0 else -1

    def timed(fn):
        for _ in range(3):
            fn()
        ts = []
        for _ in range(a.iters):
            e0, e1 = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            e0.record()
            fn()
            e1.record()
            torch.cuda.synchronize()
            ts.append(e0.elapsed_time(e1))
        return sorted(ts)[len(ts) // 2]

    keep = {}
    layer(x, pos, starts, left, -1, 0, adapters, keep)
    q, k, v, qkv, o = (keep[n] for n in ("q", "k", "v", "qkv", "o"))
    y = keep["y_shared"]
    line = {"layer": a.shape, "tokens": x.shape[0], "adapters": a.adapters, "left": left,
            "ms": timed(lambda: layer(x, pos, starts, left, -1, 0, adapters)),
            "ms_qkv": timed(lambda: layer.qkv(x)),
            "ms_norm_rope": timed(lambda: B.oq_qk_norm_rope(q, k, layer.rope, pos, layer.wq, layer.wk, norm=layer.norm)),
            "ms_attention": timed(lambda: B.oq_attention(q, k, v, starts, starts, left=left)),
            "ms_proj": timed(lambda: layer.proj(o))}
    if adapters:
        line["ms_adapter_qkv"] = timed(lambda: adapters[0].add(x, qkv, starts, adapters[2]))
        line["ms_adapter_proj"] = timed(lambda: adapters[1].add(o, y, starts, adapters[2]))
    assert B.oq_device_status() == 0
    print(json.dumps(line))


if __name__ == "__main__":
    main()
