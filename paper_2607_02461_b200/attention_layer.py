"""One self-attention layer of a diffusion transformer on quantized projections, from the library's calls:

    x -> rotate+quantize -> QKV projection -> + low-rank adapters -> q/k norms and rotation by position (in place)
      -> attention -> rotate+quantize -> output projection -> + low-rank adapters

Where the tokens come in chunks (streamed video, requests that go on), the keys and values of all chunks are held in a PagedCache in 8 or 4
bits, and attention of a chunk runs over it.

    python -m paper_2607_02461_b200.attention_layer [--shape flux|wan|small] [--adapters 2] [--window 0] [--cache fp8|fp4 [--chunk 1560]]

runs a layer of the named shape on synthetic data and prints one JSON line with the time of each step (with --cache: of a chunk's steps, once
the cache holds the shape's other tokens).
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


class PagedCache:
    """Keys and values of one layer for several requests, in 8 or 4 bits, in pages of one pool (see oq_cache_write).  The book-keeping is the
    host's: extend() and forget() take pages from the pool and give them back, table and lens on the device follow in the next step().  Positions
    count from a request's first token on, so max_tokens bounds all that it ever has, the tokens whose pages were given back included."""

    def __init__(self, n_pages, kv_heads, head_dim, requests, max_tokens, page_size=64, kind="fp8", device="cuda"):
        self.pages = B.oq_cache_alloc(n_pages, page_size, kv_heads, head_dim, kind, device)
        self.kind, self.page_size, self.max_tokens = kind, page_size, max_tokens
        self.free = list(range(n_pages - 1, -1, -1))
        self._table = torch.full((requests, -(-max_tokens // page_size)), -1, dtype=torch.int32)
        self._lens = torch.zeros(requests, dtype=torch.int32)
        self.table, self.lens = self._table.to(device), self._lens.to(device)

    def extend(self, new):
        """Room for new[r] more tokens of each request r."""
        if len(new) != len(self._lens) or min(new) < 0:
            raise B.OqError(1, "PagedCache: one number of new tokens for each request")
        ends = [int(n) + more for n, more in zip(self._lens, new)]
        if max(ends) > self.max_tokens:
            raise B.OqError(1, f"PagedCache: a request would have {max(ends)} tokens, more than {self.max_tokens}")
        wanted = [(r, p) for r, end in enumerate(ends) for p in range(-(-int(self._lens[r]) // self.page_size), -(-end // self.page_size))]
        if len(wanted) > len(self.free):
            raise B.OqError(6, f"PagedCache: {len(wanted)} pages wanted, {len(self.free)} free")
        for r, p in wanted:
            self._table[r, p] = self.free.pop()
        self._lens += torch.tensor(new, dtype=torch.int32)

    def forget(self, request, before, keep=0):
        """Gives back the pages that hold none but tokens keep .. before - 1 of a request: no later window sees them."""
        before = min(before, int(self._lens[request]))
        for p in range(-(-keep // self.page_size), before // self.page_size):
            if self._table[request, p] >= 0:
                self.free.append(int(self._table[request, p]))
                self._table[request, p] = -1

    def drop(self, request):
        """Gives a request's pages back; its place is free for another one."""
        self.free += [p for p in self._table[request].tolist() if p >= 0]
        self._table[request] = -1
        self._lens[request] = 0

    def step(self):
        """Brings table and lens to the device (the same tensors, so captured calls see them)."""
        self.table.copy_(self._table)
        self.lens.copy_(self._lens)


class AttentionLayer:
    """w_qkv: CUDA bf16 [(heads + 2 kv_heads) * head_dim, d], w_proj: [d, heads * head_dim]; both are quantized here.
    rope: Rope handle or None.  wq, wk: bf16 norm weights, norm: "head", "row" or "none" (see oq_qk_norm_rope)."""

    def __init__(self, w_qkv, w_proj, heads, kv_heads, head_dim, rope=None, wq=None, wk=None, norm="head", bits_a=4, bits_w=4,
                 block=128, seed=0):
        self.heads, self.kv_heads, self.head_dim = heads, kv_heads, head_dim
        self.rope, self.wq, self.wk, self.norm = rope, wq, wk, norm
        self.qkv, self.proj = _Projection(w_qkv, bits_a, bits_w, block, seed), _Projection(w_proj, bits_a, bits_w, block, seed)

    def __call__(self, x, pos=None, starts=None, left=-1, right=-1, sinks=0, adapters=None, keep=None, cache=None):
        """x: CUDA bf16 [T, d], the tokens of one or several requests one after the other; pos: int32 [T, axes];
        starts: int32 [requests + 1] or None (one request); left, right, sinks: the attention window of oq_attention.
        adapters: None or (Adapters of the QKV projection or None, Adapters of the output projection or None, seg_adapter
        int32 [requests]), which needs starts.  keep: a dict that receives what passes between the steps.
        cache: a PagedCache with a request for each of x's, extended by x's tokens: these are new tokens, their keys and values are written into it, and
        they see what it holds of their request (right = 0: causal; left, right, sinks count from a token's place in the whole request)."""
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
        if cache is None:
            o = B.oq_attention(q, k, v, q_start=starts, k_start=starts, left=left, right=right, sinks=sinks).flatten(1)
        else:
            form = dict(kind=cache.kind, page_size=cache.page_size)
            B.oq_cache_write(cache.pages, k, v, cache.table, cache.lens, starts, **form)
            o = B.oq_cache_attention(q, cache.pages, cache.table, cache.lens, starts, left=left, right=right, sinks=sinks, **form).flatten(1)
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
    ap.add_argument("--cache", choices=sorted(B.CACHE_KINDS), help="hold keys and values in a paged cache of this kind; the last tokens come as a chunk")
    ap.add_argument("--chunk", type=int, default=1560, help="tokens of a chunk, with --cache")
    ap.add_argument("--iters", type=int, default=10)
    a = ap.parse_args()
    if a.chunk < 1:
        ap.error("--chunk: at least one token")
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

    if a.cache:
        return stream(a, layer, x, pos, left, adapters, timed)
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


def stream(a, layer, x, pos, left, adapters, timed):
    """The shape's tokens as one request that comes in chunks: all but the last fill the cache, the last is timed."""
    total, n = x.shape[0], min(a.chunk, x.shape[0])
    cache = PagedCache(-(-total // 64), layer.kv_heads, layer.head_dim, 1, total, kind=a.cache)
    if adapters:
        adapters = (adapters[0], adapters[1], adapters[2][:1])
    keep, right = {}, n - 1                              # the tokens of a chunk see each other
    for at in range(0, total, n):
        end = min(at + n, total)
        cache.extend([end - at])
        cache.step()
        start = torch.tensor([0, end - at], device="cuda", dtype=torch.int32)
        args = (x[at:end], pos[at:end], start, left, right, 0, adapters)
        layer(*args, keep=keep, cache=cache)
    q, k, v = (keep[name] for name in ("q", "k", "v"))
    where = (cache.pages,), (cache.table, cache.lens, start)
    line = {"layer": a.shape, "tokens": total, "chunk": q.shape[0], "cache": a.cache, "cache_bytes": cache.pages.numel(), "left": left,
            "ms": timed(lambda: layer(*args, cache=cache)),
            "ms_cache_write": timed(lambda: B.oq_cache_write(*where[0], k, v, *where[1], kind=a.cache)),
            "ms_cache_attention": timed(lambda: B.oq_cache_attention(q, *where[0], *where[1], kind=a.cache, left=left, right=right)),
            "ms_cache_read": timed(lambda: B.oq_cache_read(*where[0], layer.head_dim, *where[1], q.shape[0], kind=a.cache))}
    assert B.oq_device_status() == 0
    print(json.dumps(line))


if __name__ == "__main__":
    main()
