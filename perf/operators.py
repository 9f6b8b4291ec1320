"""Workloads of the operators around the quantized projections of a diffusion transformer's attention layer.

Three operators, in the order in which a block runs them:

  adapter    low-rank adapters of several requests added to a shared (quantized) projection's output
  qk         norms of queries and keys and the rotation by position with several axes, in one pass
  attention  softmax attention with a sliding window and a few first keys that stay visible

Every case can be run in two ways: in its plain form (elementary torch operations in 32 bits, rounded once at the
end) or, when `own` is true, through this repository's entry points.  `exact` evaluates the definition in 64 bits.
"""
import functools
import math

import torch

own = False


def _binding():
    from paper_2607_02461_b200 import binding
    return binding


# ------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # the smallest call: one token of a video transformer (40 heads of 128), where launch latency is all there is
        dict(name="qk one token", op="qk", tokens=1, q_heads=40, k_heads=40, head_dim=128, axes="44,42,42", grid="21,30,52",
             text=0, norm="row", layout="pairs", dtype="bf16", theta=10000.0),
        # a small odd batch kept in fp32, grouped heads of 64, one axis, halves layout: the text encoder's form
        dict(name="qk odd fp32", op="qk", tokens=513, q_heads=16, k_heads=4, head_dim=64, axes="64", grid="257",
             text=0, norm="head", layout="halves", dtype="f32", theta=10000.0),
        # FLUX-shaped joint sequence: 512 text tokens at the origin, 64 x 64 image tokens; q and k of the fused projection
        dict(name="qk image", op="qk", tokens=4608, q_heads=24, k_heads=24, head_dim=128, axes="16,56,56", grid="1,64,64",
             text=512, norm="head", layout="pairs", dtype="bf16", theta=10000.0),
        # Wan-shaped video: 21 x 30 x 52 latent patches, 40 heads, one norm over all heads of a token
        dict(name="qk video", op="qk", tokens=32760, q_heads=40, k_heads=40, head_dim=128, axes="44,42,42", grid="21,30,52",
             text=0, norm="row", layout="pairs", dtype="bf16", theta=10000.0),
        # a prompt of 77 tokens, causal, grouped heads of 64: a short call bound by latency
        dict(name="attention short", op="attention", q_lens="77", k_lens="77", q_heads=12, k_heads=4, head_dim=64, left=-1,
             right=0, sinks=0),
        # one query token against the cached keys of a whole Wan-shaped clip: bound by reading the keys and values
        dict(name="attention one token", op="attention", q_lens="1", k_lens="32760", q_heads=40, k_heads=40, head_dim=128,
             left=-1, right=0, sinks=0),
        # five requests of different sizes packed together (one of them empty, one with fewer keys than queries), a
        # window to both sides with 64 first keys visible to all
        dict(name="attention ragged", op="attention", q_lens="1000,0,333,2049,97", k_lens="1000,128,333,2049,40", q_heads=24,
             k_heads=8, head_dim=128, left=300, right=211, sinks=64),
        # FLUX-shaped joint attention: 4608 tokens, 24 heads, every key visible
        dict(name="attention image", op="attention", q_lens="4608", k_lens="4608", q_heads=24, k_heads=24, head_dim=128,
             left=-1, right=-1, sinks=0),
        # streamed Wan-shaped video: the 1560 tokens of a new latent frame see the first frame and the last eight of
        # the 21 cached ones
        dict(name="attention stream", op="attention", q_lens="1560", k_lens="32760", q_heads=40, k_heads=40, head_dim=128,
             left=12480, right=1560, sinks=1560),
        # modulation of eight samples, one token each, every one with an adapter of its own, fp32 output
        dict(name="adapter single tokens", op="adapter", lens="1,1,1,1,1,1,1,1", ids="0,1,2,3,4,5,6,7", adapters=8, rank=16,
             d_in=3072, d_out=18432, dtype="f32"),
        # four FLUX-shaped requests of odd sizes on the fused projection, one of them without an adapter
        dict(name="adapter image", op="adapter", lens="1536,1035,1,2036", ids="2,0,-1,1", adapters=3, rank=32, d_in=3072,
             d_out=9216, dtype="bf16"),
        # a Wan-shaped clip: two requests on the fused projection, rank 64
        dict(name="adapter video", op="adapter", lens="20000,12760", ids="1,0", adapters=2, rank=64, d_in=5120, d_out=15360,
             dtype="bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cut(rng, total, parts):
    """`parts` lengths, some of them possibly zero, that add up to `total`."""
    at = sorted(rng.randint(0, total) for _ in range(parts - 1))
    return [b - a for a, b in zip([0] + at, at + [total])]


def _text(values):
    return ",".join(str(v) for v in values)


def _ints(text):
    return [int(v) for v in text.split(",")]


def draw(rng):
    op = rng.choice(["qk", "attention", "attention", "adapter"])
    if op == "qk":
        head_dim = rng.choice([64, 128])
        k_heads = rng.choice([1, 2, 4, 8, 12])
        q_heads = k_heads * rng.choice([1, 1, 2, 3])
        dtype = rng.choice(["bf16", "bf16", "f32"])
        layout = rng.choice(["pairs", "pairs", "halves"])
        if layout == "pairs":
            axes = rng.choice({64: ["16,24,24", "64", "32,32"], 128: ["16,56,56", "44,42,42", "64,64", "96"]}[head_dim])
        else:
            axes = rng.choice({64: ["64", "32,32", "32,16,16"], 128: ["128", "32,48,48", "64,64"]}[head_dim])
        grid = _text([rng.randint(1, 90) for _ in _ints(axes)])
        tokens = _log_uniform(rng, 1, 32000)
        return dict(op="qk", tokens=tokens, q_heads=q_heads, k_heads=k_heads, head_dim=head_dim, axes=axes, grid=grid,
                    text=rng.choice([0, tokens // 8]), norm=rng.choice(["head", "row"]), layout=layout, dtype=dtype,
                    theta=rng.choice([256.0, 10000.0]))
    if op == "attention":
        head_dim = rng.choice([64, 128, 128])
        k_heads = rng.choice([1, 2, 4, 8])
        q_heads = k_heads * rng.choice([1, 1, 2, 3])
        kind = rng.choice(["whole", "stream", "ragged", "few"])
        if kind == "whole":
            q = [_log_uniform(rng, 1, 6000)]
            k, left, right, sinks = q, -1, rng.choice([-1, -1, 0]), 0
        elif kind == "stream":
            q = [_log_uniform(rng, 16, 1600)]
            k = [q[0] + _log_uniform(rng, 1, 24000)]
            left, right, sinks = _log_uniform(rng, 1, k[0]), rng.choice([0, q[0]]), rng.choice([0, 4, rng.randint(1, 1600)])
        elif kind == "ragged":
            q = _cut(rng, _log_uniform(rng, 64, 6000), rng.randint(2, 9))
            k = [max(0, v + rng.choice([0, 0, rng.randint(-64, 256)])) for v in q]
            left, right, sinks = rng.choice([-1, rng.randint(0, 1500)]), rng.choice([-1, 0, rng.randint(0, 1500)]), rng.choice([0, 64])
            if sum(k) == 0:
                k[0] = 1
        else:
            q = [rng.randint(1, 8) for _ in range(rng.randint(1, 4))]
            k = [v + _log_uniform(rng, 1, 30000) for v in q]
            left, right, sinks = rng.choice([-1, rng.randint(1, 4000)]), 0, rng.choice([0, 4])
        return dict(op="attention", q_lens=_text(q), k_lens=_text(k), q_heads=q_heads, k_heads=k_heads, head_dim=head_dim,
                    left=left, right=right, sinks=sinks)
    d_in, d_out = 64 * _log_uniform(rng, 2, 128), 64 * _log_uniform(rng, 2, 128)
    parts, adapters = rng.randint(1, 8), rng.randint(1, 8)
    few = rng.random() < 0.3
    lens = [rng.randint(1, 4) for _ in range(parts)] if few else _cut(rng, _log_uniform(rng, 16, 20000), parts)
    return dict(op="adapter", lens=_text(lens), ids=_text([rng.randint(-1, adapters - 1) for _ in lens]), adapters=adapters,
                rank=rng.choice([8, 16, 24, 32, 64, 128]), d_in=d_in, d_out=d_out, dtype=rng.choice(["bf16", "bf16", "f32"]))


# ------------------------------------------------------------------------------------------------------ inputs

_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}


@functools.lru_cache(maxsize=None)
def _rope(axes, grid, theta, layout):
    """The rotation table of a model: made once, kept for the program's life."""
    dims = _ints(axes)
    return _binding().oq_make_rope(dims, [max(n, 8) for n in _ints(grid)], theta, layout)


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, device="cuda", generator=g)  # noqa: E731
    state = {"case": case}
    if case["op"] == "qk":
        T, D = case["tokens"], case["head_dim"]
        hq, hk = case["q_heads"], case["k_heads"]
        # q, k and v leave the fused projection side by side; a few channels are much larger than the others
        x = randn(T, (hq + 2 * hk) * D) * torch.exp(0.5 * randn(T, 1))
        x = x * torch.where(torch.rand(x.shape[1], device="cuda", generator=g) < 0.01, 8.0, 1.0)
        x = x.to(_DTYPE[case["dtype"]])
        grid = _ints(case["grid"])
        n, at, cols = T - case["text"], torch.arange(T, device="cuda") - case["text"], []
        at = at + int(torch.randint(0, max(1, math.prod(grid) - n), (1,), device="cuda", generator=g))
        for size in reversed(grid):
            cols.append(at % size)
            at = at // size
        pos = torch.stack(cols[::-1], 1)
        pos[: case["text"]] = 0                                        # text sits at the origin
        wide = D * (1 if case["norm"] == "head" else hq), D * (1 if case["norm"] == "head" else hk)
        state.update(q=x[:, : hq * D].view(T, hq, D), k=x[:, hq * D:(hq + hk) * D].view(T, hk, D),
                     pos=pos.to(torch.int32).contiguous(), wq=(1 + 0.2 * randn(wide[0])).bfloat16(),
                     wk=(1 + 0.2 * randn(wide[1])).bfloat16())
        if own:
            state["rope"] = _rope(case["axes"], case["grid"], case["theta"], case["layout"])
    elif case["op"] == "attention":
        ql, kl, D = _ints(case["q_lens"]), _ints(case["k_lens"]), case["head_dim"]
        hq, hk = case["q_heads"], case["k_heads"]
        # normed heads with learned gains: scores are of order one, with some heads sharper than others
        unit = lambda x: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)  # noqa: E731
        common = randn(1, hk, D)
        q = unit(randn(sum(ql), hq, D) + 0.5 * common.repeat_interleave(hq // hk, 1)) * (0.7 + 1.3 * torch.rand(1, hq, 1, device="cuda", generator=g))
        k = unit(randn(sum(kl), hk, D) + 0.5 * common)
        kv = torch.empty(sum(kl), 2, hk, D, dtype=torch.bfloat16, device="cuda")
        kv[:, 0], kv[:, 1] = k, randn(sum(kl), hk, D)
        start = lambda lens: torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32)  # noqa: E731
        state.update(q=q.bfloat16(), k=kv[:, 0], v=kv[:, 1], q_start=start(ql), k_start=start(kl))
    else:
        lens, m, d, r = _ints(case["lens"]), case["d_out"], case["d_in"], case["rank"]
        x = randn(sum(lens), d) * torch.where(torch.rand(d, device="cuda", generator=g) < 0.01, 8.0, 1.0)
        state.update(x=x.bfloat16(), a=(randn(case["adapters"], r, d) / math.sqrt(d)).bfloat16(),
                     b=(0.1 * randn(case["adapters"], m, r)).bfloat16(),
                     scale=0.5 + torch.rand(case["adapters"], device="cuda", generator=g),
                     start=torch.tensor([0] + lens, device="cuda").cumsum(0).to(torch.int32),
                     ids=torch.tensor(_ints(case["ids"]), device="cuda", dtype=torch.int32),
                     base=randn(sum(lens), m).to(_DTYPE[case["dtype"]]))
    return state


# -------------------------------------------------------------------------------------------------------- runs

def run(state):
    return {"qk": _run_qk, "attention": _run_attention, "adapter": _run_adapter}[state["case"]["op"]](state)


def _run_qk(s):
    c = s["case"]
    if own:
        q, k = _binding().oq_qk_norm_rope(s["q"], s["k"], s["rope"], s["pos"], s["wq"], s["wk"], norm=c["norm"], eps=1e-6)
        return {"q": q, "k": k}
    axes = _ints(c["axes"])
    dev = s["pos"].device
    # one angle for each pair: the axis it belongs to, and its frequency
    axis = torch.arange(len(axes), device=dev).repeat_interleave(torch.tensor(axes, device=dev) // 2)
    dims = torch.tensor(axes, device=dev)[axis]
    first = torch.cumsum(torch.tensor([0] + axes, device=dev), 0)[axis]                  # first coordinate of the axis
    i = torch.arange(axis.numel(), device=dev) - first // 2
    angle = s["pos"][:, axis].float() * torch.exp(-math.log(c["theta"]) * (2 * i).float() / dims.float())
    cos, sin = torch.cos(angle)[:, None, :], torch.sin(angle)[:, None, :]
    lo = first + (2 * i if c["layout"] == "pairs" else i)
    hi = lo + (1 if c["layout"] == "pairs" else dims // 2)

    def one(x, w):
        y = x.float()
        T, H, D = y.shape
        y = y if c["norm"] == "head" else y.reshape(T, 1, H * D)
        y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + 1e-6) * w.float()
        y = y.reshape(T, H, D)
        a, b = y[..., lo], y[..., hi]
        out = y.clone()
        out[..., lo], out[..., hi] = a * cos - b * sin, a * sin + b * cos
        return out.to(x.dtype)

    return {"q": one(s["q"], s["wq"]), "k": one(s["k"], s["wk"])}


def _run_attention(s):
    c = s["case"]
    if own:
        out, lse = _binding().oq_attention(s["q"], s["k"], s["v"], q_start=s["q_start"], k_start=s["k_start"], left=c["left"],
                                           right=c["right"], sinks=c["sinks"], want_lse=True)
        return {"out": out, "lse": lse}
    q, k, v, q_start, k_start = (s[n] for n in ("q", "k", "v", "q_start", "k_start"))
    Tq, H, D = q.shape
    Tk, Hk, _ = k.shape
    i = torch.arange(Tq, device=q.device, dtype=torch.int32)
    j = torch.arange(Tk, device=q.device, dtype=torch.int32)
    sq, sk = torch.searchsorted(q_start[1:], i, right=True), torch.searchsorted(k_start[1:], j, right=True)
    lq, lk = q_start[1:] - q_start[:-1], k_start[1:] - k_start[:-1]
    at = (i - q_start[sq] + (lk - lq)[sq])[:, None]                    # a query's place among its keys: ends are aligned
    j = (j - k_start[sk])[None, :]
    seen = sq[:, None] == sk[None, :]
    if c["right"] >= 0:
        seen &= j <= at + c["right"]
    if c["left"] >= 0:
        seen &= (j >= at - c["left"]) | (j < c["sinks"])
    qf = q.float().view(Tq, Hk, H // Hk, D).permute(1, 2, 0, 3).reshape(Hk, H // Hk * Tq, D)
    score = torch.matmul(qf, k.float().permute(1, 2, 0)).mul_(1 / math.sqrt(D)).view(H, Tq, Tk)
    score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(Hk, H // Hk * Tq, Tk), v.float().permute(1, 0, 2)).view(H, Tq, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    return {"out": o.permute(1, 0, 2).to(torch.bfloat16), "lse": (top + total.log()).squeeze(-1)}


def _run_adapter(s):
    if own:
        return _binding().oq_adapter_add(s["x"], s["a"], s["b"], s["scale"], s["start"], s["ids"], s["base"])
    T, n = s["x"].shape[0], s["a"].shape[0]
    t = torch.arange(T, device=s["x"].device, dtype=torch.int32)
    mine = s["ids"][torch.searchsorted(s["start"][1:], t, right=True)]
    chosen = (mine[:, None] == torch.arange(n, device=mine.device)[None, :]).float() * s["scale"]
    u = torch.matmul(s["x"].float(), s["a"].float().flatten(0, 1).T).view(T, n, -1) * chosen[:, :, None]
    y = torch.matmul(u.view(T, -1), s["b"].float().permute(0, 2, 1).flatten(0, 1))
    return (s["base"].float() + y).to(s["base"].dtype)


# -------------------------------------------------------------------------------------------------------- work

def _visible(case):
    """(pairs of a query and a key it sees, keys that some query sees), summed over the sequences, for one head."""
    pairs = keys = 0
    for nq, nk in zip(_ints(case["q_lens"]), _ints(case["k_lens"])):
        if not nq or not nk:
            continue
        at = torch.arange(nq) + (nk - nq)
        end = torch.full_like(at, nk) if case["right"] < 0 else (at + case["right"] + 1).clamp(0, nk)
        begin = torch.zeros_like(at) if case["left"] < 0 else (at - case["left"]).clamp(0, nk)
        begin = torch.minimum(begin, end)
        early = torch.minimum(torch.minimum(torch.full_like(at, case["sinks"]), begin), end)
        pairs += int((end - begin + early).sum())
        some = end > begin
        window = int(end.max() - begin[some].min()) if bool(some.any()) else 0
        keys += min(nk, window + int(early.max()))
    return pairs, keys


def work(case):
    if case["op"] == "qk":
        size = 2 if case["dtype"] == "bf16" else 4
        values = case["tokens"] * (case["q_heads"] + case["k_heads"]) * case["head_dim"]
        return {"bytes": 2 * size * values + 4 * case["tokens"] * len(_ints(case["axes"])), "flops": 8 * values}
    if case["op"] == "attention":
        pairs, keys = _visible(case)
        rows = sum(_ints(case["q_lens"])) * case["q_heads"]
        return {"bytes": 2 * 2 * rows * case["head_dim"] + 4 * rows + 2 * 2 * keys * case["k_heads"] * case["head_dim"],
                "flops": 4 * pairs * case["q_heads"] * case["head_dim"]}
    size = 2 if case["dtype"] == "bf16" else 4
    pairs = [(n, a) for n, a in zip(_ints(case["lens"]), _ints(case["ids"])) if n > 0]
    tokens, used = sum(n for n, a in pairs), len({a for n, a in pairs if a >= 0})
    with_one = sum(n for n, a in pairs if a >= 0)
    width = case["d_in"] + case["d_out"]
    return {"bytes": 2 * size * tokens * case["d_out"] + 2 * with_one * case["d_in"] + 2 * used * case["rank"] * width,
            "flops": 2 * with_one * case["rank"] * width}


# ------------------------------------------------------------------------------------------------------- exact

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "qk":
        axes, pos = _ints(case["axes"]), s["pos"].double()

        def one(x, w):
            x = x.double()
            over = (-1,) if case["norm"] == "head" else (-2, -1)
            x = x / torch.sqrt((x * x).mean(over, keepdim=True) + 1e-6)
            x = x * (w.double() if case["norm"] == "head" else w.double().view(x.shape[1], x.shape[2]))
            parts, at = [], 0
            for a, d in enumerate(axes):
                y = x[..., at:at + d].reshape(*x.shape[:2], d // 2, 2) if case["layout"] == "pairs" else \
                    torch.stack((x[..., at:at + d // 2], x[..., at + d // 2:at + d]), -1)
                f = torch.tensor([case["theta"] ** (-2.0 * i / d) for i in range(d // 2)], dtype=torch.float64, device=x.device)
                turn = torch.polar(torch.ones(1, dtype=torch.float64, device=x.device), pos[:, a, None] * f)
                y = torch.view_as_real(torch.view_as_complex(y.contiguous()) * turn[:, None])
                parts.append(y.flatten(-2) if case["layout"] == "pairs" else torch.cat((y[..., 0], y[..., 1]), -1))
                at += d
            return torch.cat(parts + [x[..., at:]], -1)

        return {"q": one(s["q"], s["wq"]), "k": one(s["k"], s["wk"])}
    if case["op"] == "attention":
        Tq, H, D = s["q"].shape
        out = torch.zeros(Tq, H, D, dtype=torch.float64, device="cuda")
        lse = torch.full((H, Tq), -math.inf, dtype=torch.float64, device="cuda")
        q0 = k0 = 0
        for nq, nk in zip(_ints(case["q_lens"]), _ints(case["k_lens"])):
            off, hidden = nk - nq, torch.zeros(nq, nk, dtype=torch.bool, device="cuda")
            if case["left"] >= 0:
                hidden |= torch.ones_like(hidden).tril(off - case["left"] - 1)
                hidden[:, : case["sinks"]] = False
            if case["right"] >= 0:
                hidden |= torch.ones_like(hidden).triu(off + case["right"] + 1)
            some = ~hidden.all(1) if nk else torch.zeros(nq, dtype=torch.bool, device="cuda")
            for h in range(H if nq and nk else 0):
                hk = h // (H // case["k_heads"])
                z = s["q"][q0:q0 + nq, h].double() @ s["k"][k0:k0 + nk, hk].double().T / math.sqrt(D)
                z = z.masked_fill(hidden, -math.inf)
                w = torch.logsumexp(z, 1)
                lse[h, q0:q0 + nq] = w
                z = torch.exp(z - torch.where(some, w, torch.zeros_like(w))[:, None])
                out[q0:q0 + nq, h] = z @ s["v"][k0:k0 + nk, hk].double()
            q0, k0 = q0 + nq, k0 + nk
        return {"out": out, "lse": lse}
    y, at = s["base"].double(), 0
    for n, a in zip(_ints(case["lens"]), _ints(case["ids"])):
        if a >= 0 and n:
            y[at:at + n] += s["scale"][a].double() * (s["x"][at:at + n].double() @ s["a"][a].double().T) @ s["b"][a].double().T
        at += n
    return y
