"""Workloads of the paged cache of quantized keys and values of a streaming attention layer.

Three operators, in the order in which a layer runs them on the tokens of a new chunk:

  write      keys and values of the new tokens quantized into the pages of their sequences
  attention  attention of the new tokens over all that is cached, with a window and first keys that stay visible
  read       tokens read back from the pages

The cache is a uint8 tensor [pages][kv heads][bytes of a block].  A block holds page_size tokens of one head, one part after the other:
keys [page_size][head_dim * bits / 8], values (the same), scales of the keys [page_size][head_dim / 32], scales of the values.  A scale is a
byte s and stands for 2^(s - 127), one for 32 adjacent coordinates.  Elements are e4m3 (kind "fp8") or e2m1 (kind "fp4", the even
coordinate in the low half of a byte).  A group's scale is the smallest power of two, of at least 2^-14 and at most 2^7 (fp8) or 2^13 (fp4),
with which its largest magnitude stays within the format (448, 6); elements are rounded to nearest even.  Position p of a sequence is
token p % page_size of page table[sequence][p / page_size].  The new tokens of a sequence are its last ones.

Every case can be run in two ways: in its plain form (elementary torch operations in 32 bits, rounded once at the end) or, when `own` is
true, through this repository's entry points.  `exact` evaluates the definitions in 64 bits.
"""
import math

import torch

own = False


def _binding():
    from paper_2607_02461_b200 import binding
    return binding


# ------------------------------------------------------------------------------------------------------- cases

def listed():
    return [
        # one new token of a Wan-shaped layer (40 heads of 128): the smallest write, where launch latency is all there is
        dict(name="write one token", op="write", kind="fp8", page=64, q_lens="1", k_lens="301", kv_heads=40, head_dim=128, dtype="bf16"),
        # the 1560 tokens of a new Wan-shaped latent frame, behind six that are cached; frames end inside pages
        dict(name="write frame", op="write", kind="fp8", page=64, q_lens="1560", k_lens="10920", kv_heads=40, head_dim=128,
             dtype="bf16"),
        # fp32 keys and values of five requests of odd sizes in 4 bits, small pages; what attention will see of them is read back
        dict(name="store requests", op="store", kind="fp4", page=16, q_lens="333,1,0,2049,97", k_lens="400,77,31,2049,1000", kv_heads=8,
             head_dim=64, dtype="f32"),
        # a small read of two sequences in 4 bits, as fp32
        dict(name="read odd", op="read", kind="fp4", page=32, q_lens="57,131", k_lens="200,131", kv_heads=4, head_dim=64, dtype="f32"),
        # the whole cached Wan-shaped clip read back in bf16 (21 x 30 x 52 latent patches), as when a request moves
        dict(name="read clip", op="read", kind="fp8", page=64, q_lens="32760", k_lens="32760", kv_heads=40, head_dim=128, dtype="bf16"),
        # a prompt of 77 tokens, causal, grouped heads of 64: a short call bound by latency
        dict(name="attention short", op="attention", kind="fp8", page=64, q_lens="77", k_lens="77", q_heads=12, kv_heads=4, head_dim=64,
             left=-1, right=0, sinks=0, evicted=False),
        # one new token against the cached keys of a whole clip: bound by reading the cache
        dict(name="attention one token", op="attention", kind="fp8", page=64, q_lens="1", k_lens="32760", q_heads=40, kv_heads=40,
             head_dim=128, left=-1, right=0, sinks=0, evicted=False),
        # a step of 16 requests at once, one token each, with caches from 17 to 16384 tokens in 4 bits, grouped heads
        dict(name="attention batch", op="attention", kind="fp4", page=32, q_lens=_text([1] * 16),
             k_lens="17,16384,1000,4097,9000,333,2048,12001,64,7777,5000,129,3000,15000,1,10241", q_heads=24, kv_heads=8, head_dim=128,
             left=-1, right=0, sinks=0, evicted=False),
        # four requests that check five drafted tokens each, grouped heads of 64, small pages
        dict(name="attention drafts", op="attention", kind="fp8", page=16, q_lens="5,5,5,5", k_lens="4005,1029,8000,260", q_heads=16,
             kv_heads=4, head_dim=64, left=-1, right=0, sinks=0, evicted=False),
        # new chunks of some requests beside single tokens of others (one of them idle), a window with first keys that stay visible,
        # pages that the window has left given back
        dict(name="attention mixed", op="attention", kind="fp4", page=16, q_lens="1000,1,333,0,1,97", k_lens="5000,3001,333,128,9000,40",
             q_heads=24, kv_heads=8, head_dim=128, left=2000, right=0, sinks=64, evicted=True),
        # 2048 more tokens of a long prompt, causal, behind 14337 cached ones in 4 bits
        dict(name="attention chunk", op="attention", kind="fp4", page=128, q_lens="2048", k_lens="16385", q_heads=24, kv_heads=8,
             head_dim=128, left=-1, right=0, sinks=0, evicted=False),
        # streamed Wan-shaped video: the 1560 tokens of a new latent frame see the first frame and the last eight of the 21 cached ones
        dict(name="attention stream", op="attention", kind="fp8", page=64, q_lens="1560", k_lens="32760", q_heads=40, kv_heads=40,
             head_dim=128, left=12480, right=1560, sinks=1560, evicted=True),
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
    op = rng.choice(["write", "store", "read", "attention", "attention", "attention"])
    kind, page = rng.choice(["fp8", "fp8", "fp4"]), rng.choice([16, 32, 64, 128])
    if op != "attention":
        kv_heads, head_dim = rng.choice([1, 2, 4, 8, 12, 40]), rng.choice([64, 128])
        q = _cut(rng, _log_uniform(rng, 1, min(32000, 1200000 // kv_heads)), rng.randint(1, 6))
        k = [n + rng.choice([0, rng.randint(0, 300), rng.randint(0, 3000)]) for n in q]
        # (what a write leaves behind is handed back as the buffer itself, so it is drawn in 8 bits, whose values torch has a type for)
        return dict(op=op, kind="fp8" if op == "write" else kind, page=page, q_lens=_text(q), k_lens=_text(k), kv_heads=kv_heads,
                    head_dim=head_dim, dtype=rng.choice(["bf16", "bf16", "f32"]))
    head_dim, kv_heads = rng.choice([64, 128, 128]), rng.choice([1, 2, 4, 8])
    q_heads = kv_heads * rng.choice([1, 1, 2, 3, 8])
    form = rng.choice(["tokens", "drafts", "mixed", "chunk", "stream"])
    left, right, sinks, evicted = -1, 0, 0, False
    if form == "tokens":
        k = [_log_uniform(rng, 1, 30000) for _ in range(_log_uniform(rng, 1, 16))]
        q = [1] * len(k)
    elif form == "drafts":
        k = [_log_uniform(rng, 8, 16000) for _ in range(rng.randint(1, 6))]
        q = [rng.randint(1, 8) for _ in k]
    elif form == "mixed":
        q = [rng.choice([0, 1, 1, rng.randint(2, 90), _log_uniform(rng, 90, 900)]) for _ in range(rng.randint(2, 7))]
        q[0] += 1
        k = [n + rng.choice([0, rng.randint(1, 100), rng.randint(1, 6000)]) for n in q]
        left, sinks, evicted = rng.choice([-1, rng.randint(0, 3000)]), rng.choice([0, 4, 64]), True
    elif form == "chunk":
        q = [_log_uniform(rng, 30, 2500)]
        k = [q[0] + _log_uniform(rng, 1, 14000)]
    else:
        q = [_log_uniform(rng, 30, 1600)]
        k = [q[0] + _log_uniform(rng, 1, 24000)]
        left, right, sinks, evicted = _log_uniform(rng, 1, k[0]), rng.choice([0, q[0]]), rng.choice([0, 4, rng.randint(1, 1600)]), True
    return dict(op=op, kind=kind, page=page, q_lens=_text(q), k_lens=_text(k), q_heads=q_heads, kv_heads=kv_heads, head_dim=head_dim,
                left=left, right=right, sinks=sinks, evicted=evicted)


# ------------------------------------------------------------------------------------------------------ inputs

_DTYPE = {"bf16": torch.bfloat16, "f32": torch.float32}
_BITS = {"fp8": 8, "fp4": 4}
_TOP = {"fp8": (0.875, 9, 7), "fp4": (0.75, 3, 13)}           # largest element as (f, e): f * 2^e, and the largest scale's exponent
_E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _parts(pages, case):
    """Keys, values and their scales as views of the pages: [pages, heads, page, bytes of a token]."""
    row, groups = case["head_dim"] * _BITS[case["kind"]] // 8, case["head_dim"] // 32
    ends = [0, row, 2 * row, 2 * row + groups, 2 * row + 2 * groups]
    return [pages[..., case["page"] * a:case["page"] * b].unflatten(-1, (case["page"], b - a)) for a, b in zip(ends, ends[1:])]


def _power(e):
    """2^e in 32 bits, exactly (int32 tensor, -126 .. 127)."""
    return ((e + 127) << 23).view(torch.float32)


def _encode(x, kind):
    """x: fp32 [..., head_dim] -> (bytes of the elements, bytes of the scales)."""
    g = x.unflatten(-1, (-1, 32))
    f, e = torch.frexp(g.abs().amax(-1, keepdim=True))
    part, top, most = _TOP[kind]
    k = (e - top + (f > part)).clamp(-14, most)
    y = g * _power(-k)
    if kind == "fp8":
        data = y.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).flatten(-2)
    else:
        a = y.abs()
        step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
        a = (torch.round(a / step) * step).clamp(max=6)
        code = torch.searchsorted(torch.tensor(_E2M1, device=x.device), a.contiguous()) + 8 * torch.signbit(y)
        data = (code[..., 0::2] + 16 * code[..., 1::2]).to(torch.uint8).flatten(-2)
    return data, (k + 127).to(torch.uint8).squeeze(-1)


def _decode(data, scales, kind):
    if kind == "fp8":
        y = data.view(torch.float8_e4m3fn).float()
    else:
        code = torch.stack((data & 15, data >> 4), -1).flatten(-2).long()
        y = torch.tensor(_E2M1 + tuple(-v for v in _E2M1), device=data.device)[code]
    return (y.unflatten(-1, (-1, 32)) * _power(scales.to(torch.int32) - 127)[..., None]).flatten(-2)


def _places(case, table, lens, new):
    """Page and place in it of the last `new` (by sequence) tokens of each sequence, one sequence after the other."""
    dev = table.device
    seq = torch.repeat_interleave(torch.arange(len(new), device=dev), torch.tensor(new, device=dev), output_size=sum(new))
    start = torch.tensor([0] + new, device=dev).cumsum(0)
    at = torch.arange(sum(new), device=dev) - start[seq] + (lens.long() - torch.tensor(new, device=dev))[seq]
    return table[seq, at // case["page"]].long(), at % case["page"]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    randn = lambda *shape: torch.randn(shape, device="cuda", generator=g)  # noqa: E731
    q_lens, k_lens, page = _ints(case["q_lens"]), _ints(case["k_lens"]), case["page"]
    H, D, kind = case["kv_heads"], case["head_dim"], case["kind"]
    held = [-(-n // page) for n in k_lens]
    total = sum(held) + 3
    # pages are taken from one pool by all sequences, so a sequence's pages lie anywhere in it
    order = torch.randperm(total, device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(k_lens), max(held + [1]) + 1), -1, dtype=torch.int32, device="cuda")
    for s, n in enumerate(held):
        table[s, :n] = order[sum(held[:s]):sum(held[:s]) + n]
        if case.get("evicted") and case["left"] >= 0:
            first = k_lens[s] - q_lens[s] - case["left"]              # the first key of the first new token's window
            table[s, -(-case["sinks"] // page):max(0, first) // page] = -1
    start = torch.tensor([0] + q_lens, device="cuda").cumsum(0).to(torch.int32)
    state = {"case": case, "table": table, "lens": torch.tensor(k_lens, device="cuda", dtype=torch.int32), "start": start}
    # keys are normed heads with a share that is common to all, values have a few larger channels; both are cached
    unit = lambda x: x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)  # noqa: E731
    common = randn(1, H, D)
    keys = lambda n: unit(randn(n, H, D) + 0.5 * common)  # noqa: E731
    values = lambda n: randn(n, H, D) * torch.where(torch.rand(1, H, D, device="cuda", generator=g) < 0.02, 6.0, 1.0)  # noqa: E731
    pages = torch.zeros(total, H, 2 * page * (D * _BITS[kind] // 8 + D // 32), dtype=torch.uint8, device="cuda")
    kd, vd, ks, vs = _parts(pages, case)
    for data, scales, make in ((kd, ks, keys), (vd, vs, values)):
        for at in range(0, total, 256):                                # (some pages at a time: the fp32 values are larger)
            n = min(256, total - at)
            b, s = _encode(make(n * page).view(n, page, H, D).transpose(1, 2), kind)
            data[at:at + n], scales[at:at + n] = b, s
    state["pages"] = pages
    if case["op"] in ("write", "store"):
        # they leave the fused projection side by side
        kv = torch.cat((keys(sum(q_lens)), values(sum(q_lens))), 1).to(_DTYPE[case["dtype"]])
        state["k"], state["v"] = kv[:, :H], kv[:, H:]
    elif case["op"] == "attention":
        gain = 0.7 + 1.3 * torch.rand(1, case["q_heads"], 1, device="cuda", generator=g)
        q = unit(randn(sum(q_lens), case["q_heads"], D) + 0.5 * common.repeat_interleave(case["q_heads"] // H, 1)) * gain
        state["q"] = q.bfloat16()
    return state


# -------------------------------------------------------------------------------------------------------- runs

def run(state):
    return {"write": _run_write, "store": _run_store, "read": _run_read, "attention": _run_attention}[state["case"]["op"]](state)


def _write(s):
    c = s["case"]
    if own:
        _binding().oq_cache_write(s["pages"], s["k"], s["v"], s["table"], s["lens"], s["start"], kind=c["kind"])
        return
    page, at = _places(c, s["table"], s["lens"], _ints(c["q_lens"]))
    kd, vd, ks, vs = _parts(s["pages"], c)
    kd[page, :, at], ks[page, :, at] = _encode(s["k"].float(), c["kind"])
    vd[page, :, at], vs[page, :, at] = _encode(s["v"].float(), c["kind"])


def _read(s):
    c = s["case"]
    total = sum(_ints(c["q_lens"]))
    if own:
        k, v = _binding().oq_cache_read(s["pages"], c["head_dim"], s["table"], s["lens"], s["start"], total, kind=c["kind"],
                                        out_dtype=_DTYPE[c["dtype"]])
        return {"k": k, "v": v}
    page, at = _places(c, s["table"], s["lens"], _ints(c["q_lens"]))
    kd, vd, ks, vs = _parts(s["pages"], c)
    return {"k": _decode(kd[page, :, at], ks[page, :, at], c["kind"]).to(_DTYPE[c["dtype"]]),
            "v": _decode(vd[page, :, at], vs[page, :, at], c["kind"]).to(_DTYPE[c["dtype"]])}


def _run_write(s):
    _write(s)
    kd, vd, ks, vs = _parts(s["pages"], s["case"])
    return {"k": kd.view(torch.float8_e4m3fn), "v": vd.view(torch.float8_e4m3fn), "k_scale": ks.view(torch.float8_e8m0fnu),
            "v_scale": vs.view(torch.float8_e8m0fnu)}


def _run_store(s):
    _write(s)
    return _read(s)


def _run_read(s):
    return _read(s)


def _run_attention(s):
    c = s["case"]
    q_lens, k_lens = _ints(c["q_lens"]), _ints(c["k_lens"])
    if own:
        out, lse = _binding().oq_cache_attention(s["q"], s["pages"], s["table"], s["lens"], s["start"], kind=c["kind"], left=c["left"],
                                                 right=c["right"], sinks=c["sinks"], max_q=max(q_lens), want_lse=True)
        return {"out": out, "lse": lse}
    dev, q = s["q"].device, s["q"]
    page, at = _places(c, s["table"], s["lens"], k_lens)
    kd, vd, ks, vs = _parts(s["pages"], c)
    here = page >= 0
    k = _decode(kd[page, :, at], ks[page, :, at], c["kind"])
    v = _decode(vd[page, :, at], vs[page, :, at], c["kind"])
    (Tq, H, D), (Tk, Hk, _) = q.shape, k.shape
    lq, lk = torch.tensor(q_lens, device=dev), torch.tensor(k_lens, device=dev)
    sq = torch.repeat_interleave(torch.arange(len(q_lens), device=dev), lq, output_size=Tq)
    sk = torch.repeat_interleave(torch.arange(len(k_lens), device=dev), lk, output_size=Tk)
    i = torch.arange(Tq, device=dev) - (lq.cumsum(0) - lq)[sq]
    p = (i + (lk - lq)[sq])[:, None]                               # a query's place among its keys: ends are aligned
    j = (torch.arange(Tk, device=dev) - (lk.cumsum(0) - lk)[sk])[None, :]
    seen = (sq[:, None] == sk[None, :]) & here[None, :]
    if c["right"] >= 0:
        seen &= j <= p + c["right"]
    if c["left"] >= 0:
        seen &= (j >= p - c["left"]) | (j < c["sinks"])
    qf = q.float().view(Tq, Hk, H // Hk, D).permute(1, 2, 0, 3).reshape(Hk, H // Hk * Tq, D)
    score = torch.matmul(qf, k.permute(1, 2, 0)).mul_(1 / math.sqrt(D)).view(H, Tq, Tk)
    score.masked_fill_(~seen, -math.inf)
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isinf(top), torch.zeros_like(top), top)
    w = score.sub_(top).exp_()
    total = w.sum(-1, keepdim=True)
    o = torch.matmul(w.view(Hk, H // Hk * Tq, Tk), v.permute(1, 0, 2)).view(H, Tq, D)
    o = torch.where(total > 0, o / total, torch.zeros_like(o))
    return {"out": o.permute(1, 0, 2).to(torch.bfloat16), "lse": (top + total.log()).squeeze(-1)}


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
    H, D = case["kv_heads"], case["head_dim"]
    token = 2 * H * (D * _BITS[case["kind"]] // 8 + D // 32)               # bytes of a cached token
    new = sum(_ints(case["q_lens"]))
    if case["op"] == "attention":
        pairs, keys = _visible(case)
        rows = new * case["q_heads"]
        return {"bytes": 4 * rows * D + 4 * rows + keys * token, "flops": 4 * pairs * case["q_heads"] * D}
    values = 2 * new * H * D
    plain = values * (2 if case["dtype"] == "bf16" else 4)
    once = {"write": 1, "read": 1, "store": 2}[case["op"]]
    return {"bytes": once * (plain + new * token), "flops": once * 2 * values}


# ------------------------------------------------------------------------------------------------------- exact

def _two_to(e):
    """2^e in 64 bits, from the bits of the number (a power computed in floating point may be off by a unit)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _element(code, kind):
    """Values of e4m3 bytes or e2m1 halves in 64 bits, from their fields."""
    m_bits, bias = (3, 7) if kind == "fp8" else (1, 1)
    code = code.long()
    sign = 1 - 2 * (code >> (_BITS[kind] - 1)).double()
    exponent = (code >> m_bits) & (15 if kind == "fp8" else 3)
    m = (code & ((1 << m_bits) - 1)).double() / (1 << m_bits)
    return sign * torch.where(exponent > 0, (1 + m) * _two_to(exponent - bias), m * 2.0 ** (1 - bias))


def _nearest(x, kind):
    """x [..., head_dim] in 64 bits -> (elements, exponents of the scales), by the definition."""
    most, digits, low, top = (448.0, 3, -6, 7) if kind == "fp8" else (6.0, 1, 0, 13)
    g = x.unflatten(-1, (-1, 32))
    largest = g.abs().amax(-1, keepdim=True)
    k = torch.full_like(largest, -14, dtype=torch.int64)
    for e in range(-14, top):
        k = torch.where(largest > most * 2.0 ** e, e + 1, k)
    y = g * _two_to(-k)
    unit = _two_to((torch.frexp(y).exponent - 1).clamp(min=low) - digits)
    y = (torch.round(y / unit) * unit).clamp(-most, most)
    return y.flatten(-2), k.squeeze(-1)


def _halves(data, kind):
    return data if kind == "fp8" else torch.stack((data % 16, data // 16), -1).flatten(-2)


def exact(case, seed):
    s = prepare(case, seed)
    kind, page, D = case["kind"], case["page"], case["head_dim"]
    q_lens, k_lens, table = _ints(case["q_lens"]), _ints(case["k_lens"]), s["table"].tolist()
    parts = _parts(s["pages"], case)
    if case["op"] == "write":
        names, out = ("k", "v", "k_scale", "v_scale"), {}
        for name, part in zip(names, parts):
            out[name] = _two_to(part.long() - 127) if "scale" in name else _element(part, kind)
        i = torch.tensor([[table[n][p // page], p % page] for n, (a, b) in enumerate(zip(q_lens, k_lens)) for p in range(b - a, b)],
                         device="cuda").view(-1, 2)
        for name in ("k", "v"):
            y, k = _nearest(s[name].double(), kind)
            out[name][i[:, 0], :, i[:, 1]], out[name + "_scale"][i[:, 0], :, i[:, 1]] = y, _two_to(k)
        return out
    if case["op"] == "store":
        def whole(x):
            y, k = _nearest(x.double(), kind)
            return (y.unflatten(-1, (-1, 32)) * _two_to(k)[..., None]).flatten(-2)
        return {"k": whole(s["k"]), "v": whole(s["v"])}

    def cached(n, first, last):
        """Keys and values of the tokens first .. last - 1 of sequence n, zeros where there is no page."""
        p = torch.arange(first, last, device="cuda")
        row = torch.tensor(table[n], device="cuda")[p // page]
        at = row.clamp(min=0), p % page
        both = []
        for data, scales in (parts[0::2], parts[1::2]):
            y = _element(_halves(data[at[0], :, at[1]], kind), kind).unflatten(-1, (-1, 32))
            y = (y * _two_to(scales[at[0], :, at[1]].long() - 127)[..., None]).flatten(-2)
            both.append(torch.where((row >= 0)[:, None, None], y, 0.0))
        return both[0], both[1], row >= 0

    if case["op"] == "read":
        got = [cached(n, b - a, b) for n, (a, b) in enumerate(zip(q_lens, k_lens))]
        return {"k": torch.cat([k for k, _, _ in got]), "v": torch.cat([v for _, v, _ in got])}
    Tq, H, _ = s["q"].shape
    out = torch.zeros(Tq, H, D, dtype=torch.float64, device="cuda")
    lse = torch.full((H, Tq), -math.inf, dtype=torch.float64, device="cuda")
    q0 = 0
    for n, (nq, nk) in enumerate(zip(q_lens, k_lens)):
        if nq and nk:
            k, v, here = cached(n, 0, nk)
            off, hidden = nk - nq, torch.zeros(nq, nk, dtype=torch.bool, device="cuda")
            if case["left"] >= 0:
                hidden |= torch.ones_like(hidden).tril(off - case["left"] - 1)
                hidden[:, : case["sinks"]] = False
            if case["right"] >= 0:
                hidden |= torch.ones_like(hidden).triu(off + case["right"] + 1)
            hidden |= ~here[None]
            some = ~hidden.all(1)
            for h in range(H):
                hk = h // (H // case["kv_heads"])
                z = (s["q"][q0:q0 + nq, h].double() @ k[:, hk].T / math.sqrt(D)).masked_fill(hidden, -math.inf)
                w = torch.logsumexp(z, 1)
                lse[h, q0:q0 + nq] = w
                out[q0:q0 + nq, h] = torch.exp(z - torch.where(some, w, torch.zeros_like(w))[:, None]) @ v[:, hk]
        q0 += nq
    return {"out": out, "lse": lse}
