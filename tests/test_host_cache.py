"""CPU checks of the paged cache: its oracle against torch's own types, sizes, and the refusals that need no device."""
import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2607_02461_b200 import binding as B
from paper_2607_02461_b200 import build as oqbuild


@pytest.fixture(scope="module", autouse=True)
def built():
    oqbuild.build()


def _code(fn, *a, **k):
    with pytest.raises(B.OqError) as e:
        fn(*a, **k)
    return e.value.code


def test_oracle_formats():
    """Element tables and rounding against torch's e4m3; e2m1 against its eight magnitudes and ties to even."""
    t = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    v = oc.values("fp8")
    assert np.array_equal(np.isnan(t), np.isnan(v)) and np.array_equal(t[~np.isnan(t)], v[~np.isnan(v)])
    assert oc.values("fp4").tolist()[:8] == [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    g = torch.Generator().manual_seed(1)
    x = torch.randn(200, 64, generator=g) * torch.exp(3 * torch.randn(200, 1, generator=g))
    code, scale = oc.encode(x.double().numpy(), "fp8")
    y = x.unflatten(-1, (-1, 32)) / torch.exp2(torch.from_numpy(scale.astype(np.float32)) - 127)[..., None]
    want = y.flatten(-2).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy()
    assert np.array_equal(code, want)
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 0.0] * 4) * 2.0 ** -14            # the scale stays at its least
    code, scale = oc.encode(ties, "fp4")
    assert scale.tolist() == [113] and code.tolist()[:8] == [0, 2, 2, 4, 4, 6, 6, 0]


def test_oracle_scales():
    """The smallest power of two with which the largest magnitude stays within the format, in its limits."""
    for kind, top, most in (("fp8", 448.0, 7), ("fp4", 6.0, 13)):
        for e in (-14, -3, 0, most - 1):
            for x, want in ((top * 2.0 ** e, e), (np.nextafter(top * 2.0 ** e, np.inf), e + 1)):
                assert oc.encode(np.array([x] + [0.0] * 31), kind)[1][0] == want + 127
        assert oc.encode(np.zeros(32), kind)[1][0] == 113
        code, scale = oc.encode(np.array([1e30, -1e30] + [0.0] * 30), kind)
        assert scale[0] == most + 127 and oc.decode(code, scale, kind)[:2].tolist() == [top * 2.0 ** most, -top * 2.0 ** most]


def test_block_bytes():
    for kind in ("fp8", "fp4"):
        for d in (64, 128):
            for page in (16, 32, 64, 128, 256):
                assert B.oq_cache_block_bytes(page, d, kind) == oc.block_bytes(page, d, kind)
    assert _code(B.oq_cache_block_bytes, 24, 128) == 2
    assert _code(B.oq_cache_block_bytes, 8, 128) == 2
    assert _code(B.oq_cache_block_bytes, 512, 128) == 2
    assert _code(B.oq_cache_block_bytes, 64, 96) == 2
    assert _code(B.oq_cache_block_bytes, 64, 128, "int8") == 1


def test_host_tensors_are_refused():
    pages = B.oq_cache_alloc(3, 16, 2, 64, device="cpu")
    table, lens = torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, dtype=torch.int32)
    k = torch.zeros(4, 2, 64, dtype=torch.bfloat16)
    assert _code(B.oq_cache_write, pages, k, k, table, lens) == 1
    assert _code(B.oq_cache_read, pages, 64, table, lens, None, 4) == 1
    assert _code(B.oq_cache_attention, k, pages, table, lens) == 1


def _cache(**fields):
    """An oq_cache of one sequence: 4 pages of 16 tokens of 2 heads of 64.  (The buffers are not memory: a call that is not refused for its
    arguments ends with a CUDA error, as there is no device.)"""
    if torch.cuda.is_available():
        pytest.skip("made-up buffers are for hosts without a device")
    at = dict(pages=4096, table=8192, lens=12288, ld=4, n_pages=4, page=16, heads=2, d=64, kind=8, seqs=1, max_pages=4)
    at.update(fields)
    return B._CACHE.pack(*(at[n] for n in ("pages", "table", "lens", "ld", "n_pages", "page", "heads", "d", "kind", "seqs", "max_pages")))


BAD_CACHES = [(dict(kind=7), 1), (dict(page=20), 2), (dict(d=80), 2), (dict(n_pages=-1), 1), (dict(heads=0), 1), (dict(heads=65536), 2),
              (dict(seqs=0), 1), (dict(seqs=257, ld=4), 2), (dict(max_pages=-1), 1), (dict(max_pages=(1 << 26) + 1, ld=1 << 27), 2), (dict(pages=0), 1),
              (dict(table=0), 1), (dict(lens=0), 1), (dict(seqs=2, ld=3), 1), (dict(pages=4104), 3)]


@pytest.mark.parametrize("fields,code", BAD_CACHES, ids=str)
def test_bad_caches_are_refused(fields, code):
    cache, row = _cache(**fields), B._CACHE_ROWS.pack(16384, 128, 64)
    L = B.lib()
    assert L.oq_cache_write(cache, row, row, 0, 65536, 4, None) == code
    assert L.oq_cache_read(cache, row, row, 0, 65536, 4, None) == code
    args = cache + B.struct.pack("@PqqPqqPPiiiiiif", 16384, 128, 64, 32768, 128, 64, 0, 65536, 4, 2, 0, -1, 0, 0, 0.0)
    assert L.oq_cache_attention(args, None, 0, None) == code


def test_the_longest_rows_of_a_table_are_taken():
    row = B._CACHE_ROWS.pack(16384, 128, 64)
    assert B.lib().oq_cache_write(_cache(max_pages=1 << 26, ld=1 << 26), row, row, 0, 65536, 4, None) == 4        # (no device)


@pytest.mark.parametrize("write", [True, False])
def test_bad_rows_are_refused(write):
    L, cache = B.lib(), _cache()
    def code(k=(16384, 128, 64), v=(20480, 128, 64), dtype=0, total=4, start=65536, c=cache):
        pack = lambda r: None if r is None else B._CACHE_ROWS.pack(*r)  # noqa: E731
        return (L.oq_cache_write if write else L.oq_cache_read)(c, pack(k), pack(v), dtype, start, total, None)
    assert code(total=0) == 0 and code() == 4                    # (nothing to do; no device)
    assert code(k=None, v=None) == 1
    assert code(k=None) == (1 if write else 4)
    assert code(k=(0, 128, 64)) == 1
    assert code(k=(16392, 128, 64)) == 3
    assert code(v=(20480, 132, 64)) == 3                         # 8-byte rows
    assert code(v=(20480, 132, 64), dtype=1) == 4                # which are 16 bytes of fp32
    assert code(k=(16384, 0, 0)) == (4 if write else 1)          # read rows may not lie over each other
    assert code(k=(16384, -128, 64)) == 1
    assert code(dtype=2) == 1
    assert code(total=-1) == 1
    assert code(total=(1 << 30) + 1) == 2
    assert code(c=_cache(seqs=2), start=0) == 1


def test_bad_attention_arguments_are_refused():
    names = ("Q", "qt", "qh", "out", "ot", "oh", "lse", "start", "total", "heads", "max_q", "left", "right", "sinks", "scale")
    def code(size=0, c=None, **fields):
        at = dict(Q=16384, qt=256, qh=64, out=32768, ot=256, oh=64, lse=0, start=65536, total=4, heads=4, max_q=0, left=-1, right=0, sinks=0, scale=0.0)
        at.update(fields)
        args = (c or _cache()) + B.struct.pack("@PqqPqqPPiiiiiif", *(at[n] for n in names))
        return B.lib().oq_cache_attention(args, 1 << 20 if size else None, size, None)
    assert code(total=0) == 0
    assert code() == 4                                           # no device; of 64 positions nothing is ever cut, so no workspace is wanted
    assert code(c=_cache(max_pages=32, ld=32)) == 4              # nor of 512
    long = _cache(max_pages=64, ld=64)
    assert code(c=long) == 6 and code(c=long, size=1 << 30) == 4
    for field in ("Q", "out"):
        assert code(**{field: 0}) == 1 and code(**{field: 16392}) == 3
    for field in ("qt", "qh", "ot", "oh"):
        assert code(**{field: 260}) == 3
    assert code(qt=0, qh=0) == 4 and code(qt=-256) == 1 and code(ot=56) == 1 and code(oh=0) == 1
    assert code(heads=3) == 1 and code(heads=0) == 1 and code(total=-1) == 1 and code(max_q=-1) == 1
    assert code(sinks=-1) == 1 and code(scale=-1.0) == 1 and code(scale=float("nan")) == 1 and code(scale=1e30) == 1
    assert code(total=1 << 30, heads=4) == 2
    assert code(c=_cache(seqs=2), start=0) == 1


def _rows(tokens, heads, lt, lh, d):
    return [h * lh + t * lt + c for t in range(tokens) for h in range(heads) for c in range(d)]


def _layouts(d, unit):
    """(tokens, heads, strides) with strides of at least a row: rows side by side in both orders, padded, dealt out between each other, and over each other."""
    g = np.random.default_rng(3)
    out = [(3, 2, 2 * d, d), (3, 2, d, 3 * d), (3, 2, d, d), (3, 2, d, 2 * d), (4, 3, 2 * d, 8 * d), (4, 3, 3 * d, 2 * d), (1, 4, 0, d), (4, 1, d, 0), (2, 2, d, d + unit), (3, 3, 4 * d, 2 * d)]
    return out + [(int(t), int(h), int(a) * unit, int(b) * unit) for t, h, a, b in zip(*g.integers(1, 5, (2, 40)), *g.integers(d // unit, 5 * d // unit, (2, 40)))]


@pytest.mark.parametrize("dtype", [0, 1])
def test_read_rows_over_each_other_are_refused(dtype):
    """Against all addresses: rows of one output, and keys over values."""
    d, unit, size = 64, (8, 4)[dtype], (2, 4)[dtype]
    L, pack = B.lib(), B._CACHE_ROWS.pack
    for tokens, heads, lt, lh in _layouts(d, unit):
        rows = _rows(tokens, heads, lt, lh, d)
        clash = len(set(rows)) < len(rows)
        for other in [None] + [unit * x for x in (-40, -32, -24, -16, -9, -8, -7, 0, 1, 8, 9, 16, 24, 32, 40, 96)]:
            v = None if other is None else pack((1 << 20) + size * other, lt, lh)
            meet = other is not None and bool(set(rows) & {x + other for x in rows})
            assert L.oq_cache_read(_cache(heads=heads), pack(1 << 20, lt, lh), v, dtype, 65536, tokens, None) == (1 if clash or meet else 4), (tokens, heads, lt, lh, other)
    assert L.oq_cache_read(_cache(), pack(1 << 20, 128, 64), pack(1 << 20, 256, 64), dtype, 65536, 4, None) == 1        # one beginning, other strides
    assert L.oq_cache_write(_cache(), pack(1 << 20, 0, 64), pack(1 << 20, 0, 64), dtype, 65536, 4, None) == 4           # what is only read may


def test_results_over_queries_or_each_other_are_refused():
    d, L = 64, B.lib()
    def code(tokens, heads, q, ql, out, ol):
        return L.oq_cache_attention(_cache(heads=heads) + B.struct.pack("@PqqPqqPPiiiiiif", q, *ql, out, *ol, 0, 65536, tokens, heads, 0, -1, 0, 0, 0.0), None, 0, None)
    base = 1 << 20
    for tokens, heads, lt, lh in _layouts(d, 8):
        rows = _rows(tokens, heads, lt, lh, d)
        clash = len(set(rows)) < len(rows)
        assert code(tokens, heads, 2 * base, (0, 0), base, (lt, lh)) == (1 if clash else 4)
        for other in (-256, -192, -128, -72, -64, -56, 0, 8, 64, 72, 128, 192, 256, 768):
            meet = bool(set(rows) & {x + other for x in rows})
            assert code(tokens, heads, base, (lt, lh), base + 2 * other, (lt, lh)) == (1 if clash or meet else 4), (tokens, heads, lt, lh, other)
    assert code(3, 2, base, (0, 0), base, (128, 64)) == 1        # queries broadcast from where the results begin
    assert code(1, 1, base, (999 * 8, 8), base + 128, (8, 999 * 8)) == 4      # strides of one token and one head are not used
