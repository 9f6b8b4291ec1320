"""An attention layer whose tokens come in chunks: what each step hands to the next against the fp64 form of that step, and the host's
book-keeping of pages (which needs no GPU)."""
import json

import numpy as np
import pytest
import torch

from oracle import cache as oc
from paper_2607_02461_b200 import attention_layer as al
from paper_2607_02461_b200 import binding as B


def _f64(t):
    return t.double().cpu().numpy()


def test_pages_are_taken_and_given_back():
    c = al.PagedCache(10, 2, 64, requests=3, max_tokens=100, page_size=16, device="cpu")
    c.extend([33, 0, 16])
    assert len(c.free) == 6 and c._lens.tolist() == [33, 0, 16]
    c.extend([14, 1, 0])
    assert len(c.free) == 5                                   # 47 tokens still fit three pages
    taken = c._table[c._table >= 0].tolist()
    assert len(set(taken)) == 5 and not set(taken) & set(c.free)
    with pytest.raises(B.OqError) as e:
        c.extend([0, 0, 84])                                  # six more pages
    assert e.value.code == 6 and c._lens.tolist() == [47, 1, 16] and len(c.free) == 5
    for new in ([54, 0, 0], [1, 1], [-1, 0, 0]):
        with pytest.raises(B.OqError) as e:
            c.extend(new)
        assert e.value.code == 1
    c.forget(0, 33)
    assert c._table[0, :3].tolist()[:2] == [-1, -1] and c._table[0, 2] >= 0 and len(c.free) == 7
    c.forget(0, 1000, keep=47)                                # nothing lies wholly between
    assert len(c.free) == 7
    c.drop(0)
    c.drop(2)
    assert len(c.free) == 9 and c._lens.tolist() == [0, 1, 0] and c._table[0].max() == -1
    c.step()
    assert torch.equal(c.table, c._table) and torch.equal(c.lens, c._lens)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["fp8", "fp4"])
def test_requests_that_go_on(kind):
    """Three requests, two of them in chunks beside single tokens, with adapters, a window, first keys that stay and pages that are given back."""
    layer, x, pos, _, adapters = al.make_layer("small")
    heads, d = layer.heads, layer.head_dim
    cache = al.PagedCache(40, heads, d, 3, 400, page_size=16, kind=kind)
    left, right, sinks = 60, 0, 20
    ids = torch.tensor([1, -1, 0], device="cuda", dtype=torch.int32)
    at = 0
    for new in ([100, 40, 1], [1, 1, 1], [0, 50, 1], [30, 1, 1]):
        before = cache.pages.cpu().numpy()
        cache.extend(new)
        cache.step()
        start = torch.tensor([0] + new, device="cuda").cumsum(0).to(torch.int32)
        n, keep = sum(new), {}
        y = layer(x[at:at + n], pos[at:at + n], start, left, right, sinks, (adapters[0], adapters[1], ids), keep, cache)
        assert y.shape == (n, x.shape[1]) and bool(torch.isfinite(y).all())
        table, lens = cache._table.numpy().astype(np.int64), cache._lens.tolist()
        oc.write(before, _f64(keep["k"]), _f64(keep["v"]), table, lens, new, d, kind)
        assert np.array_equal(cache.pages.cpu().numpy(), before)
        ref, _, size = oc.attention(_f64(keep["q"]), before, table, lens, new, kind, left=left, right=right, sinks=sinks)
        got = _f64(keep["o"]).reshape(ref.shape)
        assert np.all(np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + (2.0 ** -11 + 1e-4) * size + 1e-30)
        for r in range(3):
            cache.forget(r, lens[r] - left, keep=sinks)       # the next token stands at lens[r] and sees from lens[r] - left on
        at += n
    assert len(cache.free) > 40 - sum(-(-n // 16) for n in lens)
    assert B.oq_device_status() == 0


@pytest.mark.gpu
def test_a_cached_chunk_is_the_whole_sequence_at_once():
    """One chunk of a whole request through the cache is the layer without one, up to what 8 bits leave of keys and values."""
    layer, x, pos, _, _ = al.make_layer("small", n_adapters=0)
    n, plain, cached = 200, {}, {}
    layer(x[:n], pos[:n], keep=plain, right=0)
    cache = al.PagedCache(4, layer.heads, layer.head_dim, 1, 256)
    cache.extend([n])
    cache.step()
    layer(x[:n], pos[:n], keep=cached, right=0, cache=cache)
    assert torch.equal(plain["q"], cached["q"]) and torch.equal(plain["k"], cached["k"]) and torch.equal(plain["v"], cached["v"])
    # e4m3 is off by at most 2^-4 of a value: scores by 2^-4 of sum |q k| / sqrt(128) at the very worst, values by 2^-4
    q, k, v = (_f64(plain[name]) for name in ("q", "k", "v"))
    z = np.einsum("ihd,jhd->hij", np.abs(q), np.abs(k)) / np.sqrt(q.shape[2]) / 16
    bound = (np.expm1(2 * z.max()) + 1 / 16) * np.abs(v).max()
    assert np.abs(_f64(plain["o"]) - _f64(cached["o"])).max() <= bound
    first = _f64(cached["o"])[0].reshape(v[0].shape)             # the first token sees itself alone: its own value, cached
    assert np.all(np.abs(first - v[0]) <= (1 / 16 + 2.0 ** -8) * np.abs(v[0]) + 2.0 ** -10)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["fp8", "fp4"])
def test_the_command(kind, capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["attention_layer", "--shape", "small", "--cache", kind, "--chunk", "100", "--iters", "2"])
    al.main()
    line = json.loads(capsys.readouterr().out)
    assert line["cache"] == kind and line["chunk"] == 12 and line["ms_cache_attention"] > 0


@pytest.mark.gpu
def test_a_cache_of_another_head_dim_is_refused():
    layer, x, pos, _, _ = al.make_layer("small", n_adapters=0)
    cache = al.PagedCache(8, layer.heads, {64: 128, 128: 64}[layer.head_dim], 1, 256)
    cache.extend([30])
    cache.step()
    with pytest.raises(B.OqError):
        layer(x[:30], pos[:30], right=0, cache=cache)


@pytest.mark.parametrize("chunk", ["0", "-5"])
def test_chunks_of_no_tokens_are_refused(chunk, capsys, monkeypatch):
    monkeypatch.setattr("sys.argv", ["attention_layer", "--shape", "small", "--cache", "fp8", "--chunk", chunk])
    with pytest.raises(SystemExit) as e:
        al.main()
    assert e.value.code == 2 and "at least one token" in capsys.readouterr().err
