"""anpd_attention with windows, prefixes and documents where many rows share keys through LDS, heads of 64 and 128, both types, against 64 bits
(test_host_cache_operators says that these calls take that form)."""
from types import SimpleNamespace

import pytest
import torch

from cache_reference import Filled, check_attention, rows_like
from paper_2404_08698_amd import binding as B
from shared_forms import SEVERAL, cases

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def first_keys(spans, document):
    """Documents of that many positions, and rows without a key: blocks of them, single ones and the last."""
    first = torch.tensor([p // document * document for pos0, n in spans for p in range(pos0, pos0 + n)], dtype=torch.int32)
    first[40:300] = 1 << 30
    first[2000] = 1999
    first[2001] = 1 << 30
    first[-5:] = 1 << 30
    return first


def parts(pos0, n, rules):
    """Rows that are looked at, in turn: the first ones (with as many keys as a prefix has), some between, around the beginning of a document, the last."""
    least = max(0, min(rules.get("prefix", 0), pos0 + n) - pos0)
    first = min(n, max(70, least))
    yield 0, first
    for at in (n // 3, rules.get("document", 0) * 2 - 20 if "document" in rules else n // 2, 1990, n - 67):
        if first <= at < n:
            yield at, min(67, n - at)


def check(filled, spans, q, out, lse, **rules):
    first, at = rules.pop("first_key", None), 0
    for s, (pos0, n) in enumerate(spans):
        one = SimpleNamespace(heads=filled.heads, kv_heads=filled.kv_heads, dim=filled.dim, k=[filled.k[s]], v=[filled.v[s]])
        for r, some in parts(pos0, n, rules):
            rows = slice(at + r, at + r + some)
            given = {k: v for k, v in rules.items() if k != "document"}
            if first is not None:
                given["first_key"] = first[rows]
            check_attention(one, q[rows], [(pos0 + r, some)], out[rows], lse[rows], **given)
        at += n


def run(filled, spans, q, **rules):
    rules.pop("document", None)
    return B.attention(filled.kvs, 0, q, n_rows=[n for _, n in spans], pos0=[p for p, _ in spans], rules=B.AttentionRules(**rules), want_lse=True)


@pytest.mark.parametrize("shape,q,rules", cases(), ids=str)
def test_rules(shape, q, rules):
    heads, kv_heads, dim, spans = shape
    filled = Filled(heads, kv_heads, dim, [p + n for p, n in spans], seed=len(str(rules)))
    rows = rows_like(filled, sum(n for _, n in spans), DTYPES[q])
    rules = dict(rules)
    if "document" in rules:
        rules["first_key"] = first_keys(spans, rules["document"]).cuda()
    out, lse = run(filled, spans, rows, **rules)
    check(filled, spans, rows, out, lse, **rules)


@pytest.mark.parametrize("q", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_what_a_window_hides_takes_no_part(dim, q, bad):
    """An unbounded value counts for the rows whose window it lies in and for no other."""
    heads, kv_heads, spans, window, at = 32, 2, SEVERAL, 1000, 1800
    pos0, n = spans[0]
    filled = Filled(heads, kv_heads, dim, [p + m for p, m in spans])
    rows = rows_like(filled, sum(m for _, m in spans), DTYPES[q])
    want, want_lse = run(filled, spans, rows, window=window)
    v = filled.v[0][at].clone()
    v[3] = bad
    filled.put(0, at, v=v)
    k = filled.k[0][1000].clone()       # seen by none, in a tile that is visited
    k[5] = bad
    filled.put(0, 1000, k=k, v=torch.full_like(v, bad))
    out, lse = run(filled, spans, rows, window=window)
    assert torch.equal(lse, want_lse)
    got, want = out.reshape(-1, heads, dim), want.reshape(-1, heads, dim)
    # rows pos0 .. see it while at > position - window: all rows up to position at + window - 1
    see = min(n, at + window - pos0)
    assert see == n
    assert not torch.isfinite(got[:n, :heads // kv_heads, 3]).any()
    others = torch.ones_like(got, dtype=torch.bool)
    others[:n, :heads // kv_heads, 3] = False
    assert torch.equal(got[others], want[others])

    v[3] = 1.0
    filled.put(0, at, v=v)
    filled.put(0, 1300, v=torch.full_like(v, bad))      # rows up to position 2299
    out, _ = run(filled, spans, rows, window=window)
    got = out.reshape(-1, heads, dim)
    assert not torch.isfinite(got[:300]).any() and torch.isfinite(got[300:]).all()
