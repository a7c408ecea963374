"""anpd_attention where many rows share keys through LDS (test_host_cache_operators says that these shapes do)."""
import pytest
import torch

from cache_reference import SHARED_DOCUMENTS, SHARED_SHAPES, Filled, attention as reference, check_attention, rows_like
from paper_2404_08698_amd import binding as B

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def run(filled, spans, q, **rules):
    given = B.AttentionRules(**rules) if rules else None
    return B.attention(filled.kvs, filled.layer, q, n_rows=[n for _, n in spans], pos0=[p for p, _ in spans], rules=given, want_lse=True)


def check(shape, q, seed=0, **rules):
    heads, kv_heads, dim, spans = shape
    filled = Filled(heads, kv_heads, dim, [p + n for p, n in spans], seed=seed)
    rows = rows_like(filled, sum(n for _, n in spans), DTYPES[q], seed=seed + 1)
    out, lse = run(filled, spans, rows, **rules)
    check_attention(filled, rows, spans, out, lse, **rules)


@pytest.mark.parametrize("q", ["bf16", "f32"])
@pytest.mark.parametrize("shape", SHARED_SHAPES, ids=str)
def test_plain(shape, q):
    check(shape, q)


@pytest.mark.parametrize("q", ["bf16", "f32"])
@pytest.mark.parametrize("rules", [dict(window=7000), dict(prefix=1), dict(prefix=2040), dict(prefix=9000), dict(window=6900, prefix=700), dict(cap=4.0), dict(scale=0.4)], ids=str)
def test_rules(rules, q):
    check(SHARED_SHAPES[0], q, seed=3, **rules)
    if "window" not in rules:
        check(SHARED_SHAPES[3], q, seed=4, **rules)


@pytest.mark.parametrize("q", ["bf16", "f32"])
def test_distance_bias_and_documents(q):
    shape = SHARED_SHAPES[3]
    heads, kv_heads, dim, spans = shape
    slopes = torch.tensor([2.0 ** -h for h in range(heads)], device="cuda")
    first = torch.tensor([p // 611 * 611 for p0, n in spans for p in range(p0, p0 + n)], dtype=torch.int32)
    first[40:300] = 1 << 30        # whole blocks of rows without a key
    first[600:640] = 1900
    first[-5:] = 1 << 30
    check(shape, q, slopes=slopes)
    check(shape, q, first_key=first.cuda())
    check(shape, q, first_key=first.cuda(), prefix=1000)
    check(shape, q, slopes=slopes, first_key=first.cuda(), prefix=400, window=900, cap=6.0)


@pytest.mark.parametrize("prefix,window", [(0, 0), (100, 0), (100, 2500)])
@pytest.mark.parametrize("length", [611, 1700])
def test_long_documents(length, prefix, window):
    heads, kv_heads, dim, ((_, n),) = SHARED_DOCUMENTS
    filled = Filled(heads, kv_heads, dim, [n])
    rows = rows_like(filled, n)
    first = torch.arange(n, dtype=torch.int32) // length * length
    first[40:300] = 1 << 30        # whole blocks of rows without a key
    first[2000] = 1999
    first[-5:] = 1 << 30
    out, lse = run(filled, [(0, n)], rows, first_key=first.cuda(), prefix=prefix, window=window)
    for at, some in ((0, 330), (1680, 60), (1990, 20), (2900, 100)):
        part = slice(at, at + some)
        check_attention(filled, rows[part], [(at, some)], out[part], lse[part], first_key=first[part], prefix=prefix, window=window)


@pytest.mark.parametrize("q", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_hidden_contents_take_no_part(q, bad):
    heads, kv_heads, dim, spans = SHARED_SHAPES[2]
    (pos0, n), = spans
    filled = Filled(heads, kv_heads, dim, [pos0 + n])
    rows = rows_like(filled, n, DTYPES[q])
    at = pos0 + 300
    v, k = filled.v[0][at].clone(), filled.k[0][pos0 + n - 1].clone()
    v[5] = bad
    filled.put(0, at, v=v)
    k[9] = bad                      # the last key: seen by the last row alone
    filled.put(0, pos0 + n - 1, k=k)
    out, lse = run(filled, spans, rows)
    got = out.cpu().double().reshape(n, heads, dim)
    want, _, size, off, _ = reference(filled, rows, spans)
    want, size = want.reshape(n, heads, dim), size.reshape(n, heads, dim)
    others = [d for d in range(dim) if d != 5]
    assert torch.isfinite(got[:300]).all() and torch.isfinite(lse.cpu()[:n - 1]).all()
    assert not torch.isfinite(got[300:n - 1, :, 5]).any() and not torch.isfinite(got[n - 1, :, 5]).any()
    tol = size * (2.5 * off)[:, :, None] + (3 * 2.0 ** -8 * (size + want.abs()) if q == "bf16" else 0) + 1e-6
    assert ((got - want).abs() <= tol)[:n - 1][:, :, others].all()
    assert ((got - want).abs() <= tol)[:300].all()


def test_large_scores():
    for std in (0.0, 200.0, 1e6, 1e18):
        (pos0, n), = SHARED_SHAPES[2][3]
        filled = Filled(*SHARED_SHAPES[2][:3], [pos0 + n], seed=3)
        rows = rows_like(filled, n, std=std)
        out, lse = run(filled, SHARED_SHAPES[2][3], rows)
        check_attention(filled, rows, SHARED_SHAPES[2][3], out, lse)


@pytest.mark.parametrize("q", ["bf16", "f32"])
def test_replays(q):
    """A captured call, its eager twin and other work in turn: the same bits."""
    heads, kv_heads, dim, spans = SHARED_SHAPES[2]
    (pos0, n), = spans
    filled = Filled(heads, kv_heads, dim, [pos0 + n])
    rows = rows_like(filled, n, DTYPES[q])
    need = B.attention_workspace_bytes(filled.kvs, [n], [pos0])
    ws, out = torch.empty(max(256, need), dtype=torch.uint8, device="cuda"), torch.empty_like(rows)
    want = B.attention(filled.kvs[0], 0, rows, pos0=[pos0]).clone()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        B.attention(filled.kvs[0], 0, rows, pos0=[pos0], out=out, workspace=ws)
    for _ in range(4):
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert torch.equal(B.attention(filled.kvs[0], 0, rows, pos0=[pos0]), want)
