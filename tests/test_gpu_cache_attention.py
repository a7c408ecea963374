"""anpd_attention against 64 bits: types, head layouts, lengths, strides, rules of the scores, hidden contents."""
import pytest
import torch

from cache_reference import Filled, attention as reference, check_attention, rows_like
from paper_2404_08698_amd import binding as B

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def run(filled, spans, q, **rules):
    given = B.AttentionRules(**rules) if rules else None
    return B.attention(filled.kvs, filled.layer, q, n_rows=[n for _, n in spans], pos0=[p for p, _ in spans], rules=given, want_lse=True)


def check(heads, kv_heads, dim, spans, cache="bf16", q="bf16", page_tokens=16, seed=0, **rules):
    filled = Filled(heads, kv_heads, dim, [p + n for p, n in spans], cache, page_tokens, seed=seed)
    rows = rows_like(filled, sum(n for _, n in spans), DTYPES[q], seed=seed + 1)
    out, lse = run(filled, spans, rows, **rules)
    check_attention(filled, rows, spans, out, lse, **rules)


TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")]


@pytest.mark.parametrize("cache,q", TYPES)
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 64), (4, 1, 64), (2, 2, 128), (6, 2, 128), (32, 2, 128)])
@pytest.mark.parametrize("pos0,n", [(0, 1), (1, 1), (15, 1), (127, 1), (128, 1), (500, 3)])
def test_few_rows(heads, kv_heads, dim, pos0, n, cache, q):
    check(heads, kv_heads, dim, [(pos0, n)], cache, q, seed=pos0 + n)


@pytest.mark.parametrize("cache,q", TYPES)
@pytest.mark.parametrize("heads,kv_heads,dim,pos0,n", [(2, 2, 128, 0, 33), (4, 2, 64, 0, 257), (5, 1, 128, 77, 70), (2, 1, 128, 1001, 130), (1, 1, 64, 3000, 2)])
def test_chunks(heads, kv_heads, dim, pos0, n, cache, q):
    check(heads, kv_heads, dim, [(pos0, n)], cache, q, seed=n)


@pytest.mark.parametrize("cache,page_tokens", [("f32", 8), ("f32", 256), ("bf16", 8), ("bf16", 64)])
def test_pages_of_other_sizes(cache, page_tokens):
    check(4, 2, 64, [(300, 17)], cache, "f32", page_tokens)
    check(2, 2, 128, [(0, 9), (1000, 1)], cache, "bf16", page_tokens)


@pytest.mark.parametrize("cache,q", TYPES)
def test_several_sequences(cache, q):
    spans = [(0, 1), (700, 5), (3, 0), (0, 40), (1, 1), (129, 2)]
    check(4, 2, 128, spans, cache, q)
    check(8, 1, 64, [(100 * i, 1) for i in range(64)], cache, q)


RULES = [dict(cap=5.0), dict(cap=256.0), dict(cap=300.0), dict(window=1), dict(window=40), dict(window=200), dict(prefix=1), dict(prefix=130), dict(prefix=5000), dict(scale=0.3),
         dict(cap=30.0, window=33, prefix=50), dict(window=64, prefix=64)]


@pytest.mark.parametrize("cap", [1e6, 1e18, 1e30])
@pytest.mark.parametrize("cache,q", TYPES)
def test_caps_far_above_the_scores_change_nothing(cache, q, cap):
    spans = [(180, 20)]
    filled = Filled(4, 2, 64, [200], cache)
    rows = rows_like(filled, 20, DTYPES[q])
    out, lse = run(filled, spans, rows, cap=cap)
    check_attention(filled, rows, spans, out, lse)


@pytest.mark.parametrize("cache,q", TYPES)
@pytest.mark.parametrize("rules", RULES, ids=str)
def test_rules(rules, cache, q):
    check(4, 2, 64, [(290, 60)], cache, q, **rules)


@pytest.mark.parametrize("cache,q", TYPES)
def test_distance_bias_and_documents(cache, q):
    slopes = torch.tensor([0.5, 0.1, 0.01, 0.0], device="cuda")
    spans = [(190, 70), (0, 20), (60, 1)]
    first = torch.tensor([p // 37 * 37 for p0, n in spans for p in range(p0, p0 + n)], dtype=torch.int32)
    first[-1] = 1 << 30       # no key at all
    first[75:80] = 1000       # above their position: none either
    first[3] = -5
    for rules in (dict(slopes=slopes), dict(first_key=first.cuda()), dict(slopes=slopes, first_key=first.cuda(), window=20),
                  dict(first_key=first.cuda(), prefix=200), dict(slopes=slopes, first_key=first.cuda(), prefix=80, window=20, cap=4.0)):
        check(4, 2, 128, spans, cache, q, **rules)


def test_rows_without_keys_beside_rows_with_many():
    first = torch.full((130,), 1 << 30, dtype=torch.int32)
    first[64] = 0
    for cache, q in TYPES:
        check(2, 2, 64, [(600, 130)], cache, q, first_key=first.cuda())


@pytest.mark.parametrize("cache,q", TYPES)
@pytest.mark.parametrize("bad", [float("inf"), float("-inf"), float("nan")])
def test_hidden_contents_take_no_part(cache, q, bad):
    """Keys and values that a row does not see may hold anything, in tiles that other rows see as well."""
    filled = Filled(2, 1, 128, [300], cache)
    rows = rows_like(filled, 40, DTYPES[q])
    spans = [(260, 40)]
    for pos in (280, 299):       # hidden from the rows before them
        v = filled.v[0][pos].clone()
        v[5] = bad
        k = filled.k[0][pos].clone()
        if pos == 299:
            k[7] = bad
        filled.put(0, pos, k, v)
    out, lse = run(filled, spans, rows)
    want, want_lse, size, off, _ = reference(filled, rows, spans)
    got = out.cpu().double()
    assert torch.isfinite(got[:20]).all() and torch.isfinite(lse.cpu()[:39]).all()
    # rows 20 .. 38 see the first value: not finite in that dim alone; the last row also a key whose score is not
    per_head = got.reshape(40, 2, 128)
    assert not torch.isfinite(per_head[20:39, :, 5]).any()
    others = [d for d in range(128) if d != 5]
    assert torch.isfinite(per_head[:39][:, :, others]).all()
    assert not torch.isfinite(per_head[39, :, 5]).any()
    tol = size * (2.5 * off).repeat_interleave(128, 1) + (3 * 2.0 ** -8 * (size + want.abs()) if q == "bf16" else 0) + 1e-6
    assert ((got - want).abs() <= tol).reshape(40, 2, 128)[:39][:, :, others].all()


def test_what_lies_behind_the_last_key_takes_no_part():
    """A page's rest may hold what was written for rows that were taken back."""
    for cache, q in TYPES:
        filled = Filled(2, 2, 64, [200], cache)
        n = 61
        bad = torch.full((200 - 100 - n, 128), float("nan"))
        filled.kvs[0].write(0, 100 + n, bad.cuda(), bad.cuda())
        rows = rows_like(filled, n, DTYPES[q])
        out, lse = run(filled, [(100, n)], rows)
        check_attention(filled, rows, [(100, n)], out, lse)


@pytest.mark.parametrize("q", ["bf16", "f32"])
@pytest.mark.parametrize("pitch,shift", [(0, 0), (257, 0), (264, 0), (300, 1), (259, 3)])
def test_strides_and_alignment(q, pitch, shift):
    filled = Filled(2, 2, 128, [90])
    store = rows_like(filled, 31, DTYPES[q], pitch=pitch + shift)
    wide = torch.zeros(31, 256 + pitch + shift, dtype=DTYPES[q], device="cuda")
    rows = wide[:, shift:shift + 256]
    rows.copy_(store)
    keep = torch.full((33, 256 + pitch + 2 * shift), 7.0, dtype=DTYPES[q], device="cuda")
    out = keep[1:32, shift:shift + 256]
    lse = torch.empty(31, 2, device="cuda")
    got = B.attention(filled.kvs[0], 0, rows, pos0=[59], out=out, lse=lse)
    assert got[0] is out
    check_attention(filled, rows, [(59, 31)], out, lse)
    mask = torch.ones_like(keep, dtype=torch.bool)
    mask[1:32, shift:shift + 256] = False
    assert (keep[mask] == 7).all()          # what surrounds the rows is left as it was


def test_out_may_be_the_rows_themselves():
    filled = Filled(4, 2, 64, [500])
    for n, pos0 in ((1, 499), (130, 370)):
        rows = rows_like(filled, n)
        want = B.attention(filled.kvs[0], 0, rows, pos0=[pos0])
        assert torch.equal(B.attention(filled.kvs[0], 0, rows, pos0=[pos0], out=rows), want)


def test_large_scores_and_small_ones():
    """Scores far beyond the range of exp, positive and negative, and queries of zero."""
    for cache, q in TYPES:
        for std in (0.0, 1e-20, 300.0, 1e6):
            filled = Filled(2, 2, 64, [150], cache, seed=3)
            rows = rows_like(filled, 5, DTYPES[q], std=std)
            out, lse = run(filled, [(145, 5)], rows)
            check_attention(filled, rows, [(145, 5)], out, lse)


def test_scores_of_any_size():
    """One key per row wins by far: the answer is its value, however large the scores are."""
    for cache, q in TYPES:
        filled = Filled(1, 1, 64, [64], cache)
        for pos in range(64):
            k = torch.zeros(64)
            k[pos] = 1.0
            filled.put(0, pos, k)
        rows = torch.zeros(4, 64, dtype=DTYPES[q])
        for r, (pos, size) in enumerate(((3, 1e4), (60, 1e9), (17, 1e15), (31, 1e30))):
            rows[r, pos] = size
        out, lse = run(filled, [(60, 4)], rows.cuda(), scale=1.0)
        got = out.cpu().float()
        for r, pos in enumerate((3, 60, 17, 31)):
            assert torch.equal(got[r], filled.v[0][pos].to(DTYPES[q]).float()), (cache, q, r)   # (rounded once to the rows' type)
        assert torch.allclose(lse.cpu()[:, 0], rows.float().amax(1), rtol=1e-6)


def test_same_cache_twice_and_other_layers():
    filled = Filled(4, 4, 64, [300], layers=3, layer=1)
    rows = rows_like(filled, 6)
    two = B.attention([filled.kvs[0]] * 2, 1, rows, n_rows=[5, 1], pos0=[100, 299])
    a = B.attention(filled.kvs[0], 1, rows[:5], pos0=[100])
    b = B.attention(filled.kvs[0], 1, rows[5:], pos0=[299])
    # (the keys are divided among blocks by the sizes of a call: equal to rounding)
    assert (two.float() - torch.cat([a, b]).float()).abs().max() <= 2.0 ** -6
    check_attention(filled, rows, [(100, 5), (299, 1)], *run(Same(filled), [(100, 5), (299, 1)], rows))


class Same:
    """One cache as two sequences."""

    def __init__(self, filled):
        self.kvs, self.layer = filled.kvs * 2, filled.layer
        filled.k, filled.v = filled.k * 2, filled.v * 2


def test_positions_default_to_the_committed_length():
    filled = Filled(2, 2, 64, [50])
    filled.kvs[0].write(0, 0, filled.k[0].cuda(), filled.v[0].cuda())
    filled.kvs[0].truncate(50)
    filled.kvs[0].truncate(45)
    more = torch.randn(3, 128).bfloat16().float()
    filled.kvs[0].write(0, 45, more.cuda(), more.cuda())
    rows = rows_like(filled, 3)
    assert torch.equal(B.attention(filled.kvs[0], 0, rows), B.attention(filled.kvs[0], 0, rows, pos0=[45]))


def test_offsets_past_32_bits():
    """A pool of more than 2^32 bytes: the last pages of the last layer."""
    layers, n = 64, 4900
    filled = Filled(32, 32, 128, [n], layers=layers, layer=layers - 1, scattered=False)
    assert filled.kvs[0].pool.numel() > 1 << 32
    rows = rows_like(filled, 2)
    out, lse = run(filled, [(n - 2, 2)], rows)
    check_attention(filled, rows, [(n - 2, 2)], out, lse)
    filled.kvs.clear()
    torch.cuda.empty_cache()


def test_another_stream_and_a_given_workspace():
    filled = Filled(2, 1, 128, [5000])
    rows = rows_like(filled, 1)
    need = B.attention_workspace_bytes(filled.kvs, [1], [4999])
    assert need > 0
    want = B.attention(filled.kvs[0], 0, rows, pos0=[4999])
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    out = torch.empty_like(rows)
    B.attention(filled.kvs[0], 0, rows, pos0=[4999], out=out, workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(out, want)
    with pytest.raises(B.AnpdError) as e:
        B.attention(filled.kvs[0], 0, rows, pos0=[4999], workspace=ws[:256])
    assert e.value.code == B.E_CAPACITY


@pytest.mark.parametrize("cache,q", TYPES)
def test_captured_calls(cache, q):
    """Replays, with eager calls and other contents between them."""
    filled = Filled(4, 2, 128, [3000], cache)
    rows, other = rows_like(filled, 2, DTYPES[q]), rows_like(filled, 2, DTYPES[q], seed=9)
    rules = B.AttentionRules(window=2500)
    kw = dict(pos0=[2998], rules=rules)
    want = [B.attention(filled.kvs[0], 0, x, **kw).clone() for x in (rows, other)]
    static, out = rows.clone(), torch.empty_like(rows)
    ws = torch.empty(max(256, B.attention_workspace_bytes(filled.kvs, [2], [2998], rules)), dtype=torch.uint8, device="cuda")
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        B.attention(filled.kvs[0], 0, static, out=out, workspace=ws, **kw)
    s.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=s):
        B.attention(filled.kvs[0], 0, static, out=out, workspace=ws, **kw)
    for i in (0, 1, 0, 0, 1):
        static.copy_((rows, other)[i])
        out.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, want[i])
        assert torch.equal(B.attention(filled.kvs[0], 0, (rows, other)[1 - i], **kw), want[1 - i])


def test_repeated_calls_agree_bit_for_bit():
    filled = Filled(8, 2, 128, [2000])
    rows = rows_like(filled, 40)
    first = B.attention(filled.kvs[0], 0, rows, pos0=[1960])
    for _ in range(5):
        assert torch.equal(B.attention(filled.kvs[0], 0, rows, pos0=[1960]), first)


@pytest.mark.parametrize("cache,q", TYPES)
def test_the_largest_windows_and_prefixes(cache, q):
    """A window of 2^31 - 1 hides nothing; a prefix of as much is all that is cached, up to the last new row, and no more."""
    largest = (1 << 31) - 1
    spans = [(290, 60), (0, 3), (100, 1)]
    check(4, 2, 64, spans, cache, q, window=largest)
    check(4, 2, 64, spans, cache, q, prefix=largest)
    check(4, 2, 64, spans, cache, q, prefix=largest, window=largest)
    filled = Filled(4, 2, 64, [400], cache)
    with pytest.raises(ValueError):
        B.attention(filled.kvs, 0, rows_like(filled, 1, DTYPES[q]), pos0=[1 << 32])
