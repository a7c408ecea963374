"""anpd_key_mass against 64 bits."""
import math

import pytest
import torch

from cache_reference import U, Filled, attention as reference, rows_like
from paper_2404_08698_amd import binding as B

pytestmark = pytest.mark.gpu
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
TYPES = [("bf16", "bf16"), ("bf16", "f32"), ("f32", "f32"), ("f32", "bf16")]


def check(heads, kv_heads, dim, spans, cache="bf16", q="bf16", page_tokens=16, seed=0, **rules):
    filled = Filled(heads, kv_heads, dim, [p + n for p, n in spans], cache, page_tokens, seed=seed)
    rows = rows_like(filled, sum(n for _, n in spans), DTYPES[q], seed=seed + 1)
    _, lse, _, off, want = reference(filled, rows, spans, **rules)
    longest = max(p + n for p, n in spans)
    before = torch.rand(len(spans), kv_heads, longest + 5, device="cuda")
    mass = before.clone()
    given = B.AttentionRules(**rules) if rules else None
    got = B.key_mass(filled.kvs, 0, rows, lse.float().cuda(), mass, n_rows=[n for _, n in spans], pos0=[p for p, _ in spans], rules=given)
    assert got is mass
    at = 0
    for s, (p, n) in enumerate(spans):
        total = p + n if n else 0
        assert torch.equal(mass[s, :, total:], before[s, :, total:])       # left as they were
        if n == 0:
            continue
        part = off[at:at + n]
        at += n
        worst = part[torch.isfinite(part)].max().item()
        lses = lse[at - n:at]
        size = lses[torch.isfinite(lses)].abs().max().item() if torch.isfinite(lses).any() else 0.0
        exact = want[s] + before[s, :, :total].cpu().double()
        # a score's error, the rounding of the lse that the call is given, and the sums' own
        allowed = want[s] * (2 * worst + 4 * U * size + (n * heads // kv_heads + 64) * U) + 2 * U * exact + 1e-37
        diff = (mass[s, :, :total].cpu().double() - exact).abs()
        assert (diff <= allowed).all(), (s, (diff / allowed).max().item())


@pytest.mark.parametrize("cache,q", TYPES)
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 64), (4, 1, 64), (2, 2, 128), (32, 2, 128)])
@pytest.mark.parametrize("pos0,n", [(0, 1), (127, 1), (128, 2), (500, 33), (0, 150)])
def test_mass(heads, kv_heads, dim, pos0, n, cache, q):
    check(heads, kv_heads, dim, [(pos0, n)], cache, q, seed=n)


@pytest.mark.parametrize("cache,q", TYPES)
def test_rows_dealt_to_several_blocks(cache, q):
    check(8, 1, 64, [(0, 300)], cache, q)
    check(2, 1, 128, [(20, 1000)], cache, q, window=100, prefix=30)


@pytest.mark.parametrize("cache,q", TYPES)
@pytest.mark.parametrize("rules", [dict(cap=5.0), dict(window=1), dict(window=40), dict(prefix=130), dict(prefix=5000), dict(scale=0.3),
                                   dict(cap=30.0, window=33, prefix=50)], ids=str)
def test_rules(rules, cache, q):
    check(4, 2, 64, [(290, 60), (0, 3)], cache, q, **rules)


@pytest.mark.parametrize("cache,q", TYPES)
def test_sequences_bias_and_documents(cache, q):
    spans = [(190, 70), (0, 20), (5, 0), (60, 1)]
    first = torch.tensor([p // 37 * 37 for p0, n in spans for p in range(p0, p0 + n)], dtype=torch.int32)
    first[-1] = 1 << 30
    first[75:80] = 1000
    check(4, 2, 128, spans, cache, q, first_key=first.cuda(), slopes=torch.tensor([0.5, 0.1, 0.01, 0.0], device="cuda"))
    check(4, 2, 128, spans, cache, q, first_key=first.cuda(), prefix=100, window=9)


def test_hidden_keys_may_hold_anything():
    for cache, q in TYPES:
        filled = Filled(2, 1, 128, [300], cache)
        rows = rows_like(filled, 20, DTYPES[q])
        lse = torch.zeros(20, 2, device="cuda")
        bad = torch.full((30, 128), float("nan"), device="cuda")
        filled.kvs[0].write(0, 270, bad, bad)
        mass = torch.zeros(1, 300, device="cuda")
        B.key_mass(filled.kvs[0], 0, rows, lse, mass, pos0=[250])
        assert torch.isfinite(mass).all() and (mass[0, 270:] == 0).all() and (mass[0, :250] > 0).all()
        lse[3] = -math.inf
        lse[4:] = math.inf
        mass.zero_()
        B.key_mass(filled.kvs[0], 0, rows, lse, mass, pos0=[250])
        assert (mass[0, 253:] == 0).all()


def test_weights_of_all_keys_add_up_to_the_rows():
    """After attention on the same rows; and the same bits every time."""
    filled = Filled(6, 2, 128, [700, 90])
    rows = rows_like(filled, 60)
    n_rows, pos0 = [50, 10], [650, 80]
    _, lse = B.attention(filled.kvs, 0, rows, n_rows=n_rows, pos0=pos0, want_lse=True)
    mass = torch.zeros(2, 2, 700, device="cuda")
    B.key_mass(filled.kvs, 0, rows, lse, mass, n_rows=n_rows, pos0=pos0)
    for s, n in enumerate(n_rows):
        assert (mass[s].double().sum(1) - 3 * n).abs().max() < 1e-3 * n
    for _ in range(3):
        again = torch.zeros_like(mass)
        B.key_mass(filled.kvs, 0, rows, lse, again, n_rows=n_rows, pos0=pos0)
        assert torch.equal(again, mass)


@pytest.mark.parametrize("cache,q", TYPES)
@pytest.mark.parametrize("rules", [{}, dict(window=300), dict(cap=5.0)], ids=str)
def test_rows_that_add_nothing_may_hold_anything(cache, q, rules):
    """An lse of -infinity takes a row out of the sums: the bits are those of a call whose row holds zeros there.  First, last and in
    between, in row tiles of one and of several rows, and with keys that all rows see."""
    filled = Filled(4, 2, 64, [400], cache)
    given = B.AttentionRules(**rules) if rules else None
    for n, out in ((300, (0, 20, 299)), (75, (0, 20, 74)), (1, (0,)), (16, (3, 15))):
        rows = rows_like(filled, n, DTYPES[q]).clone()
        at = dict(pos0=[400 - n], rules=given)
        _, lse = B.attention(filled.kvs[0], 0, rows, want_lse=True, **at)
        masses = []
        for value in (0.0, float("nan"), float("inf"), float("-inf")):
            for r in out:
                rows[r] = value
                lse[r] = -math.inf
            masses.append(B.key_mass(filled.kvs[0], 0, rows, lse, torch.zeros(2, 400, device="cuda"), **at))
        assert torch.isfinite(masses[0]).all() and (masses[0].sum() > 0) == (n > len(out))
        for got in masses[1:]:
            assert torch.equal(got, masses[0])


def test_masses_of_sequences_between_each_others_rows():
    """[key heads][sequences][keys] seen as [sequences][key heads][keys]."""
    filled = Filled(4, 2, 64, [300, 77, 300])
    rows = rows_like(filled, 9)
    at = dict(n_rows=[2, 4, 3], pos0=[298, 60, 200])
    _, lse = B.attention(filled.kvs, 0, rows, want_lse=True, **at)
    want, store = torch.zeros(3, 2, 300, device="cuda"), torch.zeros(2, 3, 300, device="cuda")
    B.key_mass(filled.kvs, 0, rows, lse, want, **at)
    got = B.key_mass(filled.kvs, 0, rows, lse, store.transpose(0, 1), **at)
    assert torch.equal(got, want) and want.sum() > 0
