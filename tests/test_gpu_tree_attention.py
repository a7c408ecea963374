"""Attention of trees of drafted tokens over caches, against 64 bits."""
import math
import random

import pytest
import torch

from cache_reference import rows_like
from draft_reference import Caches, check_attention, random_tree
from paper_2404_08698_amd import binding as B

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32
#: (cache type, page, row type): the matrix-core form with one and three terms, both plain ones, 8 bits with one and two terms
FORMS = [("bf16", 16, BF16), ("bf16", 16, F32), ("bf16", 64, BF16), ("f32", 8, F32), ("int8", 16, BF16), ("int8", 16, F32)]
IDS = ["%s%d-%s" % (c, p, "bf16" if t == BF16 else "f32") for c, p, t in FORMS]


def run(filled, q, spans, parents, **rules):
    parent = torch.tensor([p for t in parents for p in t], dtype=torch.int32, device="cuda")
    r = {k: v for k, v in rules.items() if v is not None}
    out, lse = B.tree_attention(filled.kvs, 0, q, parent, n_rows=[n for _, n in spans], pos0=[p for p, _ in spans], rules=B.AttentionRules(**r), want_lse=True)
    check_attention(filled, q, spans, out, lse, parents=parents, **rules)
    return out, lse


def make(form, heads, kv_heads, dim, spans, seed=0, **more):
    dtype, page, rows = form
    filled = Caches(heads, kv_heads, dim, [p + n for p, n in spans], dtype=dtype, page_tokens=page, seed=seed, **more)
    return filled, rows_like(filled, sum(n for _, n in spans), rows, seed=seed + 1)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 4, 128), (8, 2, 64), (16, 1, 128)])
@pytest.mark.parametrize("pos0,n", [(0, 1), (0, 64), (15, 2), (16, 33), (127, 64), (700, 17), (2000, 31)])
def test_trees(form, heads, kv_heads, dim, pos0, n):
    filled, q = make(form, heads, kv_heads, dim, [(pos0, n)], seed=n)
    run(filled, q, [(pos0, n)], [random_tree(n, random.Random(n))])


RULES = [dict(window=1), dict(window=3), dict(window=40), dict(window=200, prefix=5), dict(prefix=7), dict(prefix=10000), dict(cap=20.0), dict(cap=500.0),
         dict(slopes=True), dict(slopes=True, window=30, prefix=3), dict(first=True), dict(first=True, window=9, prefix=90), dict(scale=0.03), dict(cap=5.0, slopes=True)]


@pytest.mark.parametrize("form", FORMS, ids=IDS)
@pytest.mark.parametrize("rule", RULES, ids=str)
def test_rules_go_by_positions(form, rule):
    rule, spans = dict(rule), [(150, 29), (0, 9), (333, 64)]
    filled, q = make(form, 8, 4, 64, spans, seed=3)
    rng = random.Random(5)
    parents = [random_tree(n, rng, 0.4) for _, n in spans]
    if rule.pop("slopes", False):
        rule["slopes"] = torch.tensor([2.0 ** (-h) for h in range(8)], device="cuda")
    if rule.pop("first", False):
        # (documents that begin in the cache, in the tree, at a row's own position, and behind everything)
        rule["first_key"] = torch.tensor([rng.choice((0, 100, 152, 160, 1, 400, 1 << 30)) for _ in range(102)], dtype=torch.int32, device="cuda")
    run(filled, q, spans, parents, **rule)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_forests_and_parents_that_are_no_earlier_rows(form):
    """-1, the row itself, a later row and numbers far outside: the row follows the cached positions."""
    spans = [(37, 12)]
    filled, q = make(form, 4, 2, 128, spans)
    run(filled, q, spans, [[-1, 0, -1, 2, 4, 9, 5, 12, -7, 1 << 30, -(1 << 31), 3]])


@pytest.mark.parametrize("form", FORMS, ids=IDS)
@pytest.mark.parametrize("shape", ["chain", "star", "comb", "binary"])
def test_shapes_of_trees(form, shape):
    n = 64
    parent = {"chain": [i - 1 for i in range(n)], "star": [-1] + [0] * (n - 1), "comb": [-1] + [i - 1 if i % 2 else max(0, i - 2) for i in range(1, n)],
              "binary": [-1] + [(i - 1) // 2 for i in range(1, n)]}[shape]
    filled, q = make(form, 4, 4, 64, [(90, n)])
    out, lse = run(filled, q, [(90, n)], [parent], window=20)
    if shape == "chain":
        # the same rows as attention over a chunk: to rounding
        want, want_lse = B.attention(filled.kvs, 0, q, n_rows=[n], pos0=[90], rules=B.AttentionRules(window=20), want_lse=True)
        check_attention(filled, q, [(90, n)], want, want_lse, window=20)


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_what_a_row_does_not_see_may_hold_anything(form):
    """Infinities, NaN and the type's largest numbers in siblings' keys and values and in cached positions outside the window."""
    spans = [(64, 16)]
    filled, q = make(form, 4, 2, 64, spans, seed=9)
    width = 2 * 64
    for pos, what in ((3, math.inf), (5, math.nan), (7, 3.0e38), (64 + 5, math.nan), (64 + 6, -math.inf), (64 + 7, 3.0e38)):
        row = torch.full((1, width), what)
        filled.fill(0, pos, row, row)
    parent = [-1] + [0] * 15
    # (rows 5, 6 and 7 see what they hold themselves, and with a huge score among a wave's the products are rounded before their exponents are formed: by 2^-24 of a score, which
    # the bound counts four times, so the others are held to 64 bits and not to the bits that they have without)
    out, _ = run(filled, q, spans, [parent], window=30)
    mine = [i for i in range(16) if i not in (5, 6, 7)]
    assert out.reshape(16, -1)[mine].isfinite().all()
    for pos in (3, 5, 7, 64 + 5, 64 + 6, 64 + 7):
        filled.fill(0, pos, torch.ones(1, width), torch.ones(1, width))
    run(filled, q, spans, [parent], window=30)


def test_many_sequences_with_and_without_rows():
    spans = [(0, 0), (5, 1), (300, 64), (17, 0), (1000, 7), (31, 33), (0, 2)]
    for form in FORMS:
        filled, q = make(form, 8, 2, 64, spans, seed=4)
        rng = random.Random(1)
        run(filled, q, spans, [random_tree(n, rng) if n else [] for _, n in spans])


def test_a_long_cache_in_splits():
    for form in (FORMS[0], FORMS[4], FORMS[5]):
        filled, q = make(form, 4, 1, 128, [(20000, 40)], seed=2)
        run(filled, q, [(20000, 40)], [random_tree(40, random.Random(3))])


@pytest.mark.parametrize("form", FORMS, ids=IDS)
def test_strides_places_and_streams(form):
    spans = [(50, 20)]
    filled, _ = make(form, 4, 4, 64, spans)
    parent = torch.tensor(random_tree(20, random.Random(2)), dtype=torch.int32, device="cuda")
    q = rows_like(filled, 20, form[2], pitch=4 * 64 + 3)       # rows that begin anywhere
    out = torch.full((20, 4 * 64 + 5), 7.0, dtype=form[2], device="cuda")
    B.tree_attention(filled.kvs, 0, q, parent, n_rows=[20], pos0=[50], out=out[:, 1:4 * 64 + 1])
    dense, lse = B.tree_attention(filled.kvs, 0, q.contiguous(), parent, n_rows=[20], pos0=[50], want_lse=True)
    check_attention(filled, q, spans, dense, lse, parents=[parent.tolist()])
    assert torch.equal(out[:, 1:4 * 64 + 1], dense)
    assert (out[:, 0] == 7).all() and (out[:, 4 * 64 + 1:] == 7).all()
    # in place, on another stream
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    mine = q.contiguous()
    B.tree_attention(filled.kvs, 0, mine, parent, n_rows=[20], pos0=[50], out=mine, stream=other)
    other.synchronize()
    assert torch.equal(mine, dense)


def test_a_captured_call_takes_the_tree_that_is_there_when_it_runs():
    spans = [(400, 30)]
    filled, q = make(FORMS[4], 8, 8, 128, spans)
    parent = torch.tensor(random_tree(30, random.Random(0)), dtype=torch.int32, device="cuda")
    out = torch.empty_like(q)
    lse = torch.empty(30, 8, device="cuda")
    ws = torch.empty(max(1, B.attention_workspace_bytes(filled.kvs, [30], [400])) + (64 << 20), dtype=torch.uint8, device="cuda")

    def call():
        B.tree_attention(filled.kvs, 0, q, parent, n_rows=[30], pos0=[400], out=out, lse=lse, workspace=ws)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for seed in range(4):
        tree = random_tree(30, random.Random(seed), 0.3)
        parent.copy_(torch.tensor(tree, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        check_attention(filled, q, spans, out, lse, parents=[tree])
        eager, eager_lse = B.tree_attention(filled.kvs, 0, q, parent, n_rows=[30], pos0=[400], want_lse=True)
        assert torch.equal(eager, out) and torch.equal(eager_lse, lse)


def test_the_model_s_own_tree_step_is_this():
    """The keys, the order and the positions of a draft tree are those of verify_tree: a window of one root and its branches, on a cache of
    the same contents, gives rows that do not depend on their siblings."""
    filled, q = make(FORMS[0], 4, 4, 64, [(100, 9)])
    parent = [-1, 0, 1, 2, 0, 4, 5, 0, 7]
    full, _ = run(filled, q, [(100, 9)], [parent])
    # each branch alone, its rows moved together
    for branch in ([0, 1, 2, 3], [0, 4, 5, 6], [0, 7, 8]):
        k, v = filled.k[0][[100 + b for b in branch]], filled.v[0][[100 + b for b in branch]]
        one = Caches(4, 4, 64, [100 + len(branch)], dtype="bf16")
        one.fill(0, 0, torch.cat([filled.k[0][:100], k]), torch.cat([filled.v[0][:100], v]))
        alone, lse = B.attention(one.kvs, 0, q[branch].contiguous(), n_rows=[len(branch)], pos0=[100], want_lse=True)
        check_attention(one, q[branch], [(100, len(branch))], alone, lse)
        assert (alone.float() - full[branch].float()).abs().max() <= 2.0 ** -6 * full.float().abs().max()


@pytest.mark.parametrize("form", FORMS, ids=IDS)
@pytest.mark.parametrize("tree", [False, True], ids=["rows", "tree"])
def test_first_keys_at_the_ends_of_32_bits(form, tree):
    spans = [(150, 29), (0, 9), (333, 64)]
    filled, q = make(form, 8, 4, 64, spans, seed=4)
    rng = random.Random(6)
    first = torch.tensor([rng.choice((-(1 << 31), -(1 << 31) + 200, -1, 0, 152, (1 << 31) - 1)) for _ in range(102)], dtype=torch.int32, device="cuda")
    for rule in (dict(first_key=first), dict(first_key=first, window=40, prefix=20), dict(first_key=first, window=(1 << 31) - 1)):
        if tree:
            run(filled, q, spans, [random_tree(n, rng) for _, n in spans], **rule)
        else:
            out, lse = B.attention(filled.kvs, 0, q, n_rows=[n for _, n in spans], pos0=[p for p, _ in spans], rules=B.AttentionRules(**rule), want_lse=True)
            check_attention(filled, q, spans, out, lse, **rule)
