"""Attention over caches of 8 bits at the ends of its numbers: long caches whose values are zeros or tiny, rows that hold no numbers."""
import math
import random

import pytest
import torch

from cache_reference import U, rows_like
from draft_reference import Caches, check_attention, empty, random_tree
from paper_2404_08698_amd import binding as B

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("rows", [BF16, F32])
@pytest.mark.parametrize("value", [0.0, 1e-37, 1.0])
def test_the_sum_of_many_weights_has_room(rows, value):
    """131072 keys of which all but a wave's first ones score 5.4 more (the largest of a score and its values decides what weights are relative to): their sum fits, and the
    values' mean comes out."""
    n, heads, seqs, late = 1 << 17, 8, 64, 5.4
    kv = empty(1, heads, heads, 64, n, "int8")
    k = torch.zeros(n, heads, 64, dtype=rows, device="cuda")
    k[128:, :, 0] = 1.0
    v = torch.full((n, heads * 64), value, dtype=rows, device="cuda")
    B.store(kv, 0, k.view(n, -1), v)
    held, also = (t[0, 0].item() for t in B.load(kv, 0, [1], pos0=[n - 1]))
    kv.truncate(n)
    q = torch.zeros(seqs, heads, 64, dtype=rows, device="cuda")
    q[:, :, 0] = late * 8
    score = q[0, 0, 0].item() / 8 * held
    # (the same cache many times: no block's keys are split then, and a wave has 2^15 of them)
    out, lse = B.attention([kv] * seqs, 0, q.view(seqs, -1), n_rows=[1] * seqs, pos0=[n - 1] * seqs, want_lse=True)
    want = math.log(128 + (n - 128) * math.exp(score))
    assert (lse.double().cpu() - want).abs().max() <= 64 * U * want, (lse[0, 0].item(), want)
    # Weights are off by 2^-11 or 2^-22 at most, all by the same here, outputs by their own rounding.  Values whose scale 2^-k is below 2^-93: a wave's weights, all
    # alike, are at least 2^(99 - k) (what follows the first keys scores 2^7.8 of them, too little to move the reference), k = 130, where fp16 ends at 2^-24: they are 0 or
    # anything up to a step.  And sums of 32 bits: a wave adds 2^15 keys to an output in 2^12 products of matrices, each off by a step at most, and to the sum of
    # weights in 2^10 steps of half a step and a few.
    near = (2.0 ** -8 + 2.0 ** -10 if rows == BF16 else 2.0 ** -20 + 1050 * U + 2.0 ** 12 * 2 * U) * abs(also) + (1.01 * abs(also) if value == 1e-37 else 0.0)
    assert (out.double().cpu() - also).abs().max() <= near, (out[0, 0].item(), also)


@pytest.mark.parametrize("tree", [False, True], ids=["rows", "tree"])
@pytest.mark.parametrize("rows", [BF16, F32])
@pytest.mark.parametrize("what", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("kind", [("int8", 16), ("bf16", 16), ("f32", 32)], ids=str)
def test_a_row_without_a_key_may_hold_anything(kind, rows, what, tree):
    """As the padding of a batch: 0 and minus infinity, whatever the row is; with a key it is no number."""
    spans = [(100, 6), (0, 40)]
    filled = Caches(4, 2, 64, [p + n for p, n in spans], dtype=kind[0], page_tokens=kind[1], seed=3)
    q = rows_like(filled, 46, rows)
    first = torch.zeros(46, dtype=torch.int32)
    none = [1, 4, 7, 20, 45]
    first[none] = 1 << 20
    first[30] = 3
    bad = none + [30]
    q[bad] = what
    q[7, :64] = 1.0
    q[9, 70] = what
    first = first.cuda()
    more, trees = {}, None
    if tree:
        trees = [random_tree(n, random.Random(n)) for _, n in spans]
        more["parent"] = torch.tensor([p for t in trees for p in t], dtype=torch.int32, device="cuda")
    out, lse = (B.tree_attention if tree else B.attention)(filled.kvs, 0, q, n_rows=[n for _, n in spans], pos0=[p for p, _ in spans],
                                                           rules=B.AttentionRules(first_key=first), want_lse=True, **more)
    assert (out[none] == 0).all() and (lse[none] == -math.inf).all()
    if kind[0] == "int8" or math.isnan(what):      # (elsewhere an infinity may leave some scores that are numbers)
        assert out[30].isnan().all() and lse[30].isnan().all() and out[9, 64:128].isnan().all()
    assert out[9, :64].isfinite().all() and out[9, 128:].isfinite().all()
    fine = [r for r in range(46) if r not in bad and r != 9]
    assert out[fine].isfinite().all() and lse[fine].isfinite().all()
    # the others are right, as beside rows of numbers (not to the bit: a wave with a row that has no reference rounds products before their exponents are formed)
    calm = q.clone()
    calm[bad] = 1.0
    calm[9] = 1.0
    also, also_lse = (B.tree_attention if tree else B.attention)(filled.kvs, 0, calm, n_rows=[n for _, n in spans], pos0=[p for p, _ in spans],
                                                                rules=B.AttentionRules(first_key=first), want_lse=True, **more)
    out[bad + [9]], lse[bad + [9]] = also[bad + [9]], also_lse[bad + [9]]
    check_attention(filled, calm, spans, out, lse, parents=trees, first_key=first)
