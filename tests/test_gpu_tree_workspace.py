"""The memory that a tree's attention asks for is what it uses: given exactly that, in a captured call, it writes nothing behind it."""
import random

import pytest
import torch

from cache_reference import rows_like
from draft_reference import Caches, check_attention, random_tree
from paper_2404_08698_amd import binding as B

pytestmark = pytest.mark.gpu

GUARD = 1 << 16


@pytest.mark.parametrize("rows", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("dtype,page", [("bf16", 16), ("int8", 16), ("f32", 16)])
@pytest.mark.parametrize("heads,kv_heads,dim,spans,rules", [(4, 4, 64, [(1500, 30)], {}), (16, 2, 128, [(3000, 64)], {}), (8, 1, 128, [(700, 3), (0, 0), (2500, 17)], {}),
                                                            (4, 2, 64, [(4000, 40)], dict(window=900)), (4, 2, 64, [(4000, 40)], dict(window=300, prefix=700)), (8, 8, 64, [(20, 5)], {})], ids=str)
def test_a_tree_s_workspace(heads, kv_heads, dim, spans, rules, dtype, page, rows):
    filled = Caches(heads, kv_heads, dim, [p + n for p, n in spans], dtype=dtype, page_tokens=page)
    n_rows, pos0, ruled = [n for _, n in spans], [p for p, _ in spans], B.AttentionRules(**rules)
    q = rows_like(filled, sum(n_rows), rows)
    rng = random.Random(1)
    trees = [random_tree(n, rng) if n else [] for n in n_rows]
    parent = torch.tensor([p for t in trees for p in t], dtype=torch.int32, device="cuda")
    need = B.tree_attention_workspace_bytes(filled.kvs, n_rows, pos0, ruled)
    assert (need > 0) == (max(pos0) > 20)
    whole = torch.full((need + GUARD,), 77, dtype=torch.uint8, device="cuda")
    out, lse = torch.empty_like(q), torch.empty(sum(n_rows), heads, device="cuda")

    def call():
        B.tree_attention(filled.kvs, 0, q, parent, n_rows=n_rows, pos0=pos0, rules=ruled, out=out, lse=lse, workspace=whole[:need] if need else None)

    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for _ in range(3):
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        check_attention(filled, q, spans, out, lse, parents=trees, **rules)
        assert (whole[need:] == 77).all()
    if need:
        with pytest.raises(B.AnpdError) as e:
            B.tree_attention(filled.kvs, 0, q, parent, n_rows=n_rows, pos0=pos0, rules=ruled, out=out, workspace=whole[:need - 256])
        # (what one type of rows takes, the other may not need)
        assert e.value.code == B.E_CAPACITY
