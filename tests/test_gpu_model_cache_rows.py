"""store, load and commit on a model's own cache: what its prompts and steps have written is read and moved, and they go on from there."""
import pytest
import torch

from draft_reference import held
from helpers import to_cuda
from paper_2404_08698_amd import binding as B
from paper_2404_08698_amd import synth

pytestmark = pytest.mark.gpu

SHAPES = {"f32": synth.TINY, "bf16": synth.TINY_BF16, "mid": synth.MID_GQA}


@pytest.fixture(scope="module", params=list(SHAPES))
def model(request):
    shape = SHAPES[request.param]
    return B.Model(shape, to_cuda(synth.make_weights(shape, 3)), max_window=16, max_positions=512)


def start(model, n=37):
    kv = B.KVCache(model, 512)
    return kv, B.prefill(model, kv, synth.workload_prompt("tiny")[:n])


def test_rows_of_a_prompt_are_read_and_written(model):
    kv, _ = start(model)
    width = kv.n_kv_heads * model.shape.head_dim
    kind = "bf16" if model.shape.dtype == "bf16" else "f32"
    for layer in range(model.shape.n_layers):
        k, v = kv.read(layer, 0, 37)
        for pos, n in ((0, 37), (5, 20), (36, 1)):
            for dtype in (torch.float32, torch.bfloat16):
                a, b = B.load(kv, layer, [n], pos0=[pos], dtype=dtype)
                assert torch.equal(a, k[pos:pos + n].to(dtype)) and torch.equal(b, v[pos:pos + n].to(dtype))
        new = torch.randn(11, width, generator=torch.Generator().manual_seed(layer)).cuda()
        B.store(kv, layer, new, -new, pos0=[30])
        k[30:37], v[30:37] = (held(t[:7].cpu(), kv.n_kv_heads, kind).cuda() for t in (new, -new))
        for have, want in zip(kv.read(layer, 0, 37), (k, v)):
            assert torch.equal(have, want)
    assert kv.length == 37


@pytest.mark.parametrize("path", [[0], [0, 1, 2], [0, 3, 9], [2, 4, 7, 11], []], ids=str)
def test_a_committed_path_is_what_its_tokens_alone_leave(model, path):
    """The keys of a path's tokens, stored among others as a tree's rows are and committed: the cache is the one that the tokens alone, appended, have left, and the next step's logits are the same."""
    one, c = start(model)
    kv, _ = start(model)
    tokens = [(c + 7 * i) % model.vocab for i in range(len(path))]
    if tokens:
        B.verify(model, one, tokens, B.APPEND)
    gen = torch.Generator().manual_seed(1)
    for layer in range(model.shape.n_layers):
        rows = [torch.randn(12, kv.n_kv_heads * model.shape.head_dim, generator=gen).cuda() for _ in range(2)]
        if path:
            for t, mine in zip(rows, B.load(one, layer, [len(path)], pos0=[37])):
                t[path] = mine
        B.store(kv, layer, *rows)
    kv.commit(path)
    assert kv.length == one.length == 37 + len(path)
    for layer in range(model.shape.n_layers):
        for a, b in zip(kv.read(layer, 0, kv.length), one.read(layer, 0, one.length)):
            assert torch.equal(a, b)
    logits = [torch.empty(3, model.vocab, device="cuda") for _ in range(2)]
    for cache, into in zip((one, kv), logits):
        B.verify(model, cache, [c, 3, 4], B.APPEND, out_logits=into)
    assert torch.equal(*logits) and kv.length == one.length
