"""Verification steps that draw their tokens, the decode loop on them, and a layer's step of a drafted tree on an 8-bit cache from the rows written to the
path committed."""
import random

import pytest
import torch

from draft_reference import check_tokens, empty, held, random_tree
from helpers import to_cuda
from paper_2404_08698_amd import binding as B
from paper_2404_08698_amd import synth

pytestmark = pytest.mark.gpu

RULES = dict(temperature=0.9, top_k=40, top_p=0.95, min_p=0.01)


@pytest.fixture(scope="module", params=["f32", "bf16", "mid"])
def model(request):
    shape = {"f32": synth.TINY, "bf16": synth.TINY_BF16, "mid": synth.MID_GQA}[request.param]
    return B.Model(shape, to_cuda(synth.make_weights(shape, 3)), max_window=16, max_positions=512)


def uniforms(n, seed=0):
    return torch.rand(n, generator=torch.Generator().manual_seed(seed)).cuda()


def one_by_one(model, prompt, u, n, rules):
    """Tokens drawn one at a time, u[i] for the one at position i; and the cache."""
    kv = B.KVCache(model, 512)
    logits = torch.empty(1, model.vocab, device="cuda")
    B.prefill(model, kv, prompt, out_logits=logits[0])
    at = len(prompt)
    tokens = [int(B.sample(logits, u[at:at + 1], rules))]
    while len(tokens) < n:
        a, nxt, drawn = B.verify_sample(model, kv, [tokens[-1]], u[at + len(tokens):at + len(tokens) + 1], rules)
        assert a == 0 and drawn == [nxt]
        tokens.append(nxt)
    return tokens, kv


def test_windows_draw_what_single_tokens_draw(model):
    """The random number of a position decides its token: drafted windows of any length, right or wrong, end in the same text, logits and cache."""
    prompt, u, rules = synth.workload_prompt("tiny")[:40], uniforms(512), B.SamplingRules(**RULES)
    want, plain = one_by_one(model, prompt, u, 40, rules)
    rng = random.Random(1)
    kv = B.KVCache(model, 512)
    B.prefill(model, kv, prompt)
    done = 1
    while done < 36:
        k = rng.randrange(0, 5)
        drafts = want[done:done + k]
        right = len(drafts)
        if k and rng.random() < 0.6:
            wrong = rng.randrange(k)
            drafts[wrong] = (drafts[wrong] + 1 + rng.randrange(model.vocab - 1)) % model.vocab
            right = wrong
        window = [want[done - 1]] + drafts
        logits = torch.empty(len(window), model.vocab, device="cuda")
        at = len(prompt) + done
        a, nxt, drawn = B.verify_sample(model, kv, window, u[at:at + len(window)].contiguous(), rules, out_logits=logits)
        assert a == right and nxt == want[done + a] and drawn[:a + 1] == want[done:done + a + 1]
        check_tokens(logits, u[at:at + len(window)], torch.tensor(drawn), None, **RULES)
        done += 1 + a
        assert kv.length == len(prompt) + done - 1
    plain.truncate(kv.length)
    for layer in range(model.shape.n_layers):
        for mine, other in zip(kv.read(layer, len(prompt), kv.length - len(prompt)), plain.read(layer, len(prompt), kv.length - len(prompt))):
            assert torch.equal(mine, other)


def test_at_temperature_0_a_step_is_verify(model):
    prompt = synth.workload_prompt("tiny")[:30]
    a, b = B.KVCache(model, 512), B.KVCache(model, 512)
    c = B.prefill(model, a, prompt)
    assert B.prefill(model, b, prompt) == c
    table = B.NgramTable(2, 4, model.vocab)
    table.update(prompt + [c])
    for _ in range(8):
        window = [c] + table.propose(5)[0]
        acc, nxt, preds = B.verify(model, a, window, want_predicts=True)
        got = B.verify_sample(model, b, window, uniforms(len(window), 4), B.SamplingRules(temperature=0.0))
        assert got == (acc, nxt, preds) and a.length == b.length
        table.update(window[1:1 + acc] + [nxt])
        c = nxt


def test_the_decode_loop(model):
    prompt = synth.workload_prompt("tiny")[:50]
    kv = B.KVCache(model, 512)
    run = lambda **more: (kv.truncate(0), B.anpd_generate(model, kv, B.NgramTable(2, 4, model.vocab), prompt, 4, 40, **more))[1]  # noqa: E731
    greedy = run()["tokens"]
    assert run(sampling=B.SamplingRules(temperature=0.0))["tokens"] == greedy
    gen = lambda s: torch.Generator(device="cuda").manual_seed(s)  # noqa: E731
    rules = B.SamplingRules(temperature=1.0, top_p=0.9)
    a, b, c = (run(sampling=rules, generator=gen(s)) for s in (1, 1, 2))
    assert a["tokens"] == b["tokens"] and a["tokens"] != c["tokens"] and len(a["tokens"]) == 40
    assert all(0 <= t < model.vocab for t in a["tokens"])
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    assert len(run(sampling=rules, generator=gen(1), stream=other)["tokens"]) == 40
    with pytest.raises(ValueError):
        run(sampling=B.SamplingRules(temperature=torch.ones(16, device="cuda")))


def test_refused_steps_leave_the_cache_as_it_is(model):
    kv = B.KVCache(model, 512)
    B.prefill(model, kv, synth.workload_prompt("tiny")[:20])
    u = uniforms(3)
    for window, rules, code in (([1, 2, 3], dict(temperature=-1.0), B.E_INVAL), ([1, 2, model.vocab], dict(), B.E_RANGE), ([1, 2, 3], dict(top_p=2.0), B.E_INVAL)):
        with pytest.raises(B.AnpdError) as e:
            B.verify_sample(model, kv, window, u, B.SamplingRules(**rules))
        assert e.value.code == code and kv.length == 20
    kv.truncate(511)
    with pytest.raises(B.AnpdError) as e:
        B.verify_sample(model, kv, [1, 2, 3], u)
    assert e.value.code == B.E_CAPACITY and kv.length == 511


def test_logits_without_a_token():
    w = to_cuda(synth.make_weights(synth.TINY, 3))
    w["lm_head"].fill_(float("nan"))
    broken = B.Model(synth.TINY, w, max_window=8, max_positions=128)
    kv = B.KVCache(broken, 128)
    kv.truncate(10)
    with pytest.raises(B.AnpdError) as e:
        B.verify_sample(broken, kv, [1, 2], uniforms(2))
    assert e.value.code == B.E_RANGE and kv.length == 10


@pytest.mark.parametrize("cache", ["int8", "bf16"])
def test_a_drafted_tree_through_one_layer(cache):
    """Rows are written, the tree is attended to, tokens are drawn from what comes out of it, the path that the draws confirm is committed: the cache then holds what
    the accepted tokens alone, one after the other, would have left, and their rows came out alike."""
    heads, kv_heads, dim, vocab = 8, 2, 128, 300
    gen = torch.Generator().manual_seed(0)
    normal = lambda *s, std=1.0: (torch.randn(*s, generator=gen) * std).cuda()  # noqa: E731
    embed, wq, wk, wv = normal(vocab, 256), normal(256, heads * dim, std=0.12), normal(256, kv_heads * dim, std=0.06), normal(256, kv_heads * dim, std=0.06)
    head = normal(heads * dim, vocab, std=0.2)
    rules, u = B.SamplingRules(temperature=0.7, top_p=0.9), uniforms(400, 7)

    # (every token's rows once: the library's product of 24 rows and of one need not have the same bits, and the caches are compared by theirs)
    of_token = [(embed.bfloat16().float() @ w).bfloat16() for w in (wq, wk, wv)]

    def project(tokens):
        return [t[torch.tensor(tokens, device="cuda")] for t in of_token]

    prompt = [i * 37 % vocab for i in range(90)]
    kv, one = empty(1, heads, kv_heads, dim, 400, cache, seed=1), empty(1, heads, kv_heads, dim, 400, cache, seed=2)
    for c in (kv, one):
        _, k, v = project(prompt)
        B.store(c, 0, k, v)
        c.truncate(90)
    text, root, rng, accepted = [], 5, random.Random(3), 0
    for step in range(6):
        # one token after the other
        chain, t, outs = [], root, []
        for i in range(5):
            q, k, v = project([t])
            B.store(one, 0, k, v)
            out = B.attention(one, 0, q)
            one.commit([0])
            outs.append(out[0])
            t = int(B.sample(out.float() @ head, u[one.length:one.length + 1].contiguous(), rules))
            chain.append(t)
        # the tree: the true continuation among others, hung under random rows
        parent = random_tree(24, rng, 0.3)
        depth = [0] * 24
        for r in range(1, 24):
            depth[r] = depth[parent[r]] + 1
        tokens, on_path = [root], [0]
        for r in range(1, 24):
            good = parent[r] == on_path[-1] and depth[r] <= 3 and depth[r] == len(on_path)
            tokens.append(chain[depth[r] - 1] if good else (chain[min(depth[r], 4)] + 1 + rng.randrange(100)) % vocab)
            if good:
                on_path.append(r)
        q, k, v = project(tokens)
        B.store(kv, 0, k, v)
        out = B.tree_attention(kv, 0, q, torch.tensor(parent, dtype=torch.int32, device="cuda"))
        at = torch.tensor([kv.length + 1 + d for d in depth], device="cuda")
        drawn = B.sample(out.float() @ head, u[at].contiguous(), rules).tolist()
        path = [0]
        while True:
            nxt = [r for r in range(24) if parent[r] == path[-1] and r and tokens[r] == drawn[path[-1]]]
            if not nxt:
                break
            path.append(nxt[0])
        length = kv.length
        kv.commit(path)
        accepted += len(path) - 1
        assert kv.length == length + len(path)
        for i, r in enumerate(path):
            # two orders of the same sums, each within 2^-7 of the row's largest number (weights and outputs rounded to bf16)
            assert (out[r].float() - outs[i].float()).abs().max() <= 2.0 ** -6 * outs[i].float().abs().max()
        assert [drawn[r] for r in path] == chain[:len(path)]
        text += [tokens[r] for r in path]
        root = drawn[path[-1]]
        one.truncate(kv.length)
    assert accepted >= 4
    for mine, other in zip(kv.read(0, 0, kv.length), one.read(0, 0, kv.length)):
        assert torch.equal(mine, other)
    _, k, _ = project(prompt + text)
    assert torch.equal(kv.read(0, 0, kv.length)[0].cpu(), held(k.float().cpu(), kv_heads, cache))
