"""The operators on caches one after another, as a program's layers and a model's own prompts use them: rows are written, attend,
say which keys they looked at, the others are evicted, and the steps go on with what is left."""
import dataclasses
import math

import numpy as np
import pytest
import torch

from cache_reference import SHARED_SHAPES, U, Filled, attention, check_attention, rows_like
from oracle import decoder as od
from paper_2404_08698_amd import binding as B
from paper_2404_08698_amd import synth

pytestmark = pytest.mark.gpu


def mass_close(got, want, off, rows):
    """off: how far a score may be from its own, at most; the sum of as many weights as there are rows and heads of the group."""
    assert ((got.cpu().double() - want).abs() <= want * (2.5 * off + rows * U) + 1e-30).all(), ((got.cpu().double() - want).abs() / (want + 1e-30)).max().item()


@pytest.mark.parametrize("dtype,page_tokens,q_dtype", [("bf16", 16, torch.bfloat16), ("bf16", 16, torch.float32), ("f32", 16, torch.float32), ("bf16", 8, torch.bfloat16)])
@pytest.mark.parametrize("rules", [{}, {"cap": 20.0, "window": 150, "prefix": 4}])
def test_prompt_eviction_and_steps(dtype, page_tokens, q_dtype, rules):
    """Two sequences of different lengths: a prompt, the weights of its last rows, an eviction each, then steps of both together."""
    heads, kv_heads, dim, lengths, keep = 8, 2, 64, (333, 700), 100
    f = Filled(heads, kv_heads, dim, lengths, dtype, page_tokens, capacity=720)
    r = B.AttentionRules(**rules)
    spans = [(0, n) for n in lengths]
    for kv, n in zip(f.kvs, lengths):
        kv.truncate(n)
    q = rows_like(f, sum(lengths), q_dtype)
    out, lse = B.attention(f.kvs, 0, q, lengths, [0, 0], r, want_lse=True)
    check_attention(f, q, spans, out, lse, **rules)

    # the last 32 rows of each prompt say what stays
    seen = [(n - 32, 32) for n in lengths]
    ends = np.cumsum(lengths)
    last = torch.cat([q[e - 32:e] for e in ends]).contiguous()
    mass = torch.zeros(2, kv_heads, max(lengths), device="cuda")
    B.key_mass(f.kvs, 0, last, torch.cat([lse[e - 32:e] for e in ends]).contiguous(), mass, [32, 32], [n - 32 for n in lengths], r)
    _, _, _, off, want = attention(f, last, seen, **rules)
    for s, n in enumerate(lengths):
        mass_close(mass[s, :, :n], want[s], off.max().item() * 2, 32 * heads // kv_heads)
        assert not mass[s, :, n:].any()
        kept, weights = B.evict(f.kvs[s], mass[s:s + 1, :, :n], keep, 4, 32)
        assert f.kvs[s].length == keep and torch.equal(weights[0], torch.gather(mass[s], 1, kept[0].long()))
        at = kept[0].cpu().long()
        for name in ("k", "v"):
            t = getattr(f, name)[s].reshape(n, kv_heads, dim)
            getattr(f, name)[s] = torch.stack([t[at[g], g] for g in range(kv_heads)], 1).reshape(keep, -1)

    # steps of one and of several rows behind what was kept
    gen = torch.Generator().manual_seed(9)
    for step in range(6):
        n = 1 + step % 3
        for s, kv in enumerate(f.kvs):
            new = [torch.randn(n, kv_heads * dim, generator=gen) for _ in range(2)]
            if dtype == "bf16":
                new = [t.bfloat16().float() for t in new]
            p = kv.length
            kv.write(0, p, new[0].cuda(), new[1].cuda())
            f.k[s], f.v[s] = torch.cat([f.k[s], new[0]]), torch.cat([f.v[s], new[1]])
        q = rows_like(f, 2 * n, q_dtype, seed=20 + step)
        out, lse = B.attention(f.kvs, 0, q, rules=r, want_lse=True)
        check_attention(f, q, [(kv.length, n) for kv in f.kvs], out, lse, **rules)
        for kv in f.kvs:
            kv.truncate(kv.length + n)


def test_captured_together():
    """Attention and mass in one graph, replayed with other calls in between, against the same calls made eagerly."""
    f = Filled(8, 2, 128, (6000,))
    kv = f.kvs[0]
    kv.truncate(6000)
    q, out, lse = rows_like(f, 32).clone(), torch.empty(32, 1024, dtype=torch.bfloat16, device="cuda"), torch.empty(32, 8, device="cuda")
    mass = torch.zeros(2, 6000, device="cuda")
    ws = torch.empty(max(256, B.attention_workspace_bytes(kv, [32], [5968])), dtype=torch.uint8, device="cuda")
    assert ws.numel() > 256     # splits that are joined
    mass_ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda")

    def run():
        mass.zero_()
        B.attention(kv, 0, q, pos0=[5968], out=out, lse=lse, workspace=ws)
        B.key_mass(kv, 0, q, lse, mass, pos0=[5968], workspace=mass_ws)
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for seed in range(4):
        q.copy_(rows_like(f, 32, seed=seed))
        run()
        want = [t.clone() for t in (out, lse, mass)]
        for t in (out, lse, mass):
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(want, (out, lse, mass)):
            assert torch.equal(a, b)


@pytest.mark.parametrize("q_dtype", [torch.bfloat16, torch.float32])
def test_pages_far_into_a_large_pool(q_dtype):
    """Where a page's offset passes 32 bits, in elements: attention of many and of few rows, mass and eviction."""
    (heads, kv_heads, dim, ((pos0, n),)), layers, capacity = SHARED_SHAPES[0], 40, 62000
    total = pos0 + n
    kv = B.LayerCache(layers, heads, dim, capacity, n_kv_heads=kv_heads)
    kv.set_page_order(list(range(kv.num_pages))[::-1])      # the first positions on the last pages
    assert (kv.num_pages - total // 16 - 1) * layers * 2 * kv_heads * 16 * dim > 1 << 32
    gen = torch.Generator().manual_seed(3)
    f = Filled(heads, kv_heads, dim, (), layer=layers - 1)
    k, v = (torch.randn(total, kv_heads * dim, generator=gen).bfloat16().float() for _ in range(2))
    f.k, f.v, f.kvs = [k], [v], [kv]
    kv.write(layers - 1, 0, k.cuda(), v.cuda())
    kv.truncate(total)
    q = rows_like(f, n, q_dtype)
    out, lse = B.attention(kv, layers - 1, q, pos0=[pos0], want_lse=True)
    last = slice(n - 32, n)
    check_attention(f, q[last], [(total - 32, 32)], out[last], lse[last])
    few, few_lse = B.attention(kv, layers - 1, q[last], pos0=[total - 32], want_lse=True)
    check_attention(f, q[last], [(total - 32, 32)], few, few_lse)
    mass = torch.zeros(layers, kv_heads, total, device="cuda")
    B.key_mass(kv, layers - 1, q[last].contiguous(), few_lse, mass[layers - 1], pos0=[total - 32])
    _, _, _, off, want = attention(f, q[last], [(total - 32, 32)])
    mass_close(mass[layers - 1], want[0], off.max().item() * 2, 32 * heads // kv_heads)
    dst = B.LayerCache(layers, heads, dim, 4000, n_kv_heads=kv_heads)
    kept, _ = B.evict(kv, mass, 4000, 4, 32, into=dst)
    at = kept[layers - 1].cpu().long()
    assert torch.equal(at, torch.cat([torch.cat([torch.arange(4), 4 + m[4:-32].argsort(descending=True, stable=True)[:4000 - 36].sort().values,
                                                 torch.arange(total - 32, total)])[None] for m in mass[layers - 1].cpu()]))
    for got, whole in zip(dst.read(layers - 1, 0, 4000), (k, v)):
        whole = whole.reshape(total, kv_heads, dim)
        assert torch.equal(got.cpu().reshape(4000, kv_heads, dim), torch.stack([whole[at[h], h] for h in range(kv_heads)], 1))


BF16 = dataclasses.replace(synth.TINY_BF16, n_layers=2)
GROUPED = dataclasses.replace(synth.MID_GQA, n_layers=2)


@pytest.mark.parametrize("before,rows,seen", [(0, 1, 32), (0, 16, 1), (0, 17, 32), (5, 12, 4), (0, 272, 16), (3, 270, 32), (0, 527, 17)])
@pytest.mark.parametrize("shape", [BF16, GROUPED], ids=["heads_of_64", "grouped"])
def test_observed_prompts(shape, before, rows, seen):
    """The prompt is the same bit for bit; the first layer's weights are those of its queries in 64 bits; every row gives 1 per head."""
    n, heads, kv_heads, dim = before + rows, shape.n_heads, getattr(shape, "n_kv_heads", 0) or shape.n_heads, shape.head_dim
    weights = synth.make_weights(shape, 5)
    # (sharper scores than N(0, 0.02) weights give)
    weights["wq"] = [t * 16 for t in weights["wq"]]
    model = B.Model(shape, {k: [t.cuda() for t in v] if isinstance(v, list) else v.cuda() for k, v in weights.items()}, max_window=8, max_positions=n)
    prompt = synth.random_tokens(shape.vocab, n, 13)
    plain, kv = B.KVCache(model, n), B.KVCache(model, n)
    a, b = (torch.empty(shape.vocab, dtype=torch.float32, device="cuda") for _ in range(2))
    for c in (plain, kv):
        if before:
            B.prefill(model, c, prompt[:before])
    mass = torch.zeros(shape.n_layers, kv_heads, n + 3, device="cuda")
    kv.observe(mass, seen)
    assert B.prefill(model, plain, prompt[before:], out_logits=a) == B.prefill(model, kv, prompt[before:], out_logits=b)
    kv.observe(None)
    assert torch.equal(a, b)
    for layer in range(shape.n_layers):
        for x, y in zip(plain.read(layer, 0, n), kv.read(layer, 0, n)):
            assert torch.equal(x, y)
    assert not mass[:, :, n:].any()
    live = min(seen, rows)
    each = live * heads // kv_heads
    # each weight to (keys + 64) half steps and what its score is off, which 2^-12 covers beside the sum's own
    assert ((mass.sum(2).cpu().double() - each).abs() <= each * 2.0 ** -12).all()

    x = weights["embed"].double()[torch.tensor(prompt[n - live:])]
    x = x / (x.pow(2).mean(1, keepdim=True) + shape.rms_eps).sqrt() * weights["attn_norm"][0].double()
    w = weights["wq"][0].double()
    q, size = (x @ w.t()).numpy(), (x.abs() @ w.abs().t()).reshape(live, heads, dim)
    q = torch.stack([torch.from_numpy(od.rope(np.ascontiguousarray(q[i]), heads, dim, n - live + i, shape.rope_base)) for i in range(live)]).reshape(live, heads, dim)
    # rows and queries as two bf16 terms each (2^-16), sums of d_model products in fp32; turning mixes two dims
    size = size + torch.cat([size[..., dim // 2:], size[..., :dim // 2]], -1)
    err = size * (3 * 2.0 ** -16 + shape.d_model * U)
    k = kv.read(0, 0, n)[0].cpu().double().reshape(n, kv_heads, dim)
    visible = torch.arange(n)[None] <= torch.arange(n - live, n)[:, None]
    for g in range(kv_heads):
        want, allowed = torch.zeros(n, dtype=torch.float64), torch.zeros(n, dtype=torch.float64)
        for h in range(g * heads // kv_heads, (g + 1) * heads // kv_heads):
            s = (q[:, h] @ k[:, g].t() / math.sqrt(dim)).masked_fill(~visible, -math.inf)
            off = (err[:, h] @ k[:, g].abs().t() / math.sqrt(dim)).amax(1, keepdim=True) + (n + 64) * U + 8 * U * s.masked_fill(~visible, 0).abs().amax(1, keepdim=True)
            p = torch.softmax(s, 1)
            want += p.sum(0)
            allowed += (p * 2.5 * off).sum(0)
        assert ((mass[0, g, :n].cpu().double() - want).abs() <= allowed + want * each * U + 1e-30).all()


@pytest.mark.parametrize("shape", [synth.TINY_BF16, synth.TINY, synth.TINY_MQA_BF16], ids=["bf16", "f32", "one_kv_head"])
def test_a_model_goes_on_after_eviction(shape):
    """In a single layer a key depends on its token and position alone: what stays of a prompt, turned to its new positions, is what the
    tokens that stay are as a prompt of their own.  The steps that follow are those of a cache with these contents."""
    shape = dataclasses.replace(shape, n_layers=1)
    n, keep, kv_heads, dim = 300, 130, getattr(shape, "n_kv_heads", 0) or shape.n_heads, shape.head_dim
    model = B.Model(shape, synth.make_weights(shape, 5, device="cuda"), max_window=8, max_positions=512)
    prompt = synth.random_tokens(shape.vocab, n, 3)
    kv, short, same = (B.KVCache(model, 512) for _ in range(3))
    B.prefill(model, kv, prompt)
    mass = torch.rand(1, 1, n, device="cuda").repeat(1, kv_heads, 1)
    kept, _ = B.evict(kv, mass, keep, 4, 16, rope_base=shape.rope_base)
    assert kv.length == keep and (kept == kept[:, :1]).all()
    B.prefill(model, short, [prompt[i] for i in kept[0, 0].tolist()])
    (k, v), (ks, vs) = kv.read(0, 0, keep), short.read(0, 0, keep)
    assert torch.equal(v, vs)
    a, b = (t.double().reshape(keep, kv_heads, dim) for t in (k, ks))
    size = b.abs() + torch.cat([b[..., dim // 2:], b[..., :dim // 2]], -1).abs()
    # rounded before the turn, after it, and in the other cache; angles in fp32 (up to `n` radians), which both sides' tables and turns are off by
    step = 2.0 ** -8 if shape.dtype == "bf16" else U
    assert ((a - b).abs() <= size * (3.1 * step + 4 * n * U)).all(), ((a - b).abs() / size).max().item()
    same.write(0, 0, k, v)
    same.truncate(keep)
    for turn in range(4):
        window = synth.random_tokens(shape.vocab, 1 + turn, 40 + turn)
        la, lb = (torch.empty(len(window), shape.vocab, dtype=torch.float32, device="cuda") for _ in range(2))
        assert B.verify(model, kv, window, B.APPEND, out_logits=la)[1] == B.verify(model, same, window, B.APPEND, out_logits=lb)[1]
        assert torch.equal(la, lb)
    assert kv.length == keep + 10


def test_observe_evict_and_generate():
    """The whole path: a prompt that is observed, its cache shortened by what the last rows looked at, decoding from there."""
    shape = BF16
    model = B.Model(shape, synth.make_weights(shape, 5, device="cuda"), max_window=8, max_positions=700)
    kv = B.KVCache(model, 700)
    prompt = synth.random_tokens(shape.vocab, 500, 3)
    mass = torch.zeros(shape.n_layers, shape.n_heads, 500, device="cuda")
    kv.observe(mass)
    with pytest.raises(B.AnpdError):
        B.prefill(model, kv, prompt + prompt[:1])     # further than the mass reaches
    assert kv.length == 0 and not mass.any()
    nxt = B.prefill(model, kv, prompt)
    kv.observe(None)
    kept, weights = B.evict(kv, mass, 200, 4, 32, rope_base=shape.rope_base)
    assert kv.length == 200 and torch.equal(weights, torch.gather(mass, 2, kept.long()))
    same = B.KVCache(model, 700)
    for layer in range(shape.n_layers):
        same.write(layer, 0, *kv.read(layer, 0, 200))
    same.truncate(200)
    tokens = []
    for c in (kv, same):
        t = [nxt]
        for _ in range(12):
            t.append(B.verify(model, c, t[-1:], B.APPEND)[1])
        tokens.append(t)
    assert tokens[0] == tokens[1]


def test_observe_refusals():
    own = B.LayerCache(1, 4, 64, 64)
    with pytest.raises(B.AnpdError) as e:
        own.observe(torch.zeros(1, 4, 64, device="cuda"))
    assert e.value.code == B.E_INVAL
    model = B.Model(synth.TINY, synth.make_weights(synth.TINY, 5, device="cuda"), max_positions=64)
    kv = B.KVCache(model, 64)
    with pytest.raises(B.AnpdError) as e:
        kv.observe(torch.zeros(2, 4, 64, device="cuda"))
    assert e.value.code == B.E_UNIMPLEMENTED
    model = B.Model(BF16, synth.make_weights(BF16, 5, device="cuda"), max_positions=64)
    kv = B.KVCache(model, 64)
    mass = torch.zeros(2, 4, 64, device="cuda")
    for bad in (mass[:, :, ::2], mass[:1], mass.double(), mass.cpu(), mass[0], mass[:, :, :60]):
        with pytest.raises(ValueError):
            kv.observe(bad)
    for rows in (0, 33, -1):
        with pytest.raises(B.AnpdError):
            kv.observe(mass, rows)
    L = B.lib()
    need = L.anpd_kv_observe_workspace_bytes(kv._h, 32)
    ws = torch.empty(need + 256, dtype=torch.uint8, device="cuda")
    p, m = ws.data_ptr(), mass.data_ptr()
    for code, args in ((B.E_INVAL, (None, m, 64, 32, p, need)), (B.E_INVAL, (kv._h, m, 0, 32, p, need)), (B.E_INVAL, (kv._h, m + 2, 64, 32, p, need)),
                       (B.E_INVAL, (kv._h, m, 64, 32, None, need)), (B.E_INVAL, (kv._h, m, 64, 32, p + 16, need)), (B.E_CAPACITY, (kv._h, m, 64, 32, p, need - 1))):
        assert L.anpd_kv_observe(*args) == code, args
    assert L.anpd_kv_observe(kv._h, m, 64, 32, p, need) == B.OK
    kv.observe(None)


def test_the_workspace_of_observed_prompts_is_nobody_elses_any_more():
    """It is taken from the current stream's memory and written by prompts on any other: what is queued on the first, and may use the
    same memory, is done when the call returns."""
    model = B.Model(BF16, synth.make_weights(BF16, 5, device="cuda"), max_positions=64)
    kv = B.KVCache(model, 64)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        mass = torch.zeros(2, 4, 64, device="cuda")
        x = torch.zeros(8192, 8192, dtype=torch.bfloat16, device="cuda")
        for _ in range(2):          # (the first time loads the product's kernel)
            kv.observe(mass)
            for _ in range(30):
                x @ x
        assert not stream.query()
        kv.observe(mass)
        assert stream.query()
    kv.observe(None)


@pytest.mark.parametrize("own", [True, False], ids=["layer_cache", "model_cache"])
def test_the_memory_of_a_cache_is_nobody_elses_any_more(own):
    """Taken from a side stream's memory and cleared on the device's default stream: what is queued on the first, and may use the
    same memory, is done before it is cleared, or unwritten positions would not read as zeros."""
    model = B.Model(BF16, synth.make_weights(BF16, 5, device="cuda"), max_positions=64)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        x = torch.zeros(8192, 8192, dtype=torch.bfloat16, device="cuda")

        def make():
            return B.LayerCache(2, 4, 64, 64) if own else B.KVCache(model, 64)
        make()
        x @ x
        stream.synchronize()
        for _ in range(30):
            x @ x
        before = stream.query()
        kv = make()
        assert not before and stream.query()
    kv.truncate(64)
    assert not any(t.any() for layer in range(2) for t in kv.read(layer, 0, 64))


def test_what_is_written_has_the_caches_width_and_type():
    """Refused by the host: other numbers of rows, widths and types would be read beyond their ends."""
    f = Filled(4, 2, 64, [40])
    kv, good = f.kvs[0], torch.ones(3, 128, device="cuda")
    for bad in (good[:2], good[:, :64].contiguous(), good.bfloat16(), good.double(), good.cpu(), good.repeat(1, 2)[:, ::2], good.reshape(-1), good.sum()):
        for k, v in ((good, bad), (bad, good)):
            with pytest.raises(ValueError):
                kv.write(0, 5, k, v)
    assert torch.equal(kv.read(0, 0, 40)[0].cpu(), f.k[0])
    kv.write(0, 5, good, good.reshape(3, 2, 64))
    kv.write(0, 8, good[:0], good[:0])
    k, v = kv.read(0, 4, 5)
    assert (k[1:4] == 1).all() and (v[1:4] == 1).all() and torch.equal(k[::4].cpu(), f.k[0][4:9:4])


def test_what_a_call_allocates_is_its_streams_memory(monkeypatch):
    """Outputs and workspaces of a call on another stream than the current one come from that stream's memory, where it follows
    what their last owner does with them."""
    model = B.Model(BF16, synth.make_weights(BF16, 5, device="cuda"), max_positions=64)
    kv, own = B.KVCache(model, 64), Filled(8, 1, 64, [3000], capacity=3001)
    own.kvs[0].truncate(2999)
    q, lse, mass = rows_like(own, 1), torch.zeros(1, 8, device="cuda"), torch.zeros(1, 1, 3000, device="cuda")
    stream, seen, empty = torch.cuda.Stream(), [], torch.empty
    torch.cuda.synchronize()
    monkeypatch.setattr(torch, "empty", lambda *a, **k: (seen.append(torch.cuda.current_stream()), empty(*a, **k))[1])

    def calls():
        yield "prefill", lambda: B.prefill(model, kv, [1, 2, 3], stream=stream), 1
        yield "read", lambda: kv.read(0, 0, 3, stream=stream), 2
        yield "attention", lambda: B.attention(own.kvs, 0, q, want_lse=True, stream=stream), 3
        yield "key_mass", lambda: B.key_mass(own.kvs, 0, q, lse, mass, stream=stream), 0
        yield "evict", lambda: B.evict(own.kvs[0], mass, 20, stream=stream), 2
    for name, call, n in calls():
        del seen[:]
        call()
        assert len(seen) == n and all(s == stream for s in seen), (name, seen)
    stream.synchronize()
