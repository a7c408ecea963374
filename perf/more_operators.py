"""Cases of the operators that follow a draft: attention of trees of drafted tokens over paged caches, caches of 8-bit keys and
values (written, read back, attended to), and the drawing of tokens from logits.

``run`` computes an operator in elementary torch operations on pages and a page table; with ``own`` set it makes the calls
that a program makes of ``paper_2404_08698_amd.binding`` on caches of the same contents.  Widths and vocabularies are those of the
repository's workloads (the tiny fp32 decoder, the LLaMA-7B, LLaMA-13B and ChatGLM3-6B shapes) and generic ones.

Attention: a sequence has ``length`` cached positions and ``rows`` new ones behind them, whose keys and values lie in the cache as
well; pages hold 16 positions and are handed out in no order.  Keys and values are N(0, 1), queries twice that, so that a row has
keys that matter and others.  Logits are N(0, 2.5) with a few tokens that stand out, as a model's that knows what may come.
"""
import math

import numpy as np
import torch

own = False

#: (heads, key / value heads, head dimension)
WIDTHS = {"7b": (32, 32, 128), "13b": (40, 40, 128), "glm6b": (32, 2, 128), "grouped": (32, 8, 128), "tiny": (4, 4, 64), "tiny_one": (4, 1, 64)}
PAGE = 16
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _attend(kind, width, rows, length, **more):
    """A case of attention: kind "tree" (rows continue one another as a tree) or "rows" (a chunk).  q, cache: types; cap, slopes,
    window, prefix: rules of the scores."""
    case = {"kind": kind, "width": width, "sequences": 1, "rows": rows, "length": length, "q": "bf16", "cache": "int8", "cap": 0.0,
            "slopes": False, "window": 0, "prefix": 0}
    return {**case, **more}


def _store(width, rows, length, **more):
    """A case of writing rows and reading them back, behind ``length`` positions."""
    return {**{"kind": "store", "width": width, "sequences": 1, "rows": rows, "length": length, "q": "bf16", "cache": "int8"}, **more}


def _sample(rows, vocab, **more):
    """A case of sampling.  q: type of the logits; masked: share of the tokens that a grammar rules out."""
    return {**{"kind": "sample", "rows": rows, "vocab": vocab, "q": "f32", "temperature": 1.0, "top_k": 0, "top_p": 1.0, "min_p": 0.0, "masked": 0.0}, **more}


def listed():
    return [
        # one token of the 7B model, the usual settings of a chat: launches and the host path are most of it
        {"name": "sample_token", **_sample(1, 32000, temperature=0.8, top_k=50, top_p=0.95)},
        # a window of k = 16 drafts, a draw for every row, the nucleus alone
        {"name": "sample_window17", **_sample(17, 32000, top_p=0.9)},
        # a serving batch over a large vocabulary, a grammar that rules out a tenth of it
        {"name": "sample_batch64", **_sample(64, 131072, q="bf16", temperature=0.7, min_p=0.02, top_p=0.98, masked=0.1)},
        # a small tree behind a short prompt
        {"name": "tree8_128", **_attend("tree", "7b", 8, 128, cache="bf16")},
        # the largest window of the step as a tree, behind a long context
        {"name": "tree32_2048", **_attend("tree", "7b", 32, 2048, cache="bf16")},
        # trees of a serving batch with grouped heads: a sliding window and first tokens that stay visible, 8-bit cache
        {"name": "trees_batch16", **_attend("tree", "grouped", 25, 3000, sequences=16, window=1024, prefix=4)},
        # the tiny fp32 decoder with a distance bias, 64 rows
        {"name": "tree64_tiny", **_attend("tree", "tiny", 64, 333, q="f32", cache="f32", slopes=True)},
        # a serving batch in plain decoding on 8-bit caches: 32 sequences of 300 to 700 tokens
        {"name": "decode8_batch32", **_attend("rows", "7b", 1, 512, sequences=32)},
        # a token behind a very long document on an 8-bit cache, grouped heads
        {"name": "decode8_65535", **_attend("rows", "grouped", 1, 65535)},
        # a piece of a prompt on an 8-bit cache, fp32 rows, 16 query heads per key / value head
        {"name": "chunk8_1001", **_attend("rows", "glm6b", 1001, 777, q="f32")},
        # a step of 32 sequences is written into 8-bit caches
        {"name": "store8_batch32", **_store("7b", 1, 512, sequences=32)},
        # the long-context workload's prompt is written into an 8-bit cache: the largest to write
        {"name": "store8_3584", **_store("7b", 3584, 0)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("sample",) * 3 + ("tree",) * 3 + ("rows",) * 2 + ("store",) * 2)
    if kind == "sample":
        vocab = rng.choice((1024, 2048, 8192, 32000, 65024, _log(rng, 32, 262144), _log(rng, 1024, 262144)))
        return _sample(_log(rng, 1, min(256, (64 * 131072) // vocab)), vocab, q=rng.choice(("f32", "f32", "bf16")), temperature=rng.choice((1.0, round(rng.uniform(0.2, 2.0), 3))),
                       top_k=rng.choice((0, 0, _log(rng, 1, min(vocab, 2000)))), top_p=rng.choice((1.0, round(rng.uniform(0.05, 0.999), 3))),
                       min_p=rng.choice((0.0, 0.0, round(rng.uniform(0.001, 0.3), 4))), masked=rng.choice((0.0, 0.0, 0.5, 0.99)))
    width = rng.choice(("7b", "7b", "13b", "glm6b", "grouped", "grouped", "tiny", "tiny_one"))
    heads, kv_heads, dim = WIDTHS[width]
    cache = rng.choice(("int8", "int8", "int8", "bf16", "f32")) if kind != "rows" else "int8"
    q = "f32" if cache == "f32" else rng.choice(("bf16", "bf16", "f32"))
    sequences = rng.choice((1, 1, _log(rng, 2, 32)))
    if kind == "store":
        rows = _log(rng, 1, max(1, 3584 * 32 // (sequences * kv_heads)) if sequences == 1 else 64)
        return _store(width, min(rows, 16384), rng.choice((0, _log(rng, 1, 1000))), sequences=sequences, q=q, cache=cache)
    rows = rng.randint(1, 64) if kind == "tree" else _log(rng, 1, 64 if sequences > 1 else 1000)
    # (what the plain form holds, and what a case costs, stay below the largest listed one)
    room = min(32768, (64 << 20) // (sequences * kv_heads * dim * 4), (1 << 28) // (4 * sequences * rows * heads) - rows)
    case = _attend(kind, width, rows, _log(rng, 1, max(16, room)), sequences=sequences, q=q, cache=cache)
    if rng.random() < 0.5:
        rule = rng.choice(("cap", "slopes", "window", "prefix"))
        case[rule] = {"cap": 30.0, "slopes": True, "window": _log(rng, 2, case["length"] + rows), "prefix": rng.randint(1, case["length"] + rows)}[rule]
        if rule == "window" and rng.random() < 0.5:
            case["prefix"] = rng.randint(1, 8)
    return case


# ------------------------------------------------------------------------------------------------------ inputs

def _lengths(case):
    """Cached positions of every sequence: one as said, several between 0.6 and 1.4 times that."""
    n, s = case["length"], case["sequences"]
    return [n] if s == 1 else [int(n * (0.6 + 0.8 * ((0.618034 * (i + 1)) % 1.0))) for i in range(s)]


def _normal(shape, dtype, gen, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen).to(dtype)


def _sample_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rows, vocab = case["rows"], case["vocab"]
    x = _normal((rows, vocab), torch.float32, gen, 2.5)
    at = torch.randint(0, vocab, (rows, 20), device="cuda", generator=gen)
    x.scatter_(1, at, 12.0 * torch.rand((rows, 20), device="cuda", generator=gen))
    if case["masked"]:
        x[torch.rand(x.shape, device="cuda", generator=gen) < case["masked"]] = -math.inf
    # (some token is left)
    x[:, vocab // 2] = 1.0
    return x.to(TYPES[case["q"]]), torch.rand(rows, device="cuda", generator=gen)


def _rows_type(case):
    """Type in which keys and values come: that of the rows, and of an unquantised cache."""
    return TYPES[case["q"] if case["cache"] == "int8" else case["cache"]]


def _inputs(case, seed):
    """queries, (keys, values) of all positions of every sequence, parent of every row, slope of every head"""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    heads, kv_heads, dim = WIDTHS[case["width"]]
    rows = case["rows"]
    q = _normal((case["sequences"] * rows, heads * dim), TYPES[case["q"]], gen, 2.0)
    caches = [(_normal((n + rows, kv_heads * dim), _rows_type(case), gen), _normal((n + rows, kv_heads * dim), _rows_type(case), gen)) for n in _lengths(case)]
    parent = slopes = None
    if case["kind"] == "tree":
        # a row goes on from the one before it, or from any earlier one: candidates of an N-gram table
        r = np.random.RandomState(seed % (1 << 32))
        p = np.array([[-1] + [i - 1 if r.rand() < 0.6 else r.randint(0, i) for i in range(1, rows)] for _ in range(case["sequences"])])
        parent = torch.from_numpy(p.astype(np.int32)).cuda()
    if case.get("slopes"):
        slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)], dtype=torch.float32, device="cuda")
    return q, caches, parent, slopes


def _store_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    _, kv_heads, dim = WIDTHS[case["width"]]
    shape = (case["sequences"] * case["rows"], kv_heads * dim)
    return _normal(shape, TYPES[case["q"]], gen), _normal(shape, TYPES[case["q"]], gen, 0.5)


def _page_order(pages, seed):
    return np.random.RandomState(seed % (1 << 32)).permutation(pages)


def _page_count(n):
    return -(-n // PAGE)


def prepare(case, seed):
    state = {"case": case}
    if case["kind"] == "sample":
        state["logits"], state["u"] = _sample_inputs(case, seed)
        if own:
            from paper_2404_08698_amd import binding as B
            state["B"], state["rules"] = B, B.SamplingRules(temperature=case["temperature"], top_k=case["top_k"], top_p=case["top_p"], min_p=case["min_p"])
        return state
    heads, kv_heads, dim = WIDTHS[case["width"]]
    lengths = _lengths(case)
    if case["kind"] == "store":
        state["k"], state["v"] = _store_inputs(case, seed)
        caches = None
    else:
        q, caches, parent, slopes = _inputs(case, seed)
        state.update(q=q, parent=parent, slopes=slopes)
    state["lengths"] = lengths
    totals = [n + case["rows"] for n in lengths]
    if own:
        from paper_2404_08698_amd import binding as B
        state["B"] = B
        state["kvs"] = []
        for i, n in enumerate(totals):
            kv = B.LayerCache(1, heads, dim, n, n_kv_heads=kv_heads, dtype=case["cache"])
            kv.set_page_order(_page_order(_page_count(n), seed + i).tolist())
            kv.truncate(n - case["rows"])
            if caches:
                # (the new rows lie in the cache and are not committed)
                kv.write(0, 0, caches[i][0].float(), caches[i][1].float())
            state["kvs"].append(kv)
        if caches:
            state["rules"] = B.AttentionRules(cap=case["cap"], slopes=state["slopes"], window=case["window"], prefix=case["prefix"])
            if state["parent"] is not None:
                state["parent"] = state["parent"].reshape(-1)
    else:
        _pages(state, caches, totals, seed)
    return state


def _pages(state, caches, totals, seed):
    """A pool [page][k | v][16][heads][dim] of the cache's elements, for 8 bits with a scale for every position and head, and the page
    tables of all sequences, padded with page 0."""
    case = state["case"]
    _, kv_heads, dim = WIDTHS[case["width"]]
    counts = [_page_count(n) for n in totals]
    order = _page_order(sum(counts), seed)
    kind = torch.int8 if case["cache"] == "int8" else TYPES[case["cache"]]
    pool = torch.zeros((sum(counts), 2, PAGE, kv_heads, dim), dtype=kind, device="cuda")
    scales = torch.zeros((sum(counts), 2, PAGE, kv_heads), dtype=torch.float32, device="cuda")
    tables, at = np.zeros((len(counts), max(counts)), dtype=np.int64), 0
    for i, c in enumerate(counts):
        tables[i, :c] = order[at:at + c]
        at += c
        for j in range(2 if caches else 0):
            t = caches[i][j].reshape(totals[i], kv_heads, dim)
            ids = torch.from_numpy(tables[i, :c]).cuda()
            full = torch.zeros((c * PAGE, kv_heads, dim), dtype=kind, device="cuda")
            if kind == torch.int8:
                codes, s = _quantised(t)
                full[:totals[i]] = codes
                each = torch.zeros((c * PAGE, kv_heads), dtype=torch.float32, device="cuda")
                each[:totals[i]] = s
                scales[ids, j] = each.reshape(c, PAGE, kv_heads)
            else:
                full[:totals[i]] = t
            pool[ids, j] = full.reshape(c, PAGE, kv_heads, dim)
    state["pool"], state["scales"], state["tables"] = pool, scales, torch.from_numpy(tables).cuda()
    # page and place in it of every new row
    p = (torch.tensor(state["lengths"])[:, None] + torch.arange(case["rows"])[None, :]).cuda()
    state["page"], state["place"] = torch.gather(state["tables"], 1, p // PAGE).reshape(-1), (p % PAGE).reshape(-1)


# -------------------------------------------------------------------------------------------------- plain forms

def _quantised(t):
    """Codes and the scale of every position and head.  The quotient in 64 bits: a value next to the middle between two codes."""
    top = t.abs().amax(-1).float()
    codes = torch.round(127.0 * t.double() / top.double().clamp(min=1e-300)[..., None])
    return codes.to(torch.int8), top / 127.0


def _plain_store(state):
    case = state["case"]
    _, kv_heads, dim = WIDTHS[case["width"]]
    t = torch.stack([state["k"], state["v"]], 1).reshape(-1, 2, kv_heads, dim)
    page, place = state["page"], state["place"]
    if case["cache"] == "int8":
        codes, s = _quantised(t)
        state["pool"][page, :, place] = codes
        state["scales"][page, :, place] = s
        back = state["pool"][page, :, place].float() * state["scales"][page, :, place][..., None]
    else:
        state["pool"][page, :, place] = t.to(state["pool"].dtype)
        back = state["pool"][page, :, place].float()
    back = back.to(t.dtype).reshape(t.shape[0], 2, -1)
    return {"k": back[:, 0], "v": back[:, 1]}


def _gathered(state, which):
    """Keys (0) or values (1), position by position: [sequences][key / value heads][positions][dim], 32 bits."""
    t = state["pool"][:, which][state["tables"]].float()
    if state["case"]["cache"] == "int8":
        t = t * state["scales"][:, which][state["tables"]][..., None]
    return t.flatten(1, 2).transpose(1, 2)


def _ancestors(parent):
    """[sequences][rows][rows]: does the row come from the other one, or is it itself?"""
    n = parent.shape[1]
    eye = torch.eye(n, dtype=torch.float64, device="cuda")
    step = (parent[:, :, None] == torch.arange(n, device="cuda")).double()
    return torch.linalg.matrix_power(eye + step, max(n, 1)) > 0


def _visible(state, n_keys):
    """Which slots a row sees, and how far away they are: [sequences][rows][slots]"""
    case, rows = state["case"], state["case"]["rows"]
    start = torch.tensor(state["lengths"], device="cuda")[:, None, None]
    j = torch.arange(n_keys, device="cuda")[None, None, :]
    if state["parent"] is None:
        p = start + torch.arange(rows, device="cuda")[None, :, None]
        seen, at = j <= p, j.expand(start.shape[0], -1, -1)
    else:
        above = _ancestors(state["parent"])
        depth = above.sum(-1) - 1
        p = start + depth[:, :, None]
        slot = (j - start).clamp(0, rows - 1)
        new = (j >= start) & (j < start + rows)
        seen = (j < start) | (new & torch.gather(above, 2, slot.expand(-1, rows, -1)))
        at = torch.where(new, start + torch.gather(depth[:, None, :], 2, slot), j)
    if case["window"]:
        seen = seen & ((at > p - case["window"]) | (at < case["prefix"]))
    elif case["prefix"] and state["parent"] is None:
        seen = seen | ((at < case["prefix"]) & (j < start + rows))
    return seen, (p - at).abs()


def _plain_attention(state):
    case = state["case"]
    heads, kv_heads, dim = WIDTHS[case["width"]]
    seqs, rows, group = case["sequences"], case["rows"], heads // kv_heads
    k = _gathered(state, 0)
    q = state["q"].float().reshape(seqs, rows, kv_heads, group, dim).permute(0, 2, 3, 1, 4)
    s = torch.matmul(q.reshape(seqs, kv_heads, group * rows, dim), k.transpose(-1, -2)) * (1.0 / math.sqrt(dim))
    s = s.reshape(seqs, kv_heads, group, rows, k.shape[2])
    if case["cap"]:
        s = case["cap"] * torch.tanh(s / case["cap"])
    seen, distance = _visible(state, k.shape[2])
    if case["slopes"]:
        s = s - state["slopes"].reshape(1, kv_heads, group, 1, 1) * distance[:, None, None]
    s = s.masked_fill(~seen[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    out = torch.matmul((p / total).reshape(seqs, kv_heads, group * rows, -1), _gathered(state, 1)).reshape(seqs, kv_heads, group, rows, dim)
    lse = (top + torch.log(total))[..., 0]
    return {"out": out.permute(0, 3, 1, 2, 4).reshape(seqs * rows, heads * dim).to(state["q"].dtype),
            "lse": lse.permute(0, 3, 1, 2).reshape(seqs * rows, heads)}


def _plain_sample(state):
    """In 64 bits: which token the random number falls on, and where the nucleus ends, are decided next to borders."""
    case = state["case"]
    a = state["logits"].double()
    a = (a - a.amax(-1, keepdim=True)) / float(np.float32(case["temperature"]))
    w = torch.exp(a)
    ranked, order = torch.sort(a, dim=-1, descending=True, stable=True)
    ranked = torch.exp(ranked)
    if case["top_k"]:
        ranked[:, case["top_k"]:] = 0.0
    before = torch.cumsum(ranked, -1) - ranked
    stays = ranked > 0
    if case["top_p"] < 1.0:
        stays &= before < float(np.float32(case["top_p"])) * ranked.sum(-1, keepdim=True)
    stays &= ranked >= float(np.float32(case["min_p"]))
    stays = torch.zeros_like(stays).scatter(1, order, stays)
    total = torch.cumsum(torch.where(stays, w, 0.0), -1)
    token = torch.searchsorted(total, state["u"].double()[:, None] * total[:, -1:], right=True)
    return {"token": token[:, 0].int(), "logprob": (torch.gather(a, 1, token) - torch.log(total[:, -1:]))[:, 0].float()}


# ---------------------------------------------------------------------------------------------------------- run

def run(state):
    case = state["case"]
    if own:
        B = state["B"]
        if case["kind"] == "sample":
            token, logprob = B.sample(state["logits"], state["u"], state["rules"], want_logprob=True)
            return {"token": token, "logprob": logprob}
        if case["kind"] == "store":
            B.store(state["kvs"], 0, state["k"], state["v"])
            k, v = B.load(state["kvs"], 0, [case["rows"]] * case["sequences"], dtype=state["k"].dtype)
            return {"k": k, "v": v}
        if case["kind"] == "tree":
            out, lse = B.tree_attention(state["kvs"], 0, state["q"], state["parent"], rules=state["rules"], want_lse=True)
        else:
            out, lse = B.attention(state["kvs"], 0, state["q"], rules=state["rules"], want_lse=True)
        return {"out": out, "lse": lse}
    return {"sample": _plain_sample, "store": _plain_store, "tree": _plain_attention, "rows": _plain_attention}[case["kind"]](state)


# --------------------------------------------------------------------------------------------------------- work

def work(case):
    el = 2 if case["q"] == "bf16" else 4
    if case["kind"] == "sample":
        n = case["rows"] * case["vocab"]
        # (a difference, a quotient and an exponential of each)
        return {"bytes": n * el + 12 * case["rows"], "flops": 16 * n}
    heads, kv_heads, dim = WIDTHS[case["width"]]
    # bytes of a position's keys and values
    each = 2 * kv_heads * {"int8": dim + 4, "bf16": 2 * dim, "f32": 4 * dim}[case["cache"]]
    rows = case["sequences"] * case["rows"]
    if case["kind"] == "store":
        # read, written, read back, written
        return {"bytes": rows * (2 * each + 4 * kv_heads * dim * el), "flops": rows * kv_heads * dim * 6}
    keys = pairs = 0
    for n in _lengths(case):
        total = n + case["rows"]
        seen = n + (case["rows"] + 1) // 2
        if case["window"]:
            seen = min(seen, case["window"] + case["prefix"])
            keys += min(total, case["window"] + case["prefix"] + case["rows"])
        else:
            keys += total
        pairs += case["rows"] * seen
    return {"bytes": rows * heads * (2 * dim * el + 4) + keys * each, "flops": 4 * dim * heads * pairs}


# -------------------------------------------------------------------------------------------------------- exact

def _values_of(case, t):
    """What a cache holds of rows [n][heads][dim], in 64 bits: 8-bit codes (the nearest, ties to the even one) times fp32 scales."""
    if case["cache"] != "int8":
        return t.to(TYPES[case["cache"]]).double()
    x = t.double()
    unit = x.abs().amax(-1, keepdim=True)
    y = torch.where(unit > 0, x / unit, 0.0) * 127.0
    # (the quotient times 127 may miss the middle between two codes that x times 127 meets)
    low = torch.floor(y - 0.25)
    rest = 2.0 * (x * 127.0 - low * unit)
    code = low + (rest > unit) + (rest > 3.0 * unit) + ((rest == unit) & (low % 2 != 0)) + ((rest == 3.0 * unit) & (low % 2 == 0))
    return code * (unit.float() / 127.0).double()


def _exact_sample(case, seed):
    logits, u = _sample_inputs(case, seed)
    x, u = logits.float().cpu().numpy().astype(np.float64), u.cpu().numpy().astype(np.float64)
    temperature, top_p, min_p = (float(np.float32(case[n])) for n in ("temperature", "top_p", "min_p"))
    token, logprob = np.empty(len(x), dtype=np.int32), np.empty(len(x), dtype=np.float64)
    for r, row in enumerate(x):
        a = (row - row.max()) / temperature
        best = np.lexsort((np.arange(len(a)), -a))
        best = best[:case["top_k"]] if case["top_k"] else best
        p = np.exp(a[best])
        if top_p < 1.0:
            reached = np.cumsum(p)
            n = int(np.searchsorted(reached, top_p * reached[-1], side="left")) + 1
            best, p = best[:n], p[:n]
        best = np.sort(best[(p >= min_p) & (p > 0)])
        reached = np.cumsum(np.exp(a[best]))
        token[r] = best[int(np.searchsorted(reached, u[r] * reached[-1], side="right"))]
        logprob[r] = a[token[r]] - math.log(reached[-1])
    return {"token": torch.from_numpy(token), "logprob": torch.from_numpy(logprob)}


def exact(case, seed):
    if case["kind"] == "sample":
        return _exact_sample(case, seed)
    heads, kv_heads, dim = WIDTHS[case["width"]]
    if case["kind"] == "store":
        return {n: _values_of(case, t.reshape(-1, kv_heads, dim)).reshape(t.shape) for n, t in zip("kv", _store_inputs(case, seed))}
    q, caches, parent, slopes = _inputs(case, seed)
    rows, group, lengths = case["rows"], heads // kv_heads, _lengths(case)
    out = torch.zeros((q.shape[0], heads * dim), dtype=torch.float64, device="cuda")
    lse = torch.zeros((q.shape[0], heads), dtype=torch.float64, device="cuda")
    for s, (n, (k, v)) in enumerate(zip(lengths, caches)):
        k, v = (_values_of(case, t.reshape(-1, kv_heads, dim)) for t in (k, v))
        if parent is None:
            hidden = torch.arange(n + rows, device="cuda")[None, :] > torch.arange(n, n + rows, device="cuda")[:, None]
            where = torch.arange(n + rows, device="cuda")
        else:
            chains = []
            for r, up in enumerate(parent[s].tolist()):
                chains.append((chains[up] if up >= 0 else []) + [r])
            hidden = torch.ones((rows, n + rows), dtype=torch.bool)
            hidden[:, :n] = False
            for r, chain in enumerate(chains):
                hidden[r, [n + c for c in chain]] = False
            hidden = hidden.cuda()
            where = torch.tensor(list(range(n)) + [n + len(c) - 1 for c in chains], device="cuda")
        p = where[n:, None]
        if case["window"]:
            hidden = hidden | ((p - where >= case["window"]) & (where >= case["prefix"]))
        elif case["prefix"] and parent is None:
            hidden = hidden & (where >= case["prefix"])
        for h in range(heads):
            mine, dims = slice(s * rows, (s + 1) * rows), slice(h * dim, (h + 1) * dim)
            t = (q[mine, dims].double() @ k[:, h // group].t().contiguous()) / math.sqrt(dim)
            if case["cap"]:
                t = torch.tanh(t / case["cap"]) * case["cap"]
            if slopes is not None:
                t = t - slopes[h].double() * (p - where).abs()
            t = t.masked_fill_(hidden, -math.inf)
            lse[mine, h] = total = torch.logsumexp(t, -1)
            out[mine, dims] = torch.exp(t - total[:, None]) @ v[:, h // group].contiguous()
    return {"out": out, "lse": lse}
