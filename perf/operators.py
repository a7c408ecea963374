"""Cases of the operators on paged caches of keys and values: attention of new rows over them, the weight that every
cached key receives, and the eviction of those that receive little.

``run`` computes an operator in elementary torch operations, in 32 bits, on pages and a page table; with ``own`` set it
makes the calls that a program makes of ``paper_2404_08698_amd.binding`` on caches of the same contents.  Widths are
those of the repository's workloads (the tiny fp32 decoder, the LLaMA-7B, LLaMA-13B and ChatGLM3-6B shapes) and a
generic one of 32 heads over 8 key / value heads.

A sequence has ``length`` cached positions and ``rows`` new ones behind them, whose keys and values lie in the cache as
well.  Pages hold 16 positions and are handed out in no order, as in a cache that has been in use.  Keys and values are
N(0, 1), as projections of normalised rows are; queries are twice that, so that a row has keys that matter and others.
"""
import math

import numpy as np
import torch

own = False

#: (heads, key / value heads, head dimension)
WIDTHS = {"7b": (32, 32, 128), "13b": (40, 40, 128), "glm6b": (32, 2, 128), "grouped": (32, 8, 128), "tiny": (4, 4, 64), "tiny_one": (4, 1, 64)}
PAGE = 16
ROPE_BASE = 10000.0
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
#: first visible key of a row that stands for no token (padding of a batch): it sees nothing
NOTHING = 1 << 30


def _case(kind, width, rows, length, **more):
    """A case of attention or key_mass.  q, cache: types; cap, slopes, window, prefix: rules of the scores; document: length
    of the documents that the positions are packed from (0: one); padding: last rows of every sequence that are no token."""
    case = {"kind": kind, "width": width, "sequences": 1, "rows": rows, "length": length, "q": "bf16", "cache": "bf16", "cap": 0.0,
            "slopes": False, "window": 0, "prefix": 0, "document": 0, "padding": 0}
    return {**case, **more}


def _evict(width, layers, length, keep, **more):
    """A case of eviction.  first, last: positions kept in any case; rotate: keys are turned to their new positions; equal:
    share of the positions whose mass is 0, so that the order decides among them."""
    case = {"kind": "evict", "width": width, "layers": layers, "length": length, "keep": keep, "first": 4, "last": 32, "cache": "bf16",
            "rotate": False, "equal": 0.2}
    return {**case, **more}


def listed():
    return [
        # a token of the 7B model behind a short prompt: launches and the host path are all there is
        {"name": "decode_128", **_case("attention", "7b", 1, 128)},
        # a serving batch in plain decoding: 32 sequences of 300 to 700 tokens
        {"name": "decode_batch32", **_case("attention", "7b", 1, 512, sequences=32)},
        # a token behind a very long document, grouped heads
        {"name": "decode_65535", **_case("attention", "grouped", 1, 65535)},
        # a window of k = 16 drafts, scores capped
        {"name": "window17_capped", **_case("attention", "7b", 17, 2048, cap=30.0)},
        # the 7B workload's prompt
        {"name": "prompt_512", **_case("attention", "7b", 512, 0)},
        # the long-context workload's prompt: the largest
        {"name": "prompt_3584", **_case("attention", "7b", 3584, 0)},
        # a ragged piece of packed documents behind what is cached, 16 query heads per key / value head, fp32 rows, padded
        {"name": "documents_1001", **_case("attention", "glm6b", 1001, 777, q="f32", document=333, padding=9)},
        # the tiny fp32 decoder with a distance bias, a sliding window and an always visible prefix
        {"name": "tiny_f32_bias", **_case("attention", "tiny", 128, 333, q="f32", cache="f32", slopes=True, window=100, prefix=40)},
        # the last rows of a prompt look at all of it, to say which keys matter
        {"name": "mass_observe_32", **_case("key_mass", "7b", 32, 4064)},
        # a whole prompt's weights, fp32 rows, 13B heads
        {"name": "mass_prompt_1800", **_case("key_mass", "13b", 1800, 0, q="f32")},
        # two layers of a prompt's cache shortened for the steps that follow, keys turned to their new positions
        {"name": "evict_3584_to_1024", **_evict("7b", 2, 3584, 1024, rotate=True)},
        # a layer of a very long cache to a quarter of it
        {"name": "evict_65536_to_16384", **_evict("grouped", 1, 65536, 16384)},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("attention",) * 4 + ("key_mass",) * 2 + ("evict",) * 2)
    width = rng.choice(("7b", "7b", "13b", "glm6b", "grouped", "grouped", "tiny", "tiny_one"))
    heads, kv_heads, dim = WIDTHS[width]
    cache = rng.choice(("bf16", "bf16", "bf16", "f32"))
    if kind == "evict":
        length = _log(rng, 64, 65536 if kv_heads <= 8 else 8192)
        keep = max(16, int(length * rng.uniform(0.1, 0.9)))
        return _evict(width, rng.randint(1, 3), length, keep, first=rng.randint(0, 8), last=rng.randint(0, 8),
                      cache=cache, rotate=rng.random() < 0.5, equal=rng.choice((0.0, 0.2, 0.9)))
    q = "f32" if cache == "f32" else rng.choice(("bf16", "bf16", "f32"))
    sequences = rng.choice((1, 1, 1, _log(rng, 2, 32)))
    # (fp32 caches and rows: pieces of up to 512 rows; what a case costs stays below the largest listed one)
    rows = _log(rng, 1, 64 if sequences > 1 else 512 if cache == "f32" else 3000)
    room = min(32768, (64 << 20) // (sequences * kv_heads * dim * 4), 3584 * 1792 * 3 // (4 * sequences * rows) - rows // 2)
    length = rng.choice((0, _log(rng, 16, room))) if rows > 1 and room > 16 else _log(rng, 16, max(17, room))
    case = _case(kind, width, rows, length, sequences=sequences, q=q, cache=cache)
    if rng.random() < 0.5:
        rule = rng.choice(("cap", "slopes", "window", "prefix", "document"))
        case[rule] = {"cap": 30.0, "slopes": True, "window": _log(rng, 8, length + rows + 8), "prefix": rng.randint(1, length + rows),
                      "document": _log(rng, 4, length + rows + 8)}[rule]
        case["padding"] = rng.randint(0, rows // 4)
    return case


# ------------------------------------------------------------------------------------------------------ inputs

def _lengths(case):
    """Cached positions of every sequence: one as said, several between 0.6 and 1.4 times that."""
    n, s = case["length"], case["sequences"]
    return [n] if s == 1 else [int(n * (0.6 + 0.8 * ((0.618034 * (i + 1)) % 1.0))) for i in range(s)]


def _first_key(case, length):
    """First visible key of every row of a sequence, or None where rows see all that is before them."""
    if not case["document"] and not case["padding"]:
        return None
    p = np.arange(length, length + case["rows"])
    first = p // case["document"] * case["document"] if case["document"] else np.zeros_like(p)
    if case["padding"]:
        first[case["rows"] - case["padding"]:] = NOTHING
    return first


def _rules(case, lengths):
    """(first visible key of every row [sequences][rows] or None, slope of every head or None)"""
    heads = WIDTHS[case["width"]][0]
    first = [_first_key(case, n) for n in lengths]
    first = None if first[0] is None else torch.from_numpy(np.stack(first).astype(np.int32)).cuda()
    slopes = torch.tensor([2.0 ** (-8.0 * (h + 1) / heads) for h in range(heads)], dtype=torch.float32, device="cuda") if case["slopes"] else None
    return first, slopes


def _normal(shape, dtype, gen, std=1.0):
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=gen).to(dtype)


def _attention_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    heads, kv_heads, dim = WIDTHS[case["width"]]
    lengths, rows = _lengths(case), case["rows"]
    q = _normal((case["sequences"] * rows, heads * dim), TYPES[case["q"]], gen, 2.0)
    caches = [(_normal((n + rows, kv_heads * dim), TYPES[case["cache"]], gen), _normal((n + rows, kv_heads * dim), TYPES[case["cache"]], gen)) for n in lengths]
    first, slopes = _rules(case, lengths)
    return lengths, q, caches, first, slopes


def _mass_inputs(case, seed):
    """Weight that the keys have received before: positive, a few of them most of it."""
    gen = torch.Generator(device="cuda").manual_seed(seed + 1)
    kv_heads = WIDTHS[case["width"]][1]
    return _normal((case["sequences"], kv_heads, max(_lengths(case)) + case["rows"]), torch.float32, gen).exp()


def _evict_inputs(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    heads, kv_heads, dim = WIDTHS[case["width"]]
    n, layers = case["length"], case["layers"]
    k = _normal((layers, n, kv_heads * dim), TYPES[case["cache"]], gen)
    v = _normal((layers, n, kv_heads * dim), TYPES[case["cache"]], gen)
    mass = _normal((layers, kv_heads, n), torch.float32, gen, 2.0).exp()
    mass[torch.rand(mass.shape, device="cuda", generator=gen) < case["equal"]] = 0.0
    return k, v, mass


def _page_order(pages, seed):
    return np.random.RandomState(seed % (1 << 32)).permutation(pages)


def _page_count(n):
    return -(-n // PAGE)


def prepare(case, seed):
    state = {"case": case}
    heads, kv_heads, dim = WIDTHS[case["width"]]
    if case["kind"] == "evict":
        k, v, mass = _evict_inputs(case, seed)
        state["mass"] = mass
        caches, lengths = [(k, v)], [case["length"]]
    else:
        lengths, q, caches, first, slopes = _attention_inputs(case, seed)
        state.update(lengths=lengths, q=q, first=first, slopes=slopes)
        if case["kind"] == "key_mass":
            state["mass"] = _mass_inputs(case, seed)
        caches = [(k[None], v[None]) for k, v in caches]
        lengths = [n + case["rows"] for n in lengths]
    if own:
        from paper_2404_08698_amd import binding as B
        state["B"] = B
        layers = case.get("layers", 1)
        state["kvs"] = []
        for i, (n, (k, v)) in enumerate(zip(lengths, caches)):
            kv = B.LayerCache(layers, heads, dim, n, n_kv_heads=kv_heads, dtype=case["cache"])
            kv.set_page_order(_page_order(_page_count(n), seed + i).tolist())
            # (the new rows lie in the cache and are not committed: giving up a length gives up its pages)
            kv.truncate(n if case["kind"] == "evict" else n - case["rows"])
            for layer in range(layers):
                kv.write(layer, 0, k[layer].float(), v[layer].float())
            state["kvs"].append(kv)
        if case["kind"] == "evict":
            state["short"] = B.LayerCache(layers, heads, dim, case["keep"], n_kv_heads=kv_heads, dtype=case["cache"])
        else:
            state["rules"] = B.AttentionRules(cap=case["cap"], slopes=state["slopes"], window=case["window"], prefix=case["prefix"],
                                              first_key=None if state["first"] is None else state["first"].reshape(-1))
    else:
        _scatter_pages(state, caches, lengths, seed)
    if case["kind"] == "key_mass":
        # what an attention call on the same rows has said; an input here
        state["lse"] = _lse(case, lengths, state["q"], caches, state["first"], state["slopes"])
    return state


def _scatter_pages(state, caches, lengths, seed):
    """pool [page][layer][k | v][16][width] and the page tables of all sequences, padded with page 0."""
    counts = [_page_count(n) for n in lengths]
    order = _page_order(sum(counts), seed)
    k0 = caches[0][0]
    pool = torch.zeros((sum(counts), k0.shape[0], 2, PAGE, k0.shape[2]), dtype=k0.dtype, device="cuda")
    tables, at = np.zeros((len(counts), max(counts)), dtype=np.int64), 0
    for i, (n, c, pair) in enumerate(zip(lengths, counts, caches)):
        tables[i, :c] = order[at:at + c]
        at += c
        ids = torch.from_numpy(tables[i, :c]).cuda()
        for j, t in enumerate(pair):
            full = torch.zeros((t.shape[0], c * PAGE, t.shape[2]), dtype=t.dtype, device="cuda")
            full[:, :n] = t
            pool[ids, :, j] = full.reshape(t.shape[0], c, PAGE, -1).transpose(0, 1)
    state["pool"], state["tables"] = pool, torch.from_numpy(tables).cuda()


# -------------------------------------------------------------------------------------------------- plain forms

def _gathered(state, which):
    """Keys (0) or values (1) of layer 0, position by position: [sequences][key / value heads][positions][dim], 32 bits."""
    _, kv_heads, dim = WIDTHS[state["case"]["width"]]
    t = state["pool"][:, 0, which][state["tables"]].float()
    return t.reshape(t.shape[0], -1, kv_heads, dim).transpose(1, 2)


def _visible(case, lengths, first, n_keys):
    """[sequences][rows][keys]"""
    rows = case["rows"]
    start = torch.tensor(lengths, device="cuda")[:, None, None]
    p = start + torch.arange(rows, device="cuda")[None, :, None]
    j = torch.arange(n_keys, device="cuda")[None, None, :]
    seen = j <= p
    if case["window"]:
        seen &= j > p - case["window"]
    if case["prefix"]:
        seen |= (j < case["prefix"]) & (j < start + rows)
    if first is not None:
        seen &= j >= first[:, :, None]
    return seen, (p - j).abs()


def _scores(state, k):
    """Scores [sequences][key / value heads][query heads of each][rows][keys] and which of them count."""
    case = state["case"]
    heads, kv_heads, dim = WIDTHS[case["width"]]
    seqs, rows, group = case["sequences"], case["rows"], heads // kv_heads
    q = state["q"].float().reshape(seqs, rows, kv_heads, group, dim).permute(0, 2, 3, 1, 4)
    s = torch.matmul(q.reshape(seqs, kv_heads, group * rows, dim), k.transpose(-1, -2)) * (1.0 / math.sqrt(dim))
    s = s.reshape(seqs, kv_heads, group, rows, k.shape[2])
    if case["cap"]:
        s = case["cap"] * torch.tanh(s / case["cap"])
    seen, distance = _visible(case, state["lengths"], state["first"], k.shape[2])
    if case["slopes"]:
        s = s - state["slopes"].reshape(1, kv_heads, group, 1, 1) * distance[:, None, None]
    return s, seen[:, None, None]


def _plain_attention(state):
    case = state["case"]
    heads, kv_heads, dim = WIDTHS[case["width"]]
    seqs, rows, group = case["sequences"], case["rows"], heads // kv_heads
    s, seen = _scores(state, _gathered(state, 0))
    top = s.masked_fill(~seen, -math.inf).amax(-1, keepdim=True).clamp(min=-3e38)
    p = torch.exp(s - top).masked_fill(~seen, 0.0)
    total = p.sum(-1, keepdim=True)
    p = p / total.clamp(min=1e-30)
    out = torch.matmul(p.reshape(seqs, kv_heads, group * rows, -1), _gathered(state, 1)).reshape(seqs, kv_heads, group, rows, dim)
    lse = (top + torch.log(total))[..., 0]
    return {"out": out.permute(0, 3, 1, 2, 4).reshape(seqs * rows, heads * dim).to(state["q"].dtype),
            "lse": lse.permute(0, 3, 1, 2).reshape(seqs * rows, heads)}


def _plain_mass(state):
    case = state["case"]
    heads, kv_heads, dim = WIDTHS[case["width"]]
    seqs, rows, group = case["sequences"], case["rows"], heads // kv_heads
    s, seen = _scores(state, _gathered(state, 0))
    lse = state["lse"].reshape(seqs, rows, kv_heads, group).permute(0, 2, 3, 1)[..., None]
    p = torch.exp(s - lse).masked_fill(~(seen & (lse > -math.inf)), 0.0)
    n = state["mass"].shape[2]
    return {"mass": state["mass"] + p.sum((2, 3))[:, :, :n]}


def _plain_evict(state):
    case, mass = state["case"], state["mass"]
    _, kv_heads, dim = WIDTHS[case["width"]]
    n, keep, layers = case["length"], case["keep"], case["layers"]
    rank = mass.clone()
    rank[:, :, :case["first"]] = math.inf
    rank[:, :, n - case["last"]:] = math.inf
    kept = torch.sort(rank, dim=-1, descending=True, stable=True).indices[:, :, :keep].sort(-1).values
    # [page][layer][k | v][16][width] -> [layer][k | v][position][head][dim]
    t = state["pool"][state["tables"][0]].permute(1, 2, 0, 3, 4).reshape(layers, 2, -1, kv_heads, dim)
    at = kept.transpose(1, 2)[..., None].expand(-1, -1, -1, dim)
    k, v = torch.gather(t[:, 0], 1, at), torch.gather(t[:, 1], 1, at)
    if case["rotate"]:
        angle = _angles(torch.arange(keep, device="cuda")[None, None, :] - kept, dim)
        c, s = torch.cos(angle).float().transpose(1, 2), torch.sin(angle).float().transpose(1, 2)
        a, b = k[..., :dim // 2].float(), k[..., dim // 2:].float()
        k = torch.cat([a * c - b * s, b * c + a * s], -1).to(v.dtype)
    return {"k": k.reshape(layers, keep, -1), "v": v.reshape(layers, keep, -1), "kept": kept.int(), "mass": torch.gather(mass, 2, kept)}


def _angles(turn, dim):
    """Angle of every rotary pair at a distance, 64 bits."""
    theta = ROPE_BASE ** (-2.0 * torch.arange(dim // 2, dtype=torch.float64, device="cuda") / dim)
    return turn.double()[..., None] * theta


# ---------------------------------------------------------------------------------------------------------- run

def run(state):
    case = state["case"]
    if own:
        B = state["B"]
        if case["kind"] == "attention":
            out, lse = B.attention(state["kvs"], 0, state["q"], rules=state["rules"], want_lse=True)
            return {"out": out, "lse": lse}
        if case["kind"] == "key_mass":
            out = torch.empty_like(state["mass"])
            out.copy_(state["mass"])
            return {"mass": B.key_mass(state["kvs"], 0, state["q"], state["lse"], out, rules=state["rules"])}
        kept, mass = B.evict(state["kvs"][0], state["mass"], case["keep"], first=case["first"], last=case["last"], into=state["short"],
                             rope_base=ROPE_BASE if case["rotate"] else 0.0)
        pairs = [state["short"].read(layer, 0, case["keep"]) for layer in range(case["layers"])]
        dtype = TYPES[case["cache"]]
        return {"k": torch.stack([k for k, _ in pairs]).to(dtype), "v": torch.stack([v for _, v in pairs]).to(dtype), "kept": kept, "mass": mass}
    return {"attention": _plain_attention, "key_mass": _plain_mass, "evict": _plain_evict}[case["kind"]](state)


# --------------------------------------------------------------------------------------------------------- work

def work(case):
    heads, kv_heads, dim = WIDTHS[case["width"]]
    el = 2 if case["cache"] == "bf16" else 4
    if case["kind"] == "evict":
        kept = case["layers"] * kv_heads * case["keep"]
        # (the mass of all positions; keys, values, mass and position of the kept ones)
        return {"bytes": 4 * case["layers"] * kv_heads * case["length"] + kept * (4 * dim * el + 8), "flops": kept * dim * 3 if case["rotate"] else 0}
    qel = 2 if case["q"] == "bf16" else 4
    keys = pairs = 0
    for n in _lengths(case):
        p = np.arange(n, n + case["rows"])
        total = n + case["rows"]
        lo = np.maximum(p - case["window"] + 1, 0) if case["window"] else np.zeros_like(p)
        pre = np.full_like(p, min(case["prefix"], total))
        first = _first_key(case, n)
        floor = np.zeros_like(p) if first is None else first
        lo = np.maximum(np.maximum(lo, pre), floor)
        seen = np.maximum(p + 1 - lo, 0) + np.maximum(pre - floor, 0)
        pairs += int(seen.sum())
        live = seen > 0
        keys += int(min(total, (p + 1 - lo)[live].clip(0).max() + (p[live].max() - p[live].min()) + pre.max())) if live.any() else 0
    rows = case["sequences"] * case["rows"]
    nbytes = rows * heads * (dim * qel + 4)
    if case["kind"] == "attention":
        return {"bytes": nbytes + rows * heads * dim * qel + 2 * keys * kv_heads * dim * el, "flops": 4 * dim * heads * pairs}
    return {"bytes": nbytes + keys * kv_heads * (dim * el + 8), "flops": 2 * dim * heads * pairs}


# -------------------------------------------------------------------------------------------------------- exact

def _each(case, lengths, q, caches, first, slopes, dtype, what):
    """what(sequence, head, scores with -inf where a key does not count, values) for every sequence and query head."""
    heads, kv_heads, dim = WIDTHS[case["width"]]
    rows, group = case["rows"], heads // kv_heads
    for s, (length, (k, v)) in enumerate(zip(lengths, caches)):
        length -= rows
        p = torch.arange(length, length + rows, device="cuda")[:, None]
        j = torch.arange(length + rows, device="cuda")[None, :]
        hidden = j > p
        if case["window"]:
            hidden = hidden | (j + case["window"] <= p)
        if case["prefix"]:
            hidden = hidden & (j >= case["prefix"])
        if first is not None:
            hidden = hidden | (j < first[s][:, None])
        for h in range(heads):
            g = h // group
            t = (q[s * rows:(s + 1) * rows, h * dim:(h + 1) * dim].to(dtype) @ k[0, :, g * dim:(g + 1) * dim].to(dtype).t().contiguous()) / math.sqrt(dim)
            if case["cap"]:
                t = torch.tanh(t / case["cap"]) * case["cap"]
            if slopes is not None:
                t = t - slopes[h].to(dtype) * (p - j).abs().to(dtype)
            what(s, h, t.masked_fill_(hidden, -math.inf), v[0, :, g * dim:(g + 1) * dim])


def _lse(case, lengths, q, caches, first, slopes):
    out = torch.empty((q.shape[0], WIDTHS[case["width"]][0]), dtype=torch.float32, device="cuda")
    rows = case["rows"]

    def one(s, h, t, v):
        out[s * rows:(s + 1) * rows, h] = torch.logsumexp(t, -1)

    _each(case, lengths, q, caches, first, slopes, torch.float32, one)
    return out


def exact(case, seed):
    heads, kv_heads, dim = WIDTHS[case["width"]]
    if case["kind"] == "evict":
        return _exact_evict(case, seed)
    lengths, q, caches, first, slopes = _attention_inputs(case, seed)
    caches = [(k[None], v[None]) for k, v in caches]
    lengths = [n + case["rows"] for n in lengths]
    rows = case["rows"]
    if case["kind"] == "attention":
        out = torch.zeros((q.shape[0], heads * dim), dtype=torch.float64, device="cuda")
        lse = torch.zeros((q.shape[0], heads), dtype=torch.float64, device="cuda")

        def one(s, h, t, v):
            lse[s * rows:(s + 1) * rows, h] = total = torch.logsumexp(t, -1)
            p = torch.exp(t - total[:, None])
            p[total == -math.inf] = 0.0
            out[s * rows:(s + 1) * rows, h * dim:(h + 1) * dim] = p @ v.double().contiguous()

        _each(case, lengths, q, caches, first, slopes, torch.float64, one)
        return {"out": out, "lse": lse}
    lse = _lse(case, lengths, q, caches, first, slopes).double()
    mass = _mass_inputs(case, seed).double()
    group = heads // kv_heads

    def add(s, h, t, v):
        of = lse[s * rows:(s + 1) * rows, h]
        live = of > -math.inf
        mass[s, h // group, :t.shape[1]] += torch.exp(t[live] - of[live][:, None]).sum(0)

    _each(case, lengths, q, caches, first, slopes, torch.float64, add)
    return {"mass": mass}


def _exact_evict(case, seed):
    _, kv_heads, dim = WIDTHS[case["width"]]
    k, v, mass = _evict_inputs(case, seed)
    n, keep, first, last, layers = case["length"], case["keep"], case["first"], case["last"], case["layers"]
    m = mass.cpu().numpy()
    kept = np.empty((layers, kv_heads, keep), dtype=np.int64)
    for l in range(layers):
        for g in range(kv_heads):
            middle = np.arange(first, n - last)
            best = middle[np.lexsort((middle, -m[l, g, first:n - last]))][:keep - first - last]
            kept[l, g] = np.concatenate([np.arange(first), np.sort(best), np.arange(n - last, n)])
    at = torch.from_numpy(kept).cuda()
    out_k = torch.empty((layers, keep, kv_heads * dim), dtype=torch.float64, device="cuda")
    out_v = torch.empty_like(out_k)
    for l in range(layers):
        for g in range(kv_heads):
            one = k[l, :, g * dim:(g + 1) * dim][at[l, g]].double()
            if case["rotate"]:
                turn = _angles(torch.arange(keep, device="cuda") - at[l, g], dim)
                z = torch.complex(one[:, :dim // 2], one[:, dim // 2:]) * torch.polar(torch.ones_like(turn), turn)
                one = torch.cat([z.real, z.imag], -1)
            out_k[l, :, g * dim:(g + 1) * dim] = one
            out_v[l, :, g * dim:(g + 1) * dim] = v[l, :, g * dim:(g + 1) * dim][at[l, g]].double()
    return {"k": out_k, "v": out_v, "kept": None, "mass": torch.gather(mass, 2, at).double()}
