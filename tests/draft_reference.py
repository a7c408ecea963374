"""The operators that follow a draft in 64 bits, on the CPU, as their definitions say: attention of trees and chunks over caches (of 8 bits too), the codes
of such caches, and the drawing of tokens."""
import math

import numpy as np
import torch

from cache_reference import Filled, U, U_BF16
from paper_2404_08698_amd import binding as B


# ----------------------------------------------------------------------------------- 8 bits

def codes(x):
    """x: [...][head_dim] float32.  (codes, scales): 127 x / max |x| to the nearest, ties to even; fp32 max |x| / 127."""
    top = x.abs().amax(-1)
    scale = (top / torch.tensor(127.0)).float()
    y = 127.0 * x.double() / top.double().clamp(min=1e-300)[..., None]      # (a quotient that is no tie is 2^-33 away from one)
    return torch.where(top[..., None] > 0, torch.round(y), 0.0), scale


def held(x, heads, dtype):
    """What a cache of this type holds of rows [n][heads * dim] (float32)."""
    if dtype == "f32":
        return x
    if dtype == "bf16":
        return x.bfloat16().float()
    t = x.reshape(x.shape[0], heads, -1)
    c, s = codes(t)
    bad = ~t.isfinite().all(-1)
    return torch.where(bad[..., None], math.nan, (c * s.double()[..., None]).float()).reshape(x.shape)


class Caches(Filled):
    """Filled, with caches of 8 bits too: k and v are what they hold."""

    def __init__(self, heads, kv_heads, dim, lengths, dtype="bf16", std=1.0, **more):
        super().__init__(heads, kv_heads, dim, lengths, dtype=dtype, **more)
        for s, kv in enumerate(self.kvs):
            if dtype == "int8" or std != 1.0:
                self.fill(s, 0, self.k[s] * std, self.v[s] * std)

    def fill(self, s, pos, k, v):
        """Overwrites positions from pos on."""
        if len(k):
            self.kvs[s].write(self.layer, pos, k.cuda().contiguous(), v.cuda().contiguous())
            self.k[s][pos:pos + len(k)] = held(k, self.kv_heads, self.dtype)
            self.v[s][pos:pos + len(v)] = held(v, self.kv_heads, self.dtype)


# -------------------------------------------------------------------------------- attention

def chains(parent):
    """Per row the rows that it sees: its ancestors and itself."""
    out = []
    for r, p in enumerate(parent):
        out.append((out[p] if 0 <= p < r else []) + [r])
    return out


def visible(pos0, n, parent=None, window=0, prefix=0, first_key=None):
    """(seen [n][pos0 + n], distance of every slot from every row)"""
    total = pos0 + n
    at = torch.arange(total)
    if parent is None:
        p = torch.arange(pos0, total)
        seen = at[None] <= p[:, None]
    else:
        rows = chains(parent)
        at[pos0:] = torch.tensor([pos0 + len(c) - 1 for c in rows])
        p = at[pos0:].clone()
        seen = torch.zeros(n, total, dtype=torch.bool)
        seen[:, :pos0] = True
        for r, c in enumerate(rows):
            seen[r, [pos0 + i for i in c]] = True
    by_rules = torch.ones(n, total, dtype=torch.bool)
    if window:
        by_rules = at[None] > p[:, None] - window
    if prefix:
        by_rules = by_rules | (at[None] < prefix)
    # (of a chunk the prefix is seen from everywhere, ahead of a row as well; a tree shows a row nothing but its own chain)
    seen = seen & by_rules if parent is not None else (seen & by_rules) | (at[None] < prefix)
    if first_key is not None:
        seen = seen & (at[None] >= first_key[:, None].cpu().long())
    return seen, (p[:, None] - at[None]).abs()


def check_attention(filled, q, spans, out, lse, parents=None, cap=0.0, slopes=None, scale=0.0, **rules):
    """Both results against 64 bits.  Off by: fp32 sums of products (their magnitudes times their number times half a step; rows of fp32 on 8 bits are two
    terms, 2^-22), which a score is, and a weight relatively; rounded weights of bf16 rows (2^-8, on 8 bits 2^-11; fp32 rows there 2^-22, and
    2^-25 of a weight of 2^6 for each key); the output's own rounding."""
    heads, dim = filled.heads, filled.dim
    group = heads // filled.kv_heads
    factor = scale or 1.0 / math.sqrt(dim)
    eight, bf16 = filled.dtype == "int8", q.dtype == torch.bfloat16
    qd, got, got_lse = q.detach().cpu().double(), out.detach().cpu().double(), lse.detach().cpu().double()
    term = 2.0 ** -22 if eight and not bf16 else 0.0
    rounding = (2.0 ** -11 if bf16 else 2.0 ** -22) if eight else (U_BF16 if bf16 else 0.0)
    at = 0
    first_key = rules.pop("first_key", None)
    for s, (pos0, n) in enumerate(spans):
        if n == 0:
            continue
        rows = slice(at, at + n)
        at += n
        seen, dist = visible(pos0, n, None if parents is None else parents[s], first_key=None if first_key is None else first_key[rows], **rules)
        live = seen.any(1)
        for h in range(heads):
            g = h // group
            k, v = (t[s][:pos0 + n, g * dim:(g + 1) * dim].double() for t in (filled.k, filled.v))
            qh = qd[rows, h * dim:(h + 1) * dim]
            kz, vz = k.nan_to_num(0.0, 0.0, 0.0), v.nan_to_num(0.0, 0.0, 0.0)
            t = (qh @ kz.t()) * factor
            err = (qh.abs() @ kz.abs().t()) * factor * ((dim + 8) * U + term)
            if cap:
                t = cap * torch.tanh(t / cap)
                err = err + cap * (8 * U if not (bf16 and cap <= 256) else 2.0 ** -22 + 8 * U)
            if slopes is not None:
                bias = slopes[h].cpu().double() * dist
                t = t - bias
                err = err + 4 * U * (bias + t.abs())
            t = t.masked_fill(~seen, -math.inf)
            total = torch.logsumexp(t, 1)
            w = torch.exp(t - total[:, None]).masked_fill(~live[:, None], 0.0)
            want, size = w @ vz, w @ vz.abs()
            off = err.masked_fill(~seen, 0.0).amax(1) + (pos0 + n + 64) * U + 4 * U * t.masked_fill(~seen, 0.0).abs().amax(1)
            allowed = size * (2.5 * off)[:, None] + size * rounding * 1.01 + 1e-30
            if eight:
                allowed = allowed + (pos0 + n) * 2.0 ** -31 * vz.abs().amax()
            allowed = allowed + (U_BF16 * (want.abs() + allowed) if bf16 else U * want.abs())
            mine = got[rows, h * dim:(h + 1) * dim]
            # rows that see something that is no number are none themselves
            huge = (kz.abs().amax(1) > 1e36) | (vz.abs().amax(1) > 1e29)
            nan = (seen & ~(k.isfinite().all(1) & v.isfinite().all(1))[None]).any(1)
            open_ = (seen & huge[None]).any(1) & ~nan    # (beyond what is promised: 2^99 in magnitude)
            bad = ~((mine - want).abs() <= allowed) & ~nan[:, None] & ~open_[:, None]
            assert not bad.any(), (s, h, bad.sum().item(), ((mine - want).abs() / allowed)[bad].max().item(), bad.nonzero()[:4].tolist())
            assert not mine[nan].isfinite().all(1).any()
            ml = got_lse[rows, h]
            fine = live & ~nan & ~open_
            assert not (ml == -math.inf)[fine].any() and (ml == -math.inf)[~live].all()
            assert ((ml - total).abs()[fine] <= (1.5 * off + 8 * U * total.abs())[fine]).all(), ((ml - total).abs() / off)[fine].max()
            assert (mine[~live] == 0).all()


def random_tree(n, rng, straight=0.6):
    return [-1] + [i - 1 if rng.random() < straight else rng.randrange(i) for i in range(1, n)]


# ----------------------------------------------------------------------------------- tokens

def kept_tokens(x, temperature, top_k, top_p, min_p):
    """(indexes that may be drawn, ascending; their weights) of a row of logits in 64 bits."""
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    if (x == np.inf).any():
        x = np.where(x == np.inf, 0.0, -np.inf)
    order = np.lexsort((np.arange(len(x)), -x))
    order = order[x[order] > -np.inf]
    if len(order) == 0:
        return order, None
    if not temperature > 0:
        return order[:1], np.ones(1)
    with np.errstate(under="ignore"):
        w = np.exp((x[order] - x[order[0]]) / min(float(np.float32(temperature)), 3.4028234e38))
    if 0 < top_k < len(order):
        order, w = order[:top_k], w[:top_k]
    if top_p < 1:
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        n = max(1, int((before < float(np.float32(top_p)) * w.sum()).sum()))
        order, w = order[:n], w[:n]
    stay = (w >= min(float(np.float32(min_p)), 1.0)) & (w > 0)
    order, w = order[stay], w[stay]
    by = np.argsort(order)
    return order[by], w[by]


def draw(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, log of its probability, how near the random number is to another token's share)"""
    at, w = kept_tokens(x, temperature, top_k, top_p, min_p)
    if len(at) == 0:
        return -1, math.nan, 1.0
    upto = np.cumsum(w)
    u = 0.0 if not u > 0 else min(float(np.float32(u)), 1.0)
    i = min(int(np.searchsorted(upto, u * upto[-1], side="right")), len(at) - 1)
    ends = np.concatenate([[0.0], upto]) / upto[-1]
    inner = ends[1:-1]
    return int(at[i]), math.log(w[i] / upto[-1]), float(np.abs(inner - u).min()) if len(inner) else 1.0


def check_tokens(logits, uniform, tokens, logprob, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Every token is the definition's; where the random number lies within 1e-12 of a border (sums of 64 bits), either side's."""
    x, u = logits.detach().float().cpu().numpy(), uniform.cpu().numpy()
    pick = lambda v, r: v[r].item() if isinstance(v, torch.Tensor) else v  # noqa: E731
    for r in range(len(x)):
        token, log_p, near = draw(x[r], u[r], *(pick(v, r) for v in (temperature, top_k, top_p, min_p)))
        assert tokens[r].item() == token or near < 1e-12, (r, tokens[r].item(), token, near)
        if logprob is not None:
            got = logprob[r].item()
            assert math.isnan(got) if math.isnan(log_p) else abs(got - log_p) <= 4 * U * max(1.0, abs(log_p)) or near < 1e-12, (r, got, log_p)


def empty(layers, heads, kv_heads, dim, max_tokens, dtype, page_tokens=16, seed=0):
    kv = B.LayerCache(layers, heads, dim, max_tokens, n_kv_heads=kv_heads, dtype=dtype, page_tokens=page_tokens)
    kv.set_page_order(torch.randperm(kv.num_pages, generator=torch.Generator().manual_seed(seed)).tolist())
    return kv
