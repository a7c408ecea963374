"""The operators on caches in 64 bits, on the CPU, key by key as their definitions say; and caches with known contents."""
import math

import torch

from paper_2404_08698_amd import binding as B

U = 2.0 ** -24      # half a step of fp32, relative
U_BF16 = 2.0 ** -8  # ... and of bf16


class Filled:
    """Caches of the same shape with N(0, 1) contents: what lies in them, and the handles."""

    def __init__(self, heads, kv_heads, dim, lengths, dtype="bf16", page_tokens=16, layers=1, layer=0, seed=0, scattered=True, capacity=None):
        gen = torch.Generator().manual_seed(seed)
        self.heads, self.kv_heads, self.dim, self.layer, self.dtype = heads, kv_heads, dim, layer, dtype
        self.k, self.v, self.kvs = [], [], []
        for n in lengths:
            kv = B.LayerCache(layers, heads, dim, max(capacity or 0, n, 1), n_kv_heads=kv_heads, dtype=dtype, page_tokens=page_tokens)
            if scattered:
                kv.set_page_order(torch.randperm(kv.num_pages, generator=gen).tolist())
            k, v = (torch.randn(n, kv_heads * dim, generator=gen) for _ in range(2))
            if dtype == "bf16":
                k, v = k.bfloat16().float(), v.bfloat16().float()
            if n:
                kv.write(layer, 0, k.cuda(), v.cuda())
            self.k.append(k)
            self.v.append(v)
            self.kvs.append(kv)

    def put(self, s, pos, k=None, v=None):
        """Overwrites a position of sequence s."""
        for name, row in (("k", k), ("v", v)):
            if row is not None:
                getattr(self, name)[s][pos] = row
        self.kvs[s].write(self.layer, pos, self.k[s][pos:pos + 1].cuda().contiguous(), self.v[s][pos:pos + 1].cuda().contiguous())


def rows_like(filled, n, dtype=torch.bfloat16, seed=1, std=2.0, pitch=0):
    """n query rows (of `pitch` elements if given), on the GPU."""
    gen = torch.Generator().manual_seed(seed)
    width = filled.heads * filled.dim
    q = (torch.randn(n, max(width, pitch), generator=gen) * std).to(dtype).cuda()
    return q[:, :width]


def visible(pos0, n, total, window=0, prefix=0, first_key=None):
    p = torch.arange(pos0, pos0 + n)[:, None]
    j = torch.arange(total)[None, :]
    seen = j <= p
    if window:
        seen = seen & (j > p - window)
    if prefix:
        seen = seen | (j < prefix)
    if first_key is not None:
        seen = seen & (j >= first_key[:, None])
    return seen, p - j


def attention(filled, q, spans, scale=0.0, cap=0.0, window=0, prefix=0, slopes=None, first_key=None):
    """spans: (pos0, rows) per sequence.  Per row and head: out, lse, and how far sums in fp32 may be from them: the error of a
    score (its products' magnitudes times their number times half a step), and the weighted magnitude of the values."""
    heads, dim = filled.heads, filled.dim
    group = heads // filled.kv_heads
    scale = scale or 1.0 / math.sqrt(dim)
    q = q.detach().cpu().double()
    out, lse = torch.zeros(q.shape[0], heads, dim, dtype=torch.float64), torch.full((q.shape[0], heads), -math.inf, dtype=torch.float64)
    size, off = torch.zeros_like(out), torch.zeros_like(lse)
    mass = [torch.zeros(filled.kv_heads, p + n, dtype=torch.float64) for p, n in spans]
    at = 0
    for s, (pos0, n) in enumerate(spans):
        total = pos0 + n
        rows = slice(at, at + n)
        at += n
        if n == 0:
            continue
        seen, dist = visible(pos0, n, total, window, prefix, None if first_key is None else first_key[rows].cpu().long())
        for h in range(heads):
            g = h // group
            k, v = (t[s][:total, g * dim:(g + 1) * dim].double() for t in (filled.k, filled.v))
            qh = q[rows, h * dim:(h + 1) * dim]
            t = (qh @ k.nan_to_num(0.0, 0.0, 0.0).t()) * scale
            err = (qh.abs() @ k.nan_to_num(0.0, 0.0, 0.0).abs().t()) * scale * ((dim + 8) * U)
            if cap:
                t = cap * torch.tanh(t / cap)
                err = err + cap * 8 * U
            if slopes is not None:
                bias = slopes[h].cpu().double() * dist.abs()
                t = t - bias
                err = err + 4 * U * (bias + t.abs())
            t = t.masked_fill(~seen, -math.inf)
            live = seen.any(1)
            total_t = torch.logsumexp(t, 1)
            w = torch.exp(t - total_t[:, None]).masked_fill(~live[:, None], 0.0)
            lse[rows, h] = total_t
            vz = v.nan_to_num(0.0, 0.0, 0.0)
            out[rows, h] = w @ vz
            size[rows, h] = w @ vz.abs()
            off[rows, h] = (err.masked_fill(~seen, 0.0).amax(1) + (total + 64) * U + 4 * U * t.masked_fill(~seen, 0.0).abs().amax(1))
            mass[s][g] += w.sum(0)
    return out.reshape(q.shape[0], -1), lse, size.reshape(q.shape[0], -1), off, mass


def check_attention(filled, q, spans, out, lse, **rules):
    """Both results against 64 bits.  A score that is off by e changes a weight by e of it, and the sum by as much: 2 e of the
    values' weighted magnitude; bf16 rows add half a step of every weight and of the output."""
    want, want_lse, size, off, _ = attention(filled, q, spans, **rules)
    got, got_lse = out.detach().cpu().double(), lse.detach().cpu().double()
    allowed = size * (2.5 * off).repeat_interleave(filled.dim, 1) + 1e-30
    if q.dtype == torch.bfloat16:
        allowed = allowed + U_BF16 * size * 1.01 + U_BF16 * (want.abs() + allowed + U_BF16 * size)
    else:
        allowed = allowed + U * want.abs()
    bad = ~((got - want).abs() <= allowed)
    assert not bad.any(), (bad.sum().item(), ((got - want).abs() / allowed).max().item(), bad.nonzero()[:4].tolist())
    dead = want_lse == -math.inf
    assert torch.equal(got_lse == -math.inf, dead)
    wrong = ~((got_lse - want_lse).abs() <= 1.5 * off + 8 * U * want_lse.abs())
    assert not wrong[~dead].any(), ((got_lse - want_lse).abs() / off)[~dead].max().item()
    if dead.any():
        assert (got.reshape(*dead.shape, -1)[dead] == 0).all()


#: (heads, key / value heads, head dim, [(pos0, rows)]) that take the form whose rows share keys through LDS, where neither caps nor biases nor a
#: short window are among the rules; with and without splits of the keys, blocks that are not full, several sequences
SHARED_SHAPES = [(32, 8, 128, [(8000, 300)]), (32, 4, 64, [(0, 2222)]), (16, 1, 128, [(9000, 500)]), (32, 2, 128, [(2000, 513), (0, 3), (2400, 777)]),
                 (48, 48, 64, [(0, 1700)])]
#: ... and with documents, bf16 rows alone
SHARED_DOCUMENTS = (32, 2, 128, [(0, 3000)])
