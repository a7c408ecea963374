"""What a drawn token and its log-probability may be: the definition in 64 bits, and how far whole weights are from it."""
import itertools
import math

import numpy as np

U = 2.0 ** -24      # half a step of fp32, relative


def resolution(vocab):
    """Half a step of the weights, of the largest: they are multiples of 2^-51, or of 2^-(62 - log2 of the vocabulary, rounded up), so that a row's sum is below 2^62."""
    return 2.0 ** -(min(51, 62 - (vocab - 1).bit_length()) + 1)


def _sets(x, temperature, top_k, top_p, min_p):
    """Every set (indexes ascending, weights) that the rules may leave, and how far its sums may be off."""
    finite = np.flatnonzero(x > -np.inf)
    order = finite[np.lexsort((finite, -x[finite]))]
    with np.errstate(under="ignore"):
        w = np.exp((x[order] - x[order[0]]) / min(float(np.float32(temperature)), 3.4028234663852886e38))
    # Equal weights are exact, and so are their sums and the products with a random number or top_p.  Others: every weight is rounded twice (to a slice's largest
    # and to the row's) and a slice of less than half a step per token counts as none, for the sum and for what lies before a token; and the roundings of sums, products
    # and exponentials in 64 bits.
    flat = bool((w == 1.0).all())
    step = 0.0 if flat else resolution(len(x))
    off = 0.0 if flat else 6 * len(order) * step + 1e-13 * w.sum()
    if 0 < top_k < len(order):
        order, w = order[:top_k], w[:top_k]
    counts, least = [len(order)], [min_p]
    if top_p < 1:
        before, goal = np.concatenate([[0.0], np.cumsum(w)[:-1]]), float(np.float32(top_p)) * w.sum()
        counts = sorted({max(1, int((before < goal + d).sum())) for d in (-off, 0.0, off)})
        off *= 3        # (those at the border: what they weigh, once more in the sum and in front of a token)
    if min_p > 0:
        at = min(float(np.float32(min_p)), 1.0)
        least = sorted({at, at - step, at + step}) if not flat else [at]
    for n, m in itertools.product(counts, least):
        stay = (np.arange(len(order)) < n) & (w >= min(m, 1.0)) & (w > 0)
        by = np.argsort(order[stay])
        yield order[stay][by], w[stay][by], off


def fits(x, u, token, logprob=None, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Whether `token` may be drawn from the row x (float32) by u, and `logprob` (None: not asked) be its own."""
    vocab = len(x)
    x = np.where(np.isnan(x), -np.inf, x.astype(np.float64))
    if (x == np.inf).any():
        x = np.where(x == np.inf, 0.0, -np.inf)
    if not (x > -np.inf).any():
        return token == -1 and (logprob is None or math.isnan(logprob))
    if not 0 <= token < vocab:
        return False
    if not temperature > 0:
        return token == int(np.argmax(x)) and logprob in (None, 0.0)
    u = 0.0 if not u > 0 else min(float(np.float32(u)), 1.0)
    for at, w, off in _sets(x, temperature, top_k, top_p, min_p):
        i = int(np.searchsorted(at, token))
        if i == len(at) or at[i] != token:
            continue
        upto = np.cumsum(w)
        total, low = upto[-1], upto[i] - w[i]
        if off == 0.0:
            if not (low <= u * total < upto[i] or (u == 1.0 and i == len(at) - 1)):
                continue
        elif not low - off <= u * total <= upto[i] + off:
            continue
        want = math.log(w[i] / total)
        if logprob is None or abs(logprob - want) <= 4 * U * max(1.0, abs(want)) + 2 * off / total:
            return True
    return False


def check_rows(logits, uniform, tokens, logprob=None, **rules):
    """All rows of a call."""
    x, u, t = logits.detach().float().cpu().numpy(), uniform.cpu().tolist(), tokens.tolist()
    p = [None] * len(t) if logprob is None else logprob.tolist()
    for r in range(len(x)):
        mine = {k: (v[r].item() if hasattr(v, "shape") else v) for k, v in rules.items()}
        assert fits(x[r], u[r], t[r], p[r], **mine), (r, u[r], t[r], p[r], mine)
