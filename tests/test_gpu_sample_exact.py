"""Drawn tokens and log-probabilities, each held to its own share: next to a border as everywhere, exactly where weights are equal."""
import math

import pytest
import torch

from paper_2404_08698_amd import binding as B
from sample_check import check_rows, resolution

pytestmark = pytest.mark.gpu

RULES = [dict(), dict(top_k=1), dict(top_k=7), dict(top_k=900), dict(top_p=0.5), dict(top_p=0.95), dict(top_p=0.99999), dict(min_p=0.1), dict(min_p=1.0), dict(temperature=0.0),
         dict(temperature=0.8, top_k=50, top_p=0.9, min_p=0.02), dict(temperature=1.7, top_k=1500, top_p=0.8), dict(temperature=2.0, top_p=0.97, min_p=1e-6)]


def run(x, u, **rules):
    token, logprob = B.sample(x, u, B.SamplingRules(**rules), want_logprob=True)
    check_rows(x, u, token, logprob, **rules)
    return token


@pytest.mark.parametrize("rules", RULES, ids=str)
@pytest.mark.parametrize("vocab", [1, 3, 100, 4097, 8193, 32000, 131072])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_every_token_is_its_share_s(vocab, rules, dtype):
    gen = torch.Generator().manual_seed(vocab)
    x = (torch.randn(6, vocab, generator=gen) * 2.5).to(dtype).cuda()
    run(x, torch.cat([torch.rand(4, generator=gen), torch.tensor([0.0, 1.0 - 2.0 ** -24])]).cuda(), **rules)


@pytest.mark.parametrize("vocab", [7, 100, 4096, 4100, 9000, 70000, 1 << 18])
def test_equal_logits_are_exact(vocab):
    """Ties of the random number with a border, of top_p with a sum: all sums are exact, so the next token is drawn, not the one before."""
    # (parts of 4 and 8, and of the number of tokens where that is a product in 32 bits)
    u = torch.tensor([0.0, 0.125, 0.25, 0.5, 0.75, 1.0 - 2.0 ** -24] + [(vocab // d) / vocab for d in (2, 3, 5)]).cuda()
    for x in (torch.zeros(vocab), torch.full((vocab,), -7.25), torch.where(torch.arange(vocab) % 4 == 1, -math.inf, 3.0), torch.where(torch.arange(vocab) % 3 == 2, math.inf, 0.0)):
        for rules in (dict(), dict(temperature=0.37), dict(top_k=4), dict(top_k=vocab // 2 + 1), dict(top_p=0.5), dict(top_p=0.25, temperature=3.0), dict(top_p=0.7), dict(min_p=1.0),
                      dict(top_k=vocab // 2 + 1, top_p=0.5), dict(temperature=0.0)):
            run(x.repeat(len(u), 1).cuda(), u, **rules)


@pytest.mark.parametrize("vocab", [2000, 20000, 131072])
def test_the_resolution_of_weights(vocab):
    """One logit far above all others, which are equal: where their weights are below half a step, none of them is drawn; from half a step on they are.  A sum over the
    row is off by half a step for each at most."""
    step = 2 * resolution(vocab)
    for part, drawn in ((0.4, False), (0.6, True), (2.0 ** 10 + 0.3, True)):
        x = torch.full((2, vocab), math.log(part * step))
        x[:, vocab - 1] = 0.0
        token = run(x.cuda(), torch.tensor([0.0, 0.5]).cuda())
        assert token.tolist() == [0 if drawn else vocab - 1, vocab - 1], part
