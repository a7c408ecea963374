"""The border between the tokens that the rules keep and the others, where it is hard to find."""
import math
import random

import numpy as np
import pytest
import torch

from paper_2404_08698_amd import binding as B
from sample_check import check_rows, fits

pytestmark = pytest.mark.gpu

TOP = np.float32(20.0)


def weight(x):
    """Of a logit, in steps of 2^-51 of the weight of TOP."""
    return int(np.rint(np.exp2((np.longdouble(x) - np.longdouble(TOP)) * np.longdouble("1.44269504088896340735992468") + 51)))


def sum_over_lanes(v):
    """Sums over a lane and those before it in 64 bits, in the order in which a wave of 64 forms them: shifts by 1, 2, 4, 8 inside rows of 16, then a row takes
    over what the one before ends with, then the two upper rows what the lower ones do."""
    v = v.copy()
    for by in (1, 2, 4, 8):
        v = v + np.array([v[i - by] if i % 16 >= by else 0.0 for i in range(64)])
    v = v + np.array([v[i // 16 * 16 - 1] if i // 16 % 2 else 0.0 for i in range(64)])
    return v + np.array([v[31] if i >= 32 else 0.0 for i in range(64)])


def half_in_front(seed):
    """(logits of a first group, those behind it): the group fills some of the 64 intervals below TOP, whose sums, rounded in a wave's order, reach half of the row's sum
    only in an interval that holds nothing; None if this seed's do not."""
    rng = random.Random(seed)
    used = sorted(rng.sample(range(1, 20), rng.randrange(3, 9)))
    front = [TOP]
    for b in used:
        for _ in range(rng.randrange(600 // len(used) // 2, 600 // len(used) * 3 // 2)):
            front.append(np.float32(20.0 - (b + rng.random() * 0.9) / 64.0 + 0.9 / 64 - 1 / 64))
    sums = [0] * 64
    for x in front:
        sums[int(np.floor(TOP * 64) - np.floor(x * np.float32(64)))] += weight(x)
    upto = sum_over_lanes(np.array([float(s) for s in sums]))
    last = max(i for i in range(64) if sums[i])
    late = [i for i in range(last + 1, 44) if (upto[:i] < upto[i]).all()]
    if not late:
        return None
    left, behind = 2 * int(upto[late[0]]) - sum(sums), []
    while left > 0 and len(behind) < 1500:
        x = np.float32(20.0 + math.log(left / 2.0 ** 51))
        if x > 20.0 - 46 / 64:
            x = np.float32(20.0 - (46 + rng.random() * 17) / 64)
        while weight(x) > left:
            x = np.nextafter(x, np.float32(-100))
        left -= weight(x)
        behind.append(x)
    return (np.array(front), np.array(behind)) if left == 0 and len(front) + len(behind) <= 2000 else None


@pytest.mark.parametrize("seed", [44, 55, 109, 179, 309, 323])
def test_half_of_a_row_is_not_reached_in_an_empty_interval(seed):
    front, behind = half_in_front(seed)
    n = len(front) + len(behind)
    # (a token that is not kept comes first)
    x = torch.from_numpy(np.concatenate([behind[::-1], front, np.full(2000 - n, -np.inf, np.float32)]).astype(np.float32))
    u = torch.tensor([0.0, 0.1, 0.5, 0.9, 0.999]).cuda()
    logits = x.repeat(len(u), 1).cuda()
    token, logprob = B.sample(logits, u, B.SamplingRules(top_p=0.5), want_logprob=True)
    check_rows(logits, u, token, logprob, top_p=0.5)
    assert ((token >= len(behind)) & (token < n)).sum() >= 4     # (the largest of those behind may be kept: the sum of the others is half but for a rounding)


def test_more_weight_than_equal_logits_have():
    """Sums of slices are of their own largest logit's resolution, the border's of the row's: a million equal logits of 1000.49 steps each are 1000.49 in the sums that say where
    top_p ends, and 1000 where they are counted, so that more of them are wanted than there are.  All of them stay, and the last slice, which has none, takes no part."""
    vocab = 1 << 20
    x = torch.full((3, vocab), float(TOP) + math.log(1000.49 / 2.0 ** 42))
    share = 2.0 ** 42 * np.exp(np.float64(x[0, 1].item()) - np.float64(TOP))
    assert 1000.4 < share < 1000.5
    x[:, vocab - (1 << 14):] = -math.inf
    x[:, 0] = float(TOP)
    u = torch.tensor([0.5, 0.9999, 0.99999]).cuda()
    logits = x.cuda()
    rules = dict(top_p=1.0 - 2.0 ** -24)
    token, logprob = B.sample(logits, u, B.SamplingRules(**rules), want_logprob=True)
    check_rows(logits, u, token, logprob, **rules)
    assert token[0] == 0 and (token[1:] > 0).all()


@pytest.mark.parametrize("rules", [dict(), dict(top_k=3), dict(top_k=60), dict(top_p=0.5), dict(min_p=0.3), dict(top_p=0.6, min_p=0.2)], ids=str)
@pytest.mark.parametrize("vocab", [100, 9000])
def test_the_largest_temperatures(vocab, rules):
    """Where 64 / temperature times a logit is below the smallest number, and where intervals end beyond the largest one."""
    largest = torch.finfo(torch.float32).max
    gen = torch.Generator().manual_seed(vocab)
    noise = torch.randn(4, vocab, generator=gen)
    rows = [torch.full((4, vocab), -1e-10), noise * 1e-12, noise * 1e-30, noise.sign() * largest, noise.clamp(-1, 1) * largest, torch.full((4, vocab), -largest), torch.full((4, vocab), largest)]
    u = torch.tensor([0.0, 0.3, 0.62, 0.97]).cuda()
    for x in rows:
        for temperature in (largest, 1e38, 2e37):
            token, logprob = torch.full((4,), -7, dtype=torch.int32, device="cuda"), torch.full((4,), 9.0, device="cuda")
            B.sample(x.cuda(), u, B.SamplingRules(temperature=temperature, **rules), tokens=token, logprob=logprob)
            check_rows(x, u, token, logprob, temperature=temperature, **rules)
        endless = torch.full((4,), math.inf, device="cuda")
        token, logprob = B.sample(x.cuda(), u, B.SamplingRules(temperature=endless, **rules), want_logprob=True)
        check_rows(x, u, token, logprob, temperature=largest, **rules)


def test_more_rows_than_a_launch_takes():
    rows = (1 << 22) + 3
    x = torch.zeros(rows, 2, device="cuda")
    x[:, 1] = math.log(3.0)
    u = torch.rand(rows, generator=torch.Generator().manual_seed(0)).cuda()
    token = B.sample(x, u)
    near = (u - 0.25).abs() < 1e-6
    assert torch.equal(token[~near], (u >= 0.25).int()[~near]) and ((token == 0) | (token == 1)).all()
