"""The check of drawn tokens itself: it takes what the definition draws, and nothing beside it (no GPU needed)."""
import math

import numpy as np
import pytest

from draft_reference import draw
from sample_check import fits, resolution


def test_ties_of_equal_logits_are_exact():
    x = np.zeros(4096, np.float32)
    right = -math.log(4096.0)
    assert fits(x, 0.25, 1024, right)
    for token, logprob in ((1023, right), (1025, right), (4095, -3.0), (1024, -3.0), (1024, right + 1e-5)):
        assert not fits(x, 0.25, token, logprob), token
    assert fits(x, 0.0, 0) and not fits(x, 0.0, 1)
    assert fits(x, 1.0, 4095) and not fits(x, 1.0, 4094)
    # half of them, by index
    assert fits(x, 0.5, 1024, math.log(1 / 2048), top_p=0.5) and not fits(x, 0.5, 1023, math.log(1 / 2048), top_p=0.5)
    assert not fits(x, 0.5, 2048, math.log(1 / 2048), top_p=0.5)
    # infinities alike
    x[::2] = np.inf
    assert fits(x, 0.5, 2048, math.log(1 / 2048)) and not fits(x, 0.5, 2046)


@pytest.mark.parametrize("rules", [dict(), dict(top_k=9), dict(top_p=0.8), dict(min_p=0.05), dict(temperature=0.4, top_k=40, top_p=0.9)], ids=str)
def test_a_mistake_is_seen(rules):
    rng = np.random.default_rng(3)
    x = (rng.standard_normal(300) * 2.5).astype(np.float32)
    for u in (0.0, 0.013, 0.4999, 0.77, 0.9999):
        token, logprob, _ = draw(x, u, **rules)
        assert fits(x, u, token, logprob, **rules)
        others = [t for t in range(300) if t != token and fits(x, u, t, **rules)]
        assert not others, (u, token, others)
        assert not fits(x, u, token, logprob + 1e-4, **rules) and not fits(x, u, -1, math.nan, **rules)


def test_rows_without_a_token_and_temperature_0():
    x = np.full(5, np.nan, np.float32)
    assert fits(x, 0.5, -1, math.nan) and not fits(x, 0.5, 0, 0.0) and not fits(x, 0.5, -1, 0.0)
    x[3] = x[4] = 1.0
    assert fits(x, 0.9, 3, 0.0, temperature=0.0) and not fits(x, 0.9, 4, 0.0, temperature=0.0)


def test_resolution():
    assert [resolution(v) for v in (1, 2048, 2049, 32000, 65536, 131072, 1 << 20)] == [2.0 ** -s for s in (52, 52, 51, 48, 47, 46, 43)]
