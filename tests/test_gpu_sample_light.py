"""Tokens whose weight is less than half a step of the sums: kept, and never drawn, by the thousand in
a slice or among heavier ones, at every row count and with every rule.

A step is 2^-shift of the largest weight, shift = 62 - log2(V rounded up to a power of two) and at most 50.
"""
import numpy as np
import pytest
import torch

from tests.test_gpu_sample import Call

pytestmark = pytest.mark.gpu


def _shift(V):
    return min(50, 62 - (V - 1).bit_length())


def _of_steps(V, steps):
    """The logit whose weight is `steps` steps, beside a largest logit of 0 at T = 1."""
    return np.float32(np.log(steps) - _shift(V) * np.log(2.0))


def _fixed(z, V):
    """Weights in steps, each rounded to a whole number."""
    return np.rint(np.exp(z.astype(np.float64)) * 2.0 ** _shift(V)).astype(np.int64)


U = [0.0, 2.0 ** -60, 2.0 ** -24, 0.5, 1 - 2.0 ** -24]
RULES = [{}, dict(top_p=0.999999), dict(top_p=0.5), dict(min_p=1e-30), dict(top_k=0, top_p=1.0, min_p=0.0),
         dict(top_k=1000), dict(temperature=1.0)]


# (few and many rows: a slice is 2,048 or 8,192 tokens)
@pytest.mark.parametrize("V, R", [(5000, 1), (5000, 520), (20003, 1), (20003, 180), (128256, 1), (128256, 40),
                                  ((1 << 20) - 3, 1), ((1 << 20) - 3, 12), ((1 << 20) + 5, 2)])
def test_all_but_the_last_token_light(V, R):
    """0.45 steps each; thousands of them in every slice in front of the one that counts."""
    z = np.full((1, V), _of_steps(V, 0.45), np.float32)
    z[0, V - 1] = 0.0
    assert _fixed(z, V)[0].nonzero()[0].tolist() == [V - 1]
    for rules in RULES:
        for u in U:
            c = Call(np.repeat(z, R, axis=0), np.full(R, u), **{
                n: np.full(R, v, np.int32 if n == "top_k" else np.float32) for n, v in rules.items()}).run()
            tokens, kept, probs, logprob = c.results()
            assert (tokens == V - 1).all(), (rules, u, tokens)
            n = 1 if rules.get("top_p", 1) < 1 else rules.get("top_k") or V
            assert (kept == n).all(), (rules, u, kept)
            # the total is off by at most half a step per token
            assert (np.abs(logprob + np.log1p((n - 1) * 0.45 * 2.0 ** -_shift(V))) <= n * 2.0 ** -_shift(V) + 1e-9).all()


@pytest.mark.parametrize("V, R", [(20003, 1), (20003, 180), (128256, 1), (128256, 40)])
def test_first_token_that_counts(V, R):
    """Light tokens, one of 0.6 steps (a whole step) in their midst, the largest at the end: u = 0 draws the
    former, any u above the light ones' sum the latter."""
    for first in (0, 300, 2047, 2048, 9000, V - 2):
        z = np.full((1, V), _of_steps(V, 0.45), np.float32)
        z[0, first], z[0, V - 1] = _of_steps(V, 0.6), 0.0
        assert _fixed(z, V)[0].nonzero()[0].tolist() == [first, V - 1]
        for u, token in ((0.0, first), (2.0 ** -24, V - 1), (1 - 2.0 ** -24, V - 1)):
            tokens, kept, probs, _ = Call(np.repeat(z, R, axis=0), np.full(R, u)).run().results()
            assert (tokens == token).all(), (first, u, tokens)
            assert (kept == V).all()


@pytest.mark.parametrize("R", [1, 40])
def test_draws_between_light_slices_have_weight(R):
    """Whatever the uniform, the token drawn is one that counts."""
    V = 128256
    rng = np.random.RandomState(4)
    z = np.full((1, V), _of_steps(V, 0.45), np.float32)
    heavy = rng.permutation(V)[:40]
    z[0, heavy] = _of_steps(V, 1.0) + rng.uniform(0, 31, 40).astype(np.float32)
    z[0, heavy[0]] = 0.0
    w = _fixed(z, V)[0]
    u = np.concatenate([2.0 ** -np.arange(1, 46.0), np.arange(1, 40) / 40])
    for a in np.array_split(u, -(-len(u) // R)):
        tokens = Call(np.repeat(z, len(a), axis=0), a).run().results()[0]
        assert (w[tokens] >= 1).all(), (a, tokens)
