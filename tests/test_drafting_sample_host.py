"""What a draft is sampled from: the distribution that verification takes it to be from.  No GPU needed."""
import numpy as np
import pytest
import torch

import drafting as D
from paper_2501_08090_amd.drafting import sample

INF, NAN = float("inf"), float("nan")


def logits_of_every_kind(g):
    z = torch.randn((7, 300), generator=g) * 3
    z[1, ::2] = -INF                       # masked tokens
    z[3, ::3] = NAN                        # count as masked
    return z


def race(p, noise):
    """a token of probability 0 has no part in it, whatever its noise"""
    with np.errstate(divide="ignore", invalid="ignore"):
        return int(np.argmax(np.where(p > 0, p / noise.double().numpy(), -1.0)))


@pytest.mark.parametrize("temperature", (1e-45, 1e-40, 1e-30, 0.3, 1.0, 4.0))
def test_sample_is_the_race_of_the_defined_probabilities(temperature):
    """the token that wins the race of the probabilities as verification defines them (the tests' 64-bit form)"""
    g = torch.Generator().manual_seed(3)
    z = logits_of_every_kind(g)
    z[2, 17] = INF                         # counts as the largest finite value
    z[4] = torch.finfo(torch.float32).min  # all the same
    z[5, 9] = torch.finfo(torch.float32).max
    noise = torch.empty((7, 300)).exponential_(generator=g)
    noise[1, 4], noise[6, int(z[6].argmax())] = 0.0, 0.0  # masked, and not
    t = torch.full((7,), temperature)
    got = sample(z, t, noise)
    assert got.dtype == torch.int32
    for r in range(7):
        with np.errstate(over="ignore", divide="ignore"):
            assert int(got[r]) == race(D.shares(z[r].numpy(), float(t[r])), noise[r]), r


@pytest.mark.parametrize("temperature", (3e38, INF))
def test_sample_at_temperatures_without_end(temperature):
    """the same for every token whose logit is above -inf"""
    g = torch.Generator().manual_seed(4)
    z = logits_of_every_kind(g)
    noise = torch.empty((7, 300)).exponential_(generator=g)
    got = sample(z, torch.full((7,), temperature), noise)
    for r in range(7):
        assert int(got[r]) == race((z[r] > -INF).double().numpy(), noise[r]), r


@pytest.mark.parametrize("temperature", (0.0, -1.0, NAN))
def test_sample_without_a_temperature_is_the_highest_logit(temperature):
    z = logits_of_every_kind(torch.Generator().manual_seed(5))
    z[2, 17] = INF
    got = sample(z, torch.full((7,), temperature), torch.ones((7, 300)))
    assert got.tolist() == np.where(np.isnan(z.numpy()), -np.inf, z.numpy()).argmax(1).tolist()


def test_sample_of_nothing_is_some_token():
    """a row without any logit above -inf: verification gives its p as 0 everywhere; the draft hands on token 0"""
    z = torch.full((2, 10), -INF)
    z[1] = NAN
    for t in (0.0, 1.0):
        assert sample(z, torch.full((2,), t), torch.ones((2, 10))).tolist() == [0, 0]
