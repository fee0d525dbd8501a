"""The choice of continuations where logits are large: a row's log-sum-exp has to keep the logarithm of the sum beside a maximum that
would swallow it, and the sum its terms, whatever the maximum rounds to.

The plain form takes the maximum off first, (x - m) - log(sum) + score in 64 bits; the bars are those of test_gpu_beam.py: an
exponential of x - m, as one difference and a product or as one fma next to the rounded maximum, is off by three roundings of x - m at most
where the residue of that maximum stays below one, and the sum of these by log V times as much."""
import math

import numpy as np
import pytest
import torch

import beam_reference as R
import paper_2412_03409_amd as P
from test_gpu_beam import LSE, select_inputs
from test_gpu_serving import BF16, DEV, F32, gen

pytestmark = pytest.mark.gpu


def candidates(logits, scores):
    """As of a prompt without ended beams, logits [W,V] f64; of a beam its W best."""
    W, V = logits.shape
    logits, scores = R.cleaned(logits), R.cleaned(scores)
    found = []
    for w in range(W):
        m = logits[w].max()
        if scores[w] == -np.inf or m == -np.inf:
            continue
        log_z = math.log(np.exp(logits[w] - m).sum())
        keep = np.nonzero(logits[w] > -np.inf)[0]
        for v in keep[np.argsort(-logits[w][keep], kind="stable")][:W]:
            found.append((((logits[w, v] - m) - log_z) + scores[w], w * V + int(v)))
    return sorted(found, key=lambda c: (-c[0], c[1]))


def check(x, scores):
    got = P.prefixkv_beam_select(x.to(DEV), scores.to(DEV))
    for s in range(x.shape[0]):
        W, V = x.shape[1:]
        found = candidates(x[s].double().numpy(), scores[s].double().numpy())
        for (a, i), (b, j) in zip(found[:W], found[1:W + 1]):
            assert i // V == j // V or a == b or a - b > 2 * LSE, "the inputs' choices are too close"
        n = min(W, len(found))
        tokens, parents, best = (t[s].cpu() for t in got[:3])
        assert (parents[:n].long() * V + tokens[:n]).tolist() == [i for _, i in found[:n]]
        want = np.array([a for a, _ in found[:n]])
        assert (np.abs(best[:n].double().numpy() - want) <= LSE + 2.0 ** -24 * np.abs(want)).all()
        assert bool((tokens[n:] == -1).all()) and bool((parents[n:] == -1).all()) and bool(torch.isneginf(best[n:]).all())


def among_ordinary_beams(V, dtype, g):
    """Two prompts of four beams: the second beam of the first prompt, and all of the second's, are for the caller to fill.  The scores are
    such that a token of the second beam comes behind the others' best with its share of an even row, and far before them if it counts whole."""
    x = torch.randn((2, 4, V), generator=g) * 2.5
    scores = torch.tensor([[-100.0, -105.3 + math.log(V), -100.7, -101.9], [-7.25, -3.5, -11.125, -3.875]])
    return x, scores


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [777, 32000, 100003])
@pytest.mark.parametrize("value", ["lowest", "largest", 1e38, -1e38, -1e30, 3e17])
def test_rows_of_one_huge_value(value, V, dtype):
    """A beam whose tokens are all hidden by the type's lowest value has each of them with the probability 1 / V."""
    x, scores = among_ordinary_beams(V, dtype, gen(V))
    value = {"lowest": torch.finfo(dtype).min, "largest": torch.finfo(dtype).max}.get(value, value)
    x[0, 1] = value
    x[1] = value
    check(x.to(dtype), scores)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V,count", [(777, 2), (777, 40), (32000, 3), (32000, 32000)])
def test_rows_with_several_infinities(V, count, dtype):
    """They share the row's weight."""
    x, scores = among_ordinary_beams(V, dtype, gen(count))
    scores[0, 1] = -104.3 + math.log(count)
    at = torch.randperm(V, generator=gen(V))[:count]
    x[0, 1, at] = float("inf")
    x[1][:, at] = float("inf")
    check(x.to(dtype), scores)


@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("V", [777, 32000])
@pytest.mark.parametrize("value", [6e4, -7e4, 1e6, -3e7, 1e9, -1e9, 6e9, 1e12, 1e17, -1e17, 1e25, -9e29])
def test_rows_around_a_large_value(value, V, dtype):
    """Logits a few steps of the type apart, where a step is less than a few units, else equal."""
    x, scores = among_ordinary_beams(V, dtype, gen(V + 1))
    x[0, 1] += value
    x[1] += value
    check(x.to(dtype), scores)


def test_values_at_the_ends():
    """Rows without a token, with +inf next to ordinary logits, with the type's largest values; scores that are NaN or +inf."""
    inf, V = float("inf"), 777
    x, scores, _ = select_inputs(3, 6, 4, V, F32)
    scores = scores.clamp(min=-200.0)
    x[0] = -inf
    x[1, 1:] = float("nan")
    x[2, 0, 5] = inf
    x[2, 1] = 3e38
    x[3, 0, 9] = -3e38
    scores[4] = torch.tensor([float("nan"), -inf, -5.0, inf])
    scores[5] = -inf
    check(x, scores)
