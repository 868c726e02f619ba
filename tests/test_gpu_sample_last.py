"""Sampled acceptance where a draw reaches the end of the weights: u[0] of 1 or
more is the last token that has weight, whatever the rounding of the sums, and
a token without weight is never the bonus."""
import numpy as np
import pytest

import kvq_reference as R
from gpu_cases import say
from test_gpu_sample import _call

pytestmark = pytest.mark.gpu

ABOVE = float(np.nextafter(np.float32(1), np.float32(2)))


def _row(rng, V, end, faint):
    """Logits N(0, 1) up to `end`, the last `faint` of them too small to move a
    sum, none behind."""
    x = np.full(V, -np.inf, np.float32)
    x[:end] = rng.standard_normal(end)
    x[end - faint:end] -= 60.0
    return x


@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("V,end", [(40, 31), (5000, 4999), (32000, 32000), (50257, 50001), (151936, 131000),
                                   (200000, 131072), (300000, 140001)])
def test_a_draw_of_one_is_the_last_token_with_weight(V, end, with_draft):
    """The sum of a row and the running sum are rounded apart: with a faint end
    the running sum passes the whole before the last token does.  Rows that end
    in an earlier group of 131072 tokens than the vocabulary; residuals after a
    rejection."""
    rng = np.random.default_rng(V)
    for trial in range(10 if V < 60000 else 4):
        logits = np.stack([_row(rng, V, end, min(end // 2, 1000)) for _ in range(2)])
        draft = np.zeros((2, V), np.float32) if with_draft else None
        if with_draft:
            draft[:, 3] = 0.9
        for u0 in (1.0, ABOVE, 7.0):
            say(f"[sample] last V={V} end={end} draft={with_draft} u0={u0}")
            one = _call([-1], [0], V, logits[:1], 1.0, None if draft is None else draft[:1], np.array([u0], np.float32))
            assert one == ([0], end - 1, 0), u0
            u = np.array([u0, 0.99], np.float32)  # node 1's token is rejected
            assert _call([-1, 0], [0, 3], V, logits, 1.0, draft, u) == ([0], end - 1, 0), u0
        # the largest draw below 1 lies 6e-8 from the end: an ordinary border
        u = np.array([np.nextafter(np.float32(1), np.float32(0)), 0.99], np.float32)
        want = R.accept_sample([-1, 0], [0, 3], V, logits, 1.0, draft, u)
        assert _call([-1, 0], [0, 3], V, logits, 1.0, draft, u)[:2] == want[:2]


def _far(V, *at):
    x = np.full((3, V), -np.inf, np.float32)
    for token, logit in at:
        x[:, token] = logit
    return x


@pytest.mark.parametrize("with_draft", [False, True])
@pytest.mark.parametrize("V", [4300, 9000, 140000])
def test_weights_below_the_smallest_count_as_none(V, with_draft):
    """A weight under e^-700 of the largest is 0.  The faint token shares its
    part of the row with a rejected child of weight e^-600, against which it
    alone would have some."""
    logits = _far(V, (5, 0.0), (4100, -600.0), (V - 50, -701.0))
    draft = None
    if with_draft:
        draft = np.zeros((3, V), np.float32)
        draft[:, 4100] = 0.5
    for u0 in (0.0, 0.5, 1.0, 7.0, float("nan")):
        got = _call([-1, 0], [0, 4100], V, logits[:2], 1.0, draft if draft is None else draft[:2],
                    np.array([u0, 0.9], np.float32))
        assert got == ([0], 5, 0), u0


@pytest.mark.parametrize("V", [4300, 9000])
def test_only_weights_below_the_smallest_are_left(V):
    """Every token that has weight is a child's, and no child is accepted: the
    bonus token is drawn from the row."""
    logits = _far(V, (7, 0.0), (4100, -600.0), (V - 50, -701.0))
    nan = float("nan")
    for u0, bonus in ((0.0, 7), (0.99, 7), (1.0, 4100)):
        got = _call([-1, 0, 0], [0, 7, 4100], V, logits, 1.0, None, np.array([u0, nan, nan], np.float32))
        assert got == ([0], bonus, 0), u0
