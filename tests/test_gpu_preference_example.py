"""The preference-tuning example: melded layers, block norms, 8-bit checkpoints, the gated MLP and the preference loss in one step."""
import math

import pytest

pytestmark = pytest.mark.gpu


def test_it_learns_the_preferences():
    from examples import preference_tuning

    losses, right = preference_tuning.train(steps=10)
    assert abs(losses[0] - math.log(2.0)) < 1e-6       # the reference is the model itself before the first step
    assert losses[-1] < 0.5 * losses[0] and right == 1.0


def test_the_adapters_alone_learn_them_too():
    from examples import preference_tuning

    losses, right = preference_tuning.train(steps=8, lr=0.5, norm_lr=0.0)
    assert losses[-1] < 0.5 * losses[0] and right == 1.0
