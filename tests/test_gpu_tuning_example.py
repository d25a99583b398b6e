"""The fine-tuning example runs its operators together: after the preference
stage more present than absent links are preferred, and after the reward stage
more drawn columns are links (both by the model's own measure; the learning
rates are far too small to overshoot and 30 steps far more than chance needs)."""
import os
import sys

import pytest

from gpu_common import require_gpu

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def test_tune_links():
    require_gpu()
    import tune_links

    r = tune_links.main(["--cells", "2048", "--steps", "40", "--pairs", "256"])
    assert r["preferred_after"] > r["preferred_before"]
    assert r["preference_loss"] < 0.69            # below that of the unchanged model, log 2
    assert r["reward_after"] > r["reward_before"]
    assert r["kl"] >= 0.0 and r["loss_after"] < 100.0


def test_tuned_factors_still_complete_the_matrix():
    """The steps are bounded (clipped to a norm of 1, rates 20 and 80, far below the factors' own norm) and the rewards
    held to the fitted model by the KL term: the completion's objective rises by less than a tenth."""
    require_gpu()
    import tune_links

    r = tune_links.main(["--cells", "2048", "--steps", "40", "--pairs", "256"])
    assert r["loss_before"] > 0.0 and r["loss_after"] < 1.1 * r["loss_before"]
