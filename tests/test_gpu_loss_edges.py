"""et_policy_loss and et_preference_loss where something is not finite: probabilities of zero, infinite logits, references without a distribution."""
import numpy as np
import pytest

from loss_util import close, half_step, rel
from oracle import losses
from test_gpu_policy_loss import KL, Case as Policy
from test_gpu_preference_loss import Case as Preference

pytestmark = pytest.mark.gpu

LOWEST = {True: -3.3895313892515355e38, False: -3.4028234663852886e38}


@pytest.mark.parametrize("eps", [0.0, 0.1, 1.0])
@pytest.mark.parametrize("row", [0, 1])
@pytest.mark.parametrize("C,offsets", [(50, False), (50, True), (3000, False)])
def test_an_infinite_margin(C, offsets, row, eps):
    """A token of probability zero in the preferred sequence (row 0) or the other: the pair's loss is 0 or infinite, its gradient finite, the other pair's as ever."""
    def edit(c):
        c.label[:] = 2
        c.x[row, 2] = -np.inf

    c = Preference([1, 1, 1, 1], C, False, edit=edit, masked=0, ref=False, eps=eps, offsets=offsets).call()
    w, R = losses.preference_loss(c.x, c.label, c.offsets, c.beta, c.eps), 4 * rel(C)
    z = w["z"][1]
    assert w["loss"] == np.inf if eps == 0.1 or (row == 0) == (eps == 0.0) else w["loss"] < 1 + abs(z)
    lp = np.array([losses.log_softmax(v)[2] for v in c.x])
    size = c.beta * sum(1 + abs(v) for v in lp[2:])             # (what the other margin is off by, and its loss and factor, whose slopes are at most 1)
    close(c.loss.item(), w["loss"], R * (size + 1), "loss")
    close(c.stats.cpu().numpy(), w["stats"], [0, 1e-6], "stats")
    assert c.logp[row].item() == -np.inf
    p = np.exp([losses.log_softmax(v) for v in c.x])
    close(c.grad.host(), w["grad"], half_step(False) * np.abs(w["grad"]) + R * c.beta / 2 * (1 + size) * np.maximum(p, np.arange(C) == 2) + 1e-37, "grad")


@pytest.mark.parametrize("rows,C,bf16,kw", [(9, 200, False, {}), (9, 6000, True, {}), (9, 140001, True, {}), (4500, 40, True, {}), (9, 200, True, dict(train=False)),
                                            (9, 5001, True, dict(in_place=True))])
def test_a_reference_that_gives_the_label_probability_zero(rows, C, bf16, kw):
    """exp(d) - d - 1 at d = -infinity is infinite, and its slope along d is -1."""
    def edit(c):
        c.label[1:3] = 0
        c.ref[1] = -np.inf

    c = Policy(rows, C, bf16, edit=edit, **kw).call().check()
    assert c.loss.item() == np.inf and (not c.grad or np.isfinite(c.grad.host()).all())
