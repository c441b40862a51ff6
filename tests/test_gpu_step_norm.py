"""The step's norm on its own: without optimizer state or an update, of changing and empty masks, and with a bound that nothing reaches."""
import numpy as np
import pytest

from oracle import losses
from synth import CONFIGS, make_workload

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["mlp", "vit_small", "mobilenet_small"])
@pytest.mark.parametrize("with_state", [False, True])
def test_the_norm_of_the_selected_tensors(name, with_state):
    import torch
    from paper_2312_14227_amd.session import Session
    cfg = CONFIGS[name]
    wl = make_workload(cfg, seed=0, init="random")
    s = Session(cfg, wl.weights, with_state=with_state)
    xt, yt = s.put_input(wl.x, wl.y)
    rng = np.random.default_rng(1)
    before = [w.clone() for w in s.w]
    for mask in (np.ones(s.n, np.uint8), (rng.random(s.n) < 0.4).astype(np.uint8), np.zeros(s.n, np.uint8), (np.arange(s.n) == s.n - 1).astype(np.uint8)):
        norm = torch.full((1,), -1.0, device="cuda")
        s.train_step(xt, yt, mask, norm=norm)
        plain = [s.grads_host(k) for k in range(s.n) if mask[k]]
        want = losses.grad_norm(plain)[0] if plain else 0.0
        assert abs(norm.item() - want) <= 2.0 ** -23 * want     # (squares in float64, the root rounded to float32)
        again = torch.full((1,), -1.0, device="cuda")
        s.train_step(xt, yt, mask, max_norm=float("inf"), norm=again)
        # (the gradients stay as computed, whatever the bound)
        assert torch.equal(norm, again) and all(np.array_equal(a, s.grads_host(k)) for a, k in zip(plain, np.flatnonzero(mask)))
    assert all(torch.equal(a, b) for a, b in zip(before, s.w))
    s.close()
