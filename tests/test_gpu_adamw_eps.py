"""AdamW with an eps that fp32 does not hold: it is above 0 all the same."""
import pytest
import torch

import paper_2607_05095_amd as fast

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("eps", [1e-60, 1e-46, 1e-44, 1e-8])
@pytest.mark.parametrize("low", [False, True], ids=["32", "8"])
def test_adamw_weights_without_gradients_stay(eps, low):
    """0 / (0 + eps) = 0: weights that no gradient has reached move by their decay alone."""
    n = 1100
    w, g = torch.randn(n, device="cuda"), torch.zeros(n, device="cuda")
    g[::7] = 0.01
    state = torch.uint8 if low else torch.float32
    m, v = torch.zeros(n, dtype=state, device="cuda"), torch.zeros(n, dtype=state, device="cuda")
    s = [[torch.zeros((n + 31) // 32, dtype=torch.uint8, device="cuda")] for _ in range(2)] if low else [None, None]
    old = w.clone()
    ts = fast.adamw_tensors([w], [g], [m], [v], *s)
    fast.fast_adamw(ts, fast.F32, fast.STATE_MXFP8 if low else fast.STATE_F32, 0.5, .9, .999, eps, 1, 3)
    still = g == 0
    assert torch.equal(w[still], old[still])
    # m / (1 - b1) = g, sqrt(v / (1 - b2)) = g: a step of lr, within the roundings of a dozen operations
    assert ((old - w)[~still] / 0.5 - 1).abs().max() < 1e-4
