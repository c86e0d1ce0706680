"""The gradient of log probabilities in rows of which nothing is asked, and without a gradient of the log probabilities (marker gpu)."""
import numpy as np
import pytest

from layer_helpers import on_gpu, torch_type
from test_gpu_layer_losses import work

pytestmark = pytest.mark.gpu


def both(t, cols, seed):
    """Seven rows, three of them not numbers, and what the forward pass says of them."""
    import torch
    from paper_2204_10562_amd import layer as pp
    x = np.random.default_rng(seed).standard_normal((7, cols))
    x[1, cols // 2], x[4, cols - 1], x[5] = np.nan, np.inf, np.nan
    mx, _ = on_gpu(x, t)
    tokens = torch.tensor([0, -1, 3, -7, -1, -1, cols + 2], dtype=torch.int32, device="cuda")
    norm, entropy, logp = torch.empty(7, 2, device="cuda"), torch.empty(7, device="cuda"), torch.empty(7, device="cuda")
    pp.pp_logprob_forward(mx, 1.0, tokens, logp, entropy, norm, None, None, work(pp.pp_logprob_workspace_bytes(torch_type(t), 7, cols, 0), t))
    return pp, torch, mx, tokens, norm, entropy, logp


@pytest.mark.parametrize("cols", [40, 5000, 150000])
@pytest.mark.parametrize("t", ["bf16", "f16", "f32"])
def test_rows_without_a_token(t, cols):
    """Their log probability is 0 whatever they hold, and so is its gradient; a gradient of the entropy of a row that is no numbers is none."""
    pp, torch, mx, tokens, norm, entropy, logp = both(t, cols, cols)
    padding = tokens < 0
    assert (logp[padding] == 0).all()
    one, dx = torch.ones(7, device="cuda"), torch.full_like(mx, 7)
    pp.pp_logprob_backward(mx, 1.0, tokens, norm, one, None, None, dx)
    assert (dx[padding] == 0).all() and torch.isfinite(dx[[0, 2]]).all() and (dx[[0, 2]] != 0).any() and torch.isnan(dx[6]).all()
    wanted = torch.where(padding, 0.0, 1.0)
    both_ways = torch.full_like(mx, 7)
    pp.pp_logprob_backward(mx, 1.0, tokens, norm, one, entropy, wanted, both_ways)
    assert (both_ways[padding] == 0).all()
    pp.pp_logprob_backward(mx, 1.0, tokens, norm, one, entropy, one, dx)
    assert torch.isnan(dx[[1, 4, 5]]).all() and torch.isfinite(dx[3]).all() and (dx[3] != 0).any()
    pp.pp_logprob_backward(mx, 1.0, tokens, norm, one, None, None, mx)      # in place
    assert (mx[padding] == 0).all()


@pytest.mark.parametrize("t", ["bf16", "f32"])
def test_tokens_without_their_gradient(t):
    """Where no gradient of the log probabilities is given, tokens are nothing to the entropy's, one outside the columns neither."""
    pp, torch, mx, tokens, norm, entropy, _ = both(t, 5000, 2)
    g = torch.randn(7, device="cuda")
    with_tokens, without = torch.empty_like(mx), torch.empty_like(mx)
    pp.pp_logprob_backward(mx, 1.0, tokens, norm, None, entropy, g, with_tokens)
    pp.pp_logprob_backward(mx, 1.0, None, norm, None, entropy, g, without)
    fine = [0, 2, 3, 6]
    assert torch.isfinite(without[fine]).all() and torch.equal(with_tokens[fine], without[fine])
    assert torch.isnan(with_tokens[[1, 4, 5]]).all()
