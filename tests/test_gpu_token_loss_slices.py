"""A long row of wedlm_token_loss that is cut into slices has one normaliser:
every lane that forms a part of the gradient joins the slices' sums to the same
bits, so that equal logits have equal gradients wherever they stand."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as T

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("R,V", [(64, 151936), (8, 151936), (3, 70001)])
def test_equal_logits_have_equal_gradients(R, V):
    from paper_2512_22737_amd import wedlm
    print(f"token loss in slices {R}x{V}", flush=True)
    g = torch.Generator(device="cuda").manual_seed(R)
    x = torch.randn(R, V, generator=g, device="cuda")
    # the slices' maxima all differ; every fourth logit is the row's own value
    x[:, ::4] = torch.randn(R, 1, generator=g, device="cuda")
    t = torch.full((R,), 1, dtype=torch.int32, device="cuda")
    loss, d = torch.empty(R, device="cuda"), torch.empty_like(x)
    wedlm.wedlm_token_loss(x, t, loss, None, d)
    same = d[:, ::4]
    assert (same == same[:, :1]).all(), [
        int(row.unique().numel()) for row in same]
    (l, dl), (bl, bd) = T.token_loss(x.double().cpu().numpy(),
                                     t.cpu().numpy(), np.ones(R))
    assert (np.abs(loss.double().cpu().numpy() - l) <= bl).all()
    assert (np.abs(d.double().cpu().numpy() - dl) <= bd).all()
