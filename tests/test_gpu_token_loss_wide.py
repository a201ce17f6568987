"""wedlm_token_loss on the longest rows that its arguments can name, 2^31 - 1
columns: the step past a row's last column passes 2^31 - 1 too.  All logits are
-inf but a few, so that the sums are short and their bounds those of a row of
those few."""
import numpy as np
import pytest
import torch

from oracle import train_oracle as T

pytestmark = pytest.mark.gpu

V = (1 << 31) - 1


@pytest.fixture(autouse=True)
def memory():
    if torch.cuda.get_device_properties(0).total_memory < 40 << 30:
        pytest.skip("needs 40 GiB")
    yield
    torch.cuda.empty_cache()


# gradients at another offset from 16 bytes than the logits, and at the same
@pytest.mark.parametrize("shift", [1, 0])
def test_row_of_the_longest_vocabulary(shift):
    from paper_2512_22737_amd import wedlm
    print(f"token loss, one row of 2^31 - 1, shift {shift}", flush=True)
    ninf = -float("inf")
    x = torch.full((1, V), ninf, dtype=torch.bfloat16, device="cuda")
    # the first columns, those around 2^30, and the last 300 (the last steps of
    # every thread); the target among the last
    at = torch.cat((torch.arange(5), (1 << 30) + torch.arange(-3, 3),
                    V - 300 + torch.arange(300))).cuda()
    values = torch.randn(len(at), generator=torch.Generator().manual_seed(1))
    x[0, at] = values.bfloat16().cuda()
    hit = len(at) - 2
    t = at[hit:hit + 1].int()
    w = torch.tensor([0.75], device="cuda")
    guard = 1024
    d = torch.full((guard + shift + V + guard,), 7.0, dtype=torch.bfloat16,
                   device="cuda")
    row = d[guard + shift:guard + shift + V].view(1, V)
    loss = torch.full((1,), float("nan"), device="cuda")
    wedlm.wedlm_token_loss(x, t, loss, w, row)
    torch.cuda.synchronize()
    (l, g), (bl, bg) = T.token_loss(
        x[0, at].double().cpu().numpy()[None], np.array([hit]),
        w.double().cpu().numpy())
    assert abs(loss.double().item() - l[0]) <= bl[0]
    # half a step of bf16
    bg = bg + T.BF16 * (np.abs(g) + bg)
    err = np.abs(row[0, at].double().cpu().numpy() - g[0])
    assert (err <= bg[0]).all(), (err / bg[0]).max()
    # nothing for the columns that are ruled out, nothing beside the row
    row[0, at] = 0.0
    for i in range(0, V, 1 << 28):
        assert not row[0, i:i + (1 << 28)].any()
    assert (d[:guard + shift] == 7.0).all() and (d[-guard:] == 7.0).all()
