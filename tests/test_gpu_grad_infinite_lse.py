"""A row whose log-sum-exp is +inf holds an infinity: its query's gradient, and those of what it sees,
are NaN and not 0."""
import pytest
import torch

from test_gpu_grad import FILL, FORMATS, grads, step
from test_gpu_tree import store_with

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("T,G", [(3, 2), (40, 4)])
@pytest.mark.parametrize("new", [True, False])
def test_an_infinite_log_sum_is_no_padding(fmt, T, G, new):
    st, n = store_with([200], 1, 1, 1, fmt, 420)
    mask = torch.ones((1, T), dtype=torch.int64, device="cuda").cumsum(1)
    mask = (torch.ones_like(mask) << (mask - 1))  # token t sees draft t alone
    x = step(st, 1, 1, 1, G, T, mask=mask, new=new)
    want = grads(st, x, 1)
    x["lse"][0, 0, 1, 0] = float("inf")
    got = grads(st, x, 1)
    assert torch.isnan(got["dq"][0, 0, 1, 0].float()).all()
    others = [t for t in range(T) if t != 1]
    assert torch.equal(got["dq"][:, :, others], want["dq"][:, :, others])
    assert torch.equal(got["dq"][0, 0, 1, 1:], want["dq"][0, 0, 1, 1:])
    if new:
        for d in ("dk", "dv"):
            assert torch.isnan(got[d][0, 0, 1].float()).all()
            assert torch.equal(got[d][:, :, others], want[d][:, :, others])
    live = (want["dk_store"].view(-1, 128) != FILL).any(1)
    assert live.sum() == n[0]
    assert torch.isnan(got["dk_store"].view(-1, 128)[live].float()).all()
