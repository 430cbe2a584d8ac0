"""The example that runs the operators on drafted tokens together: every step's
attention equals the definition on the rotated inputs and on what the store holds,
and the accepted rows are found in the store."""
import os
import sys

import numpy as np
import pytest
import torch

import drafts
from paper_2608_21541_gb300 import workloads as W

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))),
                                "examples"))
import verify_drafts  # noqa: E402

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["bf16", "fp8", "fp4"])
@pytest.mark.parametrize("T", [5, 12])
def test_every_step_matches_the_definition(fmt, T):
    wl = W.Workload("VD", B=2, L=2, Hq=8, H=2, n=1500, d=128, w=16, keep=(1, 8), kind="planted")
    seen = []

    def on_step(step, q, k, v, mask, out, store):
        counts = store.counts.cpu().numpy()
        ref = drafts.attention(q, store, counts, wl.H, k, v, mask)
        drafts.check_attention(out, None, ref)
        seen.append((k.clone(), counts))

    r = verify_drafts.run(wl, fmt, steps=3, T=T, on_step=on_step)
    store = r["store"]
    assert store.read_status() == 0 and len(seen) == 3
    real = r["packed"].real_counts.cpu().numpy() + 1
    np.testing.assert_array_equal(seen[0][1], real)
    np.testing.assert_array_equal(store.counts.cpu().numpy(), real + r["accepted"])
    # the rows appended after the last step are drafts of that step, as encoded
    k, before = seen[-1]
    n = int(store.counts[0].item()) - int(before[0])
    at = drafts.slots(store.table.cpu().numpy(), 0, int(before[0]), n)
    held = drafts.held(store, "k")["codes"][at]
    of_drafts = drafts.encode(k[0, 0, :, 0].cpu(), fmt)["codes"]
    for row in held:
        assert (row == of_drafts).all(1).any()
