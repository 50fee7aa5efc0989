"""The prompt attention's failure path: with the test hook that holds back every copy, all of its waits run out; it reports a
time-out, leaves the output alone and returns, and the next call is clean."""

import numpy as np
import pytest
import torch

from paper_2605_28803_gb300 import qvla as Q
from tests import attention_helpers as H

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens_k", [[300, 20], [1400, 1000]], ids=["short", "long"])  # long: CTAs that join their parts
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_waits_that_run_out(dim, lens_k):
    rng = np.random.default_rng(dim)
    lens = [300, 20]
    x = [H.draw_heads(rng, sum(n), h, dim, "bf16").to(H.DEV) for n, h in ((lens, 4), (lens_k, 2), (lens_k, 2))]
    want = H.prompt(*x, lens, lens_k, True)
    Q.qvla_check_device(H.stream())
    Q.qvla_debug_set_hooks(20_000_000, True)
    try:
        got = H.prompt(*x, lens, lens_k, True)
        with pytest.raises(Q.QvlaError) as e:
            Q.qvla_check_device(H.stream())
        assert e.value.status == 6
        assert torch.isnan(got.float()).all()  # nothing was written
    finally:
        Q.qvla_debug_set_hooks(0, False)
    Q.qvla_check_device(H.stream())
    assert torch.equal(H.prompt(*x, lens, lens_k, True), want)
