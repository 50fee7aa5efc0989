"""The 4-bit MLP block's refusals, without a GPU."""

import pytest
import torch

from paper_2605_28803_gb300 import qvla as Q
from paper_2605_28803_gb300.fp4_mlp import Fp4Mlp


def layer(n, k, gated, xdt=Q.BF16, ydt=Q.BF16):
    return Q.Fp4Layer(0, n, k, 1, Q.NVFP4, xdt, ydt, gated)  # no handle: nothing here reaches the library with it


def norm(dt=Q.BF16):
    return Q.BlockNorm(Q.NORM_RMS, dt)


def block(gate_up=None, down=None, before=None, after=None, tokens=4, rdt=None):
    return Fp4Mlp(gate_up or layer(256, 128, True), down or layer(128, 256, False), before or norm(), after or norm(), tokens, rdt, device="cpu")


@pytest.mark.parametrize("kw", [
    dict(gate_up=layer(256, 128, False)), dict(down=layer(128, 256, True)), dict(down=layer(128, 512, False)), dict(down=layer(256, 256, False)),
    dict(gate_up=layer(256, 128, True, xdt=Q.F32)), dict(down=layer(128, 256, False, ydt=Q.F16)), dict(before=norm(Q.F16)), dict(after=norm(Q.F16)),
    dict(rdt=Q.F16), dict(tokens=0)])
def test_what_does_not_fit_together(kw):
    with pytest.raises(ValueError):
        block(**kw)


def test_inputs_of_other_shapes():
    b = block()
    r, y = torch.zeros(3, 128, dtype=torch.bfloat16), torch.zeros(3, 128, dtype=torch.bfloat16)
    assert b._check(r, y) == 3 and b._check(r[:0], y[:0]) == 0
    for bad in ((torch.zeros(5, 128, dtype=torch.bfloat16),) * 2, (r, y[:2]), (r[:, :64], y), (r.float(), y), (r, y.half()), (r, torch.zeros(128, 3, dtype=torch.bfloat16).T)):
        with pytest.raises(ValueError):
            b._check(*bad)
    f = block(rdt=Q.F32)
    assert f._check(r.float(), y) == 3
    with pytest.raises(ValueError):
        f._check(r, y)
