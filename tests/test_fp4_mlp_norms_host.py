"""Norms whose vectors do not fit the 4-bit MLP block, refused where the block is made."""

import pytest
import torch

from paper_2605_28803_gb300 import qvla as Q
from tests.test_fp4_mlp_host import block  # 128 channels, 4 tokens


def t(*shape, dtype=torch.bfloat16):
    return torch.zeros(*shape, dtype=dtype)


def norm(**kw):
    return Q.BlockNorm(Q.NORM_RMS, Q.BF16, **kw)


WIDTHS = [dict(pre_weight=t(256)), dict(pre_weight=t(64)), dict(pre_weight=t(128), pre_bias=t(136)), dict(post_norm=True, post_weight=t(256)),
          dict(scale=t(4, 256), mod_tokens=1), dict(gate=t(4, 120), mod_tokens=1)]


@pytest.mark.parametrize("where", ["before", "after"])
@pytest.mark.parametrize("kw", WIDTHS)
def test_vectors_of_another_width(where, kw):
    with pytest.raises(ValueError, match=f"`{where}`"):
        block(**{where: norm(**kw)})


def test_vectors_of_the_blocks_width():
    mods = t(2, 384)  # a conditioning layer's output, of which each takes a third
    assert block(before=norm(pre_weight=t(128), gate=mods[:, :128], scale=mods[:, 128: 256], shift=mods[:, 256:], mod_tokens=2),
                 after=norm(post_norm=True, post_weight=t(128), pre_weight=t(128), pre_bias=t(128)))


@pytest.mark.parametrize("where", ["before", "after"])
@pytest.mark.parametrize("kw", [dict(gate=t(1, 128), mod_tokens=2), dict(shift=t(2, 128), mod_tokens=1), dict(scale=t(5, 128), mod_index=t(2, dtype=torch.int32))])
def test_more_tokens_than_a_norms_conditioning_has(where, kw):
    """Refused before any call: behind the first one the residual is no longer what it was."""
    b = block(**{where: norm(**kw)})
    assert b._check(t(2, 128), t(2, 128)) == 2
    with pytest.raises(ValueError, match=f"`{where}`"):
        b._check(t(3, 128), t(3, 128))


def test_an_index_without_conditioning_is_not_read():
    assert block(after=norm(mod_index=t(4, dtype=torch.int32)))._check(t(4, 128), t(4, 128)) == 4
