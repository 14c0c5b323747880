"""Sizes that the token-gate calls cannot take are refused before a device is looked at.  CPU only."""
import pytest

from paper_2308_10037_b200 import api
from test_gate_validation import L, NULL, P, dead   # noqa: F401 (L and dead are fixtures)


@pytest.mark.parametrize("T,n", [(4, 65535 * 256 + 1), (2 ** 31 - 1, 8191), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_embed_grad_refuses_grids_that_do_not_fit_before_anything_else(L, dead, T, n, accumulate):
    for call, base in ((L.lr_embed_grad, 256), (L.lr_embed_grad_bf16, 256)):
        assert call(dead, P, 4, P, n, T, 9, n, 1.0, -1, accumulate, P, NULL) == api.LR_ERR_SHAPE


def test_the_stated_limits_hold(L, dead):
    assert L.lr_embed(dead, P, 8388481, P, 4, 4, 9, 8388481, 1.0, P, 8388481, NULL) == api.LR_ERR_SHAPE
    assert L.lr_embed_grad(dead, P, 4, P, 8, 4, 2 ** 31 - 1, 8, 1.0, -1, 0, P, NULL) == api.LR_ERR_SHAPE
