"""What the options of the class losses become on their way into the library.  CPU only (see test_gate_validation)."""
import pytest

from test_class_validation import I32, I64, R, X, Y, ctx, fake   # noqa: F401 (ctx is a fixture)

CALLS = {
    "policy": lambda c, **k: c.policy_loss(fake(X), fake(Y, I64), fake(R), **k),
    "pref": lambda c, **k: c.pref_loss(fake(X), fake(Y, I64), fake(5, I32), **k),
    "distill": lambda c, **k: c.distill_loss(fake(X), fake((6, 2), I32), fake((6, 2)), **k),
}


@pytest.mark.parametrize("what", CALLS)
def test_a_norm_below_fp32_is_refused(ctx, what):
    """The library takes a float, whose 0 stands for the sum of the weights: no number may become that."""
    for norm in (1e-50, 7e-46, 5e-324):
        with pytest.raises(ValueError):
            CALLS[what](ctx, norm=norm)
    assert ctx.rec.calls == []
    CALLS[what](ctx, norm=1e-45)                    # fp32's smallest number
    assert len(ctx.rec.calls) == 1
