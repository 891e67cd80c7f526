"""What the calls around products of microscaled 4-bit floats refuse on the host."""
import pytest


@pytest.fixture(scope="module")
def b():
    from paper_2312_08538_b200 import build
    build.build_library()
    from paper_2312_08538_b200 import binding
    return binding


def test_waits_refusals(b):
    for args in ((-1, -1, -1), (0, -2, -1), (0, -1, -2), (0, 1 << 32, -1), (0, -1, (1 << 32) - 1)):
        assert b.lib.conef_mx4_set_waits(*args) == b.ERR_INVALID_ARG
    with pytest.raises(b.ConEFError):
        b.mx4_set_waits(-1.0)
    b.mx4_set_waits(1.0, 3, 4)
    b.mx4_set_waits()
    assert b.lib.conef_mx4_timeouts(None, None) == b.ERR_INVALID_ARG


def test_tensors_that_require_a_gradient_are_refused(b):
    """... where gradients are recorded: the result would silently have none.  (Ahead of the other checks, which CPU tensors do not pass.)"""
    import torch
    x, leaf, d = torch.zeros(4, 8), torch.zeros(4, 8, requires_grad=True), b.Draw(1, 0, 0, 0)
    calls = [lambda: b.dropout(leaf, 0.5, d), lambda: b.dropout(leaf * 2, 0.5, d), lambda: b.mx4_quantise(leaf), lambda: b.mx4_quantise(leaf, forms="both")]
    for call in calls:
        with pytest.raises(b.ConEFError, match="gradient") as e:
            call()
        assert e.value.code == b.ERR_INVALID_ARG
        with torch.no_grad(), pytest.raises(b.ConEFError, match="on a GPU"):
            call()
