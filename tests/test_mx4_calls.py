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
