"""Refusals of the token mixer's entry points that need no GPU."""
import pytest

FAKE, S = 0x10000, 0  # never dereferenced: the checks come first


@pytest.fixture(scope="module")
def vmb():
    from paper_2412_16602_gb300 import _build
    _build.build()
    import paper_2412_16602_gb300 as vmb
    return vmb


def step(vmb, q=FAKE, k=FAKE * 2, v=FAKE * 3, o=FAKE * 4):
    return vmb.lib.vmb_delta_rule_step(q, k, v, FAKE, FAKE, None, FAKE * 5, 0, o, 2, 1, 2, 2, 16, 16, 2, 0.25, 0, S)


def test_step_refuses_an_output_in_place_of_an_input(vmb):
    """The blocks of a head's other channels still read q and k."""
    for name in ("q", "k", "v"):
        assert step(vmb, **{name: FAKE * 4}) == vmb.VMB_ERR_INVALID_ARG
