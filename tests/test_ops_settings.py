"""CPU tests of the operators' process-wide settings: what is refused."""
import pytest

from paper_2609_11562_b200 import build as B

B.build()
from paper_2609_11562_b200 import entwine as E  # noqa: E402


@pytest.mark.parametrize("key,value", [(0, 1), (3, 1), (-1, 1), (1, 0), (1, -5), (1, 999_999), (2, -2), (2, 131_072), (2, 1 << 40)])
def test_settings_out_of_range_are_refused(key, value):
    with pytest.raises(E.EntwineError, match="entwine_ops_set_option") as e:
        E.ops_set_option(key, value)
    assert e.value.code == E.ERR_INVALID


def test_settings_in_range_are_taken():
    E.ops_set_option(E.OPS_OPT_WAIT_BUDGET_NS, 1_000_000)
    E.ops_set_option(E.OPS_OPT_WAIT_BUDGET_NS, 2_000_000_000)
    E.ops_set_option(E.OPS_OPT_WITHHOLD_BLOCK, 0)
    E.ops_set_option(E.OPS_OPT_WITHHOLD_BLOCK, -1)


def test_the_count_needs_a_place():
    assert E._lib.entwine_ops_failed_waits(None, None) == E.ERR_INVALID
