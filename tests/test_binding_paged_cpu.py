"""The binding of the rotations: numbers that the ABI's 32-bit fields do not hold."""
import pytest

from paper_2606_24467_amd import compresskv as C
from tests.test_abi_paged_cpu import _Here


@pytest.mark.parametrize("fields", [dict(layout=1 << 32), dict(layout=(1 << 32) + C.ROTARY_PAIRS),
                                    dict(scaling=1 << 32), dict(rotary_dim=(1 << 32) + 64),
                                    dict(head_dim=(1 << 32) + 64, rotary_dim=64)], ids=str)
def test_fields_past_32_bits_are_refused(fields):
    """(Their low bits alone would name another layout, scaling or size.)"""
    args = dict(head_dim=64, device="cpu")
    args.update(fields)
    with _Here(), pytest.raises(ValueError, match="32 bits"):
        C.Rotary(**args)
