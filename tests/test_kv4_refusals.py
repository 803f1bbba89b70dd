"""Further refusals of the calls on the 4-bit cache, on the host."""
import pytest

from test_kv4_abi import FAKE, INVALID, TABLES, lib  # noqa: F401


@pytest.mark.parametrize("B", [2, 1000])
@pytest.mark.parametrize("by", [0, 4, -4])
@pytest.mark.parametrize("input", ["context_len", "new_len"])
def test_page_tables_refuses_lengths_that_overlap(lib, input, by, B):  # noqa: F811
    """The new lengths beside, before or behind an input's first element, and at its last one."""
    other = {"context_len": "new_len", "new_len": "context_len"}[input]
    for at in (by, (B - 1) * 4 if by >= 0 else -(B - 1) * 4):
        a = {**TABLES, input: 0x100000, other: 0x200000, "total_len": 0x100000 + at, "B": B}
        assert lib.lt_page_tables(*a.values()) == INVALID
