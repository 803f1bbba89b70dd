"""The calls of the 4-bit cache, and what a user needs to call them, are the package's own names."""
import re

import paper_2607_11976_b200 as package

from test_abi import declared_functions


def test_every_call_of_the_4_bit_cache_is_in_the_package():
    names = [n for n in declared_functions() if re.match(r"lt_kv4_|lt_page_tables", n)]
    assert len(names) >= 7
    for name in names + ["alloc_kv4_pool"]:
        assert getattr(package, name, None) is getattr(package.binding, name), name
