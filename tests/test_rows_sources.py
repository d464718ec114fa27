"""Rules of the sources that no run shows reliably: a load in inline assembly in front of a store to the same place (drows may be rows itself)."""
import re

from tests.test_kernel_sources import _source


def test_loads_in_assembly_keep_their_place_among_stores():
    """Without the clobber a compiler may move an ordinary store in front of the assembly's load."""
    text = _source("rows.cuh")
    loads = re.findall(r'asm volatile\("ld\.global.*?;\s*\n', text, flags=re.S)
    assert len(loads) == 5
    for load in loads:
        assert load.rstrip().endswith(': "memory");'), load
