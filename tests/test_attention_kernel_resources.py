"""What the built kernels of the memory by attention keep in scratch memory: nothing, but for the ones whose comments say so."""
import re

import pytest
from test_kernel_resources import built, of  # noqa: F401  (the fixture)

# two blocks of rows of heads of 128; keys of heads of 128 (and one of fp32 heads of 64); rows that sixteen waves hold: bytes a lane
KNOWN = [(r"k_attn_fwdIDF16bLi128ELi2E", 176), (r"k_attn_dkvIDF16bLi128E", 172), (r"k_attn_dkvIfLi64ELi1ELb1ELi0E", 12), (r"k_norm_bwdI(f|DF16b)Li16E", 188)]


@pytest.mark.parametrize("pattern", [r"k_attn_fwd", r"k_attn_dq", r"k_attn_dkv", r"k_attn_(prepare|join)", r"k_attn_step", r"k_pages", r"k_norm"])
def test_scratch_memory(pattern, built):  # noqa: F811
    room = {n: next((most for p, most in KNOWN if re.search(p, n)), 0) for n in of(built, pattern)}
    assert {n: built[n][".private_segment_fixed_size"] for n, most in room.items() if built[n][".private_segment_fixed_size"] > most} == {}
