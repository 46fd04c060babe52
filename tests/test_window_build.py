"""How the window attention is compiled: it tells rows that see NaN from others, by comparisons and arithmetic that
a compiler may drop where it is told that no value is NaN."""

import re

from paper_2410_01651_amd import build


def test_window_attention_is_compiled_with_nan():
    flags = build.COMMON + build.PER_SOURCE["window_attn.hip"]
    assert not [f for f in flags if re.search("no-honor-nans|fast-math|finite-math|no-amdgpu-ieee|Ofast", f)]
