"""What a library whose kernels over codes cannot be set up still serves (no GPU): read off the source."""
from __future__ import annotations

import re

from tests.test_paged_start import body, code


def test_kernels_over_codes_fail_their_own_calls_alone():
    """A program with 16-bit pools does not depend on them: neither their set-up nor an error that it leaves behind reaches
    vt_paged_create or the next call."""
    capi = code("capi.cu")
    start = body(capi, "cudaError_t init_paged()")
    assert not re.search(r"g_init_paged_err\s*=\s*(init_paged_decode_(e4m3|int8)|e\b)", start)
    for name in ("e4m3", "int8"):
        assert f"= init_paged_decode_{name}()" in start and f"init_paged_prefill_{name}()" in start
        assert not re.search(rf"=\s*init_paged_prefill_{name}\(\)", start)
    last = start[start.rindex("init_paged_decode_"):start.index("});")]
    assert "cudaGetLastError()" in last and "return" not in last


def test_the_calls_over_codes_say_why_before_they_launch():
    capi = code("capi.cu")
    for call in ("vt_paged_decode_mx", "vt_paged_prefill_mx"):
        text = body(capi, f'extern "C" vt_status {call}(')
        assert text.index("VT_CUDA(g_init_codes_err[pool->format])") < text.index("launch_")
    tiles = body(capi, 'extern "C" vt_status vt_paged_prefill_mx(')
    for name in ("e4m3", "int8"):
        assert tiles.index(f"paged_tiles_error_{name}()") < tiles.index("launch_")
