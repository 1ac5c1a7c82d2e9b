"""What a library that was built otherwise still serves (no GPU): read off the source."""
from __future__ import annotations

import re
from pathlib import Path

CSRC = Path(__file__).resolve().parents[1] / "paper_2607_07046_gb300" / "csrc"


def code(name):
    return re.sub(r"//[^\n]*", "", (CSRC / name).read_text())


def test_the_tiles_kernel_alone_depends_on_its_register_count():
    """The kernel's register split needs what it is launched with to be exactly what it was planned for.  A compiler that
    gives it another count must not fail the start of the library, which every call goes through."""
    capi = code("capi.cu")
    start = capi[capi.index("cudaError_t init_library()"):]
    start = start[:start.index("\n}\n")]
    assert "g_init_err = init_paged_decode()" in start and "init_paged_prefill()" in start
    assert not re.search(r"g_init_err\s*=\s*init_paged_prefill\(\)", start)
    call = capi[capi.index('extern "C" vt_status vt_paged_prefill('):]
    call = call[:call.index("\n}\n")]
    assert "paged_tiles_error()" in call and call.index("paged_tiles_error()") < call.index("VT_CUDA(")
