"""What a library that was built otherwise still serves (no GPU): read off the source."""
from __future__ import annotations

import re
from pathlib import Path

CSRC = Path(__file__).resolve().parents[1] / "paper_2607_07046_gb300" / "csrc"


def code(name):
    return re.sub(r"//[^\n]*", "", (CSRC / name).read_text())


def body(text, head):
    text = text[text.index(head):]
    return text[:text.index("\n}\n")]


def test_the_paged_kernels_are_set_up_by_their_first_workspace():
    """Setting a kernel up loads it.  A process without a paged cache loads none of its kernels: what they displaced cost
    the fused decode token up to 7%, which never runs them."""
    capi = code("capi.cu")
    assert "paged" not in body(capi, "cudaError_t init_library()")
    assert "VT_CUDA(init_paged())" in body(capi, 'extern "C" vt_status vt_paged_create(')


def test_the_tiles_kernel_alone_depends_on_its_register_count():
    """The kernel's register split needs what it is launched with to be exactly what it was planned for.  A compiler that
    gives it another count must not fail the start of the library, which every call goes through."""
    capi = code("capi.cu")
    start = body(capi, "cudaError_t init_paged()")
    assert "g_init_paged_err = init_paged_decode()" in start and "init_paged_prefill()" in start
    assert not re.search(r"=\s*init_paged_prefill\(\)", start)
    call = body(capi, 'extern "C" vt_status vt_paged_prefill(')
    assert "paged_tiles_error()" in call and call.index("paged_tiles_error()") < call.index("VT_CUDA(")
