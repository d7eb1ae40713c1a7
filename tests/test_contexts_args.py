"""What the calls on pages, summaries, shared and sparse contexts refuse before they look at any device."""
import ctypes

import pytest

import paper_2505_00232_b200 as P
from paper_2505_00232_b200 import binding

lib, BAD = binding.lib, P.QL_ERR_INVALID_ARG
BUFFER = ctypes.create_string_buffer(4096)
AT = (ctypes.addressof(BUFFER) + 255) & ~255                              # 256-byte aligned; never read: every call below is refused
BATCH = (AT, 4, 4, AT, AT, 1, 1)


def test_no_handle():
    assert lib.qlinear_paged_pages_workspace(None) == 0
    assert lib.qlinear_paged_attention_selected_workspace(None, 8) == 0
    assert lib.qlinear_paged_attention_shared_workspace(None, 8, 1, 1, 1, 1, 1) == 0
    assert lib.qlinear_paged_fork(None, AT, AT, 4, 4, 1, AT, AT, 1, AT + 1024, 4, None) == BAD
    assert lib.qlinear_paged_release(None, AT, AT, 4, 4, 1, AT, AT, 1, None) == BAD
    assert lib.qlinear_paged_reserve(None, AT, *BATCH, AT, AT, 4096, None) == BAD
    assert lib.qlinear_paged_compact(None, AT, AT, 4, 4, 1, None, None, AT, AT, 4096, None) == BAD
    assert lib.qlinear_paged_summarise(None, *BATCH, AT, AT, None) == BAD
    assert lib.qlinear_paged_select(None, AT, 64, 1, AT, AT, *BATCH, 4, 1, 1, AT, None) == BAD
    assert lib.qlinear_paged_attention_selected(None, AT, 64, AT + 1024, 64, 1, AT, 4, *BATCH, 1.0, 0.0, AT, 4096, None) == BAD
    assert lib.qlinear_paged_attention_shared(None, AT, 64, AT + 1024, 64, 1, *BATCH, 1, AT, AT, 1, 1.0, 0.0, AT, 4096, None) == BAD


@pytest.mark.parametrize("name", ["fork", "release", "reserve", "compact", "key_bounds", "summarise", "select", "attention_selected", "attention_shared"])
def test_the_binding_documents_its_calls(name):
    assert getattr(P.PagedKV, name).__doc__
