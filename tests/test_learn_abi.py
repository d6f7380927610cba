"""CPU-side checks of the part of the library that include/gns_learn.h declares: it is exported and bound, its struct has
the header's layout, and calls without a context are refused.  No GPU work here."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2106_06150_amd", "libgns.so")
HEADER = os.path.join(ROOT, "include", "gns_learn.h")

if not os.path.exists(LIB):
    pytest.skip("libgns.so not built (run __graft_entry__.build())", allow_module_level=True)

from paper_2106_06150_amd import binding as B  # noqa: E402
from paper_2106_06150_amd import learn  # noqa: E402


def header_text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_header_functions_are_exported_and_bound():
    names = sorted(set(re.findall(r"^(?:gns_status|size_t) (gns_\w+)\(", header_text(), flags=re.M)))
    assert names == sorted(learn.EXPORTED) and len(names) == 11
    lib = ctypes.CDLL(LIB)
    for name in names:
        assert hasattr(lib, name), name
        arguments = re.search(r"\b%s\((.*?)\);" % name, header_text(), flags=re.S).group(1)
        assert len(getattr(B.lib, name).argtypes) == arguments.count(",") + 1, name


def test_constants_and_struct_match_the_header():
    text = header_text()
    for name in ("GNS_MAX_TOP", "GNS_INT8_MAX_K", "GNS_STAGE_INT8", "GNS_STAGE_CHECKPOINT", "GNS_STAGE_BACKWARD",
                 "GNS_STAGE_LOG_PROBS"):
        assert getattr(learn, name) == int(re.search(r"#define %s (\d+)" % name, text).group(1)), name
    assert ctypes.sizeof(learn.gns_rows) == 24
    assert [learn.int8_stride(k) for k in (1, 64, 65)] == [64, 64, 128]
    assert [learn.checkpoint_groups(w) for w in (1, 32, 33)] == [1, 1, 2]


def test_calls_without_a_context_are_refused():
    rows = learn.gns_rows(0x1000, 4, 4, 0)
    lib = B.lib
    assert lib.gns_quantize_rows(None, rows, None, 0x1000, 0x1000, 1, None) == B.GNS_EINVAL
    assert lib.gns_dense_int8(None, 0x1000, 0x1000, 4, 0x1000, 0x1000, None, 0, rows, 1, None) == B.GNS_EINVAL
    assert lib.gns_sage_dense_int8(None, rows, None, 0x1000, 0x1000, None, 0, rows, 1, 0x1000, 1 << 20, None) == B.GNS_EINVAL
    assert lib.gns_checkpoint_save(None, rows, 0x1000, 0x1000, None, 1, None) == B.GNS_EINVAL
    assert lib.gns_checkpoint_load(None, 0x1000, 0x1000, rows, 1, None) == B.GNS_EINVAL
    assert lib.gns_sage_dense_backward(None, rows, None, None, None, 4, None, None, 0, None, None, 0x1000, None, 1, 0x1000,
                                       1 << 20, None) == B.GNS_EINVAL
    assert lib.gns_log_probs(None, rows, None, None, 0x1000, None, 0, None, None, 1, None, 0, None) == B.GNS_EINVAL
    assert lib.gns_log_probs_backward(None, rows, None, 0x1000, None, None, None, rows, 1, None) == B.GNS_EINVAL
    assert learn.gns_sage_dense_int8_workspace_bytes(None, 64, 1) == 0
    assert learn.gns_sage_dense_backward_workspace_bytes(None, 64, 0, 64, 1) == 0
    assert learn.gns_log_probs_workspace_bytes(None, 64, 1, 1) == 0
