"""CPU-side checks of the part of the library that include/gns_layers.h declares: it is exported and bound, its structs have the
header's layout, and calls without a context are refused.  No GPU work here."""
import ctypes
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
LIB = os.path.join(ROOT, "paper_2106_06150_amd", "libgns.so")
HEADER = os.path.join(ROOT, "include", "gns_layers.h")

if not os.path.exists(LIB):
    pytest.skip("libgns.so not built (run __graft_entry__.build())", allow_module_level=True)

from paper_2106_06150_amd import binding as B  # noqa: E402
from paper_2106_06150_amd import layers, learn  # noqa: E402


def header_text():
    return re.sub(r"/\*.*?\*/", "", open(HEADER).read(), flags=re.S)


def test_header_functions_are_exported_and_bound():
    names = sorted(set(re.findall(r"^(?:gns_status|size_t) (gns_\w+)\(", header_text(), flags=re.M)))
    assert names == sorted(layers.EXPORTED) and len(names) == 10
    lib = ctypes.CDLL(LIB)
    for name in names:
        assert hasattr(lib, name), name
        arguments = re.search(r"\b%s\((.*?)\);" % name, header_text(), flags=re.S).group(1)
        assert len(getattr(B.lib, name).argtypes) == arguments.count(",") + 1, name


def test_constants_and_structs_match_the_header():
    text = header_text()
    for name in ("GNS_ACT_NONE", "GNS_ACT_RELU", "GNS_ACT_SILU", "GNS_ACT_GELU", "GNS_ORTHOGONAL_MAX", "GNS_MAX_STEPS", "GNS_FP8_BLOCK",
                 "GNS_STAGE_NORM", "GNS_STAGE_ORTHOGONAL", "GNS_STAGE_FP8"):
        assert getattr(layers, name) == int(re.search(r"#define %s (\d+)" % name, text).group(1)), name
    for name in ("GNS_MAX_SEGMENTS", "GNS_FP8_MAX_K"):
        assert getattr(layers, name) == 1 << int(re.search(r"#define %s \(1 << (\d+)\)" % name, text).group(1)), name
    assert ctypes.sizeof(layers.gns_norm) == 48
    assert ctypes.sizeof(layers.gns_orthogonal) == 24 + 12 * layers.GNS_MAX_STEPS
    assert [layers.fp8_stride(k) for k in (1, 128, 129)] == [128, 128, 256]
    assert [layers.fp8_exponents(k) for k in (1, 512, 513)] == [4, 4, 8]


def test_calls_without_a_context_are_refused():
    rows = learn.gns_rows(0x1000, 4, 4, 0)
    norm = layers.gns_norm(None, None, None, 0, 1, 2, 0, 1e-5)
    how = layers.gns_orthogonal(0.9, 1, 1e-7, 1.0, -0.1, 0)
    lib = B.lib
    assert lib.gns_group_norm(None, rows, norm, rows, None, 1, None, 0, None) == B.GNS_EINVAL
    assert lib.gns_group_norm_backward(None, rows, rows, norm, 0x1000, rows, None, None, 1, None, 0, None) == B.GNS_EINVAL
    assert lib.gns_orthogonal_update(None, rows, None, how, None, None, rows, 1, 0x1000, 1 << 20, None) == B.GNS_EINVAL
    assert lib.gns_quantize_fp8(None, rows, None, 0x1000, 0x1000, 1, None) == B.GNS_EINVAL
    assert lib.gns_dense_fp8(None, 0x1000, 0x1000, 4, 0x1000, 0x1000, None, 0, rows, 1, None) == B.GNS_EINVAL
    assert lib.gns_sage_dense_fp8(None, rows, None, 0x1000, 0x1000, None, 0, rows, 1, 0x1000, 1 << 20, None) == B.GNS_EINVAL
    assert lib.gns_group_norm_workspace_bytes(None, 4, norm, 1) == 0
    assert lib.gns_group_norm_backward_workspace_bytes(None, 4, norm, 1) == 0
    assert lib.gns_orthogonal_update_workspace_bytes(None, 4, 4) == 0
    assert lib.gns_sage_dense_fp8_workspace_bytes(None, 64, 1) == 0


def test_a_norm_counts_its_segments():
    assert layers.Norm(1, segment_rows=3).segment_count(7) == 3
    assert layers.Norm(1, segment_rows=3).segment_count(0) == 0
    how = layers.Orthogonal([(1, 2, 3), (4, 5, 6)], mu=0.5)
    assert how.struct.steps == 2 and list(how.struct.coefficients[1]) == [4, 5, 6]
