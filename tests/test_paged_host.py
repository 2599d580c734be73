"""Norms, rotary positions and the paged cache at the C boundary, without a GPU: structure layouts, calls without a context, NVTX ranges,
and the frequencies that the binding makes."""
import ctypes
import math

import pytest

import test_segment_attn_host as base
import test_tracing
from test_segment_attn_host import lib  # noqa: F401
from test_tracing import probe  # noqa: F401


@pytest.mark.parametrize("c_name,py_name", [("swam_rope", "SwamRope"), ("swam_norm_rope_args", "SwamNormRopeArgs"), ("swam_paged_cache", "SwamPagedCache"),
                                            ("swam_append_args", "SwamAppendArgs"), ("swam_paged_args", "SwamPagedArgs")])
def test_argument_structures_match_the_header(tmp_path, c_name, py_name):
    base.test_argument_structures_match_the_header(tmp_path, c_name, py_name)


@pytest.mark.parametrize("name,py_name", [("swam_norm_rope", "SwamNormRopeArgs"), ("swam_append_kv", "SwamAppendArgs"), ("swam_paged_attn", "SwamPagedArgs")])
def test_calls_without_a_context_are_refused(lib, name, py_name):  # noqa: F811
    from paper_2609_38984_b200 import swam
    args = getattr(swam, py_name)()
    assert getattr(lib, name)(None, ctypes.byref(args), None) == swam.ERR_INVALID_ARG
    assert getattr(lib, name)(None, None, None) == swam.ERR_INVALID_ARG
    bytes_ = ctypes.c_size_t(7)
    assert lib.swam_paged_attn_scratch_bytes(None, ctypes.byref(swam.SwamPagedArgs()), ctypes.byref(bytes_)) == swam.ERR_INVALID_ARG
    assert bytes_.value == 7


def test_calls_open_and_close_their_range(probe, tmp_path):  # noqa: F811
    lines = test_tracing.traced(probe, tmp_path, """
        import ctypes
        from paper_2609_38984_b200 import swam
        lib = swam.load_library()
        n = ctypes.c_size_t()
        assert lib.swam_norm_rope(None, ctypes.byref(swam.SwamNormRopeArgs()), None) == swam.ERR_INVALID_ARG
        assert lib.swam_append_kv(None, ctypes.byref(swam.SwamAppendArgs()), None) == swam.ERR_INVALID_ARG
        assert lib.swam_paged_attn(None, ctypes.byref(swam.SwamPagedArgs()), None) == swam.ERR_INVALID_ARG
        assert lib.swam_paged_attn_scratch_bytes(None, ctypes.byref(swam.SwamPagedArgs()), ctypes.byref(n)) == swam.ERR_INVALID_ARG
    """)
    assert [n for n, _ in test_tracing.tree(lines)] == ["swam_norm_rope", "swam_append_kv", "swam_paged_attn"]


def test_frequencies():
    from paper_2609_38984_b200 import swam
    plain = swam.rope_frequencies(64)
    assert len(plain) == 32 and plain[0] == 1.0
    assert all(math.isclose(f, 10000.0 ** (-i / 32), rel_tol=1e-15) for i, f in enumerate(plain))
    linear = swam.rope_frequencies(64, factor=8.0)
    assert all(math.isclose(a, b / 8, rel_tol=1e-15) for a, b in zip(linear, plain))
    mixed = swam.rope_frequencies(64, factor=8.0, trained=4096)
    for a, b in zip(mixed, plain):
        turns = 4096 * b / (2 * math.pi)
        if turns >= 32:
            assert a == b
        elif turns <= 1:
            assert math.isclose(a, b / 8, rel_tol=1e-15)
        else:
            assert b / 8 < a < b
    assert any(a == b for a, b in zip(mixed, plain)) and math.isclose(mixed[-1], plain[-1] / 8, rel_tol=1e-15)
    assert swam.rope_magnitude(1.0) == 1.0 and math.isclose(swam.rope_magnitude(8.0), 0.1 * math.log(8.0) + 1.0)
    for bad in (dict(rot_dim=7), dict(rot_dim=0), dict(rot_dim=8, base=0.0), dict(rot_dim=8, factor=0.5), dict(rot_dim=8, trained=-1),
                dict(rot_dim=8, turns_low=3.0, turns_high=3.0)):
        with pytest.raises(ValueError):
            swam.rope_frequencies(**bad)
    for bad in (([],), ([1.0], [0, 1]), ([1.0], [-1]), ([1.0], None, False, 0.0)):
        with pytest.raises(ValueError):
            swam.Rope(*bad)
