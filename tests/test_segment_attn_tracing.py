"""Cross and shared-prefix attention open their NVTX range like every launching call of the library, also when they fail; asking for
the size of their scratch launches nothing and opens none."""
import test_tracing as base
from test_tracing import probe  # noqa: F401  (the fixture that builds the probe)


def test_segment_attention_calls_open_and_close_their_range(probe, tmp_path):  # noqa: F811
    lines = base.traced(probe, tmp_path, """
        import ctypes
        from paper_2609_38984_b200 import swam
        lib = swam.load_library()
        c, p, n = swam.SwamCrossArgs(), swam.SwamPrefixArgs(), ctypes.c_size_t()
        assert lib.swam_cross_attn(None, ctypes.byref(c), None) == swam.ERR_INVALID_ARG
        assert lib.swam_cross_attn_scratch_bytes(None, ctypes.byref(c), ctypes.byref(n)) == swam.ERR_INVALID_ARG
        assert lib.swam_prefix_attn(None, ctypes.byref(p), None) == swam.ERR_INVALID_ARG
        assert lib.swam_prefix_attn_scratch_bytes(None, ctypes.byref(p), ctypes.byref(n)) == swam.ERR_INVALID_ARG
    """)
    assert [n for n, _ in base.tree(lines)] == ["swam_cross_attn", "swam_prefix_attn"]
    assert all(not kids for _, kids in base.tree(lines))
