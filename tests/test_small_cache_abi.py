"""The calls of 8-bit pages, weights and eviction refuse a missing context before anything else; no GPU is needed."""
import ctypes

from paper_2608_19662_b200 import binding

NEW = ("recache_compact_routes_q8", "recache_attend_decode_q8", "recache_attend_decode_weighted", "recache_evict_rows")


def test_null_context_is_refused():
    lib = binding.load_library()
    for name in NEW:
        args = [t(0) if t in (ctypes.c_int32, ctypes.c_int64) else None for t in binding.SIGNATURES[name][1]]
        assert getattr(lib, name)(*args) == 1, name
    assert lib.recache_decode_q8_workspace_bytes(None, 1) == -1
    assert lib.recache_decode_weighted_workspace_bytes(None, 1, 1) == -1


def test_each_call_has_its_native_entry():
    binding.load_library()
    from paper_2608_19662_b200 import _native
    for name in ("compact_q8", "decode_q8", "decode_weighted", "evict"):
        assert callable(getattr(_native, name))
        try:
            getattr(_native, name)()
        except TypeError as e:
            assert "arguments" in str(e)
