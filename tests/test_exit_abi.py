"""The diagnostic of a cluster's exit refuses a missing result before anything is launched (no GPU needed)."""
import ctypes

from paper_2310_08041_b200 import binding as B


def test_a_missing_result_is_refused():
    before = B.qllm_launch_count()
    assert B._lib.qllm_debug_exit_expiry(ctypes.c_void_p(None), None) == B.QLLM_ERR_NULL
    assert B.qllm_launch_count() == before
