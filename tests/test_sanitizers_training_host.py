"""The calls of test_training_host.py and the query of test_policy_variants.py under AddressSanitizer + UndefinedBehaviorSanitizer (CPU only)."""
from test_sanitizers import _run_pytest_under


def test_host_code_of_calls_that_launch_nothing():
    from paper_1812_07625_amd import build as hip_build
    lib = hip_build.build(sanitize=True)
    out = _run_pytest_under(hip_build.asan_runtime(), {"W2L_LIB": lib}, ["test_training_host.py", "test_policy_variants.py"])
    assert "failed" not in out
