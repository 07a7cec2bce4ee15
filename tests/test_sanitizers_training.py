"""The host side of the group norm's, the policy loss's and AdamW's entry points -- argument checks, the comparison of all operands' addresses, launch arithmetic -- under
AddressSanitizer + UndefinedBehaviorSanitizer (CPU only), as the other entry points' is."""
from test_sanitizers import _run_pytest_under


def test_host_code_of_the_training_operators():
    from paper_1812_07625_amd import build as hip_build
    lib = hip_build.build(sanitize=True)
    out = _run_pytest_under(hip_build.asan_runtime(), {"W2L_LIB": lib}, ["test_training_abi.py", "test_norm_variants.py"])
    assert "failed" not in out
