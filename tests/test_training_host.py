"""Host-only: calls of the training operators that have nothing to launch."""
import paper_1812_07625_amd as P

N = None


def test_a_step_over_empty_tensors_without_a_workspace():
    """Nothing that asks for a workspace, and no values: allowed, and nothing is launched."""
    for bits in (32, 8):
        for count in (1, 49, 200):
            a = (P.w2l_adamw_tensor * count)()
            for grad in (P.W2L_F32, P.W2L_BF16):
                assert P.raw.w2l_adamw_step(a, count, grad, bits, 1, 1e-3, 0.9, 0.999, 1e-8, 1.0, 0.0, 1, N, N, N, N, 0, N) == 0
