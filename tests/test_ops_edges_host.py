"""CPU-only checks of the training operators at their edges."""
import random

from paper_2201_06227_b200 import ops


def test_workspace_never_falls_as_a_size_grows():
    """A handle sized for the largest call takes every smaller one."""
    r = random.Random(5)

    def size(most):
        return int(2 ** r.uniform(0, most))

    for fn, most in ((ops.egeria_linear_workspace_bytes, (17, 14, 14)), (ops.egeria_norm_workspace_bytes, (17, 13))):
        for _ in range(20000):
            big = [size(m) for m in most]
            small = [r.choice((v, max(1, v - 1), r.randint(1, v))) for v in big]
            assert fn(*small) <= fn(*big), (small, big)
    assert ops.egeria_linear_workspace_bytes(13568, 768, 768) <= ops.egeria_linear_workspace_bytes(13824, 768, 768)
    assert ops.egeria_norm_workspace_bytes(9000, 1024) <= ops.egeria_norm_workspace_bytes(9000, 1025)
