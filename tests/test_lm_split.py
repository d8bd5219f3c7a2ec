"""The selective scan's workspaces are those of the split that the tests of its pieces assume."""
import random

from lm_split import workspaces
from paper_2012_15198_amd import cxlm as lm


def test_workspaces_follow_the_split():
    rng = random.Random(3)
    sizes = [(1, 1, 1, 1), (1, 16_381, 1_024, 16), (16, 2_048, 1_024, 16), (6, 1_111, 515, 10), (1, 1 << 20, 64, 16), (4_096, 40, 64, 3), (8_192, 64, 64, 3)]
    for _ in range(400):
        sizes.append((1 << rng.randint(0, 11), round(2 ** rng.uniform(0, 15)), round(2 ** rng.uniform(0, 12)), rng.randint(1, 16)))
    for B, T, D, N in sizes:
        assert (lm.cx_select_workspace(B, T, D, N), lm.cx_select_grad_workspace(B, T, D, N)) == workspaces(B, T, D, N), (B, T, D, N)
