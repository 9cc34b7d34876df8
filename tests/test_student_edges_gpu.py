"""Calls of the student block's operators at their edges: parts that are not there, values that
are not finite, extreme sizes, other streams than the current one."""
import pytest
import torch

from test_norm_gpu import Problem, check_fwd

pytestmark = pytest.mark.gpu

BF16, F32 = torch.bfloat16, torch.float32


@pytest.fixture(scope="module")
def H():
    from paper_2609_18145_gb300 import hcw
    hcw.lib()
    return hcw


@pytest.mark.parametrize("post,pre", [(0, 1), (0, 2), (1, 2), (2, 1), (2, 2), (2, 0)])
def test_without_a_branch_its_gate_and_norm_are_not_read(H, post, pre):
    p = Problem(33, 264, BF16, 7)
    check_fwd(H, p, post, pre, f=False)
    p.gate[0, 5], p.post_w[7], p.post_b[9] = float("nan"), float("inf"), float("nan")
    check_fwd(H, p, post, pre, f=False)
