"""Derivatives of the layer's functions that there are none of."""
import pytest
import torch

import workloads
from tests.gpu_util import require_gpu

pytestmark = pytest.mark.gpu
F32 = torch.float32


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def test_no_second_derivative_of_the_head_norms():
    """The gradients' kernel has none: asking for it is an error, not a missing term."""
    from paper_2307_02486_amd.layer import QKNormXPosFunction
    q, k = (workloads.make_random((1, 9, h, 32), F32, 1.0, 8, "cuda", t).requires_grad_() for t, h in enumerate((4, 2)))
    w = torch.ones(32, device="cuda", requires_grad=True)
    qo, ko = QKNormXPosFunction.apply(q, k, w, w, 1e-6, 4, 10000.0, 0.4, 512.0)
    first, = torch.autograd.grad((qo * qo).sum() + ko.sum(), q, create_graph=True)
    (plain,) = torch.autograd.grad((qo * qo).sum() + ko.sum(), q, retain_graph=True)
    assert torch.equal(first.detach(), plain) and not plain.requires_grad
    for x in (q, k, w):
        with pytest.raises(RuntimeError, match="cannot be differentiated"):
            torch.autograd.grad(first.sum() + (x * x).sum(), x, retain_graph=True)
