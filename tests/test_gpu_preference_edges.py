"""The preference loss of scores at the ends of their types."""
import numpy as np
import pytest

import paper_2110_14890_amd as sm
from gpu_common import require_gpu
from training_common import EPS32, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.mark.parametrize("n", [1, 5, 300, 3000, 9000])
@pytest.mark.parametrize("beta", [0.5, 1.0])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("kind", ["pairs", "softmax"])
def test_a_positive_at_the_lowest_value(kind, dtype, beta, n):
    """A positive masked with its type's lowest value against ordinary
    negatives: every -z is beta times that value within an ulp of it, so the
    softmax is even over the negatives and the paired slopes are 1 / n each.

    The differences take one rounding, the product with beta one, the
    logarithm of n and the sum one each, the n terms of a sum n: the shares and
    the loss are off by n + 8 half steps (and the exponents not at all: the
    differences of fp32 scores beside the lowest value are equal; of fp16 the
    negatives here are equal too)."""
    import torch
    dev = torch.device("cuda")
    t = getattr(torch, dtype)
    low = torch.finfo(t).min
    neg = torch.ones((3, n), dtype=t, device=dev)
    if dtype != "float16":
        neg.copy_(torch.as_tensor(np.random.default_rng(81).normal(size=(3, n))))
    pos = torch.tensor([low, 1.0, low], dtype=t, device=dev)
    counts = torch.tensor([n, n, (n + 1) // 2], dtype=torch.int32, device=dev)
    out = sm.preference_loss(pos, neg, n_valid=counts, kind=kind, beta=beta)
    assert all(torch.isfinite(x[1]).all() for x in out.values())
    for row, c in ((0, n), (2, (n + 1) // 2)):
        each = beta / c
        want = np.where(np.arange(n) < c, each, 0.0)
        got = out["grad_negatives"][row].double().cpu().numpy()
        assert (np.abs(got - want) <= (n + 8) * EPS32 * want + rounding(want, dtype)).all()
        gone = out["grad_positive"][row].item()
        assert abs(gone + beta) <= (2 * n + 16) * EPS32 * beta + rounding(np.float64(beta), dtype)
        size = beta * (-low + (1.0 if dtype == "float16" else 0.0))
        loss = out["loss"][row].item()
        if kind == "softmax":
            size += np.log(c) if dtype == "float16" else 0.0
            assert abs(loss - size) <= (n + 8) * EPS32 * size
        elif dtype == "float16":
            assert abs(loss - size) <= (n + 8) * EPS32 * size
        else:      # a sum of more than one such loss is no fp32 number
            assert loss == np.inf if size * c > 3.5e38 else abs(loss - size) <= (n + 8) * EPS32 * size


@pytest.mark.parametrize("kind", ["pairs", "softmax"])
def test_negatives_far_above(kind):
    """The largest of the negatives beyond 2^127 / log2(e), others far below."""
    import torch
    dev = torch.device("cuda")
    neg = torch.tensor([[3.0e38, 1.0e38, 3.0e38, 0.0]], device=dev)
    out = sm.preference_loss(torch.zeros(1, device=dev), neg, kind=kind, beta=1.0)
    want = [[0.5, 0.0, 0.5, 0.0]] if kind == "softmax" else [[0.25, 0.25, 0.25, 0.125]]
    assert np.allclose(out["grad_negatives"].cpu().numpy(), want, rtol=8 * EPS32, atol=0.0)
    if kind == "softmax":
        assert abs(out["loss"].item() - 3.0e38) <= 8 * EPS32 * 3.0e38
