"""Training calls on a stream of the caller's, the current stream busy with
other work."""
import numpy as np
import pytest

import paper_2110_14890_amd as sm
from gpu_common import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.fixture(scope="module")
def keep_busy():
    """Tens of milliseconds of work on the current stream."""
    import torch
    a = torch.ones((8192, 8192), device="cuda")

    def work():
        for _ in range(5):
            torch.mm(a, a)
    work()
    torch.cuda.synchronize()
    return work


@pytest.mark.parametrize("view", ["columns", "transposed", "expanded"])
def test_entries_that_are_views(keep_busy, view):
    """ids and coefficients that are not contiguous, on a stream that waited
    for them before the RowGrad was made: the step does not depend on what the
    current stream does in the meantime."""
    import torch
    rng = np.random.default_rng(71)
    dev = torch.device("cuda")
    ids = torch.as_tensor(rng.integers(-1, 300, size=(200, 33)), dtype=torch.int32, device=dev)
    coef = torch.as_tensor(rng.normal(size=(200, 33)), dtype=torch.float32, device=dev)
    pick = {"columns": lambda t: t[:, 1:], "transposed": lambda t: t.t(), "expanded": lambda t: t[:1].expand(200, 33)}[view]
    n = pick(ids).numel()
    vec = torch.as_tensor(rng.normal(size=(n // 8, 100)), dtype=torch.float32, device=dev)
    a, b = torch.ones((300, 100), device=dev), torch.ones((300, 100), device=dev)
    kw = dict(bits=8, seed=2, tables=(0,))
    one, two = sm.AdamW([a], **kw), sm.AdamW([b], **kw)
    two.step([sm.row_grad(pick(ids).contiguous(), vec, coef=pick(coef).contiguous(), per=8)])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    keep_busy()
    one.step([sm.row_grad(pick(ids), vec, coef=pick(coef), per=8)], stream=side)
    side.synchronize()
    with torch.cuda.stream(side):
        got = a.cpu()
    torch.cuda.synchronize()
    assert torch.equal(got, b.cpu()) and not (got == 1).all()
