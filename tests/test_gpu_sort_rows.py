"""The order of entries by table row against numpy's stable sort: whole
numbers, compared exactly."""
import numpy as np
import pytest

import paper_2110_14890_amd as sm
from gpu_common import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def check(ids, n_rows):
    import torch
    rows, order = sm.sort_rows(torch.as_tensor(ids, device="cuda"), n_rows)
    key = np.where((ids < 0) | (ids >= n_rows), n_rows, ids)
    want = np.argsort(key, kind="stable")
    assert rows.dtype == torch.int32 and order.dtype == torch.int64
    assert np.array_equal(order.cpu().numpy(), want)
    assert np.array_equal(rows.cpu().numpy(), ids[want])


# around a wavefront, a tile of either size, and where each tile stops adding
# up the others' counts itself (65,536 entries); one pass to four
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 255, 257, 1023, 1024, 1025, 4097, 65535, 65536, 65537, 200_003, 1_100_000])
@pytest.mark.parametrize("n_rows", [1, 2, 255, 256, 15_000, 400_000, 86_000_000, 2 ** 31 - 1])
def test_lengths_and_tables(n, n_rows):
    rng = np.random.default_rng(n)
    ids = rng.integers(-2, min(n_rows + 2, 2 ** 31 - 1), size=n).astype(np.int32)
    ids[0], ids[-1] = n_rows - 1, -1
    check(ids, n_rows)


@pytest.mark.parametrize("n", [1000, 70_000, 300_000])
def test_few_values(n):
    rng = np.random.default_rng(n)
    check(np.zeros(n, np.int32), 100)                                        # one run
    check(np.full(n, -1, np.int32), 100)                                     # nothing in the table
    check(np.arange(n, dtype=np.int32), n)
    check(np.arange(n, dtype=np.int32)[::-1].copy(), n)
    check(np.where(rng.random(n) < 0.5, 7, rng.integers(0, 400_000, n)).astype(np.int32), 400_000)   # a hub


def test_empty_and_in_a_step():
    import torch
    rows, order = sm.sort_rows(torch.empty(0, dtype=torch.int32, device="cuda"), 5)
    assert rows.numel() == 0 and order.numel() == 0
    rng = np.random.default_rng(3)
    ids = torch.as_tensor(rng.integers(-1, 50, size=(40, 7)), dtype=torch.int32, device="cuda")
    vec = torch.as_tensor(rng.normal(size=(40, 33)), dtype=torch.float32, device="cuda")
    a, b = torch.ones((48, 33), device="cuda"), torch.ones((48, 33), device="cuda")
    one, two = sm.AdamW([a], tables=(0,)), sm.AdamW([b], tables=(0,))
    r, o = torch.sort(ids.view(-1), stable=True)
    one.step([sm.row_grad(ids, vec, per=7)])
    two.step([sm.RowGrad(r, vec, order=o, per=7)])
    assert torch.equal(a, b) and not (a == 1).all()
    one.step([sm.row_grad(ids[:0], vec[:0], per=7)])                         # a batch without entries
    assert torch.equal(a, b) and one.steps == 2
    with pytest.raises(ValueError, match="not in order"):
        one.step([sm.RowGrad(r, vec, order=o, per=7, in_order=False)])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    one.step([sm.row_grad(ids, vec, per=7)], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    two.steps = one.steps - 1            # the step without entries counted
    two.step([sm.row_grad(ids, vec, per=7)])
    assert torch.equal(a, b)


def test_a_captured_step_sorts_its_entries():
    """Unsorted entries in a captured step: each replay sorts what the ids hold
    then; eager steps between use the same sizes."""
    import torch
    rng = np.random.default_rng(4)
    dev = torch.device("cuda")
    ids = torch.zeros((90, 11), dtype=torch.int32, device=dev)
    vec = torch.as_tensor(rng.normal(size=(90, 70)), dtype=torch.float32, device=dev)
    a, b = torch.ones((60, 70), device=dev), torch.ones((60, 70), device=dev)
    kw = dict(tables=(0,), device_step=True, bits=8, seed=1)
    graphed, eager = sm.AdamW([a], **kw), sm.AdamW([b], **kw)
    sm.AdamW([torch.ones((60, 70), device=dev)], **kw).step([sm.row_grad(ids, vec, per=11)])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        graphed.step([sm.row_grad(ids, vec, per=11)])
    for k in range(4):
        ids.copy_(torch.as_tensor(rng.integers(-1, 61, size=(90, 11))))
        graph.replay()
        torch.cuda.synchronize()
        eager.step([sm.row_grad(ids, vec, per=11)])
        assert torch.equal(a, b), k
