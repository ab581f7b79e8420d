"""Candidate scores and their gradient against 64-bit sums.

A sum of d products in fp32, in any order, is off by at most (d + 1) half
steps of the sum of the products' magnitudes; a result stored in bf16 is
rounded once more."""
import numpy as np
import pytest

import paper_2110_14890_amd as sm
from gpu_common import require_gpu
from training_common import EPS32, gathered, rounding

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def make(rng, rows, dim, batch, n, table, query):
    import torch
    t = torch.as_tensor(rng.normal(size=(rows, dim)), dtype=getattr(torch, table))
    q = torch.as_tensor(rng.normal(size=(batch, dim)), dtype=getattr(torch, query))
    ids = rng.integers(-1, rows + 1, size=(batch, n)).astype(np.int32)   # rows: one past the last entity
    return t, q, ids


def check_score(t, q, ids, got):
    x = gathered(t.double().numpy(), ids)
    qd = q.double().numpy()[:, None, :]
    want, size = (x * qd).sum(-1), np.abs(x * qd).sum(-1)
    assert (np.abs(got.double().cpu().numpy() - want) <= (t.shape[1] + 1) * EPS32 * size + 2.0 ** -126).all()


def check_grad(t, ids, g, got, dtype):
    x = gathered(t.double().numpy(), ids)
    inside = (ids >= 0) & (ids < t.shape[0])
    gd = np.where(inside, g, 0.0)[:, :, None]
    want, size = (x * gd).sum(1), np.abs(x * gd).sum(1)
    bound = (ids.shape[1] + 1) * EPS32 * size + rounding(want, dtype)
    assert (np.abs(got.double().cpu().numpy() - want) <= bound).all()


TYPES = [("float32", "float32"), ("bfloat16", "float32"), ("float32", "bfloat16"), ("bfloat16", "bfloat16")]


@pytest.mark.parametrize("table,query", TYPES)
@pytest.mark.parametrize("dim", [1, 2, 3, 7, 8, 9, 31, 64, 65, 100, 127, 129, 256, 257, 400, 513, 1025, 2051])
def test_score_and_gradient_over_widths(dim, table, query):
    import torch
    rng = np.random.default_rng(dim)
    t, q, ids = make(rng, 37, dim, 5, 19, table, query)
    g = rng.normal(size=ids.shape).astype(np.float32)
    g[ids < 0] = np.nan                       # gradients of padding are not used
    dev = torch.device("cuda")
    td, idd = t.to(dev), torch.as_tensor(ids, device=dev)
    check_score(t, q, ids, sm.score(td, q.to(dev), idd))
    check_grad(t, ids, g, sm.score_grad(td, idd, torch.as_tensor(g, device=dev), dtype=getattr(torch, query)), query)


@pytest.mark.parametrize("batch,n", [(1, 1), (1, 4097), (3, 63), (3, 64), (3, 65), (2, 129), (700, 3), (4100, 9), (33, 1000)])
def test_score_and_gradient_over_lengths(batch, n):
    import torch
    rng = np.random.default_rng(n)
    t, q, ids = make(rng, 500, 24, batch, n, "bfloat16", "float32")
    if batch > 2:
        ids[1] = -1                           # a query without candidates
    g = rng.normal(size=ids.shape).astype(np.float32)
    dev = torch.device("cuda")
    td, idd = t.to(dev), torch.as_tensor(ids, device=dev)
    got = sm.score(td, q.to(dev), idd)
    check_score(t, q, ids, got)
    grad = sm.score_grad(td, idd, torch.as_tensor(g, device=dev))
    check_grad(t, ids, g, grad, "float32")
    if batch > 2:
        assert not got[1].any() and not grad[1].any()
    # the same call gives the same bits
    assert torch.equal(got, sm.score(td, q.to(dev), idd))
    assert torch.equal(grad, sm.score_grad(td, idd, torch.as_tensor(g, device=dev)))


def test_strided_views_and_neighbours_stay():
    """Tables, queries, candidates and outputs that are columns of wider
    matrices, at odd offsets; what lies beside the outputs is kept."""
    import torch
    rng = np.random.default_rng(3)
    dev = torch.device("cuda")
    wide_t = torch.as_tensor(rng.normal(size=(50, 75)), dtype=torch.bfloat16, device=dev)
    wide_q = torch.as_tensor(rng.normal(size=(9, 90)), dtype=torch.float32, device=dev)
    wide_i = torch.as_tensor(rng.integers(-1, 50, size=(9, 40)), dtype=torch.int32, device=dev)
    t, q, ids = wide_t[:, 3:74], wide_q[:, 1:72], wide_i[:, 5:38]
    out = torch.full((9, 40), 7.0, device=dev)
    sm.score_into(t, q, ids, out[:, 2:35])
    check_score(t.cpu(), q.cpu(), ids.cpu().numpy(), out[:, 2:35])
    assert (out[:, :2] == 7).all() and (out[:, 35:] == 7).all()
    g = torch.as_tensor(rng.normal(size=(9, 41)), dtype=torch.float32, device=dev)[:, 3:36]
    dq = torch.full((9, 90), 7.0, device=dev)
    sm.score_grad_into(t, ids, g, dq[:, 1:72])
    check_grad(t.cpu(), ids.cpu().numpy(), g.cpu().numpy(), dq[:, 1:72], "float32")
    assert (dq[:, :1] == 7).all() and (dq[:, 72:] == 7).all()


def test_shared_candidates_and_empty_sets():
    import torch
    rng = np.random.default_rng(4)
    dev = torch.device("cuda")
    t, q, ids = make(rng, 60, 40, 12, 33, "float32", "float32")
    one = torch.as_tensor(ids[:1], device=dev).expand(12, 33)
    check_score(t, q, np.repeat(ids[:1], 12, 0), sm.score(t.to(dev), q.to(dev), one))
    none = torch.empty((12, 0), dtype=torch.int32, device=dev)
    assert sm.score(t.to(dev), q.to(dev), none).shape == (12, 0)
    assert not sm.score_grad(t.to(dev), none, torch.empty((12, 0), device=dev)).any()


def test_rows_far_into_a_large_table():
    """Byte offsets beyond 2^32."""
    import torch
    dev = torch.device("cuda")
    rows, dim = 3_000_000, 800                # 4.8 GB of bf16
    t = torch.zeros((rows, dim), dtype=torch.bfloat16, device=dev)
    ids = torch.tensor([[rows - 1, 0, 2_700_000, rows]], dtype=torch.int32, device=dev)
    t[rows - 1], t[2_700_000] = 1.0, 2.0
    got = sm.score(t, torch.ones((1, dim), device=dev), ids)
    assert got.tolist() == [[800.0, 0.0, 1600.0, 0.0]]
    dq = sm.score_grad(t, ids, torch.ones((1, 4), device=dev))
    assert (dq == 3.0).all()


def test_on_another_stream():
    import torch
    rng = np.random.default_rng(5)
    dev = torch.device("cuda")
    t, q, ids = make(rng, 60, 40, 12, 33, "float32", "float32")
    td, qd, idd = t.to(dev), q.to(dev), torch.as_tensor(ids, device=dev)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = sm.score(td, qd, idd, stream=side)
    grad = sm.score_grad(td, idd, got, stream=side)
    side.synchronize()
    check_score(t, q, ids, got)
    check_grad(t, ids, got.cpu().numpy().astype(np.float64), grad, "float32")


def test_gradient_is_the_slope_of_the_scores():
    """Against differences: scores are linear in the queries, so a difference
    quotient with step 1 is the gradient up to the sums' own rounding."""
    import torch
    rng = np.random.default_rng(6)
    dev = torch.device("cuda")
    t, q, ids = make(rng, 30, 5, 4, 7, "float32", "float32")
    td, idd = t.to(dev), torch.as_tensor(ids, device=dev)
    w = torch.as_tensor(rng.normal(size=(4, 7)), dtype=torch.float32, device=dev)
    grad = sm.score_grad(td, idd, w)
    for c in range(5):
        unit = torch.zeros((4, 5), device=dev)
        unit[:, c] = 1.0
        rise = (sm.score(td, unit, idd).double() * w.double()).sum(1)      # exact products of one column
        size = (sm.score(td.abs(), unit, idd).double() * w.double().abs()).sum(1)
        assert ((grad[:, c].double() - rise).abs() <= 8 * EPS32 * size).all()


def test_capture_and_replay():
    """A captured call whose queries are split over workgroups (its workspace
    lies in the graph's memory), replayed on new inputs with other calls of
    that kind between."""
    import torch
    rng = np.random.default_rng(7)
    dev = torch.device("cuda")
    t, q, ids = make(rng, 300, 72, 3, 2000, "float32", "float32")
    td, idd = t.to(dev), torch.as_tensor(ids, device=dev)
    g = torch.zeros((3, 2000), device=dev)
    sm.score_grad(td, idd, g)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = sm.score_grad(td, idd, g)
    for _ in range(4):
        g.copy_(torch.as_tensor(rng.normal(size=(3, 2000))))
        idd.copy_(torch.as_tensor(rng.integers(-1, 301, size=(3, 2000))))
        graph.replay()
        other = sm.score_grad(td, idd.flip(1).contiguous(), g)
        torch.cuda.synchronize()
        assert torch.equal(out, sm.score_grad(td, idd, g)) and not torch.equal(out, other)


def test_calls_side_by_side_on_streams():
    """Split calls that overlap do not share scratch memory."""
    import torch
    rng = np.random.default_rng(8)
    dev = torch.device("cuda")
    t, _, _ = make(rng, 3000, 400, 1, 1, "bfloat16", "float32")
    td = t.to(dev)
    ids = [torch.as_tensor(rng.integers(-1, 3000, size=(4, 4000)), dtype=torch.int32, device=dev) for _ in range(4)]
    g = [torch.as_tensor(rng.normal(size=(4, 4000)), dtype=torch.float32, device=dev) for _ in range(4)]
    want = [sm.score_grad(td, i, x) for i, x in zip(ids, g)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(4)]
    for _ in range(5):
        got = [sm.score_grad(td, i, x, stream=s) for i, x, s in zip(ids, g, streams)]
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
