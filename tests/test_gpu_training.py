"""Training steps on sampled batches: the sampler's outputs go straight into
scores, the preference loss, its gradients and AdamW, and every step is
compared with the same step in 64 bits from the state before it."""
import numpy as np
import pytest

import kgsynth
import paper_2110_14890_amd as sm
from gpu_common import require_gpu
from test_gpu_adamw import OPT, as64, check_row, check_sums, snapshot
from test_gpu_preference import check as check_loss
from training_common import EPS32, gathered, preference, valid_places

pytestmark = pytest.mark.gpu
V, R, DIM, BATCH, N = 700, 5, 144, 96, 40


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


@pytest.fixture(scope="module")
def graph():
    rng = np.random.default_rng(51)
    # dense enough that some queries are short of negatives
    return sm.Graph(kgsynth.random_tiny(rng, V, R, 60000), V, R, add_inverse=True)


@pytest.mark.parametrize("bits", [32, 8])
def test_steps_on_sampled_batches(graph, bits):
    import torch
    rng = np.random.default_rng(52)
    dev = torch.device("cuda")
    table = torch.as_tensor(rng.normal(size=(V, DIM)) * 0.3, dtype=torch.float32, device=dev)
    dense = torch.as_tensor(rng.normal(size=(DIM, DIM)) * 0.1, dtype=torch.float32, device=dev)
    opt = sm.AdamW([table, dense], **OPT, bits=bits, tables=(0,), seed=7)
    weight = 1.0 / BATCH
    for step in range(1, 4):
        batch = sm.sample(graph, "2p", BATCH, N, seed=9, query_offset=BATCH * step, neg_tries=2 * N)
        counts = batch["n_valid"]
        ids = torch.cat([batch["positive"][:, None], batch["negatives"]], 1)
        anchors = table[batch["anchors"][:, 0].clamp(min=0).long()]
        queries = (anchors @ dense).contiguous()            # the caller's own model, in torch
        before = [snapshot(p, s) for p, s in zip(opt.params, opt.states)]
        scores = sm.score(table, queries, ids)
        coef = torch.empty_like(scores)
        loss = torch.empty(BATCH, device=dev)
        sm.preference_loss_into(scores[:, 0], scores[:, 1:], {"loss": loss, "grad_positive": coef[:, 0], "grad_negatives": coef[:, 1:]},
                                n_valid=counts, kind="pairs", beta=0.5, weight=weight)
        grad_queries = sm.score_grad(table, ids, coef)
        grad_dense = anchors.t().contiguous() @ grad_queries
        opt.step([sm.row_grad(ids, queries, coef=coef, per=N + 1), grad_dense])

        # the same in 64 bits
        t64, q64, i = before[0][0], as64(queries), ids.cpu().numpy()
        n_valid = counts.cpu().numpy()
        assert (n_valid == -1).any() or (n_valid < N).any() or step > 1
        rows = gathered(t64, i)
        s64 = (rows * q64[:, None, :]).sum(-1)
        ds = (DIM + 1) * EPS32 * (np.abs(rows) * np.abs(q64)[:, None, :]).sum(-1)
        assert (np.abs(as64(scores) - s64) <= ds + 2.0 ** -126).all()
        valid = valid_places(BATCH, N, n_valid)
        l64, dpos, dneg, z = preference(s64[:, 0], s64[:, 1:], None, None, valid, "pairs", 0.5, 0.0)
        c64 = np.concatenate([dpos[:, None], dneg], 1) * weight
        # z off by the scores' bounds and its own four roundings; a slope by a quarter of that
        dz = 0.5 * (ds[:, :1] + ds[:, 1:] + 4 * EPS32 * (np.abs(s64[:, :1]) + np.abs(s64[:, 1:])))
        count = np.maximum(valid.sum(1), 1)[:, None]
        dc = np.where(valid, (dz / 4 + 16 * EPS32) / count, 0.0) * 0.5 * weight + 4 * EPS32 * np.abs(c64[:, 1:])
        dc = np.concatenate([dc.sum(1, keepdims=True) + (N + 8) * EPS32 * np.abs(c64[:, 1:]).sum(1, keepdims=True), dc], 1)
        assert (np.abs(as64(loss) - l64) <= np.where(valid, dz, 0.0).sum(1) / count[:, 0] + (N + 24) * EPS32 * l64 + 2.0 ** -126).all()
        assert (np.abs(as64(coef) - c64) <= dc + 2.0 ** -126).all()
        gq = (rows * c64[:, :, None]).sum(1)
        dgq = (np.abs(rows) * (dc + (N + 2) * EPS32 * np.abs(c64))[:, :, None]).sum(1)
        assert (np.abs(as64(grad_queries) - gq) <= dgq + 2.0 ** -126).all()

        # the table, row by row, and the dense operator as one row
        p1, s1 = snapshot(table, opt.states[0])
        sums, off = {}, {}
        for b in range(BATCH):
            for k in range(N + 1):
                r = i[b, k]
                if 0 <= r < V:
                    sums[r] = sums.get(r, 0.0) + c64[b, k] * q64[b]
                    off[r] = off.get(r, 0.0) + (dc[b, k] + 2 * EPS32 * np.abs(c64[b, k])) * np.abs(q64[b])
        assert sums
        for r in range(V):
            pick = lambda d: {k: a[r] for k, a in d.items()}
            if r in sums:
                check_sums(p1[r], pick(s1), before[0][0][r], pick(before[0][1]), sums[r], off[r], "float32", bits, step, r)
            else:
                assert np.array_equal(p1[r], before[0][0][r]) and all(np.array_equal(s1[k][r], before[0][1][k][r]) for k in s1)
        p1, s1 = snapshot(dense, opt.states[1])
        flat = lambda d: {k: a.reshape(-1) for k, a in d.items()}
        check_row(("dense", step), before[1][0].reshape(-1), flat(before[1][1]), p1.reshape(-1), flat(s1),
                  as64(grad_dense).reshape(-1), "float32", bits, step, 1, 0, 7, OPT)


def test_shared_minibatch_and_verified_candidates(graph):
    """Masks as sample_shared and verify write them, with scores of a matrix
    product."""
    import torch
    rng = np.random.default_rng(53)
    dev = torch.device("cuda")
    table = torch.as_tensor(rng.normal(size=(V, DIM)) * 0.3, dtype=torch.float32, device=dev)
    queries = torch.as_tensor(rng.normal(size=(BATCH, DIM)), dtype=torch.float32, device=dev)
    batch = sm.sample_shared(graph, "pi", BATCH, 77, seed=3)
    size = int(batch["n_shared"].item())
    assert size == 77
    negatives = queries @ table[batch["shared"].long()].t().contiguous()
    positive = sm.score(table, queries, batch["positive"][:, None])[:, 0]
    for mask in (batch["mask"], sm.verify(graph, "pi", batch["anchors"], batch["relations"],
                                          batch["shared"].expand(BATCH, 77).contiguous())["mask"]):
        for kind in ("pairs", "softmax"):
            out = sm.preference_loss(positive, negatives, mask=mask, kind=kind, beta=0.5)
            check_loss([positive, negatives, None, None], out, valid_places(BATCH, 77, mask=mask.cpu().numpy()), kind, 0.5, 0.0,
                       np.ones(BATCH), "float32")


def test_a_captured_step(graph):
    """A whole step in a graph, replayed on new batches, against eager steps:
    the operators give equal bits, so the tables are equal."""
    import torch
    rng = np.random.default_rng(54)
    dev = torch.device("cuda")
    start = torch.as_tensor(rng.normal(size=(V, DIM)) * 0.3, dtype=torch.float32, device=dev)
    ids = torch.empty((BATCH, N + 1), dtype=torch.int32, device=dev)
    counts = torch.empty(BATCH, dtype=torch.int32, device=dev)
    queries = torch.empty((BATCH, DIM), device=dev)
    rows, order = torch.empty(ids.numel(), dtype=torch.int32, device=dev), torch.empty(ids.numel(), dtype=torch.int64, device=dev)

    def step(table, opt):
        scores = sm.score(table, queries, ids)
        out = sm.preference_loss(scores[:, 0], scores[:, 1:], n_valid=counts, kind="softmax", beta=0.5, weight=1 / BATCH)
        coef = torch.cat([out["grad_positive"][:, None], out["grad_negatives"]], 1)
        grad = sm.score_grad(table, ids, coef)
        opt.step([sm.RowGrad(rows, queries, order=order, coef=coef.view(-1), per=N + 1)])
        return out["loss"], grad

    def fill(k):
        batch = sm.sample(graph, "ip", BATCH, N, seed=k)
        ids.copy_(torch.cat([batch["positive"][:, None], batch["negatives"]], 1))
        counts.copy_(batch["n_valid"])
        queries.copy_(torch.as_tensor(np.random.default_rng(k).normal(size=(BATCH, DIM))))
        r, o = torch.sort(ids.view(-1), stable=True)
        rows.copy_(r), order.copy_(o)

    fill(0)
    a, b = start.clone(), start.clone()
    kw = dict(OPT, device_step=True, seed=5, bits=8, tables=(0,))
    graphed, eager = sm.AdamW([a], **kw), sm.AdamW([b], **kw)
    step(start.clone(), sm.AdamW([start.clone()], **kw))
    torch.cuda.synchronize()
    captured = torch.cuda.CUDAGraph()
    with torch.cuda.graph(captured):
        got = step(a, graphed)
    for k in range(1, 5):
        fill(k)
        captured.replay()
        torch.cuda.synchronize()
        want = step(b, eager)
        for x, y in zip(got, want):
            assert torch.equal(x, y), k
        assert torch.equal(a, b) and all(torch.equal(graphed.states[0][n].view(torch.uint8), eager.states[0][n].view(torch.uint8))
                                         for n in ("m", "v")), k
