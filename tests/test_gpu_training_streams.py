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


def score(x, stream):
    return [sm.score(x["table"], x["queries"], x["ids"], stream=stream)]


def score_grad(x, stream):
    return [sm.score_grad(x["table"], x["ids"], x["coef"], stream=stream)]


def loss(x, stream):
    return list(sm.preference_loss(x["pos"], x["neg"], x["ref_pos"], x["ref_neg"], n_valid=x["count"], weight=x["weight"],
                                   stream=stream).values())


def masked_loss(x, stream):
    return list(sm.preference_loss(x["pos"], x["neg"], mask=x["mask"], kind="softmax", stream=stream).values())


def sort(x, stream):
    return list(sm.sort_rows(x["ids"].view(-1), 400, stream=stream))


def step(x, stream):
    """The optimizer and its moments go as well, but for the parameters."""
    import torch
    opt = sm.AdamW([x["param"], x["table"]], lr=x["rate"], bits=8, seed=3, tables=(1,))
    if stream is not None:
        stream.wait_stream(torch.cuda.current_stream())        # for the zero moments
    opt.step([x["grad"], sm.row_grad(x["ids"], x["queries"], coef=x["coef"], per=41)], grad_scale=x["scale"], stream=stream)
    return [x["param"], x["table"]]


@pytest.mark.parametrize("call", [score, score_grad, loss, masked_loss, sort, step], ids=lambda c: c.__name__)
def test_what_a_call_reads_is_kept_for_its_stream(keep_busy, call):
    """Inputs that the caller lets go of right after a call on a busy stream:
    tensors made meanwhile get other memory."""
    import torch
    rng = np.random.default_rng(72)
    dev = torch.device("cuda")
    new = lambda *s: torch.as_tensor(rng.normal(size=s), dtype=torch.float32, device=dev)
    whole = lambda lo, hi, *s: torch.as_tensor(rng.integers(lo, hi, size=s), dtype=torch.int32, device=dev)
    x = dict(table=new(400, 72), queries=new(50, 72), coef=new(50, 41), ids=whole(-1, 400, 50, 41), count=whole(-1, 41, 50),
             mask=whole(-2 ** 31, 2 ** 31, 50, 2), pos=new(50), neg=new(50, 40), ref_pos=new(50), ref_neg=new(50, 40),
             weight=new(50), scale=torch.full((1,), 0.5, device=dev), rate=torch.full((1,), 1e-3, device=dev), param=new(3000),
             grad=new(3000))
    copy = lambda: {k: t.clone() for k, t in x.items()}
    want = [t.cpu() for t in call(copy(), None)]
    side = torch.cuda.Stream()
    passing = copy()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        keep_busy()
    got = call(passing, side)
    passing.clear()
    junk = [torch.full_like(t, 7) for t in x.values() for _ in range(3)]
    junk += [torch.full((n,), 7, dtype=torch.uint8, device=dev) for n in (3000, 28800, 96, 1600) for _ in range(4)]
    torch.cuda.synchronize()
    assert all(torch.equal(a.cpu(), b) for a, b in zip(got, want)) and len(junk)


def test_capture_on_a_given_stream():
    """Calls that name the stream which a graph is captured on, replayed on
    new inputs with eager calls between."""
    import torch
    rng = np.random.default_rng(73)
    dev = torch.device("cuda")
    side = torch.cuda.Stream()
    table = torch.as_tensor(rng.normal(size=(90, 40)), dtype=torch.float32, device=dev)
    ids, queries = torch.zeros((6, 2001), dtype=torch.int32, device=dev), torch.zeros((6, 40), device=dev)
    a, b = table.clone(), table.clone()
    kw = dict(bits=8, seed=4, tables=(0,), device_step=True)
    graphed, eager = sm.AdamW([a], **kw), sm.AdamW([b], **kw)

    def run(table, opt, stream=None):
        scores = sm.score(table, queries, ids, stream=stream)
        out = sm.preference_loss(scores[:, 0], scores[:, 1:], kind="softmax", stream=stream)
        grad = sm.score_grad(table, ids[:, 1:], out["grad_negatives"], stream=stream)
        opt.step([sm.row_grad(ids[:, 1:], queries, coef=out["grad_negatives"], per=2000)], stream=stream)
        return [scores, out["loss"], grad]

    run(table.clone(), sm.AdamW([table.clone()], **kw))
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        got = run(a, graphed, side)
    for k in range(4):
        ids.copy_(torch.as_tensor(rng.integers(-1, 91, size=(6, 2001))))
        queries.copy_(torch.as_tensor(rng.normal(size=(6, 40))))
        graph.replay()
        torch.cuda.synchronize()
        want = run(b, eager)
        assert all(torch.equal(x, y) for x, y in zip(got, want)) and torch.equal(a, b), k


def test_states_that_hold_more_than_moments():
    """A checkpoint's state may carry other entries; a step on a given stream
    looks at the moments alone, as one on the current stream does."""
    import torch
    p = torch.ones(300, device="cuda")
    opt = sm.AdamW([p], lr=0.5, bits=8)
    opt.states[0]["step"] = 7
    opt.states[0]["note"] = None
    g = torch.ones(300, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    opt.step([g], stream=side)
    torch.cuda.current_stream().wait_stream(side)
    opt.step([torch.ones(300, device="cuda")])
    assert opt.steps == 2 and (p < 0.1).all()
