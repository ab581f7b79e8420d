"""Table rows with several entries, moments in 8 bits: the codes and scales of
a row do not depend on how many entries its gradient is the sum of.

Gradients are whole multiples of 2^-22 below 2^24 of them, and so are their
parts, so that every product (the coefficients are powers of two) and every sum
is exact: a row's gradient is one known fp32 number however it is added up, and
the checks are those of a dense tensor."""
import numpy as np
import pytest

import paper_2110_14890_amd as sm
from gpu_common import require_gpu
from test_gpu_adamw import OPT, as64, check_row, snapshot, start_state
from training_common import decode

pytestmark = pytest.mark.gpu
UNIT = 2.0 ** -22


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def parts_of(rng, total, count):
    """Whole numbers [count, dim] whose sum is total."""
    each = rng.integers(-(1 << 16), 1 << 16, size=(count, len(total)))
    each[-1] += total - each.sum(0)
    return each


# widths whose rows one lane, a few lanes, a block of lanes and several blocks
# hold, with lanes that hold no column beside them
WIDTHS = [1, 3, 8, 24, 40, 63, 64, 65, 100, 128, 130, 256, 300, 513]
# entries of a row: those that a wavefront's look shows, more than those, and
# stretches of 128 whose sums are made ahead
COUNTS = [1, 2, 4, 5, 20, 63, 64, 65, 128, 300, 700]


@pytest.mark.parametrize("param", ["float32", "bfloat16"])
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dim", WIDTHS)
def test_entries_add_up_to_one(dim, bits, param):
    """Gradients that oppose the moments, so that a block's largest moment is
    far below its gradient's share: each row against the formula in 64 bits,
    and all bits against the same gradients given as one entry a row."""
    import torch
    rng = np.random.default_rng(dim)
    dev = torch.device("cuda")
    rows = 3 * len(COUNTS)
    counts = np.tile(COUNTS, 3)[rng.permutation(rows)]
    p = torch.as_tensor(rng.normal(size=(rows, dim)) * 0.05, dtype=getattr(torch, param), device=dev)
    state = start_state(rng, p, bits, True)
    before = snapshot(p, state)
    m = before[1]["m"]
    if bits == 8:
        m = np.stack([decode(m[r], before[1]["m_scale"][r]) for r in range(rows)])
    # 0.1 g against 0.9 m: from half of it to a little more than all
    want = np.rint(-9.0 * m * rng.uniform(0.5, 1.05, size=m.shape) / UNIT).astype(np.int64)
    ids, vectors, coef = [], [], []
    for r in range(rows):
        scale = 2.0 ** rng.integers(-2, 3, size=counts[r]).astype(float)
        ids += [r] * counts[r]
        coef += list(scale)
        vectors.append(parts_of(rng, want[r], counts[r]) * UNIT / scale[:, None])
    vectors, order = np.concatenate(vectors), rng.permutation(len(ids))
    as_gpu = lambda a, t: torch.as_tensor(np.ascontiguousarray(a), dtype=t, device=dev)
    grads = as_gpu(vectors[order], torch.float32)
    single = p.clone()
    single_state = {k: t.clone() for k, t in state.items()}
    kw = dict(OPT, bits=bits, seed=31, steps=10)
    opt, one = sm.AdamW([p], states=[state], **kw), sm.AdamW([single], states=[single_state], **kw)
    opt.step([sm.row_grad(as_gpu(np.array(ids)[order], torch.int32), grads, coef=as_gpu(np.array(coef)[order], torch.float32))])
    total = as_gpu(want * UNIT, torch.float32)
    assert np.array_equal(as64(grads), vectors[order]) and np.array_equal(as64(total), want * UNIT)     # nothing was rounded
    one.step([sm.row_grad(torch.arange(rows, dtype=torch.int32, device=dev), total)])
    after = snapshot(p, state)
    for r in range(rows):
        row = lambda d: {k: a[r] for k, a in d.items()}
        check_row((dim, counts[r]), before[0][r], row(before[1]), after[0][r], row(after[1]), want[r] * UNIT, param, bits, 11, 0,
                  r, 31, OPT)
    alone = snapshot(single, single_state)
    assert np.array_equal(after[0], alone[0])
    for k in state:
        assert np.array_equal(after[1][k], alone[1][k]), (k, counts[(after[1][k] != alone[1][k]).any(1)])


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dim,rows", [(24, 30_000), (200, 9_000), (400, 5_000)])
def test_many_entries_add_up_to_one(dim, rows, bits):
    """The same with more than 131,072 entries, of which a wavefront looks at
    16 at a time: rows of one to 40 entries and a few of thousands, all bits
    against the gradients given as one entry a row."""
    import torch
    rng = np.random.default_rng(dim)
    dev = torch.device("cuda")
    counts = rng.integers(1, 1 + 2 * 140_000 // rows, size=rows)
    counts[rng.integers(0, rows, size=5)] = (1000, 128, 4096, 2500, 777)
    ids = np.repeat(np.arange(rows), counts)
    assert len(ids) > 131_072
    # sums of at most 4,096 whole numbers of 12 bits
    parts = torch.as_tensor(rng.integers(-2048, 2048, size=(len(ids), dim)), dtype=torch.float32, device=dev)
    order = torch.as_tensor(rng.permutation(len(ids)), device=dev)
    ids = torch.as_tensor(ids, device=dev)
    total = torch.zeros((rows, dim), dtype=torch.float64, device=dev).index_add_(0, ids, parts.double())
    p = torch.as_tensor(rng.normal(size=(rows, dim)) * 0.05, dtype=torch.bfloat16, device=dev)
    q = p.clone()
    kw = dict(OPT, bits=bits, seed=31, tables=(0,))
    many, one = sm.AdamW([p], **kw), sm.AdamW([q], **kw)
    for _ in range(2):
        many.step([sm.row_grad(ids[order].int(), parts[order] * UNIT)])
        one.step([sm.row_grad(torch.arange(rows, dtype=torch.int32, device=dev), (total * UNIT).float())])
        assert torch.equal(p, q)
        for k in many.states[0]:
            a, b = [o.states[0][k].view(torch.uint8) for o in (many, one)]
            assert torch.equal(a, b), k
