"""AdamW over dense tensors and table rows, moments in 32 and in 8 bits,
against the formula in 64 bits.

In 32 bits the bounds are those of training_common.adamw_bounds.  An 8-bit
code is the exact rounding of the moment in 64 bits unless the moment lies
within fp32's error of the border where the rounding changes: a moment
relative to its block's largest is off by at most 24 half steps of fp32 (its
own 6, the largest's 6, the scale's, a square root and two products), which
is 16 times as much of a code's step (a step is at least 1 / 16 of a value),
so codes may differ where the border is within 24 x 16 x EPS32 = 2^-15.4."""
import numpy as np
import pytest

import paper_2110_14890_amd as sm
from gpu_common import require_gpu
from training_common import (BLOCK, EPS32, adamw, adamw_bounds, code_values, decode, draws, encode, rounding)

pytestmark = pytest.mark.gpu
NEAR = 24 * 16 * EPS32
OPT = dict(lr=2e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=0.02)


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def as64(t):
    import torch
    if t.dtype == torch.float8_e4m3fn:
        return t.view(torch.uint8).cpu().numpy()
    return t.double().cpu().numpy()


def start_state(rng, p, bits, table):
    """Moments in the middle of training."""
    import torch
    state = sm.alloc_adamw_state(p, bits, table)
    m = rng.normal(size=tuple(p.shape)) * 1e-3
    root = rng.uniform(0.2, 1.5, size=tuple(p.shape)) * 1e-3
    if bits == 32:
        state["m"].copy_(torch.as_tensor(m))
        state["v"].copy_(torch.as_tensor(root * root))
        return state
    rows = [0] if not table else range(p.shape[0])
    values = code_values()
    for k, (x, least) in {"m": (m, False), "v": (root, True)}.items():
        x = x.reshape(len(rows), -1)
        for r in rows:
            scale, val, _, _ = encode(x[r], None, least)
            order = np.argsort(np.nan_to_num(values[:127]))
            code = order[np.searchsorted(values[:127][order], np.abs(val))] | np.where(val < 0, 128, 0)
            state[k].view(torch.uint8).view(len(rows), -1)[r].copy_(torch.as_tensor(code.astype(np.uint8)))
            state[k + "_scale"].view(len(rows), -1)[r].copy_(torch.as_tensor(scale))
    return state


def snapshot(p, state):
    return as64(p).copy(), {k: as64(t).copy() for k, t in state.items()}


def check_row(what, p0, s0, p1, s1, g, param, bits, step, index, row, seed, opt):
    """One row (flat arrays) before and after a step with gradient g."""
    lr, betas, eps, decay = opt["lr"], opt["betas"], opt["eps"], opt["weight_decay"]
    m0, v0 = s0["m"], s0["v"]
    if bits == 8:
        m0, v0 = decode(m0, s0["m_scale"]), decode(v0, s0["v_scale"]) ** 2
    p, m, v = adamw(p0, g, m0, v0, lr, betas, eps, decay, step)
    dp, dm, dv = adamw_bounds(p0, g, m0, v0, lr, betas, eps, decay, step)
    if bits == 8:          # the square of a decoded root: three more roundings
        dp, dv = dp + 4 * EPS32 * np.abs(p - p0), dv + 4 * EPS32 * v
    if param == "bfloat16" and seed is not None:
        share = (((draws(seed, step, index, row, len(p)) ^ np.uint64(0x85EBCA6B)) * np.uint64(0x9E3779B1)) & np.uint64(0xFFFFFFFF)) >> np.uint64(16)
        unit = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(p), 2.0 ** -126))) - 7)
        up = np.floor(np.abs(p) / unit + share.astype(float) / 65536) * unit
        sure = np.abs(np.abs(p) / unit + share.astype(float) / 65536 - np.round(np.abs(p) / unit + share.astype(float) / 65536)) > dp / unit
        assert np.array_equal(np.where(sure, p1, 0), np.where(sure, np.copysign(up, p), 0)), what
        assert (np.abs(p1 - p) <= 1.001 * unit + dp).all(), what
        assert sure.mean() > 0.9 or len(p) < 50, what
    else:
        assert (np.abs(p1 - p) <= dp + (rounding(p, param) if param == "bfloat16" else 0.0)).all(), (what, np.abs(p1 - p).max())
    if bits == 32:
        assert (np.abs(s1["m"] - m) <= dm).all() and (np.abs(s1["v"] - v) <= dv).all(), what
        return
    d = None if seed is None else draws(seed, step, index, row, len(p))
    for name, x, least, bound in (("m", m, False, dm), ("v", np.sqrt(v), True, dv / (2 * np.sqrt(v) + 1e-300))):
        share = None if d is None else ((d & np.uint64(0xFFFF)) if name == "m" else (d >> np.uint64(16))).astype(float) / 65536
        scale, val, far, code_step = encode(x, share, least)
        # a moment that is the small difference of large terms is off by more than half steps of itself (`bound`); where
        # that is the block's largest, so is the scale, and with it every value relative to it (16 steps at most)
        at = np.arange(len(x)) // BLOCK
        off = np.array([bound[at == b].max() for b in range(len(scale))])
        assert (np.abs(s1[name + "_scale"] - scale) <= off / 448 + 4 * EPS32 * scale + 2.0 ** -126).all(), (what, name)
        got = code_values()[s1[name]]
        top = np.maximum(448 * scale[at], 1e-300)
        loose = NEAR + np.where(scale[at] > 0, 448 * bound / top / code_step + 16 * off[at] / top, 0.0)
        sure = far > loose
        assert np.array_equal(np.where(sure, got, 0), np.where(sure, val, 0)), (what, name)
        assert (np.abs(got - val) <= code_step * 1.001).all() and (sure.mean() > 0.9 or len(x) < 50), (what, name)


def f32(x):
    return x.astype(np.float32)


SIZES = [(1,), (2,), (3,), (5,), (127,), (128,), (129,), (255,), (257,), (1023,), (1025,), (4095,), (4097,), (20000,), (33, 77)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float32", "float16"), ("bfloat16", "float32")])
@pytest.mark.parametrize("seed", [None, 0x123456789AB])
def test_dense_tensors(bits, param, grad, seed):
    """Many tensors of odd sizes in one call, over several steps, each
    checked from the state before it."""
    import torch
    rng = np.random.default_rng(21)
    dev = torch.device("cuda")
    params = [torch.as_tensor(rng.normal(size=s) * 0.05, dtype=getattr(torch, param), device=dev) for s in SIZES]
    states = [start_state(rng, p, bits, False) for p in params]
    opt = sm.AdamW(params, **OPT, bits=bits, seed=seed, states=states, steps=6)
    for step in (7, 8, 9):
        grads = [torch.as_tensor(rng.normal(size=s) * 1e-3, dtype=getattr(torch, grad), device=dev) for s in SIZES]
        grads[3].zero_()
        before = [snapshot(p, s) for p, s in zip(params, states)]
        opt.step(grads)
        for k, (p, s) in enumerate(zip(params, states)):
            p1, s1 = snapshot(p, s)
            flat = lambda d: {n: a.reshape(-1) for n, a in d.items()}
            check_row((step, SIZES[k]), before[k][0].reshape(-1), flat(before[k][1]), p1.reshape(-1), flat(s1),
                      as64(grads[k]).reshape(-1), param, bits, step, k, 0, seed, OPT)


def sum_entries(ids, coef, grad, per, rows):
    """Row gradients in 64 bits, and the bound of sums of products in fp32
    that are rounded once more."""
    total, size = {}, {}
    for i, r in enumerate(ids):
        if 0 <= r < rows:
            x = coef[i] * grad[i // per]
            total[r] = total.get(r, 0.0) + x
            size[r] = size.get(r, 0.0) + np.abs(x)
    return total, {r: 2 * EPS32 * size[r] for r in size}


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad", [("float32", "float32"), ("bfloat16", "float32"), ("float32", "bfloat16")])
@pytest.mark.parametrize("dim", [1, 4, 100, 129, 257, 400])
def test_table_rows(bits, param, grad, dim):
    """Entries in any order with repeats and ids outside the table; runs
    below, at and far above the length whose sums are made ahead, from odd
    places; the other rows stay as they were, bit for bit."""
    import torch
    rng = np.random.default_rng(dim)
    dev = torch.device("cuda")
    rows, per = 40, 3
    runs = {0: 1, 1: 2, 5: 63, 6: 64, 7: 65, 9: 127, 10: 128, 11: 129, 12: 300, 20: 1000, 33: 1, 39: 640}
    ids = np.concatenate([np.full(n, r) for r, n in runs.items()] + [np.full(50, -1), np.full(40, rows), np.full(3, 2 ** 31 - 1)])
    ids = rng.permutation(ids).astype(np.int32)
    n = len(ids)
    p = torch.as_tensor(rng.normal(size=(rows, dim)) * 0.05, dtype=getattr(torch, param), device=dev)
    state = start_state(rng, p, bits, True)
    opt = sm.AdamW([p], **OPT, bits=bits, seed=99, states=[state], steps=10)
    vectors = torch.as_tensor(rng.normal(size=(-(-n // per), dim)), dtype=getattr(torch, grad), device=dev)
    # one summand dominates no other: sums of few roundings' error against each moment's bound
    coef = f32(rng.uniform(0.5, 1.0, size=n) * 1e-3)
    before = snapshot(p, state)
    opt.step([sm.row_grad(torch.as_tensor(ids, device=dev), vectors, coef=torch.as_tensor(coef, device=dev), per=per)])
    p1, s1 = snapshot(p, state)
    sums, off = sum_entries(ids, coef.astype(float), as64(vectors), per, rows)
    for r in range(rows):
        row = lambda d: {k: a[r] for k, a in d.items()}
        if r not in sums:
            assert np.array_equal(p1[r], before[0][r]) and all(np.array_equal(s1[k][r], before[1][k][r]) for k in s1), r
            continue
        check_sums(p1[r], row(s1), before[0][r], row(before[1]), sums[r], off[r], param, bits, 11, r)


def check_sums(p1, s1, p0, s0, g, dg, param, bits, step, row):
    """check_row for a gradient that is itself off by up to dg: the result
    lies between (within the bounds of) those of g - dg and g + dg; moments
    in 8 bits within a code's step of theirs."""
    lr, betas = OPT["lr"], OPT["betas"]
    m0, v0 = s0["m"], s0["v"]
    if bits == 8:
        m0, v0 = decode(m0, s0["m_scale"]), decode(v0, s0["v_scale"]) ** 2
    args = (lr, betas, OPT["eps"], OPT["weight_decay"], step)
    p, m, v = adamw(p0, g, m0, v0, *args)
    dp, dm, dv = adamw_bounds(p0, g, m0, v0, *args)
    for s in (-1, 1):
        ps, ms, vs = adamw(p0, g + s * dg, m0, v0, *args)
        dp, dm, dv = dp + np.abs(ps - p), dm + np.abs(ms - m), dv + np.abs(vs - v)
    if bits == 8:          # the square of a decoded root: three more roundings
        dp, dv = dp + 4 * EPS32 * np.abs(p - p0), dv + 4 * EPS32 * v
    unit = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(p), 2.0 ** -126))) - 7) if param == "bfloat16" else 0.0
    assert (np.abs(p1 - p) <= dp + 1.001 * unit).all(), (row, np.abs(p1 - p).max())
    if bits == 32:
        assert (np.abs(s1["m"] - m) <= dm).all() and (np.abs(s1["v"] - v) <= dv).all(), row
        return
    for name, x, dx in (("m", m, dm), ("v", np.sqrt(v), dv / np.sqrt(v))):
        scale, val, _, code_step = encode(x, np.zeros(len(x)), name == "v")
        at = np.arange(len(x)) // BLOCK
        # rounding up or down: within a step (twice that where the value crosses a power of two)
        assert (np.abs(decode(s1[name], s1[name + "_scale"]) - x) <= (code_step * 2.001 * scale[at]) + dx).all(), (row, name)


@pytest.mark.parametrize("dim", [3, 24, 200, 300])
def test_a_hub_among_the_entries(dim):
    """One row with 20,000 entries (sums made ahead of more stretches than a
    wavefront looks at at once), from an odd place, among short runs."""
    import torch
    rng = np.random.default_rng(dim)
    dev = torch.device("cuda")
    rows = 200
    ids = np.concatenate([np.full(20_000, 77), rng.integers(0, rows, size=3001)]).astype(np.int32)
    rng.shuffle(ids)
    n = len(ids)
    p = torch.as_tensor(rng.normal(size=(rows, dim)) * 0.05, dtype=torch.float32, device=dev)
    state = start_state(rng, p, 32, True)
    opt = sm.AdamW([p], **OPT, states=[state], steps=10)
    vectors = torch.as_tensor(rng.normal(size=(-(-n // 7), dim)), dtype=torch.float32, device=dev)
    coef = f32(rng.uniform(0.5, 1.0, size=n) * 1e-5)
    before = snapshot(p, state)
    opt.step([sm.row_grad(torch.as_tensor(ids, device=dev), vectors, coef=torch.as_tensor(coef, device=dev), per=7)])
    p1, s1 = snapshot(p, state)
    sums, off = sum_entries(ids, coef.astype(float), as64(vectors), 7, rows)
    for r in range(rows):
        row = lambda d: {k: a[r] for k, a in d.items()}
        check_sums(p1[r], row(s1), before[0][r], row(before[1]), sums[r], off[r], "float32", 32, 11, r)


def test_rows_equal_a_dense_step():
    """Every row of a table of whole blocks named once, in a shuffled order:
    the same bits as a dense step of it."""
    import torch
    rng = np.random.default_rng(22)
    dev = torch.device("cuda")
    for bits in (32, 8):
        a = torch.as_tensor(rng.normal(size=(50, 256)), dtype=torch.bfloat16, device=dev)
        b = a.clone()
        g = torch.as_tensor(rng.normal(size=(50, 256)), dtype=torch.float32, device=dev)
        dense = sm.AdamW([a], **OPT, bits=bits, seed=3)
        by_rows = sm.AdamW([b], **OPT, bits=bits, seed=3, tables=(0,))
        ids = torch.as_tensor(rng.permutation(50), dtype=torch.int32, device=dev)
        for _ in range(3):
            dense.step([g])
            by_rows.step([sm.row_grad(ids, g[ids.long()].contiguous())])
            assert torch.equal(a, b) and torch.equal(dense.states[0]["m"].view(torch.uint8), by_rows.states[0]["m"].view(torch.uint8))


def test_stochastic_rounding_is_right_in_the_mean():
    """Moments in 8 bits from 0 under a constant gradient of 1: v reaches
    1 - b2^t.  sqrt(v) is rounded by at most a step of 1/8 of itself each
    time, up or down with mean 0; over 4096 independent elements the mean's
    spread is below 1/8 x sqrt(steps that matter / 4096): with 1 / (1 - b2) =
    100 steps, 0.02; five of those are allowed.  Rounded to the nearest the
    elements would all be the same."""
    import torch
    dev = torch.device("cuda")
    p = torch.zeros(4096, device=dev)
    opt = sm.AdamW([p], lr=1e-3, betas=(0.9, 0.99), weight_decay=0.0, bits=8, seed=5)
    g = torch.rand(4096, device=dev) * 0.5 + 0.25
    for _ in range(400):
        opt.step([g])
    s = opt.states[0]
    root = as64(s["v"])
    root = decode(root, as64(s["v_scale"]))
    want = as64(g) * np.sqrt(1 - 0.99 ** 400)
    assert abs((root / want).mean() - 1) < 0.1
    m = decode(as64(s["m"]), as64(s["m_scale"]))
    assert abs((m / as64(g)).mean() - 1) < 0.1
    assert len(np.unique(root)) > 8


def test_small_roots_do_not_vanish():
    """A sqrt(v) far below its block's largest keeps a code above 0, so that a
    later step without gradient is small."""
    import torch
    dev = torch.device("cuda")
    for seed in (None, 4):
        p = torch.zeros(128, device=dev)
        opt = sm.AdamW([p], lr=1e-2, weight_decay=0.0, bits=8, seed=seed)
        g = torch.full((128,), 1e-9, device=dev)
        g[0] = 1.0
        opt.step([g])
        assert (as64(opt.states[0]["v"]) > 0).all()
        before = p.clone()
        opt.step([torch.zeros(128, device=dev)])
        assert (p - before).abs().max().item() < 0.1


@pytest.mark.parametrize("bits", [32, 8])
def test_values_that_are_not_finite(bits):
    """A NaN gradient spoils its element, in 8 bits its block of 128, and no
    other; a gradient scale that is not finite leaves everything."""
    import torch
    dev = torch.device("cuda")
    p = torch.ones(500, device=dev)
    opt = sm.AdamW([p], **OPT, bits=bits, seed=1)
    g = torch.full((500,), 0.5, device=dev)
    opt.step([g])
    before = snapshot(p, opt.states[0])
    for bad in (float("nan"), float("inf")):
        opt.step([g], grad_scale=torch.tensor([bad], device=dev))
        after = snapshot(p, opt.states[0])
        assert np.array_equal(before[0], after[0]) and all(np.array_equal(before[1][k], after[1][k]) for k in after[1])
    assert opt.steps == 3
    g[130] = float("nan")
    opt.step([g])
    opt.step([torch.full((500,), 0.5, device=dev)])
    spoiled = np.isnan(as64(p))
    want = np.zeros(500, bool)
    want[128:256] = bits == 8
    want[130] = True
    assert np.array_equal(spoiled, want)


def test_gradient_scale_and_none():
    import torch
    dev = torch.device("cuda")
    rng = np.random.default_rng(23)
    g = torch.as_tensor(rng.normal(size=300), dtype=torch.float32, device=dev)
    a, b, c = torch.ones(300, device=dev), torch.ones(300, device=dev), torch.ones(300, device=dev)
    sm.AdamW([a], **OPT).step([g * 0.25])
    opt = sm.AdamW([b, c], **OPT)
    version = b._version
    opt.step([g, None], grad_scale=torch.tensor([0.25], device=dev))
    assert torch.equal(a, b) and (c == 1).all() and b._version > version


def test_many_tensors_and_types_in_one_call():
    """More tensors than a launch takes, types alternating, against one call
    for each."""
    import torch
    rng = np.random.default_rng(24)
    dev = torch.device("cuda")
    types = [torch.float32, torch.bfloat16]
    sizes = [int(s) for s in rng.integers(1, 6000, size=131)]
    one = [torch.as_tensor(rng.normal(size=s), dtype=types[(k // 60) % 2], device=dev) for k, s in enumerate(sizes)]
    two = [p.clone() for p in one]
    grads = [torch.as_tensor(rng.normal(size=s), dtype=types[k % 2 if k > 100 else 0], device=dev) for k, s in enumerate(sizes)]
    opt = sm.AdamW(one, **OPT)
    single = [sm.AdamW([p], **OPT) for p in two]
    for _ in range(2):
        opt.step(grads)
        for o, g in zip(single, grads):
            o.step([g])
    for k, (p, q) in enumerate(zip(one, two)):
        assert torch.equal(p, q), k


def test_capture_with_counts_on_the_device():
    """A captured step with its count and rate on the device, replayed with
    eager work between, equals eager steps bit for bit where the bias
    corrections agree; they are computed apart, so moments are compared
    exactly and parameters within their bounds."""
    import torch
    rng = np.random.default_rng(25)
    dev = torch.device("cuda")
    a = torch.as_tensor(rng.normal(size=(30, 130)), dtype=torch.float32, device=dev)
    b = a.clone()
    g = torch.empty_like(a)
    ids = torch.as_tensor(rng.integers(0, 30, size=400), dtype=torch.int32, device=dev)
    vec = torch.as_tensor(rng.normal(size=(400, 130)), dtype=torch.float32, device=dev)
    t_a = torch.as_tensor(rng.normal(size=(30, 130)), dtype=torch.float32, device=dev)
    t_b = t_a.clone()
    rate = torch.tensor([1e-3], device=dev)
    kw = dict(betas=(0.9, 0.99), weight_decay=0.0, bits=8, seed=8, tables=(1,))
    graphed = sm.AdamW([a, t_a], lr=rate, device_step=True, **kw)
    eager = sm.AdamW([b, t_b], lr=1e-3, **kw)
    rows = sm.row_grad(ids, vec)
    graph = torch.cuda.CUDAGraph()
    g.zero_()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        graphed.step([g, rows])
    for k in range(5):
        g.copy_(torch.as_tensor(rng.normal(size=(30, 130))))
        graph.replay()
        torch.cuda.synchronize()
        eager.step([g, rows])
        assert graphed.device_steps.item() == k + 1 == eager.steps
        for x, y in zip(graphed.states, eager.states):
            assert torch.equal(x["m"].view(torch.uint8), y["m"].view(torch.uint8)), k
            assert torch.equal(x["v"].view(torch.uint8), y["v"].view(torch.uint8)), k
        # rate x (5 + 5) half steps of the corrections, for each step so far
        assert (a - b).abs().max().item() <= (k + 1) * (1e-3 * 16 * 32 * EPS32 + 8 * EPS32 * 5)
        assert (t_a - t_b).abs().max().item() <= (k + 1) * (1e-3 * 16 * 32 * EPS32 + 8 * EPS32 * 5)


def test_rate_on_the_device_and_decay_per_parameter():
    """A rate in an fp32 tensor equals the same number given as one (which has
    to be an fp32 number): the step size's quotient is a product then, one
    rounding more."""
    import torch
    rng = np.random.default_rng(26)
    dev = torch.device("cuda")
    rate = 2.0 ** -9
    start = torch.as_tensor(rng.normal(size=900), dtype=torch.float32, device=dev)
    g = torch.as_tensor(rng.normal(size=900), dtype=torch.float32, device=dev)
    ps = [start.clone() for _ in range(4)]
    sm.AdamW(ps[:2], lr=rate, weight_decay=[0.0, 0.5]).step([g, g])
    lr = torch.tensor([rate], device=dev)
    opt = sm.AdamW(ps[2:], lr=lr, weight_decay=[0.0, 0.5])
    opt.step([g, g])
    for x, y in ((ps[0], ps[2]), (ps[1], ps[3])):
        assert ((x - y).abs() <= rate * 2 * EPS32 + 2 * EPS32 * x.abs()).all()
    # decay takes rate x 0.5 of the parameter: within three roundings of it
    assert ((ps[0] - ps[1] - start * (rate * 0.5)).abs() <= 4 * EPS32 * start.abs() + rate * 2 * EPS32).all()
    lr.fill_(0.0)
    before = ps[2].clone()
    opt.step([g, g])
    assert torch.equal(before, ps[2])


def test_a_parameter_that_was_replaced():
    """Addresses are not kept: a parameter's data and a state's tensors may be
    replaced between steps."""
    import torch
    dev = torch.device("cuda")
    p = torch.ones(300, device=dev)
    opt = sm.AdamW([p], **OPT)
    g = torch.full((300,), 0.5, device=dev)
    opt.step([g])
    old = p.data
    p.data = torch.full((300,), 2.0, device=dev)
    opt.states[0]["m"] = torch.zeros(300, device=dev)
    kept = old.clone()
    opt.step([g])
    assert torch.equal(old, kept) and (p < 2.0).all() and opt.states[0]["m"].any()
    p.data = torch.zeros(10, device=dev)
    with pytest.raises(ValueError, match="fits"):
        opt.step([torch.zeros(10, device=dev)])
    with pytest.raises(ValueError, match="table"):
        sm.AdamW([torch.zeros(10, device=dev)], bits=8, tables=(0,))


def test_settings_that_change_between_steps():
    """Rate, decay, betas and eps are those of the object at the step."""
    import torch
    dev = torch.device("cuda")
    p = [torch.ones(40, device=dev), torch.ones(40, device=dev)]
    opt = sm.AdamW(p, lr=0.5, weight_decay=[0.0, 0.0])
    zero = [torch.zeros(40, device=dev)] * 2
    opt.step(zero)
    assert all((x == 1.0).all() for x in p)
    opt.weight_decay[1] = 0.5
    opt.step(zero)
    assert (p[0] == 1.0).all() and (p[1] == 0.75).all()
    opt.lr, opt.weight_decay = 0.25, [1.0, 0.0]
    opt.step(zero)
    assert (p[0] == 0.75).all() and (p[1] == 0.75).all()
    opt.lr, opt.weight_decay = 1.0, 0.5
    opt.step(zero)
    assert all((x == 0.375).all() for x in p) and opt.weight_decay == [0.5, 0.5]
    opt.weight_decay = [1.0]
    with pytest.raises(ValueError, match="weight_decay"):
        opt.step(zero)
    assert all((x == 0.375).all() for x in p) and opt.steps == 4


def test_a_parameter_that_is_no_longer_contiguous():
    import torch
    dev = torch.device("cuda")
    p = torch.ones(6, 6, device=dev)
    opt = sm.AdamW([p], **OPT)
    opt.step([torch.ones(6, 6, device=dev)])
    p.data = p.data.t()
    with pytest.raises(ValueError, match="contiguous"):
        opt.step([torch.ones(6, 6, device=dev)])


def test_a_table_beyond_32_bit_offsets():
    """Rows whose elements lie behind the 2^32nd, with a run across the
    length whose sums are made ahead."""
    import torch
    dev = torch.device("cuda")
    rows, dim = 6_000_000, 800
    p = torch.zeros((rows, dim), dtype=torch.bfloat16, device=dev)
    opt = sm.AdamW([p], lr=1.0, weight_decay=0.0, bits=8, tables=(0,))
    ids = torch.cat([torch.full((300,), rows - 1), torch.tensor([5, 5_900_000])]).to(dev, torch.int32)
    opt.step([sm.row_grad(ids, torch.ones((302, dim), device=dev))])
    # the first step moves by the rate, whatever the gradient: within half a step of bf16 and 16 of fp32
    for r in (rows - 1, 5, 5_900_000):
        assert ((p[r].float() + 1.0).abs() <= 2.0 ** -8).all()
    s = opt.states[0]      # no other row was stepped
    assert s["m_scale"].count_nonzero().item() == 3 * 7
    del p, opt, s
    torch.cuda.empty_cache()


def test_refusals_on_the_device_side():
    import torch
    dev = torch.device("cuda")
    p = torch.zeros((8, 200), device=dev)
    opt = sm.AdamW([p], bits=8, tables=(0,))
    with pytest.raises(ValueError, match="RowGrad"):
        opt.step([torch.zeros_like(p)])                        # scales are per row
    with pytest.raises(ValueError, match="int32"):
        opt.step([sm.RowGrad(torch.zeros(3, dtype=torch.int64, device=dev), torch.zeros((3, 200), device=dev))])
    with pytest.raises(ValueError, match="one for each"):
        opt.step([sm.row_grad(torch.zeros(5, dtype=torch.int32, device=dev), torch.zeros((2, 200), device=dev), per=2)])
    with pytest.raises(ValueError, match="no table"):
        sm.AdamW([torch.zeros(200, device=dev)], bits=8).step([sm.row_grad(torch.zeros(1, dtype=torch.int32, device=dev),
                                                                           torch.zeros((1, 200), device=dev))])
    with pytest.raises(ValueError, match="gradients for"):
        opt.step([])
    q = torch.zeros(100, device=dev)
    with pytest.raises(sm.SmoreError, match="overlap"):
        sm.AdamW([q, q[50:]]).step([torch.zeros(100, device=dev), torch.zeros(50, device=dev)])
    with pytest.raises(ValueError, match="contiguous"):
        sm.AdamW([torch.zeros((4, 4), device=dev).t()])
    with pytest.raises(ValueError, match="fp32 or bf16"):
        sm.AdamW([torch.zeros(4, device=dev, dtype=torch.float16)])
    assert opt.steps == 0 and not p.any()
