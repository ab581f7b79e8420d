"""AdamW at the ends of fp32: second moments that are subnormal or infinite,
with an eps that leaves the root alone in the divisor."""
import numpy as np
import pytest

import paper_2110_14890_amd as sm
from gpu_common import require_gpu
from test_gpu_adamw import as64, snapshot
from training_common import EPS32, adamw, decode

pytestmark = pytest.mark.gpu
LEAST = 2.0 ** -149          # fp32's step below 2^-126


@pytest.fixture(scope="module", autouse=True)
def _gpu():
    require_gpu()


def optimizer(p, by_rows, **kw):
    return sm.AdamW([p], betas=(0.9, 0.999), weight_decay=0.0, tables=(0,) if by_rows else (), **kw)


def step(opt, g, by_rows):
    """A step of all of a matrix, densely or by its rows, the gradient of
    every other row as the sum of six entries."""
    import torch
    if not by_rows:
        return opt.step([g])
    rows = torch.arange(len(g), device=g.device)
    ids = torch.cat([rows, rows[1::2].repeat(5)]).to(torch.int32)
    opt.step([sm.row_grad(ids, torch.cat([g, torch.zeros_like(g[1::2]).repeat(5, 1)]))])


@pytest.mark.parametrize("by_rows", [False, True])
@pytest.mark.parametrize("bits,seed", [(32, None), (8, 3), (8, None)])
@pytest.mark.parametrize("eps", [0.0, 1e-30])
def test_gradients_whose_squares_are_subnormal(eps, bits, seed, by_rows):
    """Gradients from 1e-20 to 1e-16, alone and in blocks with ordinary ones:
    steps of the size of the rate, from each state to the next.

    v is off by three roundings of its terms, each at most 2^-150 where it is
    subnormal (the square, its product, a decoded root's square) beside the
    relative ones, so its root is by 2^-149 / v at most, and the step with it;
    32 half steps hold the rest (the bounds of ordinary steps)."""
    import torch
    rng = np.random.default_rng(61)
    dev = torch.device("cuda")
    rate, shape = 2e-3, (20, 300)
    p = torch.zeros(shape, device=dev)
    opt = optimizer(p, by_rows, lr=rate, eps=eps, bits=bits, seed=seed)
    scales = ("m_scale", "v_scale")
    for at in (1, 2, 3):
        g = 10.0 ** rng.uniform(-20, -16, size=shape) * rng.choice([-1, 1], size=shape)
        g[5:8, ::7] *= 1e18
        g = torch.as_tensor(g, dtype=torch.float32, device=dev)
        p0, s0 = snapshot(p, opt.states[0])
        step(opt, g, by_rows)
        m0, v0 = s0["m"].reshape(-1), s0["v"].reshape(-1)
        if bits == 8:
            per_row = [np.repeat(s0[k].reshape(20, -1), 128, 1)[:, :300].reshape(-1) if by_rows else None for k in scales]
            m0, v0 = [decode(x, s0[k]) if r is None else decode(x, np.ones(47)) * r
                      for x, k, r in zip((m0, v0), scales, per_row)]
            v0 = v0 ** 2
        want, _, v = adamw(p0.reshape(-1), as64(g).reshape(-1), m0, v0, rate, (0.9, 0.999), eps, 0.0, at)
        got = as64(p).reshape(-1)
        size = np.abs(want - p0.reshape(-1))
        # the first moment of opposed gradients is a small difference: half steps of its terms
        terms = rate * 10 * (0.9 * np.abs(m0) + 0.1 * np.abs(as64(g).reshape(-1))) / (np.sqrt(v) / np.sqrt(1 - 0.999 ** at) + eps)
        assert np.isfinite(got).all(), at
        assert (np.abs(got - want) <= size * (LEAST / v + 32 * EPS32) + 8 * EPS32 * terms + 4 * EPS32 * np.abs(want)).all(), at
        if at == 1 and eps == 0.0:
            assert (np.abs(np.abs(got) / rate - 1) < 0.01).all()


@pytest.mark.parametrize("by_rows", [False, True])
@pytest.mark.parametrize("rate", [2e-3, 0.0])
@pytest.mark.parametrize("bits,seed", [(32, None), (8, 3)])
def test_second_moments_that_are_infinite(bits, seed, rate, by_rows):
    """A gradient whose square is no fp32 number: the parameter stands still
    (a finite moment over an infinite root) in either width, and its
    neighbours take their ordinary step.  The moments of its block are lost in
    8 bits from then on, and the block's parameters NaN in the step after."""
    import torch
    dev = torch.device("cuda")
    p = torch.ones((4, 300), device=dev)
    opt = optimizer(p, by_rows, lr=rate, bits=bits, seed=seed)
    g = torch.full((4, 300), 0.5, device=dev)
    g[1, 7], g[2, 290] = 1e20, -1e25
    step(opt, g, by_rows)
    # a first step is the rate times the gradient's sign: 1 less 16 half steps of the rate and 2 of 1
    got, moved = as64(p), np.ones((4, 300), bool)
    moved[1, 7] = moved[2, 290] = False
    assert (got[~moved] == 1.0).all()
    assert (np.abs(got[moved] - (1.0 - np.float32(rate))) <= 16 * EPS32 * rate + 2 * EPS32).all()
    if bits == 32:
        assert torch.isinf(opt.states[0]["v"]).nonzero().tolist() == [[1, 7], [2, 290]]
    # in 8 bits blocks of 128 elements of a row, or of the whole matrix
    lost = ~moved
    if bits == 8:
        block = np.arange(300) // 128 + 3 * np.arange(4)[:, None] if by_rows else np.arange(1200).reshape(4, 300) // 128
        lost = np.isin(block, block[~moved])
        assert np.isnan(as64(opt.states[0]["m_scale"])).sum() == np.isnan(as64(opt.states[0]["v_scale"])).sum() == 2
    step(opt, torch.full((4, 300), 0.5, device=dev), by_rows)
    got = as64(p)
    if bits == 8:
        assert np.isnan(got[lost]).all()
    else:
        assert (got[lost] == 1.0).all()
    assert (np.abs(got[~lost] - (1.0 - 2 * rate)) <= 2 * (16 * EPS32 * rate + 2 * EPS32) + 2.0 ** -3 * rate * (bits == 8)).all()


def test_eight_bit_moments_follow_the_gradients_by_default():
    """sqrt(v) after the gradients grew from 0.05 to 0.4, one element of each
    block as large as that all the time, so that the scales stay.

    A root u is rounded by a code's step s <= u / 8 at most, up or down with
    mean 0, and returns to its value at a rate of 1 - b2 a step.  Rounded
    that way an element's variance gains (distance to the value) x (1 - b2) s
    and loses 2 (1 - b2) of itself a step, so its spread is at most s / 2, a
    sixteenth.  Of 4,064 independent elements the mean is then within
    5 / 16 / sqrt(4,064) = 0.5 %; that sqrt(b2 u^2 + ..) is convex adds half
    the variance, 0.2 %, and 0.5 % is left for the elements' finite number of
    codes.  Rounded to the nearest u would stay near 0.05."""
    import torch
    dev = torch.device("cuda")
    b2, size = 0.999, 4096
    p = torch.zeros(size, device=dev)
    opt = sm.AdamW([p], lr=1e-6, betas=(0.9, b2), weight_decay=0.0, bits=8)
    assert opt.seed is not None
    small, large = torch.full((size,), 0.05, device=dev), torch.full((size,), 0.4, device=dev)
    small[::128] = 0.4
    for _ in range(3000):
        opt.step([small])
    for _ in range(8000):
        opt.step([large])
    s = opt.states[0]
    u = decode(as64(s["v"]), as64(s["v_scale"]))
    want = np.sqrt((1 - b2 ** 8000) * 0.4 ** 2 + b2 ** 8000 * (1 - b2 ** 3000) * 0.05 ** 2)
    moved = np.arange(size) % 128 != 0
    assert abs(u[moved].mean() / want - 1) < 0.012
    assert abs((u[moved] ** 2).mean() / want ** 2 - 1) < 0.03
    assert u.min() > 0.5 * want and u.max() < 1.6 * want      # eight and ten spreads


def test_the_default_seed():
    """0 with moments in 8 bits; none with 32, where parameters in bf16 are
    rounded to the nearest.  A seed that is given is taken."""
    import torch
    rng = np.random.default_rng(62)
    dev = torch.device("cuda")
    start = torch.as_tensor(rng.normal(size=3000), dtype=torch.bfloat16, device=dev)
    grads = [torch.as_tensor(rng.normal(size=3000), dtype=torch.float32, device=dev) for _ in range(3)]

    def run(**kw):
        p = start.clone()
        opt = sm.AdamW([p], lr=1e-2, **kw)
        for g in grads:
            opt.step([g])
        return p, opt.states[0]["v"].view(torch.uint8).clone()

    same = lambda a, b: all(torch.equal(x, y) for x, y in zip(a, b))
    assert same(run(bits=8), run(bits=8, seed=0)) and same(run(bits=32), run(bits=32, seed=None))
    for other in (None, 1):
        assert not same(run(bits=8), run(bits=8, seed=other))
    assert not same(run(bits=32), run(bits=32, seed=0))


@pytest.mark.parametrize("bits,name", [(32, "m"), (32, "v"), (8, "m"), (8, "v"), (8, "m_scale"), (8, "v_scale")])
def test_moments_replaced_at_the_same_address(bits, name):
    """A state's tensor that was let go of, and a smaller one or one of another
    type in its place (which the allocator puts at the same address): looked
    at again, and refused."""
    import torch
    dev = torch.device("cuda")
    p = torch.ones(12800, device=dev)
    opt = sm.AdamW([p], lr=1e-3, bits=bits)
    g = torch.ones(12800, device=dev)
    opt.step([g])
    state = opt.states[0]
    whole = state[name].numel()
    for count, dtype in ((whole - 1, state[name].dtype), (whole * state[name].element_size() // 2, torch.float16)):
        shape = state[name].shape
        torch.cuda.synchronize()
        state[name] = None
        state[name] = torch.zeros(count, dtype=torch.uint8, device=dev).view(dtype) if dtype == torch.float8_e4m3fn else \
            torch.zeros(count, dtype=dtype, device=dev)
        with pytest.raises(ValueError, match="m_scale|fits"):
            opt.step([g])
        state[name] = torch.zeros(shape, dtype=torch.float32 if bits == 32 or "scale" in name else torch.uint8, device=dev)
        if bits == 8 and "scale" not in name:
            state[name] = state[name].view(torch.float8_e4m3fn)
        opt.step([g])
    assert torch.isfinite(p).all() and opt.steps == 3


def test_a_parameter_of_another_type_at_the_same_address():
    """A parameter's data replaced twice: its type is looked at, not only where
    it lies."""
    import torch
    dev = torch.device("cuda")
    p = torch.ones(12800, device=dev)
    opt = sm.AdamW([p], lr=0.5, weight_decay=0.0)
    g = torch.ones(12800, device=dev)
    opt.step([g])
    p.data = p.data.double()
    p.data = p.data.to(torch.bfloat16)
    opt.step([g])
    # two steps of 0.5, each off by 16 half steps of itself at most (the bound of ordinary steps): the first leaves
    # 0.5 (1 - 2^-20) to 0.5 (1 + 2^-20), which is 0.5 in bf16, the second 8 half steps of 1 beside 0, and the sum's own
    assert p.dtype == torch.bfloat16 and (p.abs() <= 10 * EPS32).all()
    p.data = p.data.double()
    with pytest.raises(ValueError, match="fp32 or bf16"):
        opt.step([g])


def test_an_optimizer_that_is_let_go_of_frees_its_tensors():
    import gc
    import weakref

    import torch
    p = torch.ones(300, device="cuda")
    opt = sm.AdamW([p], lr=0.5, bits=8)
    opt.step([torch.ones(300, device="cuda")])
    gone = [weakref.ref(t) for t in (p, *opt.states[0].values())]
    gc.disable()
    try:
        del p, opt
        assert all(r() is None for r in gone)
    finally:
        gc.enable()
