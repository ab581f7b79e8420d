"""The training operators behind a sampled batch, in cases that can be timed and compared.

`score` compares each query's vector with the embedding rows of its candidates,
`score_grad` is its gradient for the queries, `loss` is the preference loss of a
positive against its verified negatives with its gradient, `adamw` steps many
dense tensors or the rows of an embedding table that a batch touched, with
moments in 32 bits or in 8, and `step` runs them one after the other.

Batches, negatives per query and entity counts are those of the synthetic
datasets of kgsynth; 400 and 100 are the paper's embedding widths.
"""
from __future__ import annotations

import math

import torch

own = False

TYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
LR, BETAS, EPS, DECAY, SEED, AT_STEP = 3e-4, (0.9, 0.999), 1e-8, 0.01, 20211014, 1000
BLOCK = 128          # elements of a row that share one scale of their 8-bit moments
TOP = 448.0          # the largest value of an 8-bit code (e4m3)


def listed():
    return [
        # a serving process or an interactive user ranks a few candidates
        dict(name="score_tiny", op="score", rows=1000, dim=100, batch=64, n=17, table="float32", query="float32"),
        # one ogbl-wikikg2-shaped minibatch, positives and negatives, table kept in bf16
        dict(name="score_wikikg2", op="score", rows=2_500_000, dim=400, batch=8192, n=257, table="bfloat16", query="float32"),
        # the backward pass of one FB400k-shaped minibatch, table kept in 32 bits
        dict(name="score_grad_fb400k", op="score_grad", rows=400_000, dim=400, batch=4096, n=257, table="float32", query="float32"),
        # few queries with long candidate lists, as in fine-tuning on a handful of queries
        dict(name="score_grad_few", op="score_grad", rows=400_000, dim=200, batch=16, n=4001, table="bfloat16", query="bfloat16"),
        # the loss of a small call, no reference model
        dict(name="loss_tiny", op="loss", kind="pairs", form="rows", batch=64, n=16, scores="float32", reference=False,
             smoothing=0.0, grad=True, ragged=False),
        # the benchmark's batch: all negatives against the positive at once, with a
        # reference model, in bf16, queries short of negatives and without a positive
        dict(name="loss_freebase", op="loss", kind="softmax", form="rows", batch=16384, n=512, scores="bfloat16", reference=True,
             smoothing=0.0, grad=True, ragged=True),
        # a minibatch whose queries share one candidate set, with its bit mask
        dict(name="loss_shared", op="loss", kind="pairs", form="shared", batch=8192, n=512, scores="float32", reference=False,
             smoothing=0.1, grad=True, ragged=True),
        # validation loss over 1,000 filtered negatives, a ragged batch, no gradient
        dict(name="loss_eval", op="loss", kind="pairs", form="rows", batch=3001, n=1000, scores="float16", reference=True,
             smoothing=0.0, grad=False, ragged=True),
        # the dense operators of a query model of width 400
        dict(name="adamw_operators", op="adamw", sizes="6x400x400 8x400 1x237x400", param="float32", grad="float32", bits=32),
        # a text encoder of 320M parameters beside the entity table, moments in 8 bits
        dict(name="adamw_encoder_8bit", op="adamw", sizes="32x2048x2048 16x2048x5632 17x2048", param="bfloat16", grad="bfloat16",
             bits=8),
        # the rows of an FB400k-shaped table that a batch touched, moments in 8 bits
        dict(name="adamw_rows_8bit", op="adamw_rows", rows=400_000, dim=400, batch=2048, n=129, param="bfloat16", grad="float32",
             bits=8),
        # a training step of one shape of the FB15k-237-shaped configuration
        dict(name="step_fb15k237", op="step", rows=15_000, dim=400, batch=512, n=128, param="float32", bits=32),
    ]


def _between(rng, lo, hi):
    """A whole number of [lo, hi], even over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["score", "score_grad", "loss", "loss", "adamw", "adamw_rows", "step"])
    rows, dim = _between(rng, 100, 2_500_000), _between(rng, 1, 1200)
    if rng.random() < 0.5:
        dim = max(8, dim // 8 * 8)
    batch, n = _between(rng, 1, 16384), _between(rng, 1, 4096)
    while batch * n < 32:
        batch *= 2
    if op == "loss":
        while batch * n > 16384 * 512:
            batch = max(1, batch // 2)
        kind = rng.choice(["pairs", "softmax"])
        return dict(op=op, kind=kind, form=rng.choice(["rows", "rows", "shared"]), batch=batch, n=n,
                    scores=rng.choice(list(TYPES)), reference=rng.random() < 0.5, grad=rng.random() < 0.75,
                    smoothing=rng.choice([0.0, 0.1]) if kind == "pairs" else 0.0, ragged=rng.random() < 0.75)
    if op == "adamw":
        parts, left = [], 320_000_000
        for _ in range(rng.randint(1, 5)):
            size = _between(rng, 1, 4_000_000)
            count = max(1, min(rng.randint(1, 20), left // size))
            parts.append("%dx%d" % (count, size))
            left -= count * size
        return dict(op=op, sizes=" ".join(parts), param=rng.choice(["float32", "bfloat16"]), grad=rng.choice(list(TYPES)),
                    bits=rng.choice([8, 32]))
    while batch * n * dim > 4096 * 257 * 400:
        batch, n = max(1, batch // 2), max(1, n * 3 // 4)
    while rows * dim > 160_000_000:
        rows //= 2
    case = dict(op=op, rows=rows, dim=dim, batch=batch, n=n)
    if op in ("score", "score_grad"):
        case.update(table=rng.choice(["float32", "bfloat16"]), query=rng.choice(["float32", "bfloat16"]))
    elif op == "adamw_rows":
        case.update(param=rng.choice(["float32", "bfloat16"]), grad=rng.choice(list(TYPES)), bits=rng.choice([8, 32]))
    else:
        case.update(param=rng.choice(["float32", "bfloat16"]), bits=rng.choice([8, 32]))
    return case


# ----------------------------------------------------------------- inputs
def _normal(gen, shape, scale, dtype=torch.float32):
    """Normal values, made a slice at a time so that a large table's are not
    held in 32 bits as well."""
    flat = torch.empty(math.prod(shape), dtype=dtype, device="cuda")
    for at in range(0, flat.numel(), 1 << 27):
        part = flat[at:at + (1 << 27)]
        part.copy_(torch.randn(part.numel(), device="cuda", generator=gen).mul_(scale))
    return flat.view(shape)


def _entities(gen, rows, batch, n, first):
    """Candidates as the sampler leaves them: uniform entities, rows of
    queries short of negatives padded with -1, some queries without any.
    `first` leading columns hold entities in every row that has a positive."""
    ids = torch.randint(0, rows, (batch, n), dtype=torch.int32, device="cuda", generator=gen)
    count = torch.randint(0, 2 * n + 1, (batch,), dtype=torch.int32, device="cuda", generator=gen).clamp_(max=n - first)
    count[torch.rand(batch, device="cuda", generator=gen) < 1 / 64] = -1
    live = torch.arange(n, device="cuda", dtype=torch.int32) < (count + first)[:, None]
    if first:
        live &= (count >= 0)[:, None]
    return torch.where(live, ids, -1), count


def _moments(gen, shape, size, bits):
    """Moments in the middle of training: gradients of this size, and the
    moments' 8-bit codes with one scale for each BLOCK elements of a row."""
    m = _normal(gen, shape, 0.3 * size)
    root = torch.empty(shape, device="cuda").uniform_(0.5, 1.5, generator=gen).mul_(size)
    if bits == 32:
        return {"m": m, "v": root.square_()}
    m_code, m_scale = _encode(m, None, 1)
    v_code, v_scale = _encode(root, None, 1)
    return {"m": m_code, "v": v_code, "m_scale": m_scale, "v_scale": v_scale}


def _shapes(sizes):
    return [tuple(map(int, part.split("x")[1:])) for part in sizes.split() for _ in range(int(part.split("x")[0]))]


def _views(flat, shapes, per=1):
    """Contiguous tensors one after the other in a flat buffer, each from a
    multiple of BLOCK elements (of BLOCK / per) on."""
    out, at = [], 0
    for s in shapes:
        out.append(flat[at:at + math.prod(s)].view(s))
        at += -(-math.prod(s) // (BLOCK // per)) * (BLOCK // per)
    return out


def _packed(shapes):
    """Elements that tensors of these shapes take in a flat buffer."""
    return sum(-(-math.prod(s) // BLOCK) * BLOCK for s in shapes)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    op, state = case["op"], dict(case)
    if op == "loss":
        batch, n, dtype = case["batch"], case["n"], TYPES[case["scores"]]
        # scores come out of one matrix, the positive in the first column
        state["policy"] = _normal(gen, (batch, n + 1), 3.0, dtype)
        state["ref"] = _normal(gen, (batch, n + 1), 3.0, dtype) if case["reference"] else None
        state["n_valid"] = state["mask"] = None
        if case["form"] == "shared":
            word = torch.randint(-2**31, 2**31, (batch, (n + 31) // 32), device="cuda", generator=gen)
            full = torch.arange((n + 31) // 32, device="cuda")[None, :] * 32 + 32 <= n
            word = torch.where(full, word, word & ((1 << (n % 32)) - 1))
            word[torch.rand(batch, device="cuda", generator=gen) < 1 / 64] = 0
            state["mask"] = word.to(torch.int32)
        elif case["ragged"]:
            _, state["n_valid"] = _entities(gen, 2, batch, n, 0)
        # a mean over the batch; with scores in fp16 a program scales its loss
        state["weight"] = torch.rand(batch, device="cuda", generator=gen).add_(0.5).mul_((32768.0 if dtype == torch.float16 else 1.0) / batch)
        return state
    if op == "adamw":
        shapes = _shapes(case["sizes"])
        # a program keeps its parameters, and each kind of moment, in one buffer
        count = _packed(shapes)
        state["flat"] = {"param": _normal(gen, (count,), 0.05, TYPES[case["param"]]), **_moments(gen, (count,), 1e-3, case["bits"])}
        state["params"] = _views(state["flat"]["param"], shapes)
        state["grads"] = _views(_normal(gen, (count,), 1e-3, TYPES[case["grad"]]), shapes)
        flat_shapes = [(math.prod(s),) for s in shapes]
        kinds = {k: _views(state["flat"][k], flat_shapes) for k in ("m", "v")}
        if case["bits"] == 8:
            scales = [(-(-n // BLOCK),) for n, in flat_shapes]
            kinds |= {k: _views(state["flat"][k], scales, BLOCK) for k in ("m_scale", "v_scale")}
        state["moments"] = [{k: t[i] for k, t in kinds.items()} for i in range(len(shapes))]
        state["at"] = AT_STEP
        return state
    batch, n, dim, rows = case["batch"], case["n"], case["dim"], case["rows"]
    if op in ("score", "score_grad"):
        state["table_rows"] = _normal(gen, (rows, dim), 0.05, TYPES[case["table"]])
        state["queries"] = _normal(gen, (batch, dim), 0.5, TYPES[case["query"]])
        state["ids"], _ = _entities(gen, rows, batch, n, 0)
        state["upstream"] = _normal(gen, (batch, n), 1e-2)
        return state
    state["params"] = [_normal(gen, (rows, dim), 0.05, TYPES[case["param"]])]
    state["moments"] = [_moments(gen, (rows, dim), 1e-3, case["bits"])]
    state["at"] = AT_STEP
    if op == "adamw_rows":
        ids, _ = _entities(gen, rows, batch, n, 0)
        state["ids"], state["order"] = torch.sort(ids.view(-1), stable=True)
        state["vectors"] = _normal(gen, (batch, dim), 0.5, TYPES[case["grad"]])
        state["coef"] = _normal(gen, (batch * n,), 2e-3)
        return state
    state["ids"], state["n_valid"] = _entities(gen, rows, batch, n + 1, 1)
    state["queries"] = _normal(gen, (batch, dim), 0.5)
    state["weight"] = torch.full((batch,), 1.0 / batch, device="cuda")
    return state


# ------------------------------------------------------------ plain forms
def _score(table, queries, ids):
    rows = table[ids.clamp(0, table.shape[0] - 1).long()].float()
    s = (rows * queries.float()[:, None, :]).sum(-1)
    return torch.where((ids >= 0) & (ids < table.shape[0]), s, 0.0)


def _score_grad(table, ids, upstream, dtype):
    g = torch.where((ids >= 0) & (ids < table.shape[0]), upstream, 0.0)
    rows = table[ids.clamp(0, table.shape[0] - 1).long()].float()
    return (rows * g[:, :, None]).sum(1).to(dtype)


def _valid(batch, n, n_valid, mask):
    at = torch.arange(n, device="cuda")
    if mask is not None:
        return (mask[:, at // 32] >> (at % 32).to(torch.int32)) & 1 != 0
    if n_valid is not None:
        return at < n_valid[:, None]
    return torch.ones((batch, n), dtype=torch.bool, device="cuda")


def _loss(policy, ref, n_valid, mask, kind, smoothing, weight, grad, beta=0.5):
    """Loss of each row and its weighted gradient, rows without a valid
    negative 0: z = beta ((pos - ref_pos) - (neg - ref_neg))."""
    dtype = policy.dtype
    policy = policy.float() if ref is None else policy.float() - ref.float()
    batch, n = policy.shape[0], policy.shape[1] - 1
    valid = _valid(batch, n, n_valid, mask)
    z = torch.where(valid, beta * (policy[:, :1] - policy[:, 1:]), 0.0)
    if kind == "pairs":
        count = valid.sum(1, keepdim=True).clamp(min=1)
        tail = torch.log1p(torch.exp(-z.abs()))
        each = (1 - smoothing) * ((-z).clamp(min=0) + tail) + smoothing * (z.clamp(min=0) + tail)
        loss = (torch.where(valid, each, 0.0) / count).sum(1)
        slope = (smoothing - 1 / (1 + torch.exp(z))) / count          # d loss / d z
    else:
        t = torch.where(valid, -z, -math.inf)
        top = t.amax(1, keepdim=True).clamp(min=0)
        e = torch.exp(t - top)
        rest = e.sum(1, keepdim=True)
        total = torch.exp(-top) + rest
        loss = torch.where(top > 0, top + torch.log(total), torch.log1p(rest))[:, 0]
        slope = -e / total
    if not grad:
        return {"loss": loss}
    slope = torch.where(valid, slope, 0.0) * beta * weight[:, None]
    return {"loss": loss, "grad_positive": slope.sum(1).to(dtype), "grad_negatives": (-slope).to(dtype)}


def _mix(x):
    """A bijective hash of 32-bit words (held in int64, or Python ints)."""
    x = x ^ (x >> 16)
    x = x * 0x7FEB352D & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = x * 0x846CA68B & 0xFFFFFFFF
    return x ^ (x >> 16)


def _key(step, index):
    """The word that keys the roundings of one tensor in one step."""
    k = _mix(_mix(SEED & 0xFFFFFFFF) ^ SEED >> 32)
    k = _mix(_mix(k + (step & 0xFFFFFFFF) & 0xFFFFFFFF) ^ step >> 32)
    return _mix(k + index & 0xFFFFFFFF)


def _draws(key, rows, dim):
    """A 32-bit word for each element of the table rows `rows` (int64 ids)."""
    blocks = -(-dim // BLOCK)
    at = torch.arange(dim, device="cuda")
    block = (rows * blocks)[:, None] + torch.arange(blocks, device="cuda")[None, :]
    base = _mix(_mix(key ^ block & 0xFFFFFFFF) + (block >> 32) & 0xFFFFFFFF)
    return _mix(base[:, at // BLOCK] + at % BLOCK & 0xFFFFFFFF)


def _encode(x, draws, low):
    """8-bit codes (e4m3) of x relative to the largest magnitude of its block,
    and the scales.  draws: 16-bit words that round stochastically (a value
    goes up with the probability of its remainder), None to the nearest.
    low: the least code of a value that is not 0."""
    shape, dim = x.shape, x.shape[-1]
    x = x.reshape(-1, dim)
    blocks = -(-dim // BLOCK)
    at = torch.arange(dim, device="cuda") // BLOCK
    top = torch.nn.functional.pad(x.abs(), (0, blocks * BLOCK - dim)).view(-1, blocks, BLOCK).amax(2)
    top = torch.where(top < 2.0**-126, 0.0, top)
    y = x.abs() * torch.where(top > 0, TOP / top, 0.0)[:, at]
    bits = y.view(torch.int32)
    small = y * 512.0
    if draws is None:
        code = (bits + 0x7FFFF + ((bits >> 20) & 1)) >> 20
        small = torch.round(small).to(torch.int32)
    else:
        draws = draws.to(torch.int32)
        code = (bits + (draws << 4)) >> 20
        whole = torch.floor(small)
        small = whole.to(torch.int32) + ((small - whole) * 65536.0 + draws >= 65536.0).to(torch.int32)
    code = torch.where(y < 2.0**-6, small, code - (120 << 3)).clamp(max=0x7E)
    code = torch.where((x != 0) & (top > 0)[:, at], code.clamp(min=low), code)
    code = code | torch.where(x < 0, 0x80, 0)
    return code.to(torch.uint8).view(torch.float8_e4m3fn).view(shape), (top / TOP).view(*shape[:-1], blocks)


def _decode(code, scale):
    return code.float() * scale[..., torch.arange(code.shape[-1], device="cuda") // BLOCK]


def _adamw(param, grad, moments, rows, step, index, bits):
    """One step of the rows `rows` (int64 ids, None: the tensor is one row)
    of a parameter: new values of the parameter and its moments there."""
    pick = (lambda t: t.reshape(1, -1)) if rows is None else (lambda t: t[rows])
    p, g = pick(param).float(), grad.float().view(-1, param.shape[-1]) if rows is not None else grad.float().view(1, -1)
    state = {k: pick(t) for k, t in moments.items()}
    if bits == 32:
        m, v = state["m"], state["v"]
    else:
        m, v = _decode(state["m"], state["m_scale"]), _decode(state["v"], state["v_scale"]).square()
    m = BETAS[0] * m + (1 - BETAS[0]) * g
    v = BETAS[1] * v + (1 - BETAS[1]) * g.square()
    hat = m / (1 - BETAS[0] ** step) / (torch.sqrt(v / (1 - BETAS[1] ** step)) + EPS)
    p = p * (1 - LR * DECAY) - LR * hat
    d = _draws(_key(step, index), torch.zeros(1, dtype=torch.int64, device="cuda") if rows is None else rows, p.shape[1]) \
        if bits == 8 or param.dtype == torch.bfloat16 else None
    if param.dtype == torch.bfloat16:
        up = ((d ^ 0x85EBCA6B) * 0x9E3779B1 & 0xFFFFFFFF) >> 16
        p = (p.view(torch.int32) + up.to(torch.int32) & -65536).view(torch.float32).to(torch.bfloat16)
    if bits == 32:
        return p, {"m": m, "v": v}
    m_code, m_scale = _encode(m, d & 0xFFFF, 0)
    v_code, v_scale = _encode(torch.sqrt(v), d >> 16, 1)
    return p, {"m": m_code, "v": v_code, "m_scale": m_scale, "v_scale": v_scale}


def _put(param, moments, rows, p, new):
    """The new values into the parameter and its moments."""
    if rows is None:
        param.copy_(p.view(param.shape))
        [moments[k].copy_(t.view(moments[k].shape)) for k, t in new.items()]
    else:
        as_bytes = lambda t: t.view(torch.uint8) if t.dtype == torch.float8_e4m3fn else t  # noqa: E731
        param[rows] = p
        [as_bytes(moments[k]).index_copy_(0, rows, as_bytes(t)) for k, t in new.items()]


def _row_gradient(ids, order, vectors, coef, per, rows):
    """The distinct entities of the sorted `ids` and the sum of each one's
    gradients: entry i adds coef[order[i]] times vectors[order[i] // per]."""
    keep = (ids >= 0) & (ids < rows)
    ids, order = ids[keep].long(), order[keep]
    unique, count = torch.unique_consecutive(ids, return_counts=True)
    each = (vectors[order // per].float() * coef[order][:, None]).double()
    return unique, torch.segment_reduce(each, "sum", lengths=count, axis=0, unsafe=True).float()


def _plain(state):
    op = state["op"]
    if op == "score":
        return _score(state["table_rows"], state["queries"], state["ids"])
    if op == "score_grad":
        return _score_grad(state["table_rows"], state["ids"], state["upstream"], state["queries"].dtype)
    if op == "loss":
        return _loss(state["policy"], state["ref"], state["n_valid"], state["mask"], state["kind"], state["smoothing"],
                     state["weight"], state["grad"])
    state["at"] += 1
    if op == "adamw":
        new = [_put(p, m, None, *_adamw(p, g, m, None, state["at"], k, state["bits"]))
               for k, (p, g, m) in enumerate(zip(state["params"], state["grads"], state["moments"]))]
        return _stepped(state)
    table, moments = state["params"][0], state["moments"][0]
    out = {}
    if op == "step":
        ids, queries = state["ids"], state["queries"]
        scores = _score(table, queries, ids)
        got = _loss(scores, None, state["n_valid"], None, "pairs", 0.0, state["weight"], True)
        coef = torch.cat([got["grad_positive"][:, None], got["grad_negatives"]], 1)
        out = {"loss": got["loss"], "grad_queries": _score_grad(table, ids, coef, queries.dtype)}
        at, order = torch.sort(ids.view(-1), stable=True)
        unique, g = _row_gradient(at, order, queries, coef.view(-1), ids.shape[1], table.shape[0])
    else:
        unique, g = _row_gradient(state["ids"], state["order"], state["vectors"], state["coef"], state["n"], table.shape[0])
    _put(table, moments, unique, *_adamw(table, g, moments, unique, state["at"], 0, state["bits"]))
    return {**out, **_stepped(state)}


def _stepped(state):
    """The parameters and moments of a step."""
    return state["flat"] if "flat" in state else {"param": state["params"][0], **state["moments"][0]}


def run(state):
    if not own:
        return _plain(state)
    import paper_2110_14890_amd as sm
    op = state["op"]
    if op == "score":
        return sm.score(state["table_rows"], state["queries"], state["ids"])
    if op == "score_grad":
        return sm.score_grad(state["table_rows"], state["ids"], state["upstream"], dtype=state["queries"].dtype)
    if op == "loss":
        policy, ref = state["policy"], state["ref"]
        return sm.preference_loss(policy[:, 0], policy[:, 1:], None if ref is None else ref[:, 0],
                                  None if ref is None else ref[:, 1:], n_valid=state["n_valid"], mask=state["mask"],
                                  kind=state["kind"], beta=0.5, smoothing=state["smoothing"], weight=state["weight"],
                                  grad=state["grad"])
    if "optimizer" not in state:
        state["optimizer"] = sm.AdamW(state["params"], lr=LR, betas=BETAS, eps=EPS, weight_decay=DECAY, bits=state["bits"],
                                      seed=SEED, states=state["moments"], steps=state["at"])
    optimizer = state["optimizer"]
    if op == "adamw":
        optimizer.step(state["grads"])
        return _stepped(state)
    if op == "adamw_rows":
        optimizer.step([sm.RowGrad(state["ids"], state["vectors"], order=state["order"], coef=state["coef"], per=state["n"])])
        return _stepped(state)
    table, ids, queries = state["params"][0], state["ids"], state["queries"]
    scores = sm.score(table, queries, ids)
    coef = torch.empty_like(scores)
    loss = torch.empty(ids.shape[0], device="cuda")
    sm.preference_loss_into(scores[:, 0], scores[:, 1:], {"loss": loss, "grad_positive": coef[:, 0], "grad_negatives": coef[:, 1:]},
                            n_valid=state["n_valid"], kind="pairs", beta=0.5, weight=state["weight"])
    grad_queries = sm.score_grad(table, ids, coef)
    optimizer.step([sm.row_grad(ids, queries, coef=coef, per=ids.shape[1])])
    return {"loss": loss, "grad_queries": grad_queries, **_stepped(state)}


# ------------------------------------------------------- sizes of the work
def work(case):
    """What a pass cannot do without: every candidate's row once (no more
    rows than the table has), every other input once, every output once."""
    op, size = case["op"], {"float32": 4, "bfloat16": 2, "float16": 2}
    if op == "loss":
        cells = case["batch"] * (case["n"] + 1)
        arrays = 1 + case["reference"] + case["grad"]
        marks = case["batch"] * (case["n"] / 8 if case["form"] == "shared" else 4 if case["ragged"] else 0)
        return {"bytes": cells * arrays * size[case["scores"]] + marks + case["batch"] * 8, "flops": 20 * cells}
    if op == "adamw":
        count = sum(math.prod(s) for s in _shapes(case["sizes"]))
        moved = 2 * size[case["param"]] + size[case["grad"]] + (16 if case["bits"] == 32 else 4 + 16 / BLOCK)
        return {"bytes": count * moved, "flops": 16 * count}
    batch, n, dim = case["batch"], case["n"] + (op == "step"), case["dim"]
    touched = case["rows"] * -math.expm1(-0.75 * batch * n / case["rows"])  # distinct rows of that many uniform ones
    if op in ("score", "score_grad"):
        vectors = batch * dim * size[case["query"]]
        return {"bytes": touched * dim * size[case["table"]] + vectors + 8 * batch * n, "flops": 2 * batch * n * dim}
    row = 2 * size[case["param"]] + (16 if case["bits"] == 32 else 4 + 16 / BLOCK)
    moved = touched * dim * row + 16 * batch * n + batch * dim * (size[case["grad"]] if op == "adamw_rows" else 8)
    return {"bytes": moved, "flops": (2 if op == "adamw_rows" else 6) * batch * n * dim + 16 * touched * dim}


# ------------------------------------------------------------- in 64 bits
def _exact_gathered(table, ids):
    """The candidates' rows in 64 bits, 0 for ids that are no entity."""
    inside = (ids >= 0) & (ids < table.shape[0])
    rows = torch.zeros((*ids.shape, table.shape[1]), dtype=torch.float64, device="cuda")
    rows[inside] = table[ids[inside].long()].double()
    return rows


def _exact_loss(policy, ref, n_valid, mask, kind, smoothing, weight, grad):
    policy = policy.double()
    if ref is not None:
        policy = policy - ref.double()
    z = 0.5 * (policy[:, :1] - policy[:, 1:])
    batch, n = z.shape
    if mask is not None:
        bits = (mask.long()[:, :, None] >> torch.arange(32, device="cuda")) & 1
        valid = bits.reshape(batch, -1)[:, :n].bool()
    else:
        upto = torch.full((batch,), n, device="cuda") if n_valid is None else n_valid
        valid = torch.arange(n, device="cuda").expand(batch, n) < upto[:, None]
    if kind == "pairs":
        share = valid.double() / valid.double().sum(1, keepdim=True).clamp(min=1.0)
        each = -(1 - smoothing) * torch.nn.functional.logsigmoid(z) - smoothing * torch.nn.functional.logsigmoid(-z)
        loss = (share * each).sum(1)
        by_z = share * (smoothing * torch.sigmoid(z) - (1 - smoothing) * torch.sigmoid(-z))
    else:
        logits = torch.cat([torch.zeros((batch, 1), dtype=torch.float64, device="cuda"),
                            (-z).masked_fill(~valid, -math.inf)], 1)
        loss = torch.logsumexp(logits, 1)
        # a small loss from the positive's share, which keeps its digits
        others = torch.logsumexp(logits[:, 1:], 1).exp()
        loss = torch.where(loss < 1e-3, torch.log1p(others), loss)
        by_z = -torch.softmax(logits, 1)[:, 1:]
    if not grad:
        return {"loss": loss}
    by_z = 0.5 * by_z * weight.double()[:, None]
    return {"loss": loss, "grad_positive": by_z.sum(1), "grad_negatives": -by_z}


def _exact_code(x, draws, least):
    """Values of the codes of x, and the scales, in 64 bits."""
    dim = x.shape[1]
    blocks = -(-dim // BLOCK)
    scale = torch.zeros((x.shape[0], blocks), dtype=torch.float64, device="cuda")
    index = (torch.arange(dim, device="cuda") // BLOCK).expand(x.shape)
    scale.scatter_reduce_(1, index, x.abs(), "amax").div_(TOP)
    y = (x.abs() / scale.gather(1, index)).nan_to_num_(0.0)
    step = torch.exp2(torch.floor(torch.log2(y.clamp(min=2.0**-6))) - 3)
    y = (torch.floor(y / step + draws.double() / 65536.0) * step).clamp_(max=TOP)
    if least:
        y = torch.where(x != 0, y.clamp(min=2.0**-9), y)
    return torch.where(x < 0, -y, y), scale


def _exact_adamw(param, g, moments, rows, step, index, bits):
    wide = {k: t.double() for k, t in moments.items()}
    flat = rows is None
    view = (lambda t: t.reshape(1, -1)) if flat else (lambda t: t)
    param_out, wide = view(param.double()), {k: view(t) for k, t in wide.items()}
    rows = torch.zeros(1, dtype=torch.int64, device="cuda") if flat else rows
    p, g = param_out[rows], g.double().reshape(rows.numel(), -1)
    m, v = wide["m"][rows], wide["v"][rows]
    dim = p.shape[1]
    if bits == 8:
        spread = torch.arange(dim, device="cuda") // BLOCK
        m, v = m * wide["m_scale"][rows][:, spread], (v * wide["v_scale"][rows][:, spread]) ** 2
    m.lerp_(g, 1 - BETAS[0])
    v.mul_(BETAS[1]).addcmul_(g, g, value=1 - BETAS[1])
    c1, c2 = -math.expm1(step * math.log(BETAS[0])), -math.expm1(step * math.log(BETAS[1]))
    p = p - LR * (DECAY * p + (m / c1) / ((v / c2).sqrt() + EPS))
    if param.dtype == torch.bfloat16 or bits == 8:
        d = _draws(_key(step, index), rows, dim)
    if param.dtype == torch.bfloat16:
        share = (((d ^ 0x85EBCA6B) * 0x9E3779B1 & 0xFFFFFFFF) >> 16).double() / 65536.0
        unit = torch.exp2(torch.floor(torch.log2(p.abs().clamp(min=2.0**-126))) - 7)
        p = torch.where(p < 0, -1.0, 1.0) * torch.floor(p.abs() / unit + share) * unit
    param_out[rows] = p
    if bits == 32:
        wide["m"][rows], wide["v"][rows] = m, v
    else:
        wide["m"][rows], wide["m_scale"][rows] = _exact_code(m, d & 0xFFFF, False)
        wide["v"][rows], wide["v_scale"][rows] = _exact_code(v.sqrt(), d >> 16, True)
    return param_out.view(param.shape), {k: t.view(moments[k].shape) for k, t in wide.items()}


def _exact_rows(ids, vectors, coef, per, rows):
    """Distinct entities and their summed gradients in 64 bits, from the
    entries in any order."""
    keep = ((ids >= 0) & (ids < rows)).nonzero()[:, 0]
    unique, at = torch.unique(ids[keep].long(), return_inverse=True)
    g = torch.zeros((unique.numel(), vectors.shape[1]), dtype=torch.float64, device="cuda")
    for part in zip(keep.split(1 << 20), at.split(1 << 20)):
        g.index_add_(0, part[1], vectors[part[0] // per].double() * coef[part[0]].double()[:, None])
    return unique, g


def exact(case, seed):
    state = prepare(case, seed)
    op = case["op"]
    if op == "score":
        parts = [torch.bmm(_exact_gathered(state["table_rows"], i), q.double()[:, :, None])[:, :, 0]
                 for i, q in zip(state["ids"].split(1024), state["queries"].split(1024))]
        return torch.cat(parts)
    if op == "score_grad":
        parts = [torch.bmm(g.double()[:, None, :], _exact_gathered(state["table_rows"], i))[:, 0, :]
                 for i, g in zip(state["ids"].split(1024), state["upstream"].split(1024))]
        return torch.cat(parts)
    if op == "loss":
        return _exact_loss(state["policy"], state["ref"], state["n_valid"], state["mask"], case["kind"], case["smoothing"],
                           state["weight"], case["grad"])
    step = AT_STEP + 1
    if op == "adamw":
        flat = {k: t.double() for k, t in state["flat"].items()}
        shapes = _shapes(case["sizes"])
        counts = [(math.prod(s),) for s in shapes]
        for k, (p, g, m) in enumerate(zip(state["params"], state["grads"], state["moments"])):
            p, m = _exact_adamw(p, g, m, None, step, k, case["bits"])
            for name, t in {"param": p.view(-1), **m}.items():
                each = [(-(-n // BLOCK),) for n, in counts] if "scale" in name else counts
                _views(flat[name], each, BLOCK if "scale" in name else 1)[k].copy_(t)
        return flat
    table = state["params"][0]
    out = {}
    if op == "step":
        ids, queries = state["ids"], state["queries"]
        gathered = _exact_gathered(table, ids)
        scores = torch.bmm(gathered, queries.double()[:, :, None])[:, :, 0]
        got = _exact_loss(scores, None, state["n_valid"], None, "pairs", 0.0, state["weight"], True)
        coef = torch.cat([got["grad_positive"][:, None], got["grad_negatives"]], 1)
        out = {"loss": got["loss"], "grad_queries": torch.bmm(coef[:, None, :], gathered)[:, 0, :]}
        unique, g = _exact_rows(ids.view(-1), queries, coef.view(-1), ids.shape[1], table.shape[0])
    else:
        back = torch.empty_like(state["ids"])
        back[state["order"]] = state["ids"]
        unique, g = _exact_rows(back, state["vectors"], state["coef"], case["n"], table.shape[0])
    p, m = _exact_adamw(table, g, state["moments"][0], unique, step, 0, case["bits"])
    return {**out, "param": p, **m}
