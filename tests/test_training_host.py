"""Refusals of the training calls, all made on the host before anything is
launched (no GPU needed; device pointers are stand-ins that nothing reads)."""
import ctypes
import os

import pytest

import paper_2110_14890_amd as sm

P = 0x1000           # a pointer that is not NULL
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(sm.LIB_PATH):
        from paper_2110_14890_amd import build
        build.build()
    return sm.lib()


def score_args(**kw):
    a = dict(batch=4, n=3, dim=8, n_rows=10, table_stride=8, query_stride=8, candidate_stride=3, score_stride=3,
             table_type=0, query_type=0)
    a.update(kw)
    return sm.ScoreArgs(**a)


@pytest.mark.parametrize("field,value,code", [
    ("batch", 0, -1), ("n", -1, -1), ("dim", 0, -1), ("dim", 2 ** 20 + 1, -1), ("n_rows", 0, -1), ("table_stride", 7, -1),
    ("query_stride", 7, -1), ("candidate_stride", -1, -1), ("score_stride", 2, -1), ("table_type", 2, -3), ("query_type", 3, -3)])
def test_score_sizes(L, field, value, code):
    a = score_args(**{field: value})
    n = ctypes.c_size_t()
    assert L.smore_score(ctypes.byref(a), P, P, P, P, None) == code
    assert L.smore_score_grad_workspace_bytes(ctypes.byref(a), ctypes.byref(n)) == code
    assert L.smore_score_grad(ctypes.byref(a), P, P, P, P, None, 0, None) == code
    assert sm.last_error()


def test_score_pointers_and_limits(L):
    a = ctypes.byref(score_args())
    for k in range(4):
        p = [P] * 4
        p[k] = None
        assert L.smore_score(a, *p, None) == -1 and "NULL" in sm.last_error()
        assert L.smore_score_grad(a, *p, None, 0, None) == -1 and "NULL" in sm.last_error()
    assert L.smore_score(None, P, P, P, P, None) == -1
    assert L.smore_score(ctypes.byref(score_args(n=0)), None, None, None, None, None) == 0      # nothing to do
    big = score_args(batch=2 ** 23, n=64, candidate_stride=64, score_stride=64)
    assert L.smore_score(ctypes.byref(big), P, P, P, P, None) == -6
    assert L.smore_score_grad(ctypes.byref(score_args(batch=2 ** 24)), P, P, P, P, None, 0, None) == -6
    # few queries with long lists need a workspace, and are refused without
    few = score_args(batch=2, n=4096, candidate_stride=4096, score_stride=4096)
    n = ctypes.c_size_t()
    assert L.smore_score_grad_workspace_bytes(ctypes.byref(few), ctypes.byref(n)) == 0 and n.value >= 2 * 2 * 8 * 4
    assert L.smore_score_grad(ctypes.byref(few), P, P, P, P, P, n.value - 1, None) == -1 and "workspace" in sm.last_error()
    assert L.smore_score_grad_workspace_bytes(ctypes.byref(score_args(batch=4096)), ctypes.byref(n)) == 0 and n.value == 0


@pytest.mark.parametrize("n", [2 ** 30 + 1, 2 ** 31 - 8, 2 ** 31 - 7, 2 ** 31 - 1])
@pytest.mark.parametrize("batch", [1, 600])
def test_score_lists_that_are_too_long(L, n, batch):
    """Lengths whose sums with a tile's or a share's size pass 31 bits."""
    a = ctypes.byref(score_args(batch=batch, n=n, candidate_stride=0, score_stride=n))
    size = ctypes.c_size_t()
    assert L.smore_score(a, P, P, P, P, None) == -1 and "2^30" in sm.last_error()
    assert L.smore_score_grad_workspace_bytes(a, ctypes.byref(size)) == -1 and "2^30" in sm.last_error()
    assert L.smore_score_grad(a, P, P, P, P, P, 2 ** 62, None) == -1 and "2^30" in sm.last_error()


def test_the_longest_score_lists(L):
    a = ctypes.byref(score_args(batch=1, n=2 ** 30, candidate_stride=0, score_stride=2 ** 30))
    size = ctypes.c_size_t()
    assert L.smore_score(a, P, P, P, P, None) == -6
    assert L.smore_score_grad_workspace_bytes(a, ctypes.byref(size)) == 0 and size.value == 512 * 8 * 4


def preference(L, args=(), ins=(), outs=()):
    a = dict(batch=4, n=3, kind=0, score_type=0, beta=0.5, smoothing=0.0, scale=1.0, positive_stride=1, negatives_stride=3,
             ref_positive_stride=1, ref_negatives_stride=3, grad_positive_stride=1, grad_negatives_stride=3)
    a.update(args)
    i = dict(positive=P, negatives=P)
    i.update(ins)
    o = dict(loss=P)
    o.update(outs)
    return L.smore_preference_loss(ctypes.byref(sm.PreferenceArgs(**a)), ctypes.byref(sm.PreferenceIn(**i)),
                                   ctypes.byref(sm.PreferenceOut(**o)), None)


@pytest.mark.parametrize("args,code", [
    (dict(batch=0), -1), (dict(batch=2 ** 24), -6), (dict(n=-1), -1), (dict(n=2 ** 30 + 1), -1), (dict(kind=2), -1),
    (dict(score_type=3), -3), (dict(score_type=-1), -3), (dict(beta=0.0), -1), (dict(beta=-1.0), -1), (dict(beta=NAN), -1),
    (dict(beta=INF), -1), (dict(smoothing=-0.1), -1), (dict(smoothing=1.0), -1), (dict(smoothing=NAN), -1),
    (dict(kind=1, smoothing=0.1), -1), (dict(scale=NAN), -1), (dict(scale=INF), -1), (dict(negatives_stride=-1), -1)])
def test_preference_sizes(L, args, code):
    assert preference(L, args) == code and sm.last_error()


def test_preference_pointers(L):
    assert preference(L, ins=dict(positive=None)) == -1
    assert preference(L, ins=dict(negatives=None)) == -1
    assert preference(L, ins=dict(ref_positive=P)) == -1
    assert preference(L, ins=dict(n_valid=P, mask=P)) == -1 and "not both" in sm.last_error()
    assert preference(L, outs=dict(loss=None)) == -1
    assert preference(L, outs=dict(grad_positive=P)) == -1
    both = dict(grad_positive=P, grad_negatives=P)
    assert preference(L, dict(grad_negatives_stride=2), outs=both) == -1 and "overlap" in sm.last_error()
    assert preference(L, dict(grad_positive_stride=0), outs=both) == -1
    assert L.smore_preference_loss(None, None, None, None) == -1


def tensor(**kw):
    a = dict(param=P, grad=P, m=P, v=P, n_rows=4, dim=8, per=1, bits=32)
    a.update(kw)
    return sm.AdamWTensor(**a)


def adamw(L, tensors, **kw):
    a = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=1)
    a.update(kw)
    ts = (sm.AdamWTensor * max(1, len(tensors)))(*tensors)
    return L.smore_adamw(ts, len(tensors), ctypes.byref(sm.AdamWArgs(**a)), None, 0, None)


@pytest.mark.parametrize("fields,code", [
    (dict(param=None), -1), (dict(grad=None), -1), (dict(m=None), -1), (dict(v=None), -1), (dict(param_type=2), -3),
    (dict(param_type=3), -3), (dict(grad_type=3), -3), (dict(bits=16), -3), (dict(bits=8), -1), (dict(n_rows=0), -1),
    (dict(dim=0), -1), (dict(weight_decay=NAN), -1), (dict(n_rows=2 ** 33, dim=2), -6), (dict(n_rows=2 ** 62, dim=2 ** 62), -6),
    (dict(rows=P, n_entries=-1), -1), (dict(rows=P, n_entries=2 ** 26), -6), (dict(rows=P, n_entries=4, per=0), -1),
    (dict(rows=P, n_entries=4, grad=None), -1), (dict(rows=P, n_rows=2 ** 31), -6),
    (dict(rows=P, n_entries=4, dim=2 ** 20 + 1), -6)])
def test_adamw_tensors(L, fields, code):
    n = ctypes.c_size_t()
    bad = tensor(**fields)
    assert adamw(L, [tensor(param=0x100000), bad]) == code and "tensor 1" in sm.last_error()
    assert L.smore_adamw_workspace_bytes(ctypes.byref(bad), 1, ctypes.byref(n)) == code


@pytest.mark.parametrize("args", [dict(lr=-1.0), dict(lr=NAN), dict(lr=INF), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0),
                                  dict(beta2=NAN), dict(eps=-1.0), dict(eps=INF), dict(step=0), dict(flags=2)])
def test_adamw_arguments(L, args):
    assert adamw(L, [tensor()], **args) == -1


def test_adamw_overlap_and_workspace(L):
    # 4 x 8 fp32 are 128 bytes
    assert adamw(L, [tensor(), tensor(param=P + 124)]) == -1 and "overlap" in sm.last_error()
    assert adamw(L, [tensor(), tensor()]) == -1 and "overlap" in sm.last_error()
    assert adamw(L, [tensor(param=P + 64, param_type=1), tensor(param=P, param_type=1), tensor(param=P + 120)]) == -1
    t = tensor(rows=P, n_entries=1000)
    n = ctypes.c_size_t()
    assert L.smore_adamw_workspace_bytes(ctypes.byref(t), 1, ctypes.byref(n)) == 0 and n.value > 0
    assert adamw(L, [t]) == -1 and "workspace" in sm.last_error()
    assert L.smore_adamw_workspace_bytes(ctypes.byref(tensor()), 1, ctypes.byref(n)) == 0 and n.value == 0
    assert adamw(L, []) == 0                                      # nothing to do


def test_sort_rows(L):
    n = ctypes.c_size_t()
    for count, rows, code in ((-1, 5, -1), (3, 0, -1), (2 ** 26, 5, -6)):
        assert L.smore_sort_rows_workspace_bytes(count, rows, ctypes.byref(n)) == code
        assert L.smore_sort_rows(P, count, rows, P, P, P, 1 << 30, None) == code
    assert L.smore_sort_rows_workspace_bytes(1000, 5, ctypes.byref(n)) == 0 and n.value >= 16 * 1000
    assert L.smore_sort_rows(P, 1000, 5, P, P, P, n.value - 1, None) == -1 and "workspace" in sm.last_error()
    for k in range(3):
        p = [P, P, P]
        p[k] = None
        assert L.smore_sort_rows(p[0], 1000, 5, p[1], p[2], P, n.value, None) == -1 and "NULL" in sm.last_error()
    assert L.smore_sort_rows(None, 0, 5, None, None, None, 0, None) == 0                       # nothing to do


def test_binding_refuses_host_tensors_and_wrong_shapes():
    import torch
    table, q = torch.zeros(5, 4), torch.zeros(2, 4)
    ids = torch.zeros((2, 3), dtype=torch.int32)
    with pytest.raises(ValueError, match="GPU"):
        sm.score(table, q, ids)
    with pytest.raises(ValueError, match="candidates"):
        sm.score(table, q, ids.long())
    with pytest.raises(ValueError, match="queries"):
        sm.score(table, q[:1], ids)
    with pytest.raises(ValueError, match="table"):
        sm.score(table.double(), q, ids)
    with pytest.raises(ValueError, match="contiguous"):
        sm.score(torch.zeros(4, 5).t(), q, ids)
    with pytest.raises(ValueError, match="grad_scores"):
        sm.score_grad(table, ids, torch.zeros(2, 4))
    pos, neg = torch.zeros(2), torch.zeros(2, 3)
    with pytest.raises(ValueError, match="GPU"):
        sm.preference_loss(pos, neg)
    for kw, word in ((dict(kind="hinge"), "kind"), (dict(ref_positive=pos), "both"), (dict(n_valid=torch.zeros(2)), "n_valid"),
                     (dict(mask=torch.zeros((2, 2), dtype=torch.int32)), "mask"), (dict(weight=torch.zeros(3)), "weight"),
                     (dict(ref_positive=pos, ref_negatives=neg.half()), "ref_negatives")):
        with pytest.raises(ValueError, match=word):
            sm.preference_loss(pos, neg, **kw)
    with pytest.raises(ValueError, match="positive"):
        sm.preference_loss(pos[:1], neg)
    with pytest.raises(ValueError, match="fp32, bf16 or fp16"):
        sm.preference_loss(pos.double(), neg.double())
    with pytest.raises(ValueError, match="both"):
        sm.preference_loss_into(pos, neg, {"grad_positive": pos})
    with pytest.raises(ValueError, match="cuda|GPU|contiguous"):
        sm.AdamW([torch.zeros(4)])
    with pytest.raises(ValueError, match="no parameters"):
        sm.AdamW([])
    with pytest.raises(ValueError, match="8 or 32"):
        sm.AdamW([torch.zeros(4)], bits=16)
