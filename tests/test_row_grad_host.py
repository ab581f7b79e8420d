"""What a RowGrad holds (no GPU needed)."""
import paper_2110_14890_amd as sm


def test_row_grad_makes_no_copies():
    """Views stay views: a copy would be made on whatever stream is current,
    not on that of the step which reads it."""
    import torch
    ids = torch.arange(40, dtype=torch.int32).view(4, 10)
    coef = torch.rand(4, 10)
    grad = torch.rand(4, 3)
    for view in (lambda t: t, lambda t: t[:, 1:], lambda t: t.t(), lambda t: t[:, :1].expand(4, 5)):
        g = sm.row_grad(view(ids), grad, coef=view(coef), per=9)
        assert g.rows.data_ptr() == view(ids).data_ptr() and g.rows.stride() == view(ids).stride()
        assert g.coef.data_ptr() == view(coef).data_ptr() and g.coef.stride() == view(coef).stride()
        assert g.grad is grad and g.order is None and g.per == 9 and not g.in_order
    assert sm.row_grad(ids, grad).coef is None
