"""Group-scaled rows and autograd, without a GPU: the calls record nothing, so a tensor that asks for gradients is refused
where they are recorded, and a tensor given for a result counts as changed."""
import pytest
import torch

import paper_1809_10572_amd as samd
from test_group_checks import fake, rows   # noqa: F401 (a fixture)


def calls(x, w, dy, g, u):
    return {
        "quantize": lambda: samd.group_quantize(x, 4, True, 32),
        "matmul": lambda: samd.group_matmul(x, w),
        "grad": lambda: samd.group_matmul_grad(dy, w),
        "grad, second": lambda: samd.group_matmul_grad(dy.detach(), w, dy, w),
        "gated": lambda: samd.group_gated(x, w, w),
        "gated_save": lambda: samd.group_gated_save(x, w, w),
        "gated_grad": lambda: samd.group_gated_grad(dy, g, u),
        "matmul, out": lambda: samd.group_matmul(x.detach(), w, out=dy),
        "dequantize, out": lambda: samd.group_dequantize(w, out=torch.zeros(5, 70, requires_grad=dy.requires_grad)),
    }


def test_tensors_that_ask_for_gradients(fake):
    rec, _ = fake
    w, g, u = rows(5, 70), rows(3, 5, 8), rows(3, 5, 8)
    asking = calls(torch.zeros(3, 70, requires_grad=True), w, torch.zeros(3, 5, requires_grad=True), g, u)
    for name, call in asking.items():
        with pytest.raises(ValueError, match="gradients"):
            call()
        assert not rec.calls, name
    # inside a graph too, not leaves alone
    with pytest.raises(ValueError, match="gradients"):
        samd.group_matmul(2 * torch.zeros(3, 70, requires_grad=True), w)
    scale = w.scale.clone().requires_grad_()
    with pytest.raises(ValueError, match="gradients"):
        samd.group_matmul(torch.zeros(3, 70), w._replace(scale=scale))
    with pytest.raises(ValueError, match="gradients"):
        samd.group_dequantize(w._replace(scale=scale))
    # nothing is recorded here
    with torch.no_grad():
        for call in asking.values():
            call()
        samd.group_matmul(torch.zeros(3, 70), w._replace(scale=scale))
    for call in calls(torch.zeros(3, 70), w, torch.zeros(3, 5), g, u).values():
        call()
    assert len(rec.calls) == 2 * len(asking) + 1


class Product(torch.autograd.Function):
    """How a program puts a frozen projection into its graph."""
    @staticmethod
    def forward(ctx, x, w):
        ctx.w = w
        return samd.group_matmul(x, w)

    @staticmethod
    def backward(ctx, dy):
        return samd.group_matmul_grad(dy.contiguous(), ctx.w), None


def test_inside_a_function(fake):
    rec, _ = fake
    x = torch.zeros(3, 70, requires_grad=True)
    Product.apply(x, rows(5, 70)).sum().backward()
    assert [c[0] for c in rec.calls] == ["samd_group_matmul", "samd_group_matmul_grad"] and x.grad.shape == x.shape


def test_results_count_as_changes(fake):
    """A graph that saved a tensor's values refuses to go backward once a call has written into it."""
    w, a = rows(5, 70), torch.ones(3, 5, requires_grad=True)
    for write in (lambda out: samd.group_matmul(torch.zeros(3, 70), w, out=out),
                  lambda out: samd.group_gated(torch.zeros(3, 70), w, w, out=out),
                  lambda out: samd.group_matmul_grad(torch.zeros(3, 70), rows(70, 5), out=out),
                  lambda out: samd.group_gated_grad(torch.zeros(3, 5), rows(3, 5, 8), rows(3, 5, 8), out=(out, torch.zeros(3, 5))),
                  lambda out: samd.group_dequantize(rows(3, 5), out=out)):
        saved = torch.zeros(3, 5)
        y = (a * saved).sum()
        with torch.no_grad():
            write(saved)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            y.backward()
