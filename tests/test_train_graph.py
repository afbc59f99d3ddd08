"""The training operators return values without an autograd graph, and say so where a gradient would be lost."""
import warnings

import pytest
import torch

from paper_2410_05589_b200 import binding as b


def quiet(call):
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        return call()


def test_it_is_said_where_an_input_requires_a_gradient():
    leaf, plain = torch.zeros(2, requires_grad=True), torch.zeros(2)
    with pytest.warns(UserWarning, match="lm_loss: the outputs carry no autograd graph"):
        b._values_only("lm_loss", plain, leaf)
    quiet(lambda: b._values_only("lm_loss", plain, None))
    with torch.no_grad():
        quiet(lambda: b._values_only("lm_loss", leaf))


@pytest.mark.gpu
def test_calls_say_it_and_a_function_around_them_does_not():
    import paper_2410_05589_b200 as ps
    g = torch.Generator().manual_seed(3)
    x, w = (torch.randn(s, generator=g).cuda().requires_grad_() for s in ((20, 64), (50, 64)))
    ids = torch.arange(20, dtype=torch.int32, device="cuda")
    at = dict(n_ctx=[0], n_groups=[4], k_masks=4)
    q = x[:, None]
    calls = (lambda: ps.group_attention(q, q, q, **at)["out"], lambda: ps.lm_loss(x, w, ids)["loss"], lambda: ps.embed_rows(ids, w))
    for call in calls:
        with pytest.warns(UserWarning, match="no autograd graph"):
            assert not call().requires_grad
        with torch.no_grad():
            quiet(call)

    class Loss(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w):
            r = ps.lm_loss(x, w, ids)
            ctx.save_for_backward(x, w, r["lse"])
            return r["loss"]

        @staticmethod
        def backward(ctx, d):
            x, w, lse = ctx.saved_tensors
            r = ps.lm_loss_backward(x, w, ids, lse, d.contiguous())
            return r["dx"], r["dw"]

    quiet(lambda: Loss.apply(x, w).sum().backward())
    logits = torch.log_softmax(x.detach().double() @ w.detach().double().T, -1).exp()
    logits[torch.arange(20), ids.long()] -= 1
    assert (x.grad - logits @ w.detach().double()).abs().max() <= 1e-4     # (gradients of size 1 to 10, fp32 sums of 50 terms)
