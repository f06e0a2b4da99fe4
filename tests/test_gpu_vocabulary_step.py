"""The operators run together as a model uses them: a table serves as input and output end (tied weights), the hidden states are sums over
bags of ids, the loss is distillation from a teacher's top logits, and both ends' gradients meet in one matrix.  Against autograd over
the same formulas in double precision."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("one_pass", [True, False])
@pytest.mark.parametrize("m,n,p,k,top", [(70, 501, 48, 3, 9), (300, 2000, 64, 1, 40)])
def test_a_step_of_training(m, n, p, k, top, one_pass):
    from paper_2608_09713_b200 import binding as B
    g = torch.Generator(device="cuda")
    g.manual_seed(m)
    e = torch.randn((n, p), generator=g, device="cuda") * 0.3
    ids = torch.randint(-1, n, (m, k), generator=g, device="cuda", dtype=torch.int32)
    w = torch.rand((m, k), generator=g, device="cuda") + 0.5
    t_ids = torch.randint(0, n, (m, top), generator=g, device="cuda", dtype=torch.int32)
    z = 3 * torch.randn((m, top), generator=g, device="cuda")
    r = torch.full((m,), 1.0 / m, device="cuda")
    r[::5] = 0.0
    tau, scale = 2.0, p ** 0.5

    h = B.spsyrk_lookup(ids, e, weights=w, scale=scale)
    logits = h @ e.t()
    if one_pass:
        loss, _, dlogits = B.spsyrk_distill(logits, t_ids, z, row_weights=r, temperature=tau, grad=logits.clone())
    else:
        loss, lse = B.spsyrk_distill(logits, t_ids, z, row_weights=r, temperature=tau)
        dlogits = B.spsyrk_distill_grad(logits, lse, t_ids, z, row_weights=r, temperature=tau, grad=logits)
    dh = dlogits @ e
    de = dlogits.t() @ h
    B.spsyrk_lookup_grad(ids, dh, n, weights=w, scale=scale, de=de, accumulate=True)
    dw = B.spsyrk_lookup_grad_weights(ids, e, dh, scale=scale)

    e64, w64 = e.double().requires_grad_(), w.double().requires_grad_()
    held = (ids >= 0).double()[..., None]
    h64 = (e64[ids.clamp(min=0).long()] * w64[..., None] * held).sum(1) * scale
    logq = torch.log_softmax(h64 @ e64.t() / tau, 1)
    logp = torch.log_softmax(z.double() / tau, 1)
    loss64 = (tau * tau * r.double()[:, None] * logp.exp() * (logp - logq.gather(1, t_ids.long()))).sum()
    loss64.backward()
    # products of p and n terms in single precision, 2^-24 each and the exponentials' 2^-22: far below 1e-4 of the largest value
    for got, expected in ((loss.sum(), loss64.detach()), (de, e64.grad), (dw, w64.grad)):
        assert float((got.double() - expected).abs().max()) < 1e-4 * float(expected.abs().max())
