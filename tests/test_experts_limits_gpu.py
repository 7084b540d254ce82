"""The operators of a block of experts and of distillation where their ranges end: margins
between logits that no float32 exponential spans."""
import math

import pytest

from test_experts_gpu import BF16, F32, U32, gen, iso, randn, wanted, within  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

HALF = {F32: 2.0 ** -24, BF16: 2.0 ** -8}  # half a step, relative to the value


# --------------------------------------------------------------------------
# Distillation
# --------------------------------------------------------------------------

def far_reference(host, t, index, scale):
    """float64 loss with the rest as a bucket, its bound, the gradient of the sum of the losses
    and its bound, where each row has a rest and no column is listed twice: q_r and each
    column's share of it from the columns that are not listed alone.

    The sums are of float32 exponentials: d = (200 + 64 turns) u of them, the argument of a
    share is off by its own roundings (`spread` is its largest).  log q_r and q_r are off by
    d, the difference of q_r and p_r by d of both, q and p of a listed column by d and by
    their arguments'."""
    z, t = host.double() * scale, t.double()
    rows, vocab = z.shape
    p = torch.exp(t)
    p_r = 1 - p.sum(1)
    assert (p_r > 0).all()
    listed = torch.zeros(rows, vocab, dtype=torch.bool).scatter_(1, index, True)
    lse = torch.logsumexp(z, 1)
    apart = z.masked_fill(listed, -math.inf)
    log_r = torch.logsumexp(apart, 1) - lse
    share = torch.softmax(apart, 1)
    log_q = z.gather(1, index) - lse[:, None]
    loss = (p * (t - log_q)).sum(1) + p_r * (torch.log(p_r) - log_r)
    d = (200 + 64 * (vocab // 32768 + 1)) * U32
    spread = torch.nan_to_num((apart.amax(1, keepdim=True) - apart).abs(), 0.0, 0.0, 0.0).clamp(max=200)
    grad = share * (torch.exp(log_r) - p_r)[:, None]
    size = share * (torch.exp(log_r) + p_r)[:, None] * (2 * d + 8 * (spread + 8) * U32)
    grad.scatter_(1, index, torch.exp(log_q) - p)
    size.scatter_(1, index, torch.exp(log_q) * (2 * d + 8 * (log_q.abs().clamp(max=200) + 8) * U32) + p * 200 * U32)
    return loss, 2 * d + 2 * U32 * loss.abs(), grad * scale, size * scale


MARGINS = [30.0, 50.0, 60.0, 86.0, 90.0, 95.0, 100.0, 105.0, 110.0, 200.0, 300.0, 700.0]


def far_inputs(margin, dtype, scale, vocab):
    """Rows whose three listed columns lead all others by margin / scale, some of which are masked."""
    g = gen(int(min(margin, 1e6)) + vocab)
    x = randn(g, 5, vocab) / scale - margin / scale
    index = torch.stack([torch.randperm(vocab, generator=g)[:3] for _ in range(5)])
    x[:, ::7] = -math.inf
    x.scatter_(1, index, (torch.tensor([0.0, -1.0, -2.5]) / scale).expand(5, 3))
    t = torch.log(torch.tensor([0.5, 0.25, 0.15])).expand(5, 3).contiguous()
    t[1] = torch.log(torch.tensor([0.75, 0.2, 0.05 - 1e-6]))  # next to no rest
    return x.to(dtype), t, index


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("scale", [1.0, 5.0])
@pytest.mark.parametrize("vocab", [300, 4097, 100003])
def test_distill_gradient_of_a_far_rest(iso, dtype, scale, vocab):
    """The rest's gradient is p_r, shared by its columns, however far below the listed ones they lie."""
    for margin in MARGINS:
        x, t, index = far_inputs(margin, dtype, scale, vocab)
        loss, bound, grad, size = far_reference(x, t, index, scale)
        dev, td, ix = x.cuda(), t.cuda(), index.cuda()
        r = iso.distill_loss(dev, td, ix, scale=scale, rest="bucket")
        within(r.loss, loss, bound)
        d = iso.distill_loss_backward(dev, td, ix, r.stats, torch.ones(5, device="cuda"), scale=scale, rest="bucket")
        within(d, grad, size + HALF[dtype] * (grad.abs() + size) + 1e-37)
        a = wanted(dev)
        iso.distill_loss(a, td, ix, scale=scale, rest="bucket").loss.sum().backward()
        assert torch.equal(a.grad, d)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("margin", [740.0, 750.0, 800.0, 5000.0, 1e30, 3e38])
@pytest.mark.parametrize("vocab", [300, 100003])
def test_distill_of_a_rest_past_any_exponential(iso, dtype, margin, vocab):
    """The rest's term is p_r (log p_r - log q_r) also where no double holds q_r; only
    -infinity masks a column."""
    x, t, index = far_inputs(margin, dtype, 1.0, vocab)
    loss, bound, grad, size = far_reference(x, t, index, 1.0)
    dev, td, ix = x.cuda(), t.cuda(), index.cuda()
    r = iso.distill_loss(dev, td, ix, rest="bucket")
    within(r.loss, loss, bound)
    d = iso.distill_loss_backward(dev, td, ix, r.stats, torch.ones(5, device="cuda"), rest="bucket")
    within(d, grad, size + HALF[dtype] * (grad.abs() + size) + 1e-37)
    # masked: no such columns
    listed = torch.zeros(5, vocab, dtype=torch.bool).scatter_(1, index, True)
    masked = x.masked_fill(~listed, -math.inf).cuda()
    r = iso.distill_loss(masked, td, ix, rest="bucket")
    log_q = torch.log_softmax(x.double().gather(1, index), 1)
    want = (t.double().exp() * (t.double() - log_q)).sum(1)
    within(r.loss, want, 2 * 264 * U32 + 2 * U32 * want.abs())
    d = iso.distill_loss_backward(masked, td, ix, r.stats, torch.ones(5, device="cuda"), rest="bucket")
    assert torch.isfinite(d).all() and not d.cpu()[~listed].any()
