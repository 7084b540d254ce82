"""The operators of a block of experts and of distillation where their ranges end: margins
between logits that no float32 exponential spans, sums that cancel,
entries that repeat, each part of a float32 operand."""
import math

import pytest

from _expert_cases import CASES
from test_experts_gpu import BF16, F32, I32, I64, U32, gen, iso, randn, wanted, within  # noqa: F401

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


# --------------------------------------------------------------------------
# Products grouped by expert
# --------------------------------------------------------------------------

@pytest.mark.parametrize("tokens,dim,cols", [(5, 64, 32), (300, 136, 72), (700, 2048, 264), (3000, 200, 1032)])
def test_expert_gradient_of_a_token_is_rounded_once(iso, tokens, dim, cols):
    """A token's rows in bfloat16: two experts whose weights differ little but for the sign, so
    that the sum is small against its terms."""
    g = gen(dim)
    top = 3
    w = randn(g, top, cols, dim, std=cols ** -0.5, dtype=BF16)
    w[1] = (-w[0].double() * (1 + 2.0 ** -6 * torch.rand(cols, dim, generator=g))).to(BF16)
    w[2] *= 2.0 ** -6
    x, d = randn(g, tokens, dim, dtype=BF16), randn(g, tokens, cols, dtype=BF16)
    # expert e has row t of every token t but the last, which expert 2 has not
    keep = [tokens, tokens, tokens - 1]
    offsets = torch.tensor([0, *keep], dtype=I64).cumsum(0)
    token = torch.cat([torch.arange(n) for n in keep])
    row = torch.stack([offsets[e] + torch.arange(tokens) for e in range(top)], 1)
    row[-1, 2] = -1
    dout = d[token].contiguous()
    want, size = torch.zeros(tokens, dim, dtype=torch.float64), torch.zeros(tokens, dim, dtype=torch.float64)
    for e in range(top):
        n = keep[e]
        want[:n] += d[:n].double() @ w[e].double()
        size[:n] += d[:n].double().abs() @ w[e].double().abs()
    # float32 sums of cols terms and of a token's rows, and one rounding to bfloat16
    off = (cols + 8 + top) * U32 * size
    bound = off + HALF[BF16] * (want.abs() + off) + 1e-37
    for kind in (I32, I64):
        o, t, r = (v.to(kind).cuda() for v in (offsets, token, row))
        dx, dw = iso.expert_matmul_backward(x.cuda(), w.cuda(), o, dout.cuda(), token=t, row=r)
        within(dx, want, bound)
        only = iso.expert_matmul_backward(x.cuda(), w.cuda(), o, dout.cuda(), token=t, row=r, need_dw=False)
        assert torch.equal(only[0], dx)
        alone = iso.expert_matmul_backward(x.cuda(), w.cuda(), o, dout.cuda(), token=t, need_dx=False)
        assert torch.equal(alone[1], dw)
    a = wanted(x.cuda())
    iso.expert_matmul(a, w.cuda(), o, token=t, row=r).backward(dout.cuda())
    assert torch.equal(a.grad, dx)


@pytest.mark.parametrize("experts,rows,dim,cols", [c[1:5] for c in CASES if c[0] == "bf16"] + [
    (3, 70001, 1024, 40), (3, 70001, 1021, 40)])
def test_expert_gradient_of_a_token_by_every_instance(iso, experts, rows, dim, cols):
    """The same by each tile, in splits and beside the weights' gradient, and of rows that are larger
    than the caches: uneven experts, one without rows, rows behind the last one's."""
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + dim)
    share = torch.rand(experts, generator=g, device="cuda") + 0.2
    share[experts // 2] = 0.0
    last, tokens = rows - 37, rows // 2
    sizes = torch.multinomial(share, last, replacement=True, generator=g).bincount(minlength=experts)
    offsets = torch.zeros(experts + 1, dtype=I64, device="cuda")
    offsets[1:] = sizes.cumsum(0)
    row = torch.randperm(rows, generator=g, device="cuda")[:2 * tokens].view(tokens, 2)
    token = torch.zeros(rows, dtype=I64, device="cuda")
    token[row.flatten()] = torch.arange(tokens, device="cuda").repeat_interleave(2)
    x = torch.randn(tokens, dim, generator=g, device="cuda").to(BF16)
    w = (torch.randn(experts, cols, dim, generator=g, device="cuda") * cols ** -0.5).to(BF16)
    d = torch.randn(rows, cols, generator=g, device="cuda").to(BF16)
    dx, dw = iso.expert_matmul_backward(x, w, offsets, d, token=token, row=row)
    terms, sizes = (torch.zeros(rows, dim, dtype=torch.float64, device="cuda") for _ in range(2))
    for e in range(experts):
        a, b = int(offsets[e]), int(offsets[e + 1])
        terms[a:b], sizes[a:b] = d[a:b].double() @ w[e].double(), d[a:b].double().abs() @ w[e].double().abs()
    want = terms[row[:, 0]] + terms[row[:, 1]]
    off = (cols + 10) * U32 * (sizes[row[:, 0]] + sizes[row[:, 1]])
    assert ((dx.double() - want).abs() <= off + HALF[BF16] * (want.abs() + off) + 1e-37).all()
    assert torch.equal(iso.expert_matmul_backward(x, w, offsets, d, token=token, row=row.int(), need_dw=False)[0], dx)
    assert torch.equal(iso.expert_matmul_backward(x, w, offsets, d, token=token, need_dx=False)[1], dw)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_experts_without_any_token(iso, dtype):
    """Tokens of which none is routed here: no rows, and gradients of zeros."""
    x, w = wanted(torch.randn(5, 64, device="cuda").to(dtype)), wanted(torch.randn(3, 32, 64, device="cuda").to(dtype))
    o, token = torch.zeros(4, dtype=I32, device="cuda"), torch.empty(0, dtype=I32, device="cuda")
    row = torch.full((5, 2), -1, dtype=I32, device="cuda")
    h = iso.expert_matmul(x, w, o, token=token, row=row)
    y = wanted(torch.empty(0, 64, device="cuda", dtype=dtype))
    out = iso.combine_tokens(y, row)
    assert h.shape == (0, 32) and out.shape == (5, 64) and not out.any()
    (h.sum() + out.sum()).backward()
    assert x.grad.shape == x.shape and not x.grad.any() and not w.grad.any() and y.grad.shape == y.shape
    dx, dw = iso.expert_matmul_backward(x.detach(), w.detach(), o, h.detach(), token=token, row=row, need_dw=False)
    assert not dx.any() and dw is None


def test_expert_matmul_finds_a_wrong_row_at_once(iso):
    x, w = wanted(torch.randn(10, 8, device="cuda")), torch.randn(3, 5, 8, device="cuda")
    o = torch.tensor([0, 5, 15, 20], dtype=I32, device="cuda")
    t = torch.arange(20, dtype=I32, device="cuda") // 2
    row = torch.arange(20, dtype=I32, device="cuda").view(10, 2)
    for wrong in (row.flatten(), row[:9], row.float(), row.view(5, 4), row.t(), row.cpu(),
                  torch.zeros(10, 33, dtype=I32, device="cuda"), row[:, :0]):
        with pytest.raises(ValueError):
            iso.expert_matmul(x, w, o, token=t, row=wrong)
    iso.expert_matmul(x, w, o, token=t, row=row).sum().backward()


@pytest.mark.parametrize("case", [i for i, c in enumerate(CASES) if c[0] == "f32"])
def test_expert_products_of_every_part(iso, case):
    """float32 products with one term each, or few: an operand has one value that is not zero in a
    row, of 24 bits, the other is full, so that the bound is the rounding of a product and a part
    of an operand that is lost, doubled or taken for another shows.

    The parts of a and b are off by nothing, what their six products leave out is at most 2^-23
    of a b, and their sum is rounded six times, once more a split."""
    _, experts, rows, dim, cols, _ = CASES[case]
    g = torch.Generator(device="cuda")
    g.manual_seed(case)

    def full(*shape):
        return (1.0 + torch.rand(*shape, generator=g, device="cuda")) * torch.where(
            torch.rand(*shape, generator=g, device="cuda") < 0.5, -1.0, 1.0)

    def single(n, width):
        """[n, width] with one value a row, at any column, and where."""
        at = torch.randint(0, width, (n,), generator=g, device="cuda")
        out = torch.zeros(n, width, device="cuda")
        out.scatter_(1, at[:, None], full(n, 1))
        return out, at

    sizes = torch.multinomial(torch.rand(experts, generator=g, device="cuda") + 0.2, rows, replacement=True,
                              generator=g).bincount(minlength=experts)
    offsets = torch.zeros(experts + 1, dtype=I64, device="cuda")
    offsets[1:] = sizes.cumsum(0)
    expert = torch.repeat_interleave(torch.arange(experts, device="cuda"), sizes)
    w = full(experts, cols, dim)
    x, at = single(rows, dim)
    d, to = single(rows, cols)
    value = x.gather(1, at[:, None]).double()
    want = value * w[expert, :, at].double()
    got = iso.expert_matmul(x, w, offsets)
    assert ((got.double() - want).abs() <= 24 * U32 * want.abs()).all()
    want = d.gather(1, to[:, None]).double() * w[expert, to].double()
    dx = iso.expert_matmul_backward(x, w, offsets, d, need_dw=False)[0]
    assert ((dx.double() - want).abs() <= 24 * U32 * want.abs()).all()
    # a row of x adds to one column of its expert's gradient: as many terms as rows have the column
    dense = full(rows, cols)
    dw = iso.expert_matmul_backward(x, w, offsets, dense, need_dx=False)[1].double()
    for e in range(experts):
        a, b = int(offsets[e]), int(offsets[e + 1])
        X, D = x[a:b].double(), dense[a:b].double()
        n = (X != 0).sum(0)[None, :]
        size = D.abs().T @ X.abs()
        assert ((dw[e] - D.T @ X).abs() <= (24 + 6 * n) * U32 * size).all()


# --------------------------------------------------------------------------
# Combination
# --------------------------------------------------------------------------

@pytest.mark.parametrize("tokens", [3, 700, 5000])
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", [I32, I64])
def test_combine_gradient_where_entries_repeat(iso, tokens, dtype, kind):
    """A row that two entries name leaves another without any, though there are as many entries as
    rows: that one's gradient is zero, whatever dy's memory held, and those named once have theirs."""
    g = gen(tokens)
    rows = tokens * 2
    y, dout, w = randn(g, rows, 96, dtype=dtype), randn(g, tokens, 96, dtype=dtype), randn(g, tokens, 2)
    row = torch.randperm(rows, generator=g).view(tokens, 2)
    row[::3, 1] = row[::3, 0]
    row[-1, 0] = row[0, 0]
    named = torch.bincount(row.flatten(), minlength=rows)
    assert (named == 0).any() and (named > 1).any()
    want = torch.zeros(rows, 96, dtype=torch.float64)
    want[row.flatten()] = (w.double()[:, :, None] * dout.double()[:, None, :]).flatten(0, 1)
    dy = torch.full((rows, 96), math.nan, device="cuda", dtype=dtype)
    size = iso.isoloco_combine_tokens_backward_workspace_size(tokens, 2)
    ws = torch.full((size + 256,), 255, dtype=torch.uint8, device="cuda")
    at = (ws.data_ptr() + 255) // 256 * 256
    d, wd, r = dout.cuda(), w.cuda(), row.to(kind).cuda()
    for _ in range(2):
        iso.isoloco_combine_tokens_backward(
            d.data_ptr(), 96, None, 96, iso.ISOLOCO_F32 if dtype == F32 else iso.ISOLOCO_BF16, rows, 96, r.data_ptr(),
            iso.ISOLOCO_I32 if kind == I32 else iso.ISOLOCO_I64, wd.data_ptr(), tokens, 2, dy.data_ptr(), 96, None, at, size,
            torch.cuda.current_stream().cuda_stream)
        got = dy.cpu()
        assert not got[named == 0].any()
        within(got[named == 1], want[named == 1], HALF[dtype] * want[named == 1].abs() + 1e-37)
        assert torch.isfinite(got).all()


def test_combine_gradient_of_many_rows(iso):
    """More rows than the workgroups that mark them take at once on a card's 256 units."""
    rows = (1 << 26) + (1 << 18) + 5
    row = torch.arange(rows - 1, -1, -1, dtype=I32, device="cuda")
    row[12345] = row[rows - 7]
    dout, dy = torch.ones(rows, 1, dtype=BF16, device="cuda"), torch.full((rows, 1), math.nan, dtype=BF16, device="cuda")
    size = iso.isoloco_combine_tokens_backward_workspace_size(rows, 1)
    ws = torch.full((size + 256,), 255, dtype=torch.uint8, device="cuda")
    iso.isoloco_combine_tokens_backward(
        dout.data_ptr(), 1, None, 1, iso.ISOLOCO_BF16, rows, 1, row.data_ptr(), iso.ISOLOCO_I32, None, rows, 1,
        dy.data_ptr(), 1, None, (ws.data_ptr() + 255) // 256 * 256, size, torch.cuda.current_stream().cuda_stream)
    assert dy[rows - 1 - 12345] == 0
    dy[rows - 1 - 12345] = 1
    assert (dy == 1).all()


# --------------------------------------------------------------------------
# Routing
# --------------------------------------------------------------------------

@pytest.mark.parametrize("tokens", [5, 200])
@pytest.mark.parametrize("normalize", [True, False])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_route_of_nan_and_infinity(iso, tokens, normalize, dtype):
    """Each makes all of its token's weights NaN, and the gradient of the scores that they depend
    on; other tokens' stay as they are."""
    g = gen(1)
    s, dw = randn(g, tokens, 40, dtype=dtype), randn(g, tokens, 4)
    clean = iso.route_tokens(s.cuda(), 4, normalize=normalize)
    s[1, 7] = math.nan
    s[3, 9] = math.inf
    r = iso.route_tokens(s.cuda(), 4, normalize=normalize)
    odd, fine = [1, 3], [t for t in range(tokens) if t not in (1, 3)]
    assert torch.isnan(r.weight[odd]).all()
    assert torch.equal(r.weight[fine], clean.weight[fine]) and torch.equal(r.expert[fine], clean.expert[fine])
    d = iso.route_tokens_backward(s.cuda(), r.expert, dw.cuda(), normalize=normalize)
    want = iso.route_tokens_backward(s[fine].cuda(), r.expert[fine].contiguous(), dw[fine].cuda(), normalize=normalize)
    assert torch.equal(d[fine], want)
    if normalize:
        assert torch.isnan(d[odd].gather(1, r.expert[odd].long())).all()
    else:
        assert torch.isnan(d[odd]).all()


def test_combine_gradient_in_a_graph_follows_its_rows(iso):
    """Many slots, marked and cleared anew at each replay."""
    g = gen(4)
    tokens, rows = 6000, 12000
    dout, w = randn(g, tokens, 72, dtype=BF16).cuda(), randn(g, tokens, 2).cuda()
    y = randn(g, rows, 72, dtype=BF16).cuda()
    kinds = []
    for drop in (0.0, 0.3, 1.0, 0.0):
        r = torch.randperm(rows, generator=g).view(tokens, 2)
        r[torch.rand(tokens, 2, generator=g) < drop] = -1
        kinds.append(r.int().cuda())
    row = kinds[0].clone()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        iso.combine_tokens_backward(dout, y, row, w)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        dy, dweight = iso.combine_tokens_backward(dout, y, row, w)
    for r in kinds * 2:
        row.copy_(r)
        dy.fill_(math.nan)
        graph.replay()
        torch.cuda.synchronize()
        want = iso.combine_tokens_backward(dout, y, r, w)
        assert torch.equal(dy, want[0]) and torch.equal(dweight, want[1])
