"""The operators of a block of experts and of distillation against plain implementations
in 64 bits (CPU), at the sizes, strides and masks where they can go wrong.

Tolerances.  u = 2^-24 is the rounding of float32 (half a step) and 2^-9 that of
bfloat16; ROUND is twice that, for a result's rounding and the float32 value before it.
A sum of n float32 terms is off by at most n u times the sum of their magnitudes; each
test says the rest of its own.
"""
import math

import pytest

from _expert_cases import CASES

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
F32, BF16 = torch.float32, torch.bfloat16
I32, I64 = torch.int32, torch.int64
ROUND = {F32: 2 * U32, BF16: 2.0 ** -8}


@pytest.fixture(scope="module")
def iso():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    import paper_2607_03011_amd as iso
    return iso


def gen(seed):
    g = torch.Generator()
    g.manual_seed(seed)
    return g


def randn(g, *shape, std=1.0, dtype=F32):
    return (torch.randn(*shape, generator=g, dtype=torch.float64) * std).to(dtype)


def within(got, want, bound):
    """got within bound (elementwise) of want; NaN and infinities where want has them."""
    got, want = got.detach().cpu().double(), want.double()
    assert got.shape == want.shape
    bound = torch.as_tensor(bound, dtype=torch.float64).expand_as(want)
    odd = ~torch.isfinite(want)
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    sure = odd & ~torch.isnan(want)
    assert torch.equal(got[sure], want[sure])
    far = ((got - want).abs() - bound)[~odd]
    assert far.numel() == 0 or far.max().item() <= 0, "off by %g more than the bound" % far.max().item()


def at_offset(t, offset, dev="cuda"):
    """A contiguous copy of t whose first element is `offset` elements into an allocation."""
    flat = torch.empty(t.numel() + offset, dtype=t.dtype, device=dev)
    out = flat[offset:].view(t.shape)
    out.copy_(t)
    return out


def strided(t, pad, dev="cuda"):
    """A copy of t (2 or 3 dimensions) whose rows are `pad` elements further apart, NaN between them."""
    big = torch.full((*t.shape[:-1], t.shape[-1] + pad), math.nan, dtype=t.dtype, device=dev)
    big[..., :t.shape[-1]].copy_(t)
    return big[..., :t.shape[-1]]


# --------------------------------------------------------------------------
# Routing
# --------------------------------------------------------------------------

def scores_of(g, tokens, experts, dtype, kind):
    s = randn(g, tokens, experts, std=2.0)
    if kind == "ties":
        s = (s * 1.5).round()
    if kind == "masked":
        s[torch.rand(tokens, experts, generator=g) < 0.5] = -math.inf
        s[::5] = -math.inf
        if tokens > 2:
            s[2, : experts // 2 + 1] = -math.inf
    return s.to(dtype)


def route_reference(scores, top, normalize):
    """float64 weights and their bound, and the whole numbers."""
    x = scores.double()
    tokens, experts = x.shape
    order = torch.sort(x, dim=1, descending=True, stable=True)
    z, expert = order.values[:, :top], order.indices[:, :top]
    none = z == -math.inf
    m = torch.where(none[:, :1], 0.0, z[:, :1])
    e = torch.exp(z - m)
    all_e = torch.exp(x - m)
    total = (e if normalize else all_e).sum(1, keepdim=True)
    weight = torch.where(none, 0.0, e / total)
    # an exponential is off by its argument's rounding, |z - m| u, and 2 ulps; the sum by
    # those, weighted, and one u a term
    far = (z - m).abs().masked_fill(none, 0.0)
    spread = torch.nan_to_num((all_e * torch.where(x == -math.inf, 0.0, (x - m).abs())).sum(1, keepdim=True) / total, 0.0)
    bound = weight * (far + spread + experts + 12) * U32
    group = torch.where(none, experts, expert).flatten()
    slot = torch.sort(group, stable=True).indices
    row = torch.empty_like(slot)
    row[slot] = torch.arange(slot.numel())
    offsets = torch.zeros(experts + 1, dtype=I64)
    offsets[1:] = torch.bincount(group, minlength=experts + 1)[:experts].cumsum(0)
    return weight, bound, torch.where(none, -1, expert), row.view(tokens, top), slot // top, offsets


ROUTES = [(1, 1, 1), (1, 5, 5), (3, 64, 8), (4, 1024, 32), (64, 8, 2), (65, 8, 2), (130, 65, 3), (257, 64, 8), (300, 256, 6),
          (1000, 300, 1), (97, 1024, 32), (700, 33, 32), (5000, 16, 4)]


@pytest.mark.parametrize("tokens,experts,top", ROUTES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("kind", ["any", "ties", "masked"])
def test_route(iso, tokens, experts, top, dtype, kind):
    s = scores_of(gen(tokens + experts), tokens, experts, dtype, kind)
    for normalize in (True, False):
        weight, bound, *whole = route_reference(s, top, normalize)
        for dev in (s.cuda(), strided(s, 3), at_offset(s, 1)):
            r = iso.route_tokens(dev, top, normalize=normalize)
            assert all(t.dtype == I32 for t in r[1:])
            for got, want in zip(r[1:], whole):
                assert torch.equal(got.cpu().long(), want)
            within(r.weight, weight, bound + 1e-37)
        # the places are a permutation, and row and token are each other's inverse
        flat = r.row.flatten().long()
        assert torch.equal(flat.sort().values.cpu(), torch.arange(tokens * top))
        assert torch.equal(r.token[flat].cpu().long(), torch.arange(tokens * top) // top)


def test_route_of_nothing(iso):
    r = iso.route_tokens(torch.empty(0, 7, device="cuda"), 2)
    assert r.weight.shape == (0, 2) and r.token.numel() == 0 and not r.offsets.any()
    d = iso.route_tokens_backward(torch.empty(0, 7, device="cuda"), r.expert, r.weight)
    assert d.shape == (0, 7)
    none = torch.full((100, 7), -math.inf, device="cuda")
    r = iso.route_tokens(none, 3)
    assert not r.weight.any() and (r.expert == -1).all() and not r.offsets.any()
    assert torch.equal(r.row.flatten().cpu(), torch.arange(300, dtype=I32))
    assert not iso.route_tokens_backward(none, r.expert, torch.ones(100, 3, device="cuda")).any()


@pytest.mark.parametrize("tokens", [5, 200])
@pytest.mark.parametrize("normalize", [True, False])
def test_route_nonfinite(iso, tokens, normalize):
    s = randn(gen(1), tokens, 40)
    s[1, 7] = math.nan
    s[3, 9] = math.inf
    r = iso.route_tokens(s.cuda(), 4, normalize=normalize)
    clean = [t for t in range(tokens) if t not in (1, 3)]
    assert torch.isnan(r.weight[[1, 3]]).all(1).cpu().any() and torch.isfinite(r.weight[clean]).all()
    assert r.expert[1, 0] == 7 and r.expert[3, 0] == 9
    want = iso.route_tokens(s[clean].cuda(), 4, normalize=normalize)
    assert torch.equal(r.weight[clean], want.weight) and torch.equal(r.expert[clean], want.expert)
    assert torch.equal(r.row.flatten().long().sort().values.cpu(), torch.arange(tokens * 4))


def route_grad_reference(scores, expert, g, normalize):
    x = scores.double()
    ok = (expert >= 0) & (expert < x.shape[1])
    at = torch.where(ok, expert, 0).long()
    g = torch.where(ok, g.double(), 0.0)
    z = torch.where(ok, x.gather(1, at), -math.inf)
    w = torch.nan_to_num(torch.softmax(z if normalize else x, 1))
    p = w if normalize else w.gather(1, at) * ok
    inner = (p * g).sum(1, keepdim=True)
    size = (p * g.abs()).sum(1, keepdim=True)
    d = torch.zeros_like(x)
    d.scatter_add_(1, at, p * (g - inner) if normalize else p * g)
    b = torch.zeros_like(x)
    b.scatter_add_(1, at, p * (g.abs() + size))
    if not normalize:
        d -= w * inner
        b += w * size
    return d, b


@pytest.mark.parametrize("tokens,experts,top", ROUTES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("normalize", [True, False])
def test_route_backward(iso, tokens, experts, top, dtype, normalize):
    g = gen(tokens * 3 + experts)
    for kind in ("any", "masked"):
        s, dw = scores_of(g, tokens, experts, dtype, kind), randn(g, tokens, top)
        expert = route_reference(s, top, normalize)[2]
        want, size = route_grad_reference(s, expert, dw, normalize)
        # the weights are off by (|z - m| <= 40, the terms of the sum) u, the differences by a few more
        bound = size * 3 * (experts + 60) * U32 + ROUND[dtype] * want.abs() + 1e-37
        for dev in (s.cuda(), strided(s, 5), at_offset(s, 1)):
            within(iso.route_tokens_backward(dev, expert.int().cuda(), dw.cuda(), normalize=normalize), want, bound)


@pytest.mark.parametrize("normalize", [True, False])
def test_route_backward_of_other_experts(iso, normalize):
    """Experts that the caller names: the same one twice, and some outside."""
    g = gen(8)
    s, dw = randn(g, 50, 12), randn(g, 50, 4)
    expert = torch.randint(-2, 15, (50, 4), generator=g)
    expert[7] = 3
    expert[9] = -1
    want, size = route_grad_reference(s, expert, dw, normalize)
    got = iso.route_tokens_backward(s.cuda(), expert.int().cuda(), dw.cuda(), normalize=normalize)
    within(got, want, size * 3 * 72 * U32 + ROUND[F32] * want.abs() + 1e-37)


def test_route_against_differences(iso):
    g = gen(2)
    s, dw, v = (t.cuda() for t in (randn(g, 90, 20), randn(g, 90, 3), randn(g, 90, 20)))
    for normalize in (True, False):
        r = iso.route_tokens(s, 3, normalize=normalize)
        # small enough to leave the choice, and its error (h^2) and rounding (u / h) 1e-5 and 2e-5 of a term
        h = 2.0 ** -8
        up, down = (iso.route_tokens(s + e * h * v, 3, normalize=normalize) for e in (1, -1))
        same = (up.expert == r.expert).all(1) & (down.expert == r.expert).all(1)
        assert same.sum() > 60
        slope = ((up.weight - down.weight) * dw).double().sum(1) / (2 * h)
        d = (iso.route_tokens_backward(s, r.expert, dw, normalize=normalize) * v).double().sum(1)
        # |third derivative| <= |dw| |v|^3 of a softmax
        bound = dw.abs().sum(1) * ((v.abs().amax(1) ** 3) * 4 * h * h + 8 * U32 / h)
        assert ((slope - d).abs() <= bound)[same].all()


# --------------------------------------------------------------------------
# Products grouped by expert
# --------------------------------------------------------------------------

EXPERTS = [
    # tokens, experts, top, dim, cols
    (1, 1, 1, 1, 1), (1, 4, 2, 64, 64), (3, 8, 8, 33, 65), (7, 64, 8, 128, 96), (16, 2, 1, 256, 40), (40, 5, 2, 72, 200),
    (65, 3, 1, 256, 130), (130, 130, 2, 40, 31), (300, 6, 2, 264, 392), (513, 4, 2, 613, 257), (700, 2, 1, 520, 136),
    (33, 1000, 4, 16, 24), (260, 3, 3, 1032, 72),
]


def grouped(g, tokens, experts, top, dropped=True):
    """A random grouping, uneven, with experts that have no rows and rows of no expert:
    offsets, token, row."""
    want = torch.rand(experts, generator=g) ** 3 + 1e-3
    if experts > 2:
        want[experts // 2] = 0
    chosen = torch.multinomial(want.expand(tokens, -1) + 1e-9, min(top, experts), generator=g)
    if dropped:
        chosen[torch.rand(chosen.shape, generator=g) < 0.1] = experts
    flat = chosen.flatten()
    slot = torch.sort(flat, stable=True).indices
    row = torch.empty_like(slot)
    row[slot] = torch.arange(slot.numel())
    offsets = torch.zeros(experts + 1, dtype=I64)
    offsets[1:] = torch.bincount(flat, minlength=experts + 1)[:experts].cumsum(0)
    return offsets, slot // chosen.shape[1], row.view(tokens, -1)


def expert_reference(x, w, offsets, dout=None):
    """float64 out (dout None) or dx and dw, and the sums of magnitudes."""
    x, w = x.double(), w.double()
    at = offsets.tolist()
    if dout is None:
        out, size = (torch.zeros(x.shape[0], w.shape[1], dtype=torch.float64) for _ in range(2))
        for e, (a, b) in enumerate(zip(at[:-1], at[1:])):
            out[a:b], size[a:b] = x[a:b] @ w[e].T, x[a:b].abs() @ w[e].abs().T
        return out, size
    d = dout.double()
    dx, dxs, dw, dws = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(w), torch.zeros_like(w)
    for e, (a, b) in enumerate(zip(at[:-1], at[1:])):
        dx[a:b], dxs[a:b] = d[a:b] @ w[e], d[a:b].abs() @ w[e].abs()
        dw[e], dws[e] = d[a:b].T @ x[a:b], d[a:b].abs().T @ x[a:b].abs()
    return dx, dxs, dw, dws


def expert_inputs(tokens, experts, top, dim, cols, dtype, seed):
    g = gen(seed)
    offsets, token, row = grouped(g, tokens, experts, top)
    return (offsets, token, row, randn(g, tokens, dim, dtype=dtype),
            randn(g, experts, cols, dim, std=dim ** -0.5, dtype=dtype), randn(g, token.numel(), cols, dtype=dtype))


@pytest.mark.parametrize("tokens,experts,top,dim,cols", EXPERTS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_expert_matmul(iso, tokens, experts, top, dim, cols, dtype):
    offsets, token, _, x, w, _ = expert_inputs(tokens, experts, top, dim, cols, dtype, tokens + cols)
    want, size = expert_reference(x[token], w, offsets)
    bound = (dim + 8) * U32 * size + ROUND[dtype] * want.abs() + 1e-37
    rows, kinds = x[token], (I32, I64)
    for i, place in enumerate((lambda t: t.cuda(), lambda t: strided(t, 5), lambda t: strided(t, 8),
                               lambda t: at_offset(t, 3))):
        o, t = (v.to(kinds[i % 2]).cuda() for v in (offsets, token))
        within(iso.expert_matmul(place(x), place(w), o, token=t), want, bound)
        within(iso.expert_matmul(place(rows), place(w), o), want, bound)
    out = strided(torch.zeros(rows.shape[0], cols, dtype=dtype), 3)
    iso.expert_matmul(x.cuda(), w.cuda(), o, token=t, out=out)
    within(out, want, bound)
    assert torch.isnan(out.as_strided((rows.shape[0], 3), (cols + 3, 1), cols)[:-1]).all()
    # some of a larger tensor's rows and experts
    part = torch.full((experts, cols + 4, dim), math.nan, dtype=dtype, device="cuda")
    part[:, 2:cols + 2].copy_(w)
    within(iso.expert_matmul(x.cuda(), part[:, 2:cols + 2], o, token=t), want, bound)


@pytest.mark.parametrize("tokens,experts,top,dim,cols", EXPERTS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_expert_matmul_backward(iso, tokens, experts, top, dim, cols, dtype):
    offsets, token, row, x, w, d = expert_inputs(tokens, experts, top, dim, cols, dtype, 3 * tokens + cols)
    dx, dxs, dw, dws = expert_reference(x[token], w, offsets, d)
    n = torch.diff(offsets).double()[:, None, None]
    bx = (cols + 8) * U32 * dxs + ROUND[dtype] * dx.abs() + 1e-37
    bw = (n + 8) * U32 * dws + ROUND[dtype] * dw.abs() + 1e-37
    # a token's rows are added after their rounding
    sums, bs = dx[row].sum(1), (bx[row] + (top + 1) * U32 * dx[row].abs()).sum(1)
    bs = bs + ROUND[dtype] * (sums.abs() + bs)
    first, kinds = None, (I32, I64)
    for i, place in enumerate((lambda t: t.cuda(), lambda t: strided(t, 5), lambda t: strided(t, 8),
                               lambda t: at_offset(t, 1))):
        o, t, r = (v.to(kinds[i % 2]).cuda() for v in (offsets, token, row))
        got = iso.expert_matmul_backward(place(x), place(w), o, place(d), token=t, row=r)
        within(got[0], sums, bs)
        within(got[1], dw, bw)
        flat = iso.expert_matmul_backward(place(x[token]), place(w), o, place(d))
        within(flat[0], dx, bx)
        within(flat[1], dw, bw)
        first = first or flat
    rows = x[token].cuda()
    only = iso.expert_matmul_backward(rows, w.cuda(), o, d.cuda(), need_dw=False)
    assert torch.equal(only[0], first[0]) and only[1] is None
    only = iso.expert_matmul_backward(rows, w.cuda(), o, d.cuda(), need_dx=False)
    assert only[0] is None and torch.equal(only[1], first[1])


def test_expert_matmul_of_nothing(iso):
    w = torch.randn(3, 5, 8, device="cuda")
    o = torch.zeros(4, dtype=I32, device="cuda")
    assert iso.expert_matmul(torch.empty(0, 8, device="cuda"), w, o).shape == (0, 5)
    dx, dw = iso.expert_matmul_backward(torch.empty(0, 8, device="cuda"), w, o, torch.empty(0, 5, device="cuda"))
    assert dx.shape == (0, 8) and dw.shape == w.shape and not dw.any()
    # rows, but no expert has any
    x, d = torch.full((70, 8), math.nan, device="cuda"), torch.full((70, 5), math.nan, device="cuda")
    assert not iso.expert_matmul(x, w, o).any()
    dx, dw = iso.expert_matmul_backward(x, w, o, d)
    assert not dx.any() and not dw.any()
    # tokens that are none
    t = torch.full((70,), -1, dtype=I32, device="cuda")
    t[3] = 70
    o[1:] = 70
    assert not iso.expert_matmul(x, w, o, token=t).any()


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tokens", [6, 150])
def test_expert_matmul_rows_of_no_expert_do_not_matter(iso, tokens, dtype):
    """Rows behind the last expert's hold anything, and tokens outside x are rows of zeros."""
    offsets, token, row, x, w, d = expert_inputs(tokens, 4, 2, 72, 136, dtype, 5)
    offsets[2:] = offsets[2]
    last, n = int(offsets[-1]), token.numel()
    assert 0 < last < n - 2
    rows, d = x[token].clone(), d.clone()
    rows[last:] = math.nan
    d[last:] = math.inf
    o = offsets.int().cuda()
    want = iso.expert_matmul(x[token].cuda(), w.cuda(), o)
    got = iso.expert_matmul(rows.cuda(), w.cuda(), o)
    assert torch.equal(got, want) and not got[last:].any()
    dx, dw = iso.expert_matmul_backward(rows.cuda(), w.cuda(), o, d.cuda())
    wx, ww = iso.expert_matmul_backward(x[token].cuda(), w.cuda(), o, torch.where(torch.isinf(d), 1.0, d).to(dtype).cuda())
    assert torch.equal(dx, wx) and torch.equal(dw, ww) and not dx[last:].any() and not dw[2:].any()
    outside = token.clone()
    outside[::3] = torch.tensor([-1, tokens, 2 ** 31 - 1, -2 ** 31])[torch.arange(len(outside[::3])) % 4]
    zeroed = x[token].clone()
    zeroed[::3] = 0
    args = (w.cuda(), o)
    assert torch.equal(iso.expert_matmul(x.cuda(), *args, token=outside.int().cuda()), iso.expert_matmul(zeroed.cuda(), *args))
    d = torch.where(torch.isinf(d), 1.0, d).to(dtype).cuda()
    a = iso.expert_matmul_backward(x.cuda(), *args, d, token=outside.int().cuda(), row=row.int().cuda())[1]
    assert torch.equal(a, iso.expert_matmul_backward(zeroed.cuda(), *args, d)[1])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tokens", [9, 300])
def test_expert_matmul_nonfinite_stays_in_its_row(iso, tokens, dtype):
    offsets, token, row, x, w, d = expert_inputs(tokens, 3, 1, 136, 72, dtype, 9)
    o = offsets.int().cuda()
    at = int(offsets[1]) // 2
    rows = x[token].clone()
    want = iso.expert_matmul(rows.cuda(), w.cuda(), o)
    wx, ww = iso.expert_matmul_backward(rows.cuda(), w.cuda(), o, d.cuda())
    rows[at, 5] = math.nan
    got = iso.expert_matmul(rows.cuda(), w.cuda(), o)
    keep = torch.arange(tokens) != at
    assert torch.isnan(got[at]).all() and torch.equal(got[keep], want[keep])
    # in the weights' gradient: one column of its own expert
    dw = iso.expert_matmul_backward(rows.cuda(), w.cuda(), o, d.cuda())[1]
    assert torch.isnan(dw[0, :, 5]).all() and torch.equal(dw[1:], ww[1:])
    cols = torch.arange(136) != 5
    assert torch.equal(dw[0][:, cols], ww[0][:, cols])
    d[at, 7] = math.nan
    dx, dw = iso.expert_matmul_backward(x[token].cuda(), w.cuda(), o, d.cuda())
    assert torch.isnan(dx[at]).all() and torch.equal(dx[keep], wx[keep])
    assert torch.isnan(dw[0, 7]).all() and torch.equal(dw[1:], ww[1:])


def test_expert_matmul_offsets_outside(iso):
    """Offsets past the rows end at them, and negative ones at none: nothing else is touched."""
    x, w = torch.randn(50, 40, device="cuda"), torch.randn(3, 24, 40, device="cuda")
    d = torch.randn(50, 24, device="cuda")
    for wrong, right in (([0, 20, 999, 2 ** 31 - 1], [0, 20, 50, 50]), ([0, -7, 30, 50], [0, 0, 30, 50])):
        a, b = (torch.tensor(v, dtype=I32, device="cuda") for v in (wrong, right))
        assert torch.equal(iso.expert_matmul(x, w, a), iso.expert_matmul(x, w, b))
        for p, q in zip(iso.expert_matmul_backward(x, w, a, d), iso.expert_matmul_backward(x, w, b, d)):
            assert torch.equal(p, q)


@pytest.mark.parametrize("experts,rows", [(3, 40), (70, 900), (5, 3000)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_expert_matmul_offsets_of_any_kind(iso, experts, rows, dtype):
    """Offsets that fall and lie anywhere: what is around the results stays as it was."""
    g = gen(experts)
    offsets = torch.randint(-rows, 2 * rows, (experts + 1,), generator=g).cuda()
    token = torch.randint(-5, 60, (rows,), generator=g).cuda()
    x, w = randn(g, 50, 72, dtype=dtype).cuda(), randn(g, experts, 136, 72, dtype=dtype).cuda()
    around = torch.full((rows + 20, 136 + 16), 7.0, dtype=dtype, device="cuda")
    out = around[10:rows + 10, 8:144]
    out.zero_()
    iso.expert_matmul(x, w, offsets, token=token, out=out)
    assert torch.isfinite(out).all()
    out.fill_(7.0)
    assert (around == 7.0).all()
    dx, dw = iso.expert_matmul_backward(x[token.clamp(0, 49)], w, offsets, randn(g, rows, 136, dtype=dtype).cuda())
    # (dw is each expert's own; rows that two experts claim are one's, those that none does are any)
    assert dx.shape == (rows, 72) and torch.isfinite(dw).all()


def test_expert_matmul_against_differences(iso):
    """The products are linear in each operand: a difference of any step is the slope."""
    offsets, token, row, x, w, d = expert_inputs(60, 5, 2, 48, 56, F32, 4)
    o, t, r = (v.int().cuda() for v in (offsets, token, row))
    x, w, d = x.cuda(), w.cuda(), d.cuda()
    dx, dw = iso.expert_matmul_backward(x, w, o, d, token=t, row=r)
    g = gen(5)
    vx, vw = randn(g, *x.shape).cuda(), randn(g, *w.shape).cuda()
    for a, b, want in ((vx, w, (dx * vx).double().sum()), (x, vw, (dw * vw).double().sum())):
        y = iso.expert_matmul(a, b, o, token=t).double() * d.double()
        # 120 rows of 56 terms, each off by (48 + 8 + 120) u of |x| |w|'s sums (<= 48 of 4 std)
        assert abs((y.sum() - want).item()) <= 200 * U32 * (y.abs().sum().item() + 120 * 56 * 48)


# --------------------------------------------------------------------------
# Combination
# --------------------------------------------------------------------------

COMBINES = [(1, 1, 1), (1, 8, 64), (3, 2, 33), (50, 3, 100), (64, 9, 513), (129, 8, 256), (33, 32, 72), (200, 1, 1030),
            (70, 4, 4100), (300, 6, 8)]


@pytest.mark.parametrize("tokens,top,dim", COMBINES)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("more", [0, 7])
def test_combine(iso, tokens, top, dim, dtype, more):
    """`more`: rows that no token has; some entries are outside then."""
    g = gen(tokens + dim)
    rows = tokens * top + more
    y, weight, dout = randn(g, rows, dim, dtype=dtype), randn(g, tokens, top), randn(g, tokens, dim, dtype=dtype)
    row = torch.randperm(rows, generator=g)[:tokens * top].view(tokens, top)
    if more:
        row[torch.rand(tokens, top, generator=g) < 0.2] = -1
        row[0, 0] = rows
    inside = (row >= 0) & (row < rows)
    picked = torch.where(inside[:, :, None], y.double()[row.clamp(0, rows - 1)], 0.0)
    for weights in (weight, None):
        w = torch.ones(tokens, top) if weights is None else weight
        terms = picked * w.double()[:, :, None]
        want = terms.sum(1)
        bound = (top + 2) * U32 * terms.abs().sum(1) + ROUND[dtype] * want.abs() + 1e-37
        dy = torch.zeros(rows, dim, dtype=torch.float64)
        dy[row[inside]] = (w.double()[:, :, None] * dout.double()[:, None, :])[inside]
        dweight = (picked * dout.double()[:, None, :]).sum(2)
        size = (picked * dout.double()[:, None, :]).abs().sum(2)
        for i, place in enumerate((lambda t: t.cuda(), lambda t: strided(t, 3), lambda t: strided(t, 8),
                                   lambda t: at_offset(t, 1))):
            r = row.to((I32, I64)[i % 2]).cuda()
            wd = None if weights is None else weights.cuda()
            within(iso.combine_tokens(place(y), r, wd), want, bound)
            got = iso.combine_tokens_backward(place(dout), place(y), r, wd)
            within(got[0], dy, ROUND[dtype] * dy.abs() + 1e-37)
            if weights is None:
                assert got[1] is None
            else:
                within(got[1], dweight, (dim + 8) * U32 * size + 1e-37)
                only = iso.combine_tokens_backward(place(dout), place(y), r, wd, need_dy=False)
                assert only[0] is None and torch.equal(only[1], got[1])
                only = iso.combine_tokens_backward(place(dout), place(y), r, wd, need_dweight=False)
                assert only[1] is None and torch.equal(only[0], got[0])
    out = strided(torch.zeros(tokens, dim, dtype=dtype), 5)
    iso.combine_tokens(y.cuda(), r, out=out)
    assert torch.equal(out, iso.combine_tokens(y.cuda(), r))
    assert torch.isnan(out.as_strided((tokens, 5), (dim + 5, 1), dim)[:-1]).all()


@pytest.mark.parametrize("tokens", [3, 700, 5000])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_combine_gradient_of_rows_without_a_token(iso, tokens, dtype):
    """Slots that are dropped leave rows that no slot names: their gradient is zero, also where
    there are as many rows as slots and dy's memory held something."""
    g = gen(tokens)
    y, dout, w = randn(g, tokens * 2, 96, dtype=dtype), randn(g, tokens, 96, dtype=dtype), randn(g, tokens, 2)
    row = torch.randperm(tokens * 2, generator=g).view(tokens, 2)
    row[torch.rand(tokens, 2, generator=g) < 0.3] = -1
    row[0, 0], row[-1, 1] = 2 ** 31 - 1, -1
    want = torch.zeros(tokens * 2, 96, dtype=torch.float64)
    ok = (row >= 0) & (row < tokens * 2)
    want[row[ok]] = (w.double()[:, :, None] * dout.double()[:, None, :])[ok]
    filler = [torch.full_like(y, math.nan, device="cuda") for _ in range(8)]
    del filler
    r = row.int().cuda()
    got = iso.combine_tokens_backward(dout.cuda(), y.cuda(), r, w.cuda())[0]
    within(got, want, ROUND[dtype] * want.abs() + 1e-37)
    dy = torch.full((tokens * 2, 96), 7.0, device="cuda", dtype=dtype)
    ws = torch.empty(4096, dtype=torch.uint8, device="cuda")
    at = (ws.data_ptr() + 255) // 256 * 256
    d, wd = dout.cuda(), w.cuda()
    iso.isoloco_combine_tokens_backward(d.data_ptr(), 96, None, 96, iso.ISOLOCO_F32 if dtype == F32 else iso.ISOLOCO_BF16,
                                        tokens * 2, 96, r.data_ptr(), iso.ISOLOCO_I32, wd.data_ptr(), tokens, 2,
                                        dy.data_ptr(), 96, None, at, 2048, torch.cuda.current_stream().cuda_stream)
    assert torch.equal(dy, got)
    a = wanted(y.cuda())
    iso.combine_tokens(a, r, wd).backward(d)
    assert torch.equal(a.grad, got)


def test_combine_of_nothing(iso):
    y = torch.randn(5, 8, device="cuda")
    row = torch.zeros(0, 2, dtype=I32, device="cuda")
    assert iso.combine_tokens(y, row).shape == (0, 8)
    dy, dweight = iso.combine_tokens_backward(torch.empty(0, 8, device="cuda"), y, row, torch.empty(0, 2, device="cuda"))
    assert not dy.any() and dweight.shape == (0, 2)
    empty = torch.full((3, 2), 1, dtype=I32, device="cuda")
    assert not iso.combine_tokens(torch.empty(0, 8, device="cuda"), empty).any()


# --------------------------------------------------------------------------
# Distillation
# --------------------------------------------------------------------------

def distill_reference(host, t, index, scale, rest, dloss=None):
    """float64 loss, its bound, lse; and with dloss the gradient and its bound.

    The sum over the vocabulary is of float32 exponentials: a thread adds at most 64 a turn
    of 32768 columns, each is off by three roundings of its argument, weighted: d = (200 + 64
    turns) u of it (arguments of more than 40 weigh nothing).  log q and log q_r are off by
    that.  In the gradient q is off by d and its own argument's roundings, the rest's factor
    by 2 d of p_r / q_r, and p_i by its argument's."""
    x, t = host.double(), t.double()
    rows, vocab = x.shape
    z = x * scale
    ok = (index >= 0) & (index < vocab)
    at = torch.where(ok, index, 0).long()
    some = ok.any(1, keepdim=True)
    t = torch.where(ok, t, -math.inf)
    if rest == "drop":
        log_p = t - torch.logsumexp(t, 1, keepdim=True)
        log_p = torch.where(torch.isinf(t), -math.inf, log_p)
    else:
        log_p = t
    p = torch.exp(log_p)
    logq = torch.log_softmax(z, 1)
    lse = torch.logsumexp(z, 1)
    logq = torch.where((z == -math.inf) & ~torch.isnan(lse)[:, None], -math.inf, logq)
    terms = torch.where(p == 0, 0.0, p * (log_p - logq.gather(1, at)))
    loss = terms.sum(1)
    weight = p.sum(1)
    listed = torch.zeros(rows, vocab + 1, dtype=torch.bool)
    listed[torch.arange(rows)[:, None].expand_as(at), torch.where(ok, at, vocab)] = True
    listed = listed[:, :vocab]
    full = torch.zeros(rows, vocab, dtype=torch.float64).scatter_add_(1, at, torch.where(ok, p, 0.0))
    ratio = torch.zeros(rows, dtype=torch.float64)
    p_r = torch.zeros(rows, dtype=torch.float64)
    if rest == "bucket":
        log_r = torch.logsumexp(logq.masked_fill(listed, -math.inf), 1)
        left = 1 - weight
        use = (left > 0) & (log_r > -math.inf)
        loss = loss + torch.where(use, left * (torch.log(left.clamp(min=1e-300)) - log_r), 0.0)
        loss = torch.where(torch.isnan(log_r), log_r, loss)
        p_r = torch.where(use, left, 0.0)
        ratio = torch.where(use, left / torch.exp(log_r), 0.0)
        weight = torch.where(use, 1.0, weight)
    d = (200 + 64 * (vocab // 32768 + 1)) * U32
    loss = torch.where(some[:, 0], loss, 0.0)
    bound = 2 * d * weight + 2 * U32 * loss.abs() + 1e-30
    if dloss is None:
        return loss, bound, lse
    q = torch.exp(logq)
    none = ~some | (lse == -math.inf)[:, None] | (dloss == 0)[:, None]
    grad = q * weight[:, None] - full - torch.where(listed, 0.0, q * ratio[:, None])
    c = dloss.double()[:, None] * scale
    far = torch.nan_to_num((z - z.amax(1, keepdim=True)).abs(), 0.0, 0.0, 0.0).clamp(max=200)
    tail = torch.where(listed, 0.0, q * ratio[:, None])
    size = (q * weight[:, None] + tail) * (2 * d + 8 * (far + 8) * U32) + full * 200 * U32
    want = torch.where(none, 0.0, grad * c)
    return want, torch.nan_to_num(torch.where(none, 0.0, size * c.abs()))


def distill_inputs(rows, vocab, top, dtype, scale, seed, odd=False):
    g = gen(seed)
    x = randn(g, rows, vocab, std=2.0)
    x[:, vocab - vocab // 50:] = -math.inf
    t = x.double() + randn(g, rows, vocab).double() * 0.5
    t, index = torch.log_softmax(t * scale, 1).topk(top, dim=1)
    t = t.float()
    if odd:
        index[::7, top // 2] = -1                  # fewer entries
        index[1::7] = torch.tensor(-3)             # none
        index[2::7, top // 3] = vocab              # outside
        t[3::7, 0] = -math.inf                     # no probability
        if top > 1:
            index[4::7, 1] = index[4::7, 0]        # a column twice
            t[4::7, 1] -= 1.0
        x[5::7] = -math.inf                        # a student without a column
    return x.to(dtype), t, index


DISTILLS = [(1, 1, 1), (1, 3, 2), (3, 40, 40), (5, 100, 8), (9, 128, 128), (4, 511, 5), (16, 4096, 32), (7, 4097, 64),
            (5, 16385, 8), (3, 32000, 128), (130, 1000, 20), (2, 70000, 32), (1, 140001, 8), (3, 33000, 1), (3, 100003, 128), (600, 5001, 8),
            (130, 131080, 4)]


@pytest.mark.parametrize("rows,vocab,top", DISTILLS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rest", ["drop", "bucket"])
@pytest.mark.parametrize("odd", [False, True])
def test_distill(iso, rows, vocab, top, dtype, rest, odd):
    scale = 0.7 if odd else 1.0
    x, t, index = distill_inputs(rows, vocab, top, dtype, scale, rows + vocab, odd)
    g = gen(3)
    dloss = randn(g, rows)
    dloss[rows // 2] = 0.0 if odd else 1.0
    want, bound, lse = distill_reference(x, t, index, scale, rest)
    grad, size = distill_reference(x, t, index, scale, rest, dloss)
    size = size + ROUND[dtype] * grad.abs() + 1e-37
    first = None
    for i, place in enumerate((lambda v: v.cuda(), lambda v: strided(v, 3), lambda v: strided(v, 8),
                               lambda v: at_offset(v, 1))):
        dev, td, ix = place(x), t.cuda(), index.to((I64, I32)[i % 2]).cuda()
        r = iso.distill_loss(dev, td, ix, scale=scale, rest=rest)
        within(r.loss, want, bound)
        d = iso.distill_loss_backward(dev, td, ix, r.stats, dloss.cuda(), scale=scale, rest=rest)
        within(d, grad, size)
        first = first or (r, d)
        assert torch.equal(r.loss, first[0].loss) and torch.equal(d, first[1])
    there = (index >= 0).any(1) & (index < vocab).any(1) & torch.isfinite(lse)
    within(first[0].stats[:, 6].cpu()[there], lse[there], (300 * U32 + 2 * U32 * lse.abs())[there])
    # in place
    dev = x.cuda()
    d = iso.distill_loss_backward(dev, td, ix, first[0].stats, dloss.cuda(), scale=scale, rest=rest, out=dev)
    assert d is dev and torch.equal(dev, first[1])


@pytest.mark.parametrize("rest", ["drop", "bucket"])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_distill_nonfinite(iso, rest, dtype):
    """A NaN or +infinity among a row's logits or a NaN among its teacher's makes its results
    NaN; a masked column that the teacher wants, an infinite loss; other rows are as before."""
    x, t, index = distill_inputs(12, 300, 6, dtype, 1.0, 4)
    dloss = torch.ones(12, device="cuda")
    clean = iso.distill_loss(x.cuda(), t.cuda(), index.cuda(), rest=rest)
    grad = iso.distill_loss_backward(x.cuda(), t.cuda(), index.cuda(), clean.stats, dloss, rest=rest)
    x[1, 299 - 50] = math.nan
    x[2, index[2, 0]] = math.nan
    x[3, 17] = math.inf
    x[4, index[4, 1]] = math.inf
    t[5, 2] = math.nan
    x[6, index[6, 3]] = -math.inf
    x[7] = math.nan
    t[8] = math.nan
    r = iso.distill_loss(x.cuda(), t.cuda(), index.cuda(), rest=rest)
    d = iso.distill_loss_backward(x.cuda(), t.cuda(), index.cuda(), r.stats, dloss, rest=rest)
    bad, fine = [1, 2, 3, 4, 5, 7, 8], [0, 9, 10, 11]
    assert torch.isnan(r.loss[bad]).all() and torch.isnan(d[bad]).all(1).sum() >= 5 and torch.isnan(d[bad]).any(1).all()
    assert r.loss[6] == math.inf and torch.isfinite(d[6]).all()
    assert torch.equal(r.loss[fine], clean.loss[fine]) and torch.equal(d[fine], grad[fine])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("value", [-1e30, -3e38])
def test_distill_large_finite_masks(iso, dtype, value):
    """Masks that are written as a large number weigh nothing, and logits far from zero are
    as exact as others."""
    x, t, index = distill_inputs(6, 500, 8, F32, 1.0, 6)
    x = x.to(dtype)
    masked = torch.where(torch.isinf(x), torch.full_like(x, value), x)
    dloss = torch.ones(6, device="cuda")
    for rest in ("drop", "bucket"):
        a, b = (iso.distill_loss(v.cuda(), t.cuda(), index.cuda(), rest=rest) for v in (x, masked))
        assert torch.equal(a.loss, b.loss)
        da, db = (iso.distill_loss_backward(v.cuda(), t.cuda(), index.cuda(), r.stats, dloss, rest=rest)
                  for v, r in ((x, a), (masked, b)))
        assert torch.equal(da, db)
    if dtype == F32:
        # logits of multiples of 2^-6 are moved by 2^17 exactly
        y = (x * 64).round() / 64
        for rest in ("drop", "bucket"):
            a, b = (iso.distill_loss(v.cuda(), t.cuda(), index.cuda(), rest=rest) for v in (y, y + 2.0 ** 17))
            assert torch.equal(a.loss, b.loss)
            da, db = (iso.distill_loss_backward(v.cuda(), t.cuda(), index.cuda(), r.stats, dloss, rest=rest)
                      for v, r in ((y, a), (y + 2.0 ** 17, b)))
            assert torch.equal(da, db)


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rest", ["drop", "bucket"])
def test_distill_small_scale(iso, dtype, rest):
    """Masked columns weigh nothing at a scale that leaves nothing of the others' differences."""
    scale, up = 2.0 ** -123, 2.0 ** 100
    x, t, index = distill_inputs(6, 500, 8, dtype, 1.0, 8)
    t = torch.log_softmax(torch.arange(8.0).expand(6, 8), 1) - 0.5  # their sum is e^-0.5
    dloss = torch.full((6,), up)
    want, bound, _ = distill_reference(x, t, index, scale, rest)
    r = iso.distill_loss(x.cuda(), t.cuda(), index.cuda(), scale=scale, rest=rest)
    within(r.loss, want, bound)
    grad, size = distill_reference(x, t, index, scale, rest, dloss)
    d = iso.distill_loss_backward(x.cuda(), t.cuda(), index.cuda(), r.stats, dloss.cuda(), scale=scale, rest=rest)
    within(d, grad, size + ROUND[dtype] * grad.abs() + 1e-37)


def test_distill_small_rest(iso):
    """A rest of 1e-12 of the student's probability is as exact as any."""
    x = torch.full((1, 1000), -30.0)
    x[0, :4] = torch.tensor([3.0, 2.0, 1.0, 0.0])
    index = torch.arange(4)[None]
    t = torch.log(torch.tensor([[0.5, 0.25, 0.125, 0.0625]]))
    want, bound, _ = distill_reference(x, t, index, 1.0, "bucket")
    r = iso.distill_loss(x.cuda(), t.cuda(), index.cuda(), rest="bucket")
    within(r.loss, want, bound)
    grad, size = distill_reference(x, t, index, 1.0, "bucket", torch.ones(1))
    within(iso.distill_loss_backward(x.cuda(), t.cuda(), index.cuda(), r.stats, torch.ones(1, device="cuda"),
                                     rest="bucket"), grad, size + 2 * U32 * grad.abs())


def test_distill_of_the_teacher_itself(iso):
    """What token_logprobs gives of the same logits: no loss with the rest as a bucket, and
    no gradient beyond the rounding of the probabilities; without it what the listed tokens
    leave of one."""
    z = randn(gen(7), 40, 3000, std=3.0).cuda()
    for k in (1, 8, 32):
        teacher = iso.token_logprobs(z, scale=0.5, top_k=k)
        for rest in ("drop", "bucket"):
            r = iso.distill_loss(z, teacher.top_logprob, teacher.top_index, scale=0.5, rest=rest)
            none = torch.zeros(40, dtype=torch.float64)
            want = none if rest == "bucket" else -torch.logsumexp(teacher.top_logprob.cpu().double(), 1)
            # log p is off by (200 + 64) u, times what sums to 1, in either call
            within(r.loss, want, 600 * U32 + 2 * U32 * want.abs())
            within(r.stats[:, 6], teacher.lse.cpu(), 4 * U32 * teacher.lse.abs().cpu() + 300 * U32)
            if rest == "bucket":
                d = iso.distill_loss_backward(z, teacher.top_logprob, teacher.top_index, r.stats,
                                              torch.ones(40, device="cuda"), scale=0.5, rest=rest)
                assert d.abs().max().item() <= 1000 * U32


def test_distill_against_differences(iso):
    x, t, index = distill_inputs(30, 200, 6, F32, 1.0, 11)
    v = randn(gen(12), 30, 200).cuda()
    x, t, index = x.cuda(), t.cuda(), index.cuda()
    one = torch.ones(30, device="cuda")
    h = 2.0 ** -7
    for rest in ("drop", "bucket"):
        r = iso.distill_loss(x, t, index, rest=rest)
        up, down = (iso.distill_loss(x + e * h * v, t, index, rest=rest).loss for e in (1, -1))
        slope = (up - down).double() / (2 * h)
        d = iso.distill_loss_backward(x, t, index, r.stats, one, rest=rest).double()
        along = (torch.where(torch.isinf(x), 0.0, d) * v.double()).sum(1)
        # third cumulants of a softmax along v (|v| <= 5), and rounding of the losses and of x + h v
        bound = 2 * h * h * v.abs().amax(1).double() ** 3 + (8 * r.loss.abs().double() + 40) * U32 / h
        assert ((slope - along).abs() <= bound).all()


def test_distill_shapes(iso):
    z = torch.randn(2, 3, 50, device="cuda")
    teacher = iso.token_logprobs(torch.randn(2, 3, 50, device="cuda"), top_k=4)
    r = iso.distill_loss(z, teacher.top_logprob, teacher.top_index)
    assert r.loss.shape == (2, 3) and r.stats.shape == (2, 3, iso.ISOLOCO_DISTILL_STATS)
    e = iso.distill_loss(z[:0], teacher.top_logprob[:0], teacher.top_index[:0])
    assert e.loss.shape == (0, 3)
    with pytest.raises(ValueError):
        iso.distill_loss(z, teacher.top_logprob[..., :2], teacher.top_index)
    with pytest.raises(ValueError):
        iso.distill_loss(z, teacher.top_logprob, teacher.top_index, rest="other")


# --------------------------------------------------------------------------
# Together
# --------------------------------------------------------------------------

def _step(iso, s, row_type=I32):
    """A block of experts and the distillation of its logits, with every gradient."""
    r = iso.route_tokens(s["scores"], 3)
    h = iso.expert_matmul(s["x"], s["w1"], r.offsets, token=r.token)
    y = iso.expert_matmul(h, s["w2"], r.offsets)
    out = iso.combine_tokens(y, r.row, r.weight)
    teacher = iso.token_logprobs(s["teacher"], top_k=6)
    loss = iso.distill_loss(out, teacher.top_logprob, teacher.top_index, rest="bucket")
    dout = iso.distill_loss_backward(out, teacher.top_logprob, teacher.top_index, loss.stats, s["dl"], rest="bucket")
    dy, dweight = iso.combine_tokens_backward(dout, y, r.row, r.weight)
    dh, dw2 = iso.expert_matmul_backward(h, s["w2"], r.offsets, dy)
    dx, dw1 = iso.expert_matmul_backward(s["x"], s["w1"], r.offsets, dh, token=r.token, row=r.row)
    dscores = iso.route_tokens_backward(s["scores"], r.expert, dweight)
    norm = iso.clip_grads([dw1, dw2], 1e-3)
    return [*r, h, y, out, loss.loss, loss.stats, dout, dy, dweight, dh, dw2, dx, dw1, dscores, norm]


def _state(dtype, tokens):
    g = gen(6)
    scores = randn(g, tokens, 9, dtype=dtype)
    scores[0] = -math.inf
    return {k: v.cuda() for k, v in dict(
        scores=scores, x=randn(g, tokens, 72, dtype=dtype), w1=randn(g, 9, 136, 72, std=0.1, dtype=dtype),
        w2=randn(g, 9, 200, 136, std=0.1, dtype=dtype), teacher=randn(g, tokens, 200, dtype=dtype),
        dl=randn(g, tokens)).items()}


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tokens", [3, 300])
def test_streams_and_determinism(iso, dtype, tokens):
    s = _state(dtype, tokens)
    first = _step(iso, s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = _step(iso, s)
    side.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)
    third = iso.expert_matmul(s["x"], s["w1"], first[4], token=first[3], stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(third, first[5])


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tokens", [2, 300])
def test_graph_replays(iso, dtype, tokens):
    """The grouping is read on the device: replays follow scores that change it."""
    s = _state(dtype, tokens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(iso, s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = _step(iso, s)
    for turn in range(4):
        s["scores"].copy_(randn(gen(50 + turn), tokens, 9, std=1.0 + turn, dtype=dtype))
        s["dl"].mul_(-1.5)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        eager = _step(iso, s)
        torch.cuda.synchronize()
        for a, b in zip(got, eager):
            assert torch.equal(a, b)


def wanted(t):
    return t.detach().clone().requires_grad_()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_autograd_reaches_every_operand(iso, dtype):
    s = _state(dtype, 200)
    scores, x, w1, w2 = (wanted(s[k]) for k in ("scores", "x", "w1", "w2"))
    r = iso.route_tokens(scores, 3)
    h = iso.expert_matmul(x, w1, r.offsets, token=r.token, row=r.row)
    y = iso.expert_matmul(h, w2, r.offsets)
    out = iso.combine_tokens(y, r.row, r.weight)
    teacher = iso.token_logprobs(s["teacher"], top_k=6)
    loss = iso.distill_loss(out, teacher.top_logprob, teacher.top_index, rest="bucket")
    assert not r.row.requires_grad and not loss.stats.requires_grad
    (loss.loss * s["dl"]).sum().backward()
    got = _step(iso, s)
    assert torch.equal(out, got[7]) and torch.equal(loss.loss, got[8])
    norm = got[-1]
    for leaf, want in ((w2, got[14]), (x, got[15]), (w1, got[16]), (scores, got[17])):
        if leaf.dim() == 3:  # clipped in place by the step
            assert torch.equal(iso.clip_grads([w1.grad.clone(), w2.grad.clone()], 1e-3), norm)
            continue
        assert torch.equal(leaf.grad, want)


def test_autograd_against_64_bits(iso):
    """The chain in float32 against torch's gradients of the same formulas in 64 bits.  Each
    of its 12 products and sums is off by less than 250 u of its norm, and the loss's
    curvature carries an error on with a factor of at most 2 a stage: 12 * 250 * 2^4 u = 2.9e-3
    in the worst case, of which rounding errors that are independent leave their square root's
    share: 1e-4."""
    s = _state(F32, 120)
    scores, x, w1, w2 = (wanted(s[k][1:] if k in ("scores", "x") else s[k]) for k in ("scores", "x", "w1", "w2"))
    teacher = iso.token_logprobs(s["teacher"][1:], top_k=6)
    r = iso.route_tokens(scores, 3)
    h = torch.nn.functional.silu(iso.expert_matmul(x, w1, r.offsets, token=r.token, row=r.row))
    out = iso.combine_tokens(iso.expert_matmul(h, w2, r.offsets), r.row, r.weight)
    iso.distill_loss(out, teacher.top_logprob, teacher.top_index, rest="drop").loss.sum().backward()
    S, X, A, B = (t.detach().cpu().double().requires_grad_() for t in (scores, x, w1, w2))
    z, e = S.topk(3, dim=1)
    rows = torch.einsum("tjfd,td->tjf", A[e], X)
    o = (torch.einsum("tjdf,tjf->tjd", B[e], torch.nn.functional.silu(rows)) * torch.softmax(z, 1)[:, :, None]).sum(1)
    logp = torch.log_softmax(teacher.top_logprob.cpu().double(), 1)
    logq = torch.log_softmax(o, 1).gather(1, teacher.top_index.cpu())
    (torch.exp(logp) * (logp - logq)).sum().backward()
    for got, want in ((scores, S), (x, X), (w1, A), (w2, B)):
        rel = (got.grad.cpu().double() - want.grad).norm() / want.grad.norm()
        assert rel.item() < 1e-4


def test_autograd_of_some_operands(iso):
    s = _state(F32, 40)
    r = iso.route_tokens(s["scores"], 2)
    t = dict(token=r.token, row=r.row)
    d = torch.randn(136, 80, device="cuda").t()
    dx, dw = iso.expert_matmul_backward(s["x"], s["w1"], r.offsets, d.contiguous(), **t)
    x = wanted(s["x"])
    iso.expert_matmul(x, s["w1"], r.offsets, **t).backward(d)
    assert torch.equal(x.grad, dx)
    w = wanted(s["w1"])
    iso.expert_matmul(s["x"], w, r.offsets, token=r.token).backward(d)
    assert torch.equal(w.grad, dw)
    y = torch.randn(80, 30, device="cuda")
    g = torch.randn(30, 40, device="cuda").t()
    dy, dweight = iso.combine_tokens_backward(g.contiguous(), y, r.row, r.weight)
    a, b = wanted(y), wanted(r.weight)
    iso.combine_tokens(a, r.row, r.weight).backward(g)
    iso.combine_tokens(y, r.row, b).backward(g)
    assert torch.equal(a.grad, dy) and torch.equal(b.grad, dweight)
    a = wanted(y)
    iso.combine_tokens(a, r.row).backward(g)
    assert torch.equal(a.grad, iso.combine_tokens_backward(g.contiguous(), y, r.row)[0])
    z = wanted(torch.randn(2, 3, 50, device="cuda"))
    teacher = iso.token_logprobs(torch.randn(2, 3, 50, device="cuda"), top_k=4)
    loss = iso.distill_loss(z, teacher.top_logprob, teacher.top_index)
    loss.loss.mean().backward()
    want = iso.distill_loss_backward(z.detach(), teacher.top_logprob, teacher.top_index, loss.stats,
                                     torch.full((2, 3), 1 / 6, device="cuda"))
    assert torch.equal(z.grad, want)


def test_autograd_refuses_what_it_lacks(iso):
    s = _state(F32, 10)
    r = iso.route_tokens(s["scores"], 2)
    x = wanted(s["x"])
    with pytest.raises(ValueError):
        iso.expert_matmul(x, s["w1"], r.offsets, token=r.token)
    with pytest.raises(ValueError):
        iso.expert_matmul(x, s["w1"], r.offsets, token=r.token, row=r.row, out=torch.empty(20, 136, device="cuda"))
    with pytest.raises(ValueError):
        iso.combine_tokens(wanted(s["x"]), r.row, out=torch.empty(10, 72, device="cuda"))
    z = wanted(torch.randn(10, 50, device="cuda"))
    top, index = torch.randn(10, 3, device="cuda"), torch.zeros(10, 3, dtype=I64, device="cuda")
    with pytest.raises(ValueError):
        iso.distill_loss(z, wanted(top), index)
    # a result may be written before its gradient is formed
    loss = iso.distill_loss(z, top, index).loss
    loss.mul_(2.0)
    loss.sum().backward()
    r = iso.distill_loss(z.detach(), top, index)
    assert torch.equal(z.grad, iso.distill_loss_backward(z.detach(), top, index, r.stats, torch.full((10,), 2.0, device="cuda")))
    # but not what the gradient takes
    q = wanted(torch.randn(10, 50, device="cuda")) * 1.0
    loss = iso.distill_loss(q, top, index).loss.sum()
    iso.distill_loss_backward(q.detach(), top, index, r.stats, torch.ones(10, device="cuda"), out=q.detach())
    with pytest.raises(RuntimeError):
        loss.backward()


# --------------------------------------------------------------------------
# Past 32 bits
# --------------------------------------------------------------------------

def test_distill_past_32_bits(iso):
    rows, vocab = 70000, 32003
    z = torch.empty(rows, vocab, dtype=BF16, device="cuda")
    for a in range(0, rows, 7000):
        z[a:a + 7000].normal_()
    pick = torch.tensor([0, 1, 33000, 67106, 67108, rows - 1], device="cuda")
    index = torch.randint(0, vocab, (rows, 4), device="cuda")
    t = torch.log_softmax(torch.randn(rows, 4, device="cuda"), 1)
    dl = torch.randn(rows, device="cuda")
    r = iso.distill_loss(z, t, index)
    part = iso.distill_loss(z[pick], t[pick], index[pick])
    # (few rows may be split: their sums are added in another order)
    assert (r.loss[pick] - part.loss).abs().max().item() <= 600 * U32 * 10
    d = iso.distill_loss_backward(z, t, index, r.stats, dl)
    want = iso.distill_loss_backward(z[pick], t[pick], index[pick], r.stats[pick], dl[pick])
    assert torch.equal(d[pick], want)


def test_expert_rows_past_32_bits(iso):
    """x, out and dx of more than 2^32 bytes, gathered and grouped."""
    rows, dim, cols = 1100000, 2048, 16
    x = torch.empty(rows, dim, dtype=BF16, device="cuda")
    for a in range(0, rows, 100000):
        x[a:a + 100000].normal_()
    w = torch.randn(3, cols, dim, device="cuda").to(BF16)
    o = torch.tensor([0, 300000, 1090000, rows], dtype=I32, device="cuda")
    out = iso.expert_matmul(x, w, o)
    pick = torch.tensor([0, 5, 299999, 300000, 1089999, 1090000, rows - 1], device="cuda")
    po = torch.tensor([0, 3, 5, 7], dtype=I32, device="cuda")
    want, size = expert_reference(x[pick].cpu(), w.cpu(), po.cpu())
    bound = (dim + 8) * U32 * size + ROUND[BF16] * want.abs()
    within(out[pick], want, bound)
    token = torch.randint(rows - 1000, rows, (500,), device="cuda", dtype=I32)
    go = torch.tensor([0, 100, 100, 500], dtype=I32, device="cuda")
    got = iso.expert_matmul(x, w, go, token=token)
    want, size = expert_reference(x[token.long()].cpu(), w.cpu(), go.cpu())
    within(got, want, (dim + 8) * U32 * size + ROUND[BF16] * want.abs())
    d = torch.randn(rows, cols, device="cuda").to(BF16)
    dx, dw = iso.expert_matmul_backward(x, w, o, d)
    px = expert_reference(x[pick].cpu(), w.cpu(), po.cpu(), d[pick].cpu())
    within(dx[pick], px[0], (cols + 8) * U32 * px[1] + ROUND[BF16] * px[0].abs())
    tail = slice(1090000, rows)
    want = d[tail].double().t() @ x[tail].double()
    # 10000 terms of |d| |x|, each of about 0.64 on average
    assert (dw[2].double() - want).abs().max().item() <= (10000 + 8) * U32 * 10000 + 2 ** -8 * want.abs().max().item()
    dwg = iso.expert_matmul_backward(x, w, go, d[:500], token=token, need_dx=False)[1]
    want = d[100:500].double().t() @ x[token[100:].long()].double()
    assert (dwg[2].double() - want).abs().max().item() <= 408 * U32 * 400 * 4 + 2 ** -8 * want.abs().max().item()


def test_combine_past_32_bits(iso):
    rows, dim = 1100000, 2048
    y = torch.empty(rows, dim, dtype=BF16, device="cuda")
    for a in range(0, rows, 100000):
        y[a:a + 100000].normal_()
    row = torch.randperm(rows, device="cuda").view(-1, 2).int()
    w = torch.rand(rows // 2, 2, device="cuda")
    out = iso.combine_tokens(y, row, w)
    pick = torch.tensor([0, 77, rows // 2 - 1], device="cuda")
    want = iso.combine_tokens(y[row[pick].long().flatten()], torch.arange(6, device="cuda").view(3, 2), w[pick])
    assert torch.equal(out[pick], want)
    dy, dweight = iso.combine_tokens_backward(out, y, row, w)
    small = iso.combine_tokens_backward(out[pick], y[row[pick].long().flatten()], torch.arange(6, device="cuda").view(3, 2),
                                        w[pick])
    assert torch.equal(dy[row[pick].long().flatten()], small[0]) and torch.equal(dweight[pick], small[1])


# --------------------------------------------------------------------------
# Every instance of the products
# --------------------------------------------------------------------------

@pytest.mark.parametrize("case", range(len(CASES)))
def test_expert_products(iso, case):
    """Larger products against torch's in 64 bits on the GPU: uneven experts, one without rows,
    some rows behind the last one's, rows as they lie and gathered."""
    kind, experts, rows, dim, cols, _ = CASES[case]
    dtype = BF16 if kind == "bf16" else F32
    g = torch.Generator(device="cuda")
    g.manual_seed(case)

    def randn(*shape, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    want = torch.rand(experts, generator=g, device="cuda") + 0.2
    want[experts // 2] = 0.0
    sizes = torch.multinomial(want, rows - 37, replacement=True, generator=g).bincount(minlength=experts)
    offsets = torch.zeros(experts + 1, dtype=I64, device="cuda")
    offsets[1:] = sizes.cumsum(0)
    tokens, last = rows // 2 + 1, rows - 37
    x, token = randn(tokens, dim), torch.randint(0, tokens, (rows,), generator=g, device="cuda")
    w, d = randn(experts, cols, dim, std=dim ** -0.5), randn(rows, cols)
    flat = x[token].contiguous()
    out = iso.expert_matmul(flat, w, offsets)
    assert torch.equal(iso.expert_matmul(x, w, offsets, token=token), out)
    dx, dw = iso.expert_matmul_backward(flat, w, offsets, d)
    assert torch.equal(iso.expert_matmul_backward(x, w, offsets, d, token=token, need_dx=False)[1], dw)
    assert torch.equal(iso.expert_matmul_backward(flat, w, offsets, d, need_dw=False)[0], dx)
    row = torch.full((tokens, 1), -1, dtype=I64, device="cuda")
    assert torch.equal(iso.expert_matmul_backward(x, w, offsets, d, token=token, row=row)[1], dw)
    assert not out[last:].any() and not dx[last:].any()
    for e in range(experts):
        a, b = int(offsets[e]), int(offsets[e + 1])
        X, W, D = flat[a:b].double(), w[e].double(), d[a:b].double()
        for got, want, size, n in ((out[a:b], X @ W.T, X.abs() @ W.abs().T, dim), (dx[a:b], D @ W, D.abs() @ W.abs(), cols),
                                   (dw[e], D.T @ X, D.abs().T @ X.abs(), b - a)):
            # (float32: the 6 products of parts are as many sums)
            bound = ((6 if dtype == F32 else 1) * n + 8) * U32 * size + ROUND[dtype] * want.abs() + 1e-37
            assert ((got.double() - want).abs() <= bound).all()


def test_expert_matmul_wide_experts(iso):
    """More experts than a wave has lanes, on the tiles: experts are found 64 at a time."""
    g = gen(12)
    experts, rows = 300, 9000
    offsets, token, row = grouped(g, rows, experts, 1)
    x, w, d = randn(g, rows, 64, dtype=BF16), randn(g, experts, 72, 64, std=0.125, dtype=BF16), randn(g, rows, 72, dtype=BF16)
    want, size = expert_reference(x[token], w, offsets)
    o, t, r = (v.int().cuda() for v in (offsets, token, row))
    within(iso.expert_matmul(x.cuda(), w.cuda(), o, token=t), want, 72 * U32 * size + ROUND[BF16] * want.abs())
    dx, dxs, dw, dws = expert_reference(x[token], w, offsets, d)
    got = iso.expert_matmul_backward(x[token].cuda(), w.cuda(), o, d.cuda())
    within(got[0], dx, 80 * U32 * dxs + ROUND[BF16] * dx.abs())
    n = torch.diff(offsets).double()[:, None, None]
    within(got[1], dw, (n + 8) * U32 * dws + ROUND[BF16] * dw.abs() + 1e-37)
