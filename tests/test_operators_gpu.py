"""The inner step's operators against plain implementations in 64 bits (CPU), at
the sizes, strides and masks where they can go wrong.

Tolerances.  u = 2^-24 is the rounding of float32 and 2^-9 that of bfloat16.  A sum
of n float32 terms is off by at most n u times the sum of their magnitudes, so the
bounds of products are those of the absolute values' products; each test says the
rest of its own.
"""
import math

import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

U32 = 2.0 ** -24
ROUND = {torch.float32: 2 * U32, torch.bfloat16: 2.0 ** -8}  # of an output, doubled for the float32 value before it
F32, BF16 = torch.float32, torch.bfloat16


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
    """A copy of the matrix t whose rows are `pad` elements further apart, NaN between them."""
    big = torch.full((t.shape[0], t.shape[1] + pad), math.nan, dtype=t.dtype, device=dev)
    big[:, :t.shape[1]].copy_(t)
    return big[:, :t.shape[1]]


# --------------------------------------------------------------------------
# Clipping
# --------------------------------------------------------------------------

def clip_reference(grads, max_norm):
    """float64: the norm, the coefficient and the scaled tensors."""
    norm = math.sqrt(sum(float(g.double().square().sum()) for g in grads))
    coef = max_norm / norm if max_norm < norm < math.inf else 1.0
    return norm, coef, [g.double() * coef for g in grads]


CLIP_SETS = {
    "one element": ([(1,)], [F32]),
    "an empty tensor among others": ([(0,), (7, 3), (0, 5), (16,)], [F32, BF16, BF16, F32]),
    "odd sizes": ([(5, 7), (33,), (1,), (1023, 3), (129,), (2049, 17)], [F32, BF16, F32, BF16, F32, F32]),
    "a chunk and its neighbours": ([(8191,), (8192,), (8193,), (16383,), (16384,), (16385,)], [F32, F32, F32, BF16, BF16, BF16]),
    "more tensors than a launch takes": ([(3 + i % 5, 11) for i in range(300)], [F32, BF16, BF16]),
    "large": ([(2048, 2048), (300, 1000), (4097,)], [BF16, F32, F32]),
}


@pytest.mark.parametrize("name", sorted(CLIP_SETS))
@pytest.mark.parametrize("in_place", [False, True])
def test_clip(iso, name, in_place):
    shapes, dtypes = CLIP_SETS[name]
    g = gen(3)
    host = [randn(g, *s, dtype=dtypes[i % len(dtypes)]) for i, s in enumerate(shapes)]
    norm, _, _ = clip_reference(host, 1.0)
    for max_norm in (0.25 * norm, 4.0 * norm, 0.0, math.inf):
        # every tensor at an alignment of its own
        dev = [at_offset(t, i % 8) for i, t in enumerate(host)]
        outs = None if in_place else [at_offset(torch.full_like(t, 7.0), (3 * i) % 8) for i, t in enumerate(host)]
        got = iso.clip_grads(dev, max_norm, out=outs)
        norm, coef, want = clip_reference(host, max_norm)
        # the norm and the coefficient are formed in 64 bits and rounded once
        within(got, torch.tensor([norm, coef], dtype=torch.float64), 2 * U32 * torch.tensor([norm, coef]))
        for t, h, w in zip(dev if in_place else outs, host, want):
            within(t, w, ROUND[h.dtype] * w.abs() + 1e-38)
            if coef == 1.0:
                assert torch.equal(t.cpu(), h)
        if not in_place:
            assert all(torch.equal(t.cpu(), h) for t, h in zip(dev, host))


def test_clip_neighbours_untouched(iso):
    """Clipping views of a flat buffer leaves what stands between them."""
    flat = torch.full((1000,), 5.0, device="cuda", dtype=BF16)
    views = [flat[1:38], flat[41:42], flat[77:910]]
    for v in views:
        v.fill_(2.0)
    iso.clip_grads(views, 1.0)
    keep = torch.ones(1000, dtype=torch.bool)
    for a, b in ((1, 38), (41, 42), (77, 910)):
        keep[a:b] = False
    host = flat.cpu().float()
    assert (host[keep] == 5.0).all() and (host[~keep] < 0.1).all()


@pytest.mark.parametrize("value", [1e30, 1e-30, 3e38])
def test_clip_range(iso, value):
    """Squares that leave the range of 32 bits."""
    t = torch.full((1000,), value, device="cuda")
    norm = iso.clip_grads([t], value)
    want = value * math.sqrt(1000.0)
    got = norm.cpu().double()
    if want > 3.4e38:
        assert got[0].item() == math.inf
    else:
        assert abs(got[0].item() / want - 1) <= 1e-6
    assert abs(got[1].item() * math.sqrt(1000.0) - 1) <= 1e-6
    within(t, torch.full((1000,), value / math.sqrt(1000.0), dtype=torch.float64), 1e-6 * value)


@pytest.mark.parametrize("max_norm", [1.0, 1e-3, 1e-10, 1e-37])
@pytest.mark.parametrize("in_place", [False, True])
def test_clip_small_coefficients(iso, max_norm, in_place):
    """Coefficients below float32's normal range, applied to gradients near its top (and to
    some that vanish)."""
    g = gen(4)
    host = [randn(g, 1000, std=1e38).clamp(-3e38, 3e38), randn(g, 37, std=1e38, dtype=BF16),
            torch.tensor([1e-10, 1.0, 1e30, -3e38, 0.0])]
    norm, coef, want = clip_reference(host, float(torch.tensor(max_norm, dtype=F32)))
    assert coef < 2.0 ** -126
    dev = [t.cuda() for t in host]
    outs = None if in_place else [torch.empty_like(t) for t in dev]
    got = iso.clip_grads(dev, max_norm, out=outs)
    within(got[1:], torch.tensor([coef], dtype=torch.float64), 2.0 ** -149)
    for t, h, w in zip(dev if in_place else outs, host, want):
        # two products, then the result's own rounding; below 2^-126 a value's steps are 2^-149 (2^-133) apart
        within(t, w, (ROUND[h.dtype] + 2 * U32) * w.abs() + (2.0 ** -148 if h.dtype == F32 else 2.0 ** -133))


@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_clip_nonfinite(iso, bad):
    host = [randn(gen(1), 100), randn(gen(2), 40, dtype=BF16)]
    host[1][17] = bad
    dev = [t.cuda() for t in host]
    norm = iso.clip_grads(dev, 1.0).cpu()
    assert (math.isnan(norm[0].item()) if math.isnan(bad) else norm[0].item() == math.inf) and norm[1].item() == 1.0
    for t, h in zip(dev, host):
        assert torch.equal(t.cpu().view(torch.int16), h.view(torch.int16))


@pytest.mark.parametrize("name", sorted(CLIP_SETS))
def test_clip_norm_only(iso, name):
    """Without results the norm has a launch of its own, and nothing is scaled."""
    shapes, dtypes = CLIP_SETS[name]
    g = gen(12)
    host = [randn(g, *s, dtype=dtypes[i % len(dtypes)]) for i, s in enumerate(shapes)]
    dev = [at_offset(t, i % 8) for i, t in enumerate(host)]
    types = [iso.ISOLOCO_F32 if t.dtype == F32 else iso.ISOLOCO_BF16 for t in dev]
    ws = torch.empty(iso.isoloco_clip_workspace_size(len(dev)), dtype=torch.uint8, device="cuda")
    for share in (0.25, 4.0):
        norm, coef, _ = clip_reference(host, share * clip_reference(host, 1.0)[0])
        got = torch.empty(2, device="cuda")
        iso.isoloco_clip_grads([t.data_ptr() for t in dev], None, [t.numel() for t in dev], types, share * norm,
                               got.data_ptr(), ws.data_ptr(), ws.numel(), torch.cuda.current_stream().cuda_stream)
        within(got, torch.tensor([norm, coef], dtype=torch.float64), 2 * U32 * torch.tensor([norm, coef]))
        assert all(torch.equal(t.cpu(), h) for t, h in zip(dev, host))


def test_clip_of_nothing(iso):
    """Tensors that hold no element: norm 0, coefficient 1."""
    empty = torch.empty(0, 5, device="cuda")
    assert iso.clip_grads([empty, empty.bfloat16()], 1.0).tolist() == [0.0, 1.0]


def test_clip_past_32_bits(iso):
    n = 2 ** 31 + 4099
    t = torch.zeros(n, dtype=BF16, device="cuda")
    t[0], t[2 ** 31 + 5], t[n - 1] = 3.0, 4.0, 12.0
    out = torch.empty_like(t)
    norm = iso.clip_grads([t], 6.5, out=[out]).cpu()
    assert norm.tolist() == [13.0, 0.5]
    assert [out[i].item() for i in (0, 2 ** 31 + 5, n - 1)] == [1.5, 2.0, 6.0]
    assert out.count_nonzero().item() == 3


# --------------------------------------------------------------------------
# Embedding
# --------------------------------------------------------------------------

def some_ids(g, n, vocab, dtype=torch.int64):
    """Skewed ids, some of them no tokens."""
    ids = (torch.rand(n, generator=g, dtype=torch.float64).pow(3) * vocab).long().clamp(max=vocab - 1)
    if n > 4:
        ids[n // 3], ids[n // 2] = -1, vocab
    return ids.to(dtype)


@pytest.mark.parametrize("dim", [1, 7, 64, 511, 513, 768, 1030])
@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (F32, BF16), (BF16, BF16), (BF16, F32)])
def test_embedding(iso, dim, dtype, out_dtype):
    g = gen(dim)
    vocab, n = 301, 75
    table, ids = randn(g, vocab, dim, dtype=dtype), some_ids(g, n, vocab, torch.int32 if dim % 2 else torch.int64)
    ok = (ids >= 0) & (ids < vocab)
    want = torch.where(ok[:, None], table[ids.long().clamp(0, vocab - 1)].double() * 0.7, 0.0)
    bound = ROUND[out_dtype] * want.abs() + U32 * 0.7 * want.abs()  # 0.7 is rounded too
    for t in (table.cuda(), at_offset(table, 1), strided(table, 3)):
        out = iso.embedding(t, ids.cuda(), scale=0.7, out_dtype=out_dtype)
        within(out, want, bound)
    into = strided(torch.zeros(n, dim, dtype=out_dtype), 5)
    assert iso.embedding(t, ids.cuda(), scale=0.7, out=into) is into
    within(into, want, bound)
    assert torch.isnan(into.as_strided((n, 5), (dim + 5, 1), dim)[:-1]).all()


@pytest.mark.parametrize("n", [0, 1])
def test_embedding_few(iso, n):
    table = randn(gen(0), 10, 20).cuda()
    ids = torch.full((n,), 9, device="cuda")
    assert torch.equal(iso.embedding(table, ids), table[ids])
    ids = torch.full((2, n, 3), 4, device="cuda")
    assert torch.equal(iso.embedding(table, ids), table[ids])


def embedding_grad_reference(ids, dout, vocab, scale, base=None):
    """float64 gradient and the bound of its rounding: a row's sum of c terms."""
    ok = (ids >= 0) & (ids < vocab)
    i = ids[ok].long()
    d = torch.zeros(vocab, dout.shape[1], dtype=torch.float64)
    a, c = d.clone(), torch.zeros(vocab, 1, dtype=torch.float64)
    d.index_add_(0, i, dout[ok].double())
    a.index_add_(0, i, dout[ok].double().abs())
    c.index_add_(0, i, torch.ones(len(i), 1, dtype=torch.float64))
    d, a = d * scale, a * abs(scale)
    if base is not None:
        d, a = d + base.double(), a + base.double().abs()
    return d, (c + 3) * U32 * a


EMBED_GRADS = [
    # n, vocab, dim
    (0, 10, 8), (1, 1, 1), (1, 300, 33), (64, 5, 16), (65, 1, 130), (200, 257, 7),
    (1000, 3, 513), (4000, 32000, 64), (5000, 70, 96), (3000, 1500000, 2), (20000, 1000, 40),
]


@pytest.mark.parametrize("n,vocab,dim", EMBED_GRADS)
@pytest.mark.parametrize("dtype,out_dtype", [(F32, F32), (BF16, F32), (BF16, BF16), (F32, BF16)])
def test_embedding_backward(iso, n, vocab, dim, dtype, out_dtype):
    g = gen(n + dim)
    ids, dout = some_ids(g, n, vocab, torch.int32 if n % 2 else torch.int64), randn(g, n, dim, dtype=dtype)
    want, bound = embedding_grad_reference(ids, dout, vocab, 1.5)
    bound = bound + ROUND[out_dtype] * want.abs()
    got = iso.embedding_backward(ids.cuda(), dout.cuda(), vocab, scale=1.5, out_dtype=out_dtype)
    within(got, want, bound)
    again = iso.embedding_backward(ids.cuda(), strided(dout, 1), vocab, scale=1.5, out_dtype=out_dtype)
    assert torch.equal(got, again)
    if vocab < 100000:
        base = randn(g, vocab, dim, dtype=out_dtype)
        into = strided(base, 2)
        iso.embedding_backward(ids.cuda(), dout.cuda(), vocab, scale=1.5, out=into, accumulate=True)
        want, bound = embedding_grad_reference(ids, dout, vocab, 1.5, base)
        within(into, want, bound + ROUND[out_dtype] * want.abs())


@pytest.mark.parametrize("n", [63, 64, 65, 128, 129, 4097, 70000])
def test_embedding_backward_one_id(iso, n):
    """All tokens the same, and two ids that share pieces of the order at every offset."""
    dim, vocab = 10, 600
    dout = randn(gen(n), n, dim)
    for ids in (torch.full((n,), 3), torch.where(torch.arange(n) < n // 3, 3, 3 + 256),
                torch.where(torch.arange(n) % 3 == 1, 599, 87)):
        want, bound = embedding_grad_reference(ids, dout, vocab, 1.0)
        within(iso.embedding_backward(ids.cuda(), dout.cuda(), vocab), want, bound + 2 * U32 * want.abs())


def test_embedding_backward_no_tokens(iso):
    """Ids that hold no token give no gradient, whatever stands in their rows."""
    ids = torch.tensor([-1, 2, -7, 10, 2 ** 40], device="cuda")
    dout = torch.full((5, 4), math.nan, device="cuda")
    dout[1] = 1.0
    got = iso.embedding_backward(ids, dout, 10).cpu()
    assert torch.equal(got.nonzero()[:, 0].unique(), torch.tensor([2])) and (got[2] == 1).all()
    ids.fill_(-1)
    assert iso.embedding_backward(ids, dout, 10).count_nonzero().item() == 0


def test_embedding_past_32_bits(iso):
    vocab, dim = 1050000, 2048
    table = torch.zeros(vocab, dim, dtype=BF16, device="cuda")
    table[vocab - 1] = 3.0
    ids = torch.tensor([vocab - 1, 0, vocab - 1], device="cuda")
    out = iso.embedding(table, ids, scale=2.0)
    assert (out[0] == 6).all() and (out[1] == 0).all() and (out[2] == 6).all()
    iso.embedding_backward(ids, out, vocab, out=table)
    assert (table[vocab - 1] == 12).all() and table[:vocab - 1].count_nonzero().item() == 0


def test_embedding_gradient_against_differences(iso):
    """The lookup is linear in the table: <w, out(T + V)> - <w, out(T)> = <grad, V>."""
    g = gen(8)
    table, v = randn(g, 50, 24), randn(g, 50, 24)
    ids, w = some_ids(g, 90, 50).cuda(), randn(g, 90, 24)
    a, b = (iso.embedding(t.cuda(), ids, scale=1.3).cpu().double() for t in (table, table + v))
    grad = iso.embedding_backward(ids, w.cuda(), 50, scale=1.3).cpu().double()
    lhs, rhs = ((b - a) * w.double()).sum(), (grad * v.double()).sum()
    assert abs(lhs - rhs) <= 90 * 24 * 8 * U32 * (w.double().abs() * (a.abs() + b.abs() + 1)).mean()


# --------------------------------------------------------------------------
# Token log probabilities
# --------------------------------------------------------------------------

def logprob_reference(logits, targets, scale, top):
    z = logits.double() * float(torch.tensor(scale, dtype=F32))
    m = z.amax(1)
    m = torch.where(m == -math.inf, torch.zeros_like(m), m)
    log_s = torch.logsumexp(z - m[:, None], 1)  # (infinity less itself: NaN)
    lse = m + log_s
    logp = (z - m[:, None]) - log_s[:, None]
    p = logp.exp()
    h = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    h = torch.where(torch.isnan(lse), lse, h)
    empty = lse == -math.inf
    h[empty] = 0.0
    logp[empty] = -math.inf
    ok = (targets >= 0) & (targets < logits.shape[1])
    lp = logp.gather(1, targets.long().clamp(0, logits.shape[1] - 1)[:, None])[:, 0]
    lp = torch.where(ok, lp, torch.zeros_like(lp))
    # stable: equal values keep the order of their indices
    key = torch.where(torch.isnan(z), torch.full_like(z, math.inf), z)
    index = torch.sort(key, dim=1, descending=True, stable=True).indices[:, :top]
    return z, lse, logp, p, h, lp, index


def logprob_bounds(z, lse, h, vocab):
    """A term's exponential is off by (|d| + 2) u of itself, d its distance from the
    maximum, and |d| e^d < 0.37; the sums have at most vocab / 1024 + 32 terms in a row."""
    n = vocab / 1024 + 40
    size = torch.nan_to_num(lse.abs(), 0, 0, 0)
    zmax = torch.nan_to_num(z, 0, 0, 0).abs().amax(1)
    return n * U32 * (1 + size + zmax), n * U32 * (2 + math.log(vocab) + torch.nan_to_num(h, 0, 0, 0)) * 2


LOGPROBS = [
    # rows, vocab, top, scale
    (1, 1, 1, 1.0), (3, 2, 2, 1.0), (5, 7, 3, 0.5), (2, 63, 32, 1.0), (4, 500, 5, 1.0), (3, 1001, 20, 1.25),
    (2, 4099, 8, 1.0), (7, 8200, 1, 0.7), (2, 32000, 8, 1.0), (1, 50257, 32, 1.0), (3, 128000, 5, 1.0),
    (300, 97, 4, 1.0), (1, 300000, 8, 1.0), (33, 2048, 0, 1.0), (64, 32000, 3, 1.0),
]


def check_logprobs(iso, host, targets, scale, top, pad=None):
    dev = host.cuda() if pad is None else strided(host, pad)
    r = iso.token_logprobs(dev, targets.cuda(), scale=scale, top_k=top)
    z, lse, logp, p, h, lp, index = logprob_reference(host, targets, scale, top)
    near, near_h = logprob_bounds(z, lse, h, host.shape[1])
    within(r.lse, lse, near)
    within(r.entropy, h, near_h)
    within(r.logprob, lp, near)
    if top:
        assert torch.equal(r.top_index.cpu(), index)
        within(r.top_logprob, logp.gather(1, index), near[:, None])
    else:
        assert r.top_logprob is None and r.top_index is None
    return r


@pytest.mark.parametrize("rows,vocab,top,scale", LOGPROBS)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_logprobs(iso, rows, vocab, top, scale, dtype):
    g = gen(vocab)
    host = randn(g, rows, vocab, std=3.0, dtype=dtype)
    targets = torch.randint(0, vocab, (rows,), generator=g, dtype=torch.int64 if rows % 2 else torch.int32)
    targets[rows // 2] = (-1, vocab, targets[rows // 2])[rows % 3]
    a = check_logprobs(iso, host, targets, scale, top)
    b = check_logprobs(iso, host, targets, scale, top, pad=3)
    for x, y in zip(a, b):
        assert x is None or torch.equal(x, y)


def odd_rows(vocab, dtype):
    """Rows of masks, ties and values at the ends of the range."""
    g = gen(5)
    low, most = torch.finfo(dtype).min, torch.finfo(dtype).max
    t = randn(g, 17, vocab, dtype=dtype)
    t[0] = -math.inf
    t[1] = 0.0
    t[2] = -math.inf
    t[2, vocab // 2] = 1.0
    t[3] = low
    t[3, vocab - 1] = 2.0
    t[4] = low
    t[5, ::2] = -math.inf
    t[6, 0] = math.nan
    t[7, vocab // 3] = math.inf
    t[8] = torch.arange(vocab).to(dtype) / vocab
    t[9] = t[8].flip(0)
    t[10] = most
    t[11] = torch.where(torch.arange(vocab) % 2 == 0, 0.0, -0.0).to(dtype)
    t[12] = 30000.0
    t[12, 3:5] = 30080.0
    t[13, : vocab // 2] = low
    t[14] = math.nan
    t[15] = -math.inf
    t[15, 0] = low
    # the largest values all stand 64 vectors apart
    t[16, :: 64 * (4 if dtype == F32 else 8)] += 50.0
    return t


@pytest.mark.parametrize("vocab,top", [(5, 2), (130, 9), (1111, 32), (33000, 6), (200000, 32)])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_logprobs_odd_rows(iso, vocab, top, dtype):
    t = odd_rows(vocab, dtype)
    check_logprobs(iso, t, torch.full((17,), vocab // 2), 1.0, top)
    check_logprobs(iso, t, torch.zeros(17, dtype=torch.int32), 1.0, 1)


def test_token_logprobs_alternatives_in_one_group(iso):
    """More large values where one thread reads them than a workgroup keeps: rows that
    rise in steps of every size that a reader may take."""
    vocab = 60000
    rows = []
    for step in (4, 8, 64 * 4, 64 * 8, 1024 * 4, 1024 * 8):
        r = torch.arange(vocab, dtype=torch.float64)
        rows.append(torch.where((r // step) % 64 == 5, 10.0 + r / vocab, r / vocab))
    host = torch.stack(rows).to(F32)
    check_logprobs(iso, host, torch.zeros(len(rows), dtype=torch.int64), 1.0, 32)
    check_logprobs(iso, host.to(BF16), torch.zeros(len(rows), dtype=torch.int64), 1.0, 7)


def test_token_logprobs_shapes(iso):
    """Leading shapes, no targets, no rows."""
    g = gen(2)
    t = randn(g, 2, 3, 50).cuda()
    r = iso.token_logprobs(t, torch.zeros(2, 3, dtype=torch.int64, device="cuda"), top_k=4)
    assert r.logprob.shape == (2, 3) and r.top_index.shape == (2, 3, 4)
    s = iso.token_logprobs(t)
    assert s.logprob is None and torch.equal(s.lse, r.lse) and torch.equal(s.entropy, r.entropy)
    e = iso.token_logprobs(t[:0], torch.zeros(0, 3, dtype=torch.int64, device="cuda"))
    assert e.logprob.shape == (0, 3)


def logprob_grad_reference(host, targets, scale, dl, de, dtype):
    """float64 gradient and its bound: p is off by (|z| + |lse| + |log p| + 60) u of
    itself (the rounding of z - lse and of its exponential, and the lse given), the
    result is rounded once."""
    z, lse, logp, p, h, _, _ = logprob_reference(host, targets, scale, 1)
    ok = (targets >= 0) & (targets < host.shape[1])
    dl = torch.where(ok, dl.double(), 0.0)
    one = torch.zeros_like(p)
    one[ok.nonzero()[:, 0], targets[ok].long()] = 1.0
    lph = torch.where(p > 0, logp + h[:, None], torch.zeros_like(p))
    d = scale * (dl[:, None] * (one - p) - de.double()[:, None] * p * lph)
    none = (lse == -math.inf) | ((dl == 0) & (de == 0))
    d[none] = 0.0
    size = torch.nan_to_num(z.abs(), 0, 0, 0) + torch.nan_to_num(lse.abs(), 0, 0, 0)[:, None] + 60
    part = p * (dl.abs()[:, None] + de.double().abs()[:, None] * (lph.abs() + 1)) + one * dl.abs()[:, None]
    return d, torch.nan_to_num(2 * size * U32 * scale * part, 0, 0, 0) + ROUND[dtype] * torch.nan_to_num(d.abs(), 0, 0, 0) + 1e-37


@pytest.mark.parametrize("rows,vocab,top,scale", [c for c in LOGPROBS if c[0] * c[1] <= 2 ** 19])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_logprobs_backward(iso, rows, vocab, top, scale, dtype):
    g = gen(vocab + 1)
    host = randn(g, rows, vocab, std=3.0, dtype=dtype)
    targets = torch.randint(0, vocab, (rows,), generator=g)
    targets[rows // 2] = (-1, vocab, targets[rows // 2])[rows % 3]
    dl, de = randn(g, rows), randn(g, rows, std=0.1)
    de[rows // 3:] = 0.0
    for pad in (None, 3):
        dev = host.cuda() if pad is None else strided(host, pad)
        r = iso.token_logprobs(dev, targets.cuda(), scale=scale)
        want, bound = logprob_grad_reference(host, targets, scale, dl, de, dtype)
        got = iso.token_logprobs_backward(dev, targets.cuda(), r.lse, dl.cuda(), entropy=r.entropy,
                                          dentropy=de.cuda(), scale=scale)
        within(got, want, bound)
        only = iso.token_logprobs_backward(dev, targets.cuda(), r.lse, dl.cuda(), scale=scale)
        want, bound = logprob_grad_reference(host, targets, scale, dl, torch.zeros(rows), dtype)
        within(only, want, bound)
        ent = iso.token_logprobs_backward(dev, None, r.lse, None, entropy=r.entropy, dentropy=dl.cuda(), scale=scale)
        want, bound = logprob_grad_reference(host, targets, scale, torch.zeros(rows), dl, dtype)
        within(ent, want, bound)
        # in place
        assert iso.token_logprobs_backward(dev, targets.cuda(), r.lse, dl.cuda(), scale=scale, out=dev) is dev
        assert torch.equal(dev, only)


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_logprobs_backward_odd_rows(iso, dtype):
    host = odd_rows(1111, dtype)
    targets = torch.full((17,), 555)
    dl, de = torch.ones(17), torch.full((17,), 0.5)
    r = iso.token_logprobs(host.cuda(), targets.cuda())
    got = iso.token_logprobs_backward(host.cuda(), targets.cuda(), r.lse, dl.cuda(), entropy=r.entropy,
                                      dentropy=de.cuda())
    want, bound = logprob_grad_reference(host, targets, 1.0, dl, de, dtype)
    within(got, want, bound)
    # an ignored row hands back zeros, whatever its logits
    got = iso.token_logprobs_backward(host.cuda(), torch.full((17,), -1, device="cuda"), r.lse, dl.cuda())
    assert got.count_nonzero().item() == 0


def test_token_logprobs_against_differences(iso):
    g = gen(4)
    z, v = randn(g, 6, 40), randn(g, 6, 40)
    t = torch.randint(0, 40, (6,), generator=g).cuda()
    wl, wh = randn(g, 6), randn(g, 6)

    def loss(x):
        r = iso.token_logprobs(x.cuda(), t, scale=1.2)
        return (r.logprob.cpu().double() * wl + r.entropy.cpu().double() * wh).sum().item(), r

    eps = 2.0 ** -6
    slope = (loss(z + eps * v)[0] - loss(z - eps * v)[0]) / (2 * eps)
    r = loss(z)[1]
    grad = iso.token_logprobs_backward(z.cuda(), t, r.lse, wl.cuda(), entropy=r.entropy, dentropy=wh.cuda(),
                                       scale=1.2).cpu().double()
    # the third derivative's part of the slope is below eps^2 times the loss' size, the rounding below 1e-5 / eps
    assert abs(slope - (grad * v).sum().item()) <= 100 * eps * eps + 1e-5 / eps


def test_token_logprobs_past_32_bits(iso):
    rows, vocab = 70000, 32000
    t = torch.zeros(rows, vocab, dtype=BF16, device="cuda")
    t[rows - 1, vocab - 1] = 20.0
    targets = torch.full((rows,), vocab - 1, device="cuda", dtype=torch.int32)
    r = iso.token_logprobs(t, targets, top_k=1)
    assert r.top_index[rows - 1, 0].item() == vocab - 1 and r.top_index[:rows - 1].count_nonzero().item() == 0
    assert abs(r.lse[0].item() - math.log(vocab)) <= 1e-5
    d = iso.token_logprobs_backward(t, targets, r.lse, torch.ones(rows, device="cuda"), out=t)
    assert d[rows - 2, vocab - 1].item() == 1.0 and abs(d[rows - 2, 5].item() * vocab + 1) <= 2.0 ** -8
    assert 0 < d[rows - 1, vocab - 1].item() < 1e-3


# Large finite logits under a scale that rounds the products: masks written as a number.

MASK_SCALES = [1.0, 0.7, 0.9, 1.25, 1 / 1.3]


def masked_rows(vocab, dtype):
    """Rows with large finite values on some columns, on all but one and on all, where
    whole threads, waves and splits hold nothing else."""
    g = gen(vocab)
    low = torch.finfo(dtype).min
    rows = []
    for fill in (-1e4, -1e9, -1e10, -1e30, low, 1e10):
        normal = randn(g, vocab, std=3.0, dtype=dtype)
        some = torch.full((vocab,), fill, dtype=dtype)
        some[torch.randperm(vocab, generator=g)[:50]] = normal[:50]
        one = torch.full((vocab,), fill, dtype=dtype)
        one[vocab // 3] = 2.5
        half = normal.clone()
        half[:vocab // 2] = fill
        rows += [some, one, half, torch.full((vocab,), fill, dtype=dtype)]
    mixed = torch.full((vocab,), low, dtype=dtype)
    mixed[::3], mixed[1::3] = -math.inf, -1e10
    rows += [mixed, torch.where(torch.arange(vocab) == vocab - 1, low, -math.inf).to(dtype)]
    return torch.stack(rows)


def as_float32(t):
    """float64 values that float32 rounds to infinity are infinite."""
    return torch.where(t.float().isinf(), t.float().double(), t)


def masked_reference(host, targets, scale, top):
    """float64 results and their bounds.  A term e^d, d = scale (x - max), is off by
    (4 |d| + 2) u of itself, where |d| e^d < 0.37, so the sum's logarithm is off by 4 u for
    each of the terms that follow each other; a log probability is d less that logarithm,
    off by 4 u |d| more, and the log-sum-exp is rounded once."""
    z, lse, logp, p, h, lp, index = logprob_reference(host, targets, scale, top)
    vocab = host.shape[1]
    n = vocab / 1024 + 40
    logs = (n * 4 + 2 * math.log(vocab + 1)) * U32
    near = lambda t: logs + 4 * U32 * torch.nan_to_num(t, 0, 0, 0).abs()  # noqa: E731
    near_h = n * U32 * (2 + math.log(vocab) + h) * 2
    return (z, lse, logp, p, h, lp, index), (near(lse), near_h, near(lp), near(logp))


@pytest.mark.parametrize("vocab,top", [(130, 9), (1111, 32), (32000, 5), (33000, 6), (200000, 8)])
@pytest.mark.parametrize("scale", MASK_SCALES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_logprobs_large_finite_masks(iso, vocab, top, scale, dtype):
    host = masked_rows(vocab, dtype)
    for column in (vocab // 3, vocab - 1):
        targets = torch.full((len(host),), column)
        (z, lse, logp, p, h, lp, index), (near_lse, near_h, near_lp, near_logp) = masked_reference(host, targets, scale, top)
        r = iso.token_logprobs(host.cuda(), targets.cuda(), scale=scale, top_k=top)
        within(r.lse, as_float32(lse), near_lse)
        within(r.entropy, h, near_h)
        within(r.logprob, as_float32(lp), near_lp)
        assert torch.equal(r.top_index.cpu(), index)
        within(r.top_logprob, as_float32(logp.gather(1, index)), near_logp.gather(1, index))


# |lse| up to which its rounding to float32 may show in the gradient (2^-24 |lse| of p)
SURE_LSE = {F32: 256.0, BF16: 8192.0}


def large_lse_reference(host, targets, scale, dl, de):
    """float64 gradient and its bound.  p = e^q with q = log p is off by (6 |q| + 2) u of itself
    for q's own roundings and the exponential, 4 u for each term that follows another in the
    sum, and lse's rounding up to SURE_LSE; the entropy that is handed back has its own error."""
    dtype = host.dtype
    (z, lse, logp, p, h, lp, index), (_, near_h, _, _) = masked_reference(host, targets, scale, 1)
    want, _ = logprob_grad_reference(host, targets, scale, dl, de, dtype)
    n = host.shape[1] / 1024 + 40
    q = torch.nan_to_num(logp, 0, 0, 0).abs().clamp(max=150)
    near_q = U32 * (6 * q + 4 * n + 64 + 2 * torch.nan_to_num(lse, 0, SURE_LSE[dtype], 0).abs().clamp(max=SURE_LSE[dtype])[:, None])
    ok = (targets >= 0) & (targets < host.shape[1])
    one = torch.zeros_like(p)
    one[ok.nonzero()[:, 0], targets[ok].long()] = 1.0
    dl, de = torch.where(ok, dl.double(), 0.0).abs()[:, None], de.double().abs()[:, None]
    lph = torch.where(p > 0, (logp + h[:, None]).abs(), torch.zeros_like(p))
    part = p * dl * (near_q + 4 * U32) + one * dl * 4 * U32 + de * p * (lph * (near_q + 4 * U32) + near_q + near_h[:, None])
    return want, scale * torch.nan_to_num(part, 0, 0, 0) * 1.01 + ROUND[dtype] * torch.nan_to_num(want, 0, 0, 0).abs() + 1e-37


@pytest.mark.parametrize("vocab", [3, 130, 1111, 33000])
@pytest.mark.parametrize("scale", MASK_SCALES)
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_logprobs_backward_large_lse(iso, vocab, scale, dtype):
    """Rows whose log-sum-exp is so large that its rounding hides the sum."""
    g = gen(vocab + 7)
    shifts = torch.tensor([-1e6, -5e4, -3000.0, -500.0, -90.0, 90.0, 500.0, 3000.0, 5e4, 1e6, 1e20, 3e38])
    # (bfloat16 rounds the larger ones together: rows of a few distinct values)
    shifted = (randn(g, len(shifts), vocab, std=3.0) + shifts[:, None]).to(dtype)
    host = torch.cat([shifted] + ([masked_rows(vocab, dtype)] if vocab > 50 else []) + [odd_rows(vocab, dtype)])
    rows = len(host)
    targets = torch.randint(0, vocab, (rows,), generator=g)
    targets[::5] = -1
    dl, de = randn(g, rows), randn(g, rows, std=0.1)
    de[::3] = 0.0
    for pad in (None, 3):
        dev = host.cuda() if pad is None else strided(host, pad)
        r = iso.token_logprobs(dev, targets.cuda(), scale=scale)
        got = iso.token_logprobs_backward(dev, targets.cuda(), r.lse, dl.cuda(), entropy=r.entropy, dentropy=de.cuda(),
                                          scale=scale)
        within(got, *large_lse_reference(host, targets, scale, dl, de))
        again = iso.token_logprobs_backward(dev, targets.cuda(), r.lse, dl.cuda(), entropy=r.entropy,
                                            dentropy=de.cuda(), scale=scale, out=dev)
        assert again is dev and torch.equal(got.view(torch.uint8), again.contiguous().view(torch.uint8))


@pytest.mark.parametrize("shift", [0.0, 300.0, -3000.0, 20000.0])
@pytest.mark.parametrize("dtype", [F32, BF16])
def test_token_logprobs_backward_of_a_part(iso, dtype, shift):
    """Rows that are parts of longer ones, with the log-sum-exp of the whole: p is e^(z - lse)
    with the lse that is given, off by (6 |log p| + 64) u of itself and, where p is formed from
    z and lse as they stand, by the rounding of lse."""
    g = gen(31)
    rows, vocab = 9, 700
    whole = (randn(g, rows, 3 * vocab, std=3.0) + shift).to(dtype)
    lse = torch.logsumexp(whole.double() * 0.75, 1).to(F32)
    dl = randn(g, rows)
    for at in range(3):
        host = whole[:, at * vocab:(at + 1) * vocab].contiguous()
        targets = torch.randint(-vocab, vocab, (rows,), generator=g)
        got = iso.token_logprobs_backward(host.cuda(), targets.cuda(), lse.cuda(), dl.cuda(), scale=0.75)
        q = host.double() * 0.75 - lse.double()[:, None]
        p, ok = q.exp(), targets >= 0
        one = torch.zeros_like(p)
        one[ok.nonzero()[:, 0], targets[ok]] = 1.0
        d = torch.where(ok, dl.double(), 0.0)[:, None]
        want = 0.75 * d * (one - p)
        near = U32 * (6 * q.abs().clamp(max=150) + 64 + 2 * lse.double().abs().clamp(max=SURE_LSE[dtype])[:, None])
        within(got, want, 0.75 * d.abs() * (p * near + one * 4 * U32) * 1.01 + ROUND[dtype] * want.abs() + 1e-37)


def test_token_logprobs_backward_large_lse_of_large_results(iso):
    """The same where the result is stored past the caches: the bits of calls of few rows."""
    rows, vocab = 4200, 32003
    t = torch.randn(rows, vocab, device="cuda")
    t[::7] += 5e4
    t[3::7] = -1e10
    t = t.to(BF16)
    targets = torch.arange(rows, device="cuda") * 7 % vocab
    w = torch.randn(2, rows, device="cuda")
    r = iso.token_logprobs(t, targets, scale=0.7)
    d = iso.token_logprobs_backward(t, targets, r.lse, w[0], entropy=r.entropy, dentropy=w[1], scale=0.7)
    assert d.numel() * d.element_size() > 256 << 20 and torch.isfinite(d).all()
    for a in range(0, rows, 500):
        b = min(rows, a + 500)
        part = iso.token_logprobs_backward(t[a:b], targets[a:b], r.lse[a:b], w[0, a:b], entropy=r.entropy[a:b],
                                           dentropy=w[1, a:b], scale=0.7)
        assert torch.equal(d[a:b], part)


# --------------------------------------------------------------------------
# Gated feed-forward block
# --------------------------------------------------------------------------

def act_of(g, act):
    if act == "silu":
        s = torch.sigmoid(g)
        return g * s, s * (1 + g * (1 - s))
    cdf = torch.special.ndtr(g)
    return g * cdf, cdf + g * torch.exp(-0.5 * g * g) / math.sqrt(2 * math.pi)


FFNS = [
    # tokens, dim, hidden
    (1, 1, 1), (1, 64, 64), (1, 200, 333), (2, 33, 65), (5, 128, 96), (16, 256, 130), (17, 72, 200), (31, 100, 64),
    (64, 640, 128), (65, 65, 129), (127, 31, 40), (200, 264, 392), (300, 613, 257), (513, 128, 1000), (1000, 96, 136),
]


def ffn_inputs(tokens, dim, hidden, dtype, seed):
    g = gen(seed)
    return (randn(g, tokens, dim, dtype=dtype), randn(g, hidden, dim, std=dim ** -0.5, dtype=dtype),
            randn(g, hidden, dim, std=dim ** -0.5, dtype=dtype), randn(g, tokens, hidden, dtype=dtype))


def ffn_reference(x, wg, wu, act):
    """float64 result, and bounds of g's and u's error and of the result's."""
    x, wg, wu = x.double(), wg.double(), wu.double()
    g, u = x @ wg.T, x @ wu.T
    n = (x.shape[1] + 8) * U32
    eg, eu = n * (x.abs() @ wg.abs().T), n * (x.abs() @ wu.abs().T)
    a, da = act_of(g, act)
    # |act'| <= 1.13; the activation itself is off by a few ulps of max(|g|, 1)
    ea = 1.13 * eg + 8 * U32 * (1 + g.abs())
    return g, u, a, da, eg, eu, ea


@pytest.mark.parametrize("tokens,dim,hidden", FFNS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_ffn(iso, tokens, dim, hidden, dtype, act):
    x, wg, wu, _ = ffn_inputs(tokens, dim, hidden, dtype, tokens + hidden)
    g, u, a, da, eg, eu, ea = ffn_reference(x, wg, wu, act)
    want = a * u
    bound = ea * u.abs() + a.abs() * eu + ea * eu + ROUND[dtype] * want.abs() + 1e-37
    within(iso.gated_ffn(x.cuda(), wg.cuda(), wu.cuda(), act=act), want, bound)
    # rows further apart than they are long, and operands that start anywhere
    xs, gs, us = (strided(t, 5) for t in (x, wg, wu))
    out = strided(torch.zeros(tokens, hidden, dtype=dtype), 3)
    iso.gated_ffn(xs, gs, us, act=act, out=out)
    within(out, want, bound)
    assert torch.isnan(out.as_strided((tokens, 3), (hidden + 3, 1), hidden)[:-1]).all()
    within(iso.gated_ffn(strided(x, 8), strided(wg, 8), strided(wu, 8), act=act), want, bound)
    within(iso.gated_ffn(*(at_offset(t, i + 1) for i, t in enumerate((x, wg, wu))), act=act), want, bound)


@pytest.mark.parametrize("tokens,dim,hidden", FFNS)
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("act", ["silu", "gelu"])
def test_gated_ffn_backward(iso, tokens, dim, hidden, dtype, act):
    x, wg, wu, dh = ffn_inputs(tokens, dim, hidden, dtype, tokens * 3 + hidden)
    g, u, a, da, eg, eu, ea = ffn_reference(x, wg, wu, act)
    X, G, W, D = (t.double() for t in (x, wg, wu, dh))
    dg, du = D * u * da, D * a
    # |act''| <= 0.8; in bfloat16 both are rounded once
    rnd = ROUND[dtype] if dtype == BF16 else 4 * U32
    edg = D.abs() * ((da.abs() + 1e-6) * eu + u.abs() * (0.8 * eg + 16 * U32) + 0.8 * eg * eu) + rnd * dg.abs()
    edu = D.abs() * ea + rnd * du.abs()
    nk, nt = (2 * hidden + 8) * U32, (tokens + 8) * U32
    want = [dg @ G + du @ W, dg.T @ X, du.T @ X]
    bound = [edg @ G.abs() + edu @ W.abs() + nk * (dg.abs() @ G.abs() + du.abs() @ W.abs()),
             edg.T @ X.abs() + nt * (dg.abs().T @ X.abs()), edu.T @ X.abs() + nt * (du.abs().T @ X.abs())]
    first = None
    for place in (lambda t: t.cuda(), lambda t: strided(t, 3), lambda t: strided(t, 8), lambda t: at_offset(t, 1)):
        got = iso.gated_ffn_backward(*(place(t) for t in (x, wg, wu, dh)), act=act)
        for r, w, b in zip(got, want, bound):
            within(r, w, 1.01 * b + ROUND[dtype] * w.abs() + 1e-37)
        first = first or got
    only = iso.gated_ffn_backward(x.cuda(), wg.cuda(), wu.cuda(), dh.cuda(), act=act, need_dw=False)
    assert torch.equal(only[0], first[0]) and only[1] is None and only[2] is None
    only = iso.gated_ffn_backward(x.cuda(), wg.cuda(), wu.cuda(), dh.cuda(), act=act, need_dx=False)
    assert only[0] is None and torch.equal(only[1], first[1]) and torch.equal(only[2], first[2])


# Sizes of bfloat16 products on larger tiles and in splits (the instances one by one, with
# the tiles that each takes: _ffn_cases.py): forward on 256-square tiles in the first two,
# on 192 x 256 in the fifth, on 128-square ones, in 4 splits in the sixth, in the others; dx
# on 256-square tiles in the third, on 192 x 256 in the last; in the others dx shares a
# launch with the weights' gradients, on 256-square tiles in the seventh.
FFN_TILES = [(6200, 136, 1000), (3000, 264, 4400), (8192, 2048, 256), (256, 2048, 4096), (4100, 520, 2056),
             (64, 2048, 5632), (700, 1032, 3000), (6144, 2048, 200)]


@pytest.mark.parametrize("tokens,dim,hidden", FFN_TILES)
def test_gated_ffn_tiles(iso, tokens, dim, hidden):
    x, wg, wu, dh = (t.cuda() for t in ffn_inputs(tokens, dim, hidden, BF16, 11))
    out = iso.gated_ffn(x, wg, wu).cpu()
    grads = [t.cpu() for t in iso.gated_ffn_backward(x, wg, wu, dh)]
    # the same bounds as above, in float64 on the GPU
    g, u, a, da, eg, eu, ea = ffn_reference(x, wg, wu, "silu")
    X, G, W, D = (t.double() for t in (x, wg, wu, dh))
    within(out, (a * u).cpu(), (ea * u.abs() + a.abs() * eu + ea * eu + ROUND[BF16] * (a * u).abs() + 1e-37).cpu())
    dg, du = D * u * da, D * a
    edg = D.abs() * ((da.abs() + 1e-6) * eu + u.abs() * (0.8 * eg + 16 * U32) + 0.8 * eg * eu) + ROUND[BF16] * dg.abs()
    edu = D.abs() * ea + ROUND[BF16] * du.abs()
    nk, nt = (2 * hidden + 8) * U32, (tokens + 8) * U32
    want = [dg @ G + du @ W, dg.T @ X, du.T @ X]
    bound = [edg @ G.abs() + edu @ W.abs() + nk * (dg.abs() @ G.abs() + du.abs() @ W.abs()),
             edg.T @ X.abs() + nt * (dg.abs().T @ X.abs()), edu.T @ X.abs() + nt * (du.abs().T @ X.abs())]
    for r, w, b in zip(grads, want, bound):
        within(r, w.cpu(), (1.01 * b + ROUND[BF16] * w.abs() + 1e-37).cpu())
        # the rounding of da and du and of the result, as random errors: far below the bound's worst case
        assert ((r.cuda().double() - w).norm() / w.norm()).item() <= 2.0 ** -8


@pytest.mark.parametrize("far", ["x", "weights"])
def test_gated_ffn_rows_far_apart(iso, far):
    """Operands that are columns of a matrix of more than 2^22: past the tiles' offsets."""
    tokens, dim, hidden, apart = 40, 24, 16, (1 << 22) + 8
    x, wg, wu, dh = ffn_inputs(tokens, dim, hidden, BF16, 2)
    want = iso.gated_ffn(x.cuda(), wg.cuda(), wu.cuda())
    grads = iso.gated_ffn_backward(x.cuda(), wg.cuda(), wu.cuda(), dh.cuda())
    if far == "x":
        ops = [strided(x, apart - dim), wg.cuda(), wu.cuda()]
    else:
        ops = [x.cuda(), strided(wg, apart - dim), strided(wu, apart - dim)]
    assert torch.equal(iso.gated_ffn(*ops), want)
    for a, b in zip(iso.gated_ffn_backward(*ops, dh.cuda()), grads):
        assert torch.equal(a, b)


def test_gated_ffn_no_tokens(iso):
    w = torch.ones(6, 4, device="cuda")
    x = torch.empty(0, 4, device="cuda")
    assert iso.gated_ffn(x, w, w).shape == (0, 6)
    dx, dg, du = iso.gated_ffn_backward(x, w, w, torch.empty(0, 6, device="cuda"))
    assert dx.shape == (0, 4) and dg.count_nonzero().item() == 0 and du.count_nonzero().item() == 0


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("tokens", [3, 150])
def test_gated_ffn_nonfinite_stays_in_its_row(iso, tokens, dtype):
    """A NaN or infinity of one token reaches that token's row only, one of a weight's
    row that column only; sizes that leave parts of every tile empty."""
    x, wg, wu, dh = ffn_inputs(tokens, 100, 90, dtype, 1)
    x[1, 50], wu[7, 99] = math.nan, math.inf
    out = iso.gated_ffn(x.cuda(), wg.cuda(), wu.cuda()).cpu()
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[1], want[:, 7] = True, True
    assert torch.equal(bad, want)


@pytest.mark.parametrize("tokens", [1, 64, 65, 200])
def test_gated_ffn_infinite_operand(iso, tokens):
    """In float32 an infinity, or a value past bfloat16's range, is taken as it is by up to 64
    tokens and gives NaN by more; in bfloat16 an infinity is always taken as it is."""
    few = tokens <= 64
    for dtype in (F32, BF16):
        x, wg, wu, _ = ffn_inputs(tokens, 48, 40, dtype, 3)
        x[0] = 0.0
        x[0, 5] = math.inf
        wg[:, 5], wu[:, 5] = 0.5, torch.where(torch.arange(40) % 2 == 0, 1.0, -1.0)
        out = iso.gated_ffn(x.cuda(), wg.cuda(), wu.cuda()).cpu()
        assert torch.isfinite(out[1:]).all()
        if few or dtype == BF16:
            assert torch.equal(out[0], torch.where(torch.arange(40) % 2 == 0, math.inf, -math.inf).to(dtype))
        else:
            assert torch.isnan(out[0]).all()
    x, wg, wu, _ = ffn_inputs(tokens, 48, 40, F32, 3)
    x[0], wg[:], wu[:] = 0.0, 0.0, 0.0
    x[0, 5], wg[:, 5], wu[:, 5] = 3.4e38, 1e-37, 1e-37
    out = iso.gated_ffn(x.cuda(), wg.cuda(), wu.cuda()).cpu()
    if few:
        within(out[0], torch.full((40,), 34.0 * 34.0 / (1 + math.exp(-34.0)), dtype=torch.float64), 1156 * 1e-5)
    else:
        assert torch.isnan(out[0]).all()


def test_gated_ffn_against_differences(iso):
    g = gen(9)
    ts = [randn(g, 20, 30), randn(g, 40, 30, std=0.2), randn(g, 40, 30, std=0.2)]
    vs = [randn(g, *t.shape, std=0.2) for t in ts]
    w = randn(g, 20, 40)
    grads = iso.gated_ffn_backward(*(t.cuda() for t in ts), w.cuda(), act="gelu")
    eps = 2.0 ** -7

    def loss(sign):
        out = iso.gated_ffn(*((t + sign * eps * v).cuda() for t, v in zip(ts, vs)), act="gelu")
        return (out.cpu().double() * w).sum().item()

    slope = (loss(1) - loss(-1)) / (2 * eps)
    want = sum((d.cpu().double() * v).sum().item() for d, v in zip(grads, vs))
    # the third derivative's part is below 100 eps^2 of the loss' terms, the rounding below 1e-4 / eps
    assert abs(slope - want) <= 100 * eps * eps + 1e-4 / eps


def test_gated_ffn_past_32_bits(iso):
    tokens, dim, hidden = 540000, 64, 4096
    x = torch.zeros(tokens, dim, dtype=BF16, device="cuda")
    w = torch.zeros(hidden, dim, dtype=BF16, device="cuda")
    x[tokens - 1], w[hidden - 1] = 1.0, 0.125
    out = iso.gated_ffn(x, w, w)
    assert abs(out[tokens - 1, hidden - 1].item() - 64 / (1 + math.exp(-8.0))) <= 0.25
    assert out.count_nonzero().item() == 1
    dx, dg, du = iso.gated_ffn_backward(x, w, w, out)
    assert dx[tokens - 1].min().item() > 0 and dx[:tokens - 1].count_nonzero().item() == 0
    assert dg[hidden - 1].min().item() > 0 and dg[:hidden - 1].count_nonzero().item() == 0


# --------------------------------------------------------------------------
# Streams, graphs, determinism
# --------------------------------------------------------------------------

def _step(iso, s):
    out = iso.embedding(s["table"], s["ids"], scale=2.0)
    h = iso.gated_ffn(out, s["wg"], s["wu"])
    r = iso.token_logprobs(h, s["targets"], top_k=3)
    dh = iso.token_logprobs_backward(h, s["targets"], r.lse, s["dl"])
    dx, dwg, dwu = iso.gated_ffn_backward(out, s["wg"], s["wu"], dh)
    dt = iso.embedding_backward(s["ids"], dx, s["table"].shape[0], scale=2.0)
    norm = iso.clip_grads([dwg, dwu, dt], 1e-3)
    return [out, h, r.logprob, r.entropy, r.lse, r.top_logprob, r.top_index, dh, dx, dwg, dwu, dt, norm]


def _state(dtype, tokens=300):
    g = gen(6)
    ids = some_ids(g, tokens, 400)
    return {k: v.cuda() for k, v in dict(
        table=randn(g, 400, 136, dtype=dtype), ids=ids, wg=randn(g, 520, 136, std=0.1, dtype=dtype),
        wu=randn(g, 520, 136, std=0.1, dtype=dtype), targets=torch.randint(0, 520, (tokens,), generator=g),
        dl=randn(g, tokens)).items()}


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_streams_and_determinism(iso, dtype):
    s = _state(dtype)
    first = _step(iso, s)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        second = _step(iso, s)
    side.synchronize()
    for a, b in zip(first, second):
        assert torch.equal(a, b)
    third = iso.gated_ffn(first[0], s["wg"], s["wu"], stream=side.cuda_stream)
    side.synchronize()
    assert torch.equal(third, first[1])


@pytest.mark.parametrize("tokens", [2, 300])
def test_graph_replays(iso, tokens):
    s = _state(BF16, tokens)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _step(iso, s)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = _step(iso, s)
    for turn in range(4):
        s["table"].copy_(randn(gen(50 + turn), 400, 136, dtype=BF16))
        s["dl"].mul_(-1.5)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in captured]
        eager = _step(iso, s)
        torch.cuda.synchronize()
        for a, b in zip(got, eager):
            assert torch.equal(a, b)


# --------------------------------------------------------------------------
# Autograd
# --------------------------------------------------------------------------

def wanted(t):
    return t.detach().clone().requires_grad_()


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_autograd_reaches_every_operand(iso, dtype):
    """The gradients are those of the functions that form them, given what a chain of the
    operators hands back; without a wish for one nothing is attached."""
    s = _state(dtype)
    table, wg, wu = (wanted(s[k]) for k in ("table", "wg", "wu"))
    x = iso.embedding(table, s["ids"], scale=2.0)
    h = iso.gated_ffn(x, wg, wu, act="gelu")
    r = iso.token_logprobs(h, s["targets"], scale=0.8, top_k=2)
    (r.logprob * s["dl"] + 0.25 * r.entropy).sum().backward()
    x0 = iso.embedding(s["table"], s["ids"], scale=2.0)
    h0 = iso.gated_ffn(x0, s["wg"], s["wu"], act="gelu")
    r0 = iso.token_logprobs(h0, s["targets"], scale=0.8, top_k=2)
    assert not x0.requires_grad and not h0.requires_grad and not r0.logprob.requires_grad
    assert torch.equal(x, x0) and torch.equal(h, h0) and all(torch.equal(a, b) for a, b in zip(r, r0))
    dh = iso.token_logprobs_backward(h0, s["targets"], r0.lse, s["dl"], entropy=r0.entropy,
                                     dentropy=torch.full_like(s["dl"], 0.25), scale=0.8)
    dx, dwg, dwu = iso.gated_ffn_backward(x0, s["wg"], s["wu"], dh, act="gelu")
    dt = iso.embedding_backward(s["ids"], dx, 400, scale=2.0, out_dtype=dtype)
    assert torch.equal(wg.grad, dwg) and torch.equal(wu.grad, dwu) and torch.equal(table.grad, dt)


def test_autograd_of_some_operands(iso):
    """One operand alone; results nobody uses; gradients that arrive expanded or strided;
    leading shapes; no targets."""
    s = _state(F32, 24)
    x0 = iso.embedding(s["table"], s["ids"]).view(2, 3, 4, 136)
    w = torch.randn(2, 3, 520, 4, device="cuda").transpose(-1, -2)
    for which in range(3):
        ts = [x0.clone(), s["wg"].clone(), s["wu"].clone()]
        ts[which].requires_grad_()
        iso.gated_ffn(*ts).backward(w)
        want = iso.gated_ffn_backward(x0, s["wg"], s["wu"], w.contiguous())[which]
        assert torch.equal(ts[which].grad, want) and all(ts[i].grad is None for i in range(3) if i != which)
    x = wanted(x0)
    iso.gated_ffn(x, s["wg"], s["wu"]).sum().backward()
    assert torch.equal(x.grad, iso.gated_ffn_backward(x0, s["wg"], s["wu"], torch.ones(2, 3, 4, 520, device="cuda"))[0])
    z = wanted(torch.randn(2, 3, 50, device="cuda"))
    r = iso.token_logprobs(z)
    r.entropy.mean().backward()
    want = iso.token_logprobs_backward(z.detach(), None, r.lse.detach(), None, entropy=r.entropy.detach(),
                                       dentropy=torch.full((2, 3), 1 / 6, device="cuda"))
    assert torch.equal(z.grad, want)
    # a float32 table looked up in bfloat16: the gradient has the table's type
    table = wanted(s["table"])
    iso.embedding(table, s["ids"], out_dtype=BF16).float().sum().backward()
    assert table.grad.dtype == F32 and table.grad.sum().item() == 136 * ((s["ids"] >= 0) & (s["ids"] < 400)).sum().item()


def test_autograd_does_not_drop_what_it_lacks(iso):
    """The log-sum-exp and the alternatives hand back no gradient, and say so; results
    written into a given tensor carry none."""
    z = wanted(torch.randn(4, 50, device="cuda"))
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    for pick in (lambda r: r.lse, lambda r: r.top_logprob, lambda r: r.logprob[:, None] + r.top_logprob):
        with pytest.raises(NotImplementedError):
            pick(iso.token_logprobs(z, t, top_k=2)).sum().backward()
    assert z.grad is None
    w = wanted(torch.randn(6, 50, device="cuda"))
    with pytest.raises(ValueError):
        iso.gated_ffn(z, w, w, out=torch.empty(4, 6, device="cuda"))
    with pytest.raises(ValueError):
        iso.embedding(w, t, out=torch.empty(4, 50, device="cuda"))
    with torch.no_grad():
        out = torch.empty(4, 6, device="cuda")
        assert iso.gated_ffn(z, w, w, out=out) is out and not out.requires_grad


def test_autograd_of_results_written_in_place(iso):
    """A result may be written, as a mask over the log probabilities does it; one that the
    backward pass needs is found out."""
    z0 = torch.randn(6, 40, device="cuda")
    t = torch.arange(6, device="cuda")
    z = wanted(z0)
    lp = iso.token_logprobs(z, t, scale=1.1, top_k=1).logprob
    lp.masked_fill_(t < 2, 0.0)
    lp[5] *= 3.0
    lp.sum().backward()
    w = torch.tensor([0.0, 0.0, 1.0, 1.0, 1.0, 3.0], device="cuda")
    lse = iso.token_logprobs(z0, t, scale=1.1).lse
    assert torch.equal(z.grad, iso.token_logprobs_backward(z0, t, lse, w, scale=1.1))
    r = iso.token_logprobs(wanted(z0), t)
    r.entropy.mul_(2.0)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        r.entropy.sum().backward()


@pytest.mark.parametrize("call", ["clip", "clip out", "embedding", "embedding gradient", "logits' gradient", "ffn"])
def test_autograd_sees_what_is_written(iso, call):
    """A tensor that was saved for a backward pass and is then written by an operator is
    found out."""
    a = torch.ones(8, 8, device="cuda")
    x = wanted(a)
    kept = torch.ones(8, 8, device="cuda")
    y = (x * kept).sum()
    version = kept._version
    ids = torch.arange(8, device="cuda")
    v = torch.ones(8, device="cuda")
    if call == "clip":
        iso.clip_grads([a, kept], 1.0)
    elif call == "clip out":
        iso.clip_grads([a], 1.0, out=[kept])
    elif call == "embedding":
        iso.embedding(a, ids, out=kept)
    elif call == "embedding gradient":
        iso.embedding_backward(ids, a, 8, out=kept, accumulate=True)
    elif call == "logits' gradient":
        iso.token_logprobs_backward(a, ids, v, v, out=kept)
    else:
        iso.gated_ffn(a, a, a, out=kept)
    assert kept._version == version + 1
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        y.backward()


# --------------------------------------------------------------------------
# Results larger than the caches, which are stored past them
# --------------------------------------------------------------------------

def test_clip_of_large_results(iso):
    """The scaled elements one by one, at odd alignments and with a shorter last chunk."""
    flat = torch.randn(36_000_011, device="cuda")
    grads = [flat[1:30_000_000], flat[30_000_000:], torch.randn(5_000_001, device="cuda").to(BF16)[1:]]
    outs = [torch.empty(g.numel() + 3, device="cuda", dtype=g.dtype)[3:] for g in grads]
    for max_norm in (1.0, 1e9):
        coef = iso.clip_grads(grads, max_norm, out=outs)[1]
        for g, o in zip(grads, outs):
            assert torch.equal(o, (g.float() * coef).to(g.dtype))


@pytest.mark.parametrize("rows,vocab,dtype", [(4200, 32003, BF16), (1100, 64001, F32)])
def test_token_logprobs_backward_of_large_results(iso, rows, vocab, dtype):
    """The same bits as in calls of few rows, whose results stay in the caches."""
    t = torch.randn(rows, vocab, device="cuda").to(dtype)
    targets = torch.arange(rows, device="cuda") * 7 % vocab
    w = torch.randn(2, rows, device="cuda")
    r = iso.token_logprobs(t, targets)
    d = iso.token_logprobs_backward(t, targets, r.lse, w[0], entropy=r.entropy, dentropy=w[1])
    assert d.numel() * d.element_size() > 256 << 20
    for a in range(0, rows, 500):
        b = min(rows, a + 500)
        part = iso.token_logprobs_backward(t[a:b], targets[a:b], r.lse[a:b], w[0, a:b], entropy=r.entropy[a:b],
                                           dentropy=w[1, a:b])
        assert torch.equal(d[a:b], part)


# Sizes at which dx and the weights' products share a launch: of 256-square tiles in 16
# and in 4 splits, of 256-square and 192 x 256 tiles, of 128-square ones; in float32 of
# 256-square ones in 8 splits and of 128-square ones.
@pytest.mark.parametrize("tokens,dim,hidden,dtype", [
    (130, 1500, 8000, BF16), (1024, 2048, 5632, BF16), (1500, 1500, 4000, BF16), (1100, 1300, 2900, BF16),
    (700, 1032, 3000, F32), (640, 1544, 4104, F32),
])
def test_gated_ffn_gradients_together(iso, tokens, dim, hidden, dtype):
    x, wg, wu, dh = (t.cuda() for t in ffn_inputs(tokens, dim, hidden, dtype, 12))
    grads = iso.gated_ffn_backward(x, wg, wu, dh)
    g, u, a, da, eg, eu, ea = ffn_reference(x, wg, wu, "silu")
    X, G, W, D = (t.double() for t in (x, wg, wu, dh))
    dg, du = D * u * da, D * a
    rnd = ROUND[dtype] if dtype == BF16 else 4 * U32
    edg = D.abs() * ((da.abs() + 1e-6) * eu + u.abs() * (0.8 * eg + 16 * U32) + 0.8 * eg * eu) + rnd * dg.abs()
    edu = D.abs() * ea + rnd * du.abs()
    nk, nt = (2 * hidden + 8) * U32, (tokens + 8) * U32
    want = [dg @ G + du @ W, dg.T @ X, du.T @ X]
    bound = [edg @ G.abs() + edu @ W.abs() + nk * (dg.abs() @ G.abs() + du.abs() @ W.abs()),
             edg.T @ X.abs() + nt * (dg.abs().T @ X.abs()), edu.T @ X.abs() + nt * (du.abs().T @ X.abs())]
    for r, w, b in zip(grads, want, bound):
        within(r.cpu(), w.cpu(), (1.01 * b + ROUND[dtype] * w.abs() + 1e-37).cpu())
        # random errors: far below the bound's worst case
        assert ((r.double() - w).norm() / w.norm()).item() <= (2.0 ** -8 if dtype == BF16 else 2.0 ** -20)
    # one of them alone: the same bits
    assert torch.equal(iso.gated_ffn_backward(x, wg, wu, dh, need_dw=False)[0], grads[0])
    only = iso.gated_ffn_backward(x, wg, wu, dh, need_dx=False)
    assert torch.equal(only[1], grads[1]) and torch.equal(only[2], grads[2])
