"""What the operators of a block of experts and of distillation refuse, before anything
is enqueued (no GPU needed: the calls end in the argument checks, and the addresses are
never read)."""
import math

import pytest

iso = pytest.importorskip("paper_2607_03011_amd")
torch = pytest.importorskip("torch")

INVALID, ALIGN, ALIAS, WORKSPACE, UNSUPPORTED = -1, -3, -4, -5, -7
A, B, C, D, E, F, WS = (0x10000000 * (i + 1) for i in range(7))  # addresses far apart
BIG = 1 << 27


def refused(status, f, *args):
    with pytest.raises(iso.IsoLoCoError) as ei:
        f(*args)
    assert ei.value.status == status
    assert iso.isoloco_last_error() != ""


def changed(good, **change):
    return [change.get(k, v) for k, v in good.items()]


ROUTE = dict(scores=A, ld=16, dtype=1, tokens=100, experts=16, top_k=4, normalize=1, weight=B, expert=C, row=D, token=E,
             offsets=F, workspace=WS, ws_bytes=BIG)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(scores=0)), (INVALID, dict(weight=0)), (INVALID, dict(expert=0)), (INVALID, dict(row=0)),
    (INVALID, dict(token=0)), (INVALID, dict(offsets=0)), (INVALID, dict(dtype=2)), (INVALID, dict(tokens=-1)),
    (INVALID, dict(experts=0)), (INVALID, dict(experts=1025, ld=1025)), (INVALID, dict(top_k=0)), (INVALID, dict(top_k=17)),
    (INVALID, dict(experts=64, ld=64, top_k=33)), (INVALID, dict(ld=15)), (INVALID, dict(tokens=1 << 29)),
    (ALIGN, dict(scores=A + 1)), (ALIGN, dict(weight=B + 2)), (ALIGN, dict(offsets=F + 1)),
    (ALIAS, dict(weight=A)), (ALIAS, dict(row=C + 16)), (ALIAS, dict(token=D)), (ALIAS, dict(offsets=WS)),
    (WORKSPACE, dict(workspace=0)), (WORKSPACE, dict(ws_bytes=16)), (WORKSPACE, dict(workspace=WS + 128)),
])
def test_route_refuses(status, change):
    refused(status, iso.isoloco_route_tokens, *changed(ROUTE, **change))


ROUTE_GRAD = dict(scores=A, ld=16, dtype=0, tokens=10, experts=16, top_k=4, normalize=0, expert=B, dweight=C, dscores=D,
                  ld_d=16)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(scores=0)), (INVALID, dict(expert=0)), (INVALID, dict(dweight=0)), (INVALID, dict(dscores=0)),
    (INVALID, dict(ld_d=15)), (INVALID, dict(dtype=-1)), (INVALID, dict(top_k=20)), (ALIGN, dict(dscores=D + 2)),
    (ALIGN, dict(expert=B + 2)), (ALIAS, dict(dscores=A)), (ALIAS, dict(dscores=C)), (ALIAS, dict(dscores=B - 64)),
])
def test_route_backward_refuses(status, change):
    refused(status, iso.isoloco_route_tokens_backward, *changed(ROUTE_GRAD, **change))


# 20 tokens in 40 rows, 5 experts of 32 x 64
EXPERTS = dict(x=A, ld_x=64, tokens=20, token=B, w=C, ld_w=64, stride_w=2048, dtype=1, offsets=D, index_type=0,
               experts=5, rows=40, dim=64, cols=32, out=E, ld_out=32, workspace=WS, ws_bytes=BIG)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(x=0)), (INVALID, dict(w=0)), (INVALID, dict(offsets=0)), (INVALID, dict(out=0)),
    (INVALID, dict(token=0)), (INVALID, dict(ld_x=63)), (INVALID, dict(ld_w=63)), (INVALID, dict(ld_out=31)),
    (INVALID, dict(stride_w=2047)), (INVALID, dict(dtype=2)), (INVALID, dict(index_type=2)), (INVALID, dict(experts=0)),
    (INVALID, dict(experts=1025)), (INVALID, dict(rows=-1)), (INVALID, dict(tokens=-1)), (INVALID, dict(dim=0)),
    (INVALID, dict(cols=0)), (INVALID, dict(dim=1 << 22, ld_x=1 << 22, ld_w=1 << 22, stride_w=1 << 28)),
    (ALIGN, dict(x=A + 1)), (ALIGN, dict(w=C + 1)), (ALIGN, dict(out=E + 1)), (ALIGN, dict(offsets=D + 2)),
    (ALIGN, dict(token=B + 1)), (ALIAS, dict(out=A)), (ALIAS, dict(out=C + 64)), (ALIAS, dict(out=B)),
    (ALIAS, dict(out=D)),
    # (float32, and rows of 60: copies, once the rows are many)
    (WORKSPACE, dict(dtype=0, rows=1000, workspace=0)), (WORKSPACE, dict(dim=60, rows=1000, ws_bytes=64)),
    (WORKSPACE, dict(dtype=0, rows=1000, workspace=WS + 8)), (ALIAS, dict(dtype=0, rows=1000, out=WS + 256)),
])
def test_expert_matmul_refuses(status, change):
    refused(status, iso.isoloco_expert_matmul, *changed(EXPERTS, **change))


EXPERTS_GRAD = dict(x=A, ld_x=64, tokens=20, token=B, w=C, ld_w=64, stride_w=2048, dtype=0, offsets=D, index_type=1,
                    experts=5, rows=40, dim=64, cols=32, dout=E, ld_dout=32, dx=F, ld_dx=64, dw=F + 65536, ld_dw=64,
                    stride_dw=2048, workspace=WS, ws_bytes=BIG)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(x=0)), (INVALID, dict(w=0)), (INVALID, dict(offsets=0)), (INVALID, dict(dout=0)),
    (INVALID, dict(token=0)), (INVALID, dict(ld_dx=10)), (INVALID, dict(ld_dw=10)), (INVALID, dict(ld_dout=31)),
    (INVALID, dict(stride_dw=100)), (INVALID, dict(index_type=-1)), (ALIGN, dict(dx=F + 2)), (ALIGN, dict(dw=F + 65537)),
    (ALIGN, dict(offsets=D + 4)), (ALIAS, dict(dx=A)), (ALIAS, dict(dw=F)), (ALIAS, dict(dw=E)), (ALIAS, dict(dx=C)),
    (WORKSPACE, dict(workspace=0)), (WORKSPACE, dict(ws_bytes=64)), (WORKSPACE, dict(workspace=WS + 16)),
])
def test_expert_matmul_backward_refuses(status, change):
    refused(status, iso.isoloco_expert_matmul_backward, *changed(EXPERTS_GRAD, **change))


COMBINE = dict(y=A, ld_y=64, dtype=1, rows=40, dim=64, row=B, index_type=0, weight=C, tokens=20, top_k=2, out=D, ld_out=64)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(y=0)), (INVALID, dict(row=0)), (INVALID, dict(out=0)), (INVALID, dict(ld_y=63)),
    (INVALID, dict(ld_out=63)), (INVALID, dict(dtype=5)), (INVALID, dict(index_type=5)), (INVALID, dict(top_k=0)),
    (INVALID, dict(top_k=33)), (INVALID, dict(rows=-1)), (INVALID, dict(tokens=-1)), (INVALID, dict(dim=0)),
    (ALIGN, dict(y=A + 1)), (ALIGN, dict(weight=C + 2)), (ALIGN, dict(row=B + 2)), (ALIAS, dict(out=A)),
    (ALIAS, dict(out=B)), (ALIAS, dict(out=C)),
])
def test_combine_refuses(status, change):
    refused(status, iso.isoloco_combine_tokens, *changed(COMBINE, **change))


COMBINE_GRAD = dict(dout=A, ld_dout=64, y=B, ld_y=64, dtype=1, rows=40, dim=64, row=C, index_type=1, weight=D, tokens=20,
                    top_k=2, dy=E, ld_dy=64, dweight=F, workspace=WS, ws_bytes=BIG)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(dout=0)), (INVALID, dict(y=0)), (INVALID, dict(row=0)), (INVALID, dict(weight=0)),
    (INVALID, dict(ld_dy=10)), (INVALID, dict(ld_dout=10)), (ALIGN, dict(dy=E + 1)), (ALIGN, dict(dweight=F + 1)),
    (ALIGN, dict(row=C + 4)), (ALIAS, dict(dy=A)), (ALIAS, dict(dy=B)), (ALIAS, dict(dweight=D)), (ALIAS, dict(dweight=E)),
    # (slots that are counted apart)
    (WORKSPACE, dict(tokens=5000, workspace=0)), (WORKSPACE, dict(tokens=5000, ws_bytes=512)),
    (WORKSPACE, dict(tokens=5000, workspace=WS + 8)), (ALIAS, dict(tokens=5000, dweight=WS + 256)),
])
def test_combine_backward_refuses(status, change):
    refused(status, iso.isoloco_combine_tokens_backward, *changed(COMBINE_GRAD, **change))


DISTILL = dict(logits=A, ld=1000, dtype=1, rows=3, vocab=1000, top_logprob=B, top_index=C, index_type=1, top_k=8, scale=1.0,
               rest=1, loss=D, stats=E, workspace=WS, ws_bytes=BIG)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(logits=0)), (INVALID, dict(top_logprob=0)), (INVALID, dict(top_index=0)), (INVALID, dict(loss=0)),
    (INVALID, dict(stats=0)), (INVALID, dict(rows=-1)), (INVALID, dict(vocab=0)), (INVALID, dict(ld=999)),
    (INVALID, dict(dtype=2)), (INVALID, dict(index_type=2)), (INVALID, dict(top_k=0)), (INVALID, dict(top_k=129)),
    (INVALID, dict(rest=2)), (INVALID, dict(scale=0.0)), (INVALID, dict(scale=-1.0)), (INVALID, dict(scale=math.nan)),
    (INVALID, dict(scale=math.inf)), (ALIGN, dict(logits=A + 1)), (ALIGN, dict(top_logprob=B + 2)),
    (ALIGN, dict(top_index=C + 4)), (ALIGN, dict(stats=E + 2)), (ALIAS, dict(loss=A)), (ALIAS, dict(stats=B)),
    (ALIAS, dict(loss=C)), (ALIAS, dict(stats=D - 8)),
    # (two rows of 100000: split, so that a workspace is needed)
    (WORKSPACE, dict(rows=2, vocab=100000, ld=100000, workspace=0)),
    (WORKSPACE, dict(rows=2, vocab=100000, ld=100000, ws_bytes=8)),
    (ALIAS, dict(rows=2, vocab=100000, ld=100000, loss=WS)),
])
def test_distill_refuses(status, change):
    refused(status, iso.isoloco_distill_loss, *changed(DISTILL, **change))


DISTILL_GRAD = dict(logits=A, ld=1000, dtype=1, rows=3, vocab=1000, top_logprob=B, top_index=C, index_type=0, top_k=8,
                    scale=1.0, rest=0, stats=D, dloss=E, dlogits=F, ld_d=1000)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(logits=0)), (INVALID, dict(stats=0)), (INVALID, dict(dloss=0)), (INVALID, dict(dlogits=0)),
    (INVALID, dict(top_index=0)), (INVALID, dict(ld_d=10)), (INVALID, dict(scale=0.0)), (INVALID, dict(rest=-1)),
    (ALIGN, dict(dlogits=F + 1)), (ALIGN, dict(dloss=E + 2)), (ALIAS, dict(dlogits=A, ld_d=1008)),
    (ALIAS, dict(dlogits=A + 16)), (ALIAS, dict(dlogits=B)), (ALIAS, dict(dlogits=C)), (ALIAS, dict(dlogits=D)),
    (ALIAS, dict(dlogits=E)),
])
def test_distill_backward_refuses(status, change):
    refused(status, iso.isoloco_distill_loss_backward, *changed(DISTILL_GRAD, **change))


def test_workspace_sizes_refuse():
    refused(INVALID, iso.isoloco_route_tokens_workspace_size, -1, 8)
    refused(INVALID, iso.isoloco_route_tokens_workspace_size, 5, 0)
    refused(INVALID, iso.isoloco_expert_matmul_workspace_size, 5, 5, 0, 8, 8, 8, 0, 0)
    refused(INVALID, iso.isoloco_expert_matmul_workspace_size, 5, 5, 1, 8, 8, 8, 0, 8)
    refused(INVALID, iso.isoloco_distill_loss_workspace_size, 5, 0)
    refused(INVALID, iso.isoloco_combine_tokens_backward_workspace_size, -1, 2)
    refused(INVALID, iso.isoloco_combine_tokens_backward_workspace_size, 5, 0)


def test_workspace_of_experts_covers_every_alignment():
    """Without the flag the size is enough whichever operands are aligned: one row of x far
    from the next, so that gathered rows are copied, and weights that are too."""
    need = iso.isoloco_expert_matmul_workspace_size
    tokens, rows, far = 1000, 8000, 1 << 22
    whole = need(tokens, rows, 8, 64, 64, far, 1, 4)
    # the gathered rows, the weights' copy
    assert whole >= rows * 64 * 2 + 8 * 64 * 64 * 2
    assert need(tokens, rows, 8, 64, 64, 64, 1, 4 | 2) < whole


def test_nothing_is_nothing():
    """Calls without rows end before any launch."""
    iso.isoloco_expert_matmul(*changed(EXPERTS, rows=0))
    iso.isoloco_combine_tokens(*changed(COMBINE, tokens=0))
    iso.isoloco_combine_tokens_backward(*changed(COMBINE_GRAD, dy=0, dweight=0, workspace=0))
    iso.isoloco_distill_loss(*changed(DISTILL, rows=0))
    iso.isoloco_route_tokens_backward(*changed(ROUTE_GRAD, tokens=0))


def test_launches_past_32_bits_of_threads_are_refused():
    refused(UNSUPPORTED, iso.isoloco_distill_loss_backward, *changed(
        DISTILL_GRAD, rows=1 << 25, ld=1, ld_d=1, vocab=1, top_k=1, top_logprob=1 << 40, top_index=1 << 41, stats=1 << 42,
        dloss=1 << 43, dlogits=1 << 44))
    refused(UNSUPPORTED, iso.isoloco_combine_tokens, *changed(
        COMBINE, tokens=1 << 28, dim=256, ld_y=256, ld_out=256, row=1 << 40, weight=1 << 41, out=1 << 42))


def test_tiles_past_32_bits_are_refused():
    far = dict(x=1 << 60, w=1 << 58, out=1 << 59, offsets=64, token=1 << 44)
    refused(UNSUPPORTED, iso.isoloco_expert_matmul, *changed(
        EXPERTS, **far, rows=1 << 30, cols=1 << 20, ld_out=1 << 20, stride_w=1 << 26, dim=64))
    refused(UNSUPPORTED, iso.isoloco_expert_matmul_workspace_size, 5, 5, 1, 4000000, 4000000, 4000000, 1, 0)


def test_tensors_on_the_host_are_refused():
    t, w, i = torch.zeros(4, 8), torch.zeros(2, 3, 8), torch.zeros(3, dtype=torch.int32)
    rows = torch.zeros(2, 2, dtype=torch.int32)
    for f in (lambda: iso.route_tokens(t, 2), lambda: iso.route_tokens_backward(t, rows, t),
              lambda: iso.expert_matmul(t, w, i), lambda: iso.expert_matmul_backward(t, w, i, torch.zeros(4, 3)),
              lambda: iso.combine_tokens(t, rows), lambda: iso.combine_tokens_backward(t, t, rows),
              lambda: iso.distill_loss(t, t, i), lambda: iso.distill_loss_backward(t, t, i, t, t)):
        with pytest.raises(ValueError):
            f()
