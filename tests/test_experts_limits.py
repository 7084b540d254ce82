"""What the entry points refuse and what they take where their ranges end (no GPU needed: the
calls end before anything is enqueued, and the addresses are never read)."""
import pytest

from test_experts_refusals import (ALIAS, ALIGN, BIG, EXPERTS, EXPERTS_GRAD, INVALID, WORKSPACE, WS, A, B, C, D, E,  # noqa: F401
                                   F, changed, iso, refused)

G, H = 0x90000000, 0xa0000000

# 20 tokens in 40 rows, 5 experts of 32 x 64, float32
TOKENS_GRAD = dict(x=A, ld_x=64, tokens=20, token=B, row=G, row_type=0, top_k=2, w=C, ld_w=64, stride_w=2048, dtype=0,
                   offsets=D, index_type=1, experts=5, rows=40, dim=64, cols=32, dout=E, ld_dout=32, dx=F, ld_dx=64,
                   dx_rows=H, dw=F + 65536, ld_dw=64, stride_dw=2048, workspace=WS, ws_bytes=BIG)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(x=0)), (INVALID, dict(w=0)), (INVALID, dict(offsets=0)), (INVALID, dict(dout=0)),
    (INVALID, dict(token=0)), (INVALID, dict(row=0)), (INVALID, dict(dx=0)), (INVALID, dict(dx_rows=0)),
    (INVALID, dict(dw=0, token=0)), (INVALID, dict(row_type=2)), (INVALID, dict(index_type=-1)), (INVALID, dict(top_k=0)),
    (INVALID, dict(top_k=33)), (INVALID, dict(ld_dx=10)), (INVALID, dict(ld_dw=10)), (INVALID, dict(ld_dout=31)),
    (INVALID, dict(dtype=2)), (ALIGN, dict(dx=F + 2)), (ALIGN, dict(row=G + 2)), (ALIGN, dict(row_type=1, row=G + 4)),
    (ALIGN, dict(dx_rows=H + 2)), (ALIAS, dict(dx=A)), (ALIAS, dict(dx=G)), (ALIAS, dict(dx_rows=E)),
    (ALIAS, dict(dx_rows=F)), (ALIAS, dict(dx_rows=F + 65536)), (ALIAS, dict(dx_rows=WS)),
    (WORKSPACE, dict(workspace=0)), (WORKSPACE, dict(ws_bytes=64)), (WORKSPACE, dict(workspace=WS + 16)),
])
def test_expert_matmul_backward_tokens_refuses(status, change):
    refused(status, iso.isoloco_expert_matmul_backward_tokens, *changed(TOKENS_GRAD, **change))


def test_expert_gradients_of_neither_operand_read_nothing():
    """Neither dx nor dw wanted: no operand is read and no workspace needed, whatever the sizes."""
    for rows in (40, 1000, 100000):
        iso.isoloco_expert_matmul_backward(*changed(EXPERTS_GRAD, rows=rows, x=0, w=0, dx=0, dw=0, workspace=0))
    # and a gradient of no token is none
    iso.isoloco_expert_matmul_backward_tokens(*changed(TOKENS_GRAD, rows=1000, tokens=0, x=0, dx=0, row=0, dw=0, workspace=0))


def test_no_rows_of_some_tokens_are_nothing():
    """No place of the grouped order names any token: an empty tensor has no address."""
    iso.isoloco_expert_matmul(*changed(EXPERTS, rows=0, token=0, out=0))
    iso.isoloco_expert_matmul_backward(*changed(EXPERTS_GRAD, rows=0, token=0, dout=0, dx=0, dw=0, workspace=0))
