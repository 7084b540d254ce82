"""What the inner step's operators refuse, before anything is enqueued (no GPU
needed: the calls end in the argument checks, and the addresses are never read)."""
import ctypes
import math

import pytest

iso = pytest.importorskip("paper_2607_03011_amd")
torch = pytest.importorskip("torch")

INVALID, ALIGN, ALIAS, WORKSPACE = -1, -3, -4, -5
A, B, C, D, E, F, WS = (0x10000000 * (i + 1) for i in range(7))  # addresses far apart
BIG = 1 << 27


def refused(status, f, *args):
    with pytest.raises(iso.IsoLoCoError) as ei:
        f(*args)
    assert ei.value.status == status
    assert iso.isoloco_last_error() != ""


def changed(good, **change):
    return [change.get(k, v) for k, v in good.items()]


CLIP = dict(src=[A, B], dst=[A, B], counts=[100, 7], dtypes=[0, 1], max_norm=1.0, norm=C, workspace=WS, ws_bytes=BIG)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(norm=0)), (INVALID, dict(max_norm=-1.0)), (INVALID, dict(max_norm=math.nan)),
    (INVALID, dict(counts=[-1, 7])), (INVALID, dict(dtypes=[0, 2])), (INVALID, dict(src=[0, B])),
    (INVALID, dict(dst=[A, 0])), (ALIGN, dict(src=[A + 2, B], dst=[A + 2, B])), (ALIGN, dict(dst=[A, B + 1])),
    (ALIGN, dict(norm=C + 2)), (ALIAS, dict(dst=[A + 4, B])), (ALIAS, dict(norm=A + 8)), (ALIAS, dict(src=[WS, B])),
    (WORKSPACE, dict(workspace=0)), (WORKSPACE, dict(ws_bytes=16)), (WORKSPACE, dict(workspace=WS + 128)),
])
def test_clip_refuses(status, change):
    refused(status, iso.isoloco_clip_grads, *changed(CLIP, **change))


EMBED = dict(table=A, ld=64, dtype=0, vocab=10, dim=64, ids=B, id_type=1, n=5, scale=1.0, out=C, ld_out=64, out_dtype=1)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(table=0)), (INVALID, dict(ids=0)), (INVALID, dict(out=0)), (INVALID, dict(dtype=2)),
    (INVALID, dict(out_dtype=-1)), (INVALID, dict(id_type=2)), (INVALID, dict(vocab=0)), (INVALID, dict(dim=0)),
    (INVALID, dict(n=-1)), (INVALID, dict(ld=63)), (INVALID, dict(ld_out=60)), (INVALID, dict(n=1 << 40)),
    (ALIGN, dict(table=A + 2)), (ALIGN, dict(ids=B + 4)), (ALIGN, dict(out=C + 1)),
    (ALIAS, dict(out=A + 128)), (ALIAS, dict(out=B)),
])
def test_embedding_refuses(status, change):
    refused(status, iso.isoloco_embedding, *changed(EMBED, **change))


EMBED_GRAD = dict(ids=A, id_type=0, n=5, dout=B, ld=64, dtype=1, vocab=10, dim=64, scale=1.0, accumulate=0, dtable=C,
                  ld_dtable=64, dtable_dtype=0, workspace=WS, ws_bytes=BIG)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(ids=0)), (INVALID, dict(dout=0)), (INVALID, dict(dtable=0)), (INVALID, dict(dtype=3)),
    (INVALID, dict(dtable_dtype=3)), (INVALID, dict(id_type=-1)), (INVALID, dict(vocab=-3)), (INVALID, dict(ld=10)),
    (INVALID, dict(ld_dtable=10)), (ALIGN, dict(dout=B + 1)), (ALIGN, dict(dtable=C + 2)), (ALIAS, dict(dtable=B)),
    (ALIAS, dict(dtable=A)), (ALIAS, dict(dout=WS)), (WORKSPACE, dict(workspace=0)), (WORKSPACE, dict(ws_bytes=100)),
    (WORKSPACE, dict(workspace=WS + 8)),
])
def test_embedding_backward_refuses(status, change):
    refused(status, iso.isoloco_embedding_backward, *changed(EMBED_GRAD, **change))


LOGPROB = dict(logits=A, ld=100, dtype=1, rows=3, vocab=100, targets=B, target_type=1, scale=1.0, top_k=2, logprob=C,
               entropy=C + 64, lse=C + 128, top=C + 256, index=C + 512, workspace=WS, ws_bytes=BIG)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(logits=0)), (INVALID, dict(targets=0)), (INVALID, dict(logprob=0)), (INVALID, dict(rows=-1)),
    (INVALID, dict(vocab=0)), (INVALID, dict(ld=99)), (INVALID, dict(dtype=9)), (INVALID, dict(target_type=9)),
    (INVALID, dict(scale=0.0)), (INVALID, dict(scale=-1.0)), (INVALID, dict(scale=math.nan)),
    (INVALID, dict(scale=math.inf)), (INVALID, dict(top_k=-1)), (INVALID, dict(top_k=33)),
    (INVALID, dict(vocab=1, ld=1, top_k=2)), (INVALID, dict(top=0)), (INVALID, dict(index=0)),
    (ALIGN, dict(logits=A + 1)), (ALIGN, dict(entropy=C + 66)), (ALIGN, dict(index=C + 516)),
    (ALIAS, dict(lse=A + 8)), (ALIAS, dict(entropy=C)), (ALIAS, dict(logprob=B)),
])
def test_token_logprobs_refuses(status, change):
    refused(status, iso.isoloco_token_logprobs, *changed(LOGPROB, **change))


LOGPROB_GRAD = dict(logits=A, ld=100, dtype=1, rows=3, vocab=100, targets=B, target_type=1, scale=1.0, lse=C,
                    entropy=C + 64, dlogprob=C + 128, dentropy=C + 256, dlogits=D, ld_d=100)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(logits=0)), (INVALID, dict(dlogits=0)), (INVALID, dict(lse=0)), (INVALID, dict(targets=0)),
    (INVALID, dict(dlogprob=0)), (INVALID, dict(entropy=0)), (INVALID, dict(scale=0.0)), (INVALID, dict(ld_d=50)),
    (ALIGN, dict(dlogits=D + 1)), (ALIGN, dict(lse=C + 2)), (ALIAS, dict(dlogits=A, ld_d=104)),
    (ALIAS, dict(dlogits=A + 16)), (ALIAS, dict(dlogits=C - 16)),
])
def test_token_logprobs_backward_refuses(status, change):
    refused(status, iso.isoloco_token_logprobs_backward, *changed(LOGPROB_GRAD, **change))


FFN = dict(x=A, ld_x=64, wg=B, wu=C, ld_w=64, dtype=1, tokens=5, dim=64, hidden=32, act=0, out=D, ld_out=32,
           workspace=WS, ws_bytes=BIG)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(x=0)), (INVALID, dict(wg=0)), (INVALID, dict(wu=0)), (INVALID, dict(out=0)), (INVALID, dict(act=2)),
    (INVALID, dict(dtype=2)), (INVALID, dict(tokens=-1)), (INVALID, dict(dim=0)), (INVALID, dict(hidden=0)),
    (INVALID, dict(ld_x=63)), (INVALID, dict(ld_w=63)), (INVALID, dict(ld_out=31)), (ALIGN, dict(x=A + 1)),
    (ALIGN, dict(out=D + 1)), (ALIAS, dict(out=A)), (ALIAS, dict(out=C + 64)),
])
def test_gated_ffn_refuses(status, change):
    refused(status, iso.isoloco_gated_ffn, *changed(FFN, **change))


FFN_GRAD = dict(x=A, ld_x=64, wg=B, wu=C, ld_w=64, dtype=1, tokens=5, dim=64, hidden=32, act=0, dout=D, ld_dout=32,
                dx=E, ld_dx=64, dwg=F, dwu=F + 8192, ld_dw=64, workspace=WS, ws_bytes=BIG)


@pytest.mark.parametrize("status,change", [
    (INVALID, dict(x=0)), (INVALID, dict(dout=0)), (INVALID, dict(dwg=0)), (INVALID, dict(dwu=0)),
    (INVALID, dict(ld_dx=10)), (INVALID, dict(ld_dw=10)), (INVALID, dict(act=-1)), (ALIGN, dict(dx=E + 1)),
    (ALIAS, dict(dx=A)), (ALIAS, dict(dwu=F)), (ALIAS, dict(dwg=D)), (WORKSPACE, dict(workspace=0)),
    (WORKSPACE, dict(ws_bytes=64)), (WORKSPACE, dict(workspace=WS + 16)),
])
def test_gated_ffn_backward_refuses(status, change):
    refused(status, iso.isoloco_gated_ffn_backward, *changed(FFN_GRAD, **change))


def test_workspace_sizes_refuse():
    refused(INVALID, iso.isoloco_clip_workspace_size, -1)
    refused(INVALID, iso.isoloco_embedding_backward_workspace_size, 5, 0, 8)
    refused(INVALID, iso.isoloco_token_logprobs_workspace_size, 5, 10, 11)
    refused(INVALID, iso.isoloco_gated_ffn_workspace_size, 5, 0, 8, 0, 0)
    lib = ctypes.CDLL(iso.LIB_PATH)
    assert lib.isoloco_clip_workspace_size(1, None) == INVALID


def test_tensors_on_the_host_are_refused():
    t = torch.zeros(4, 8)
    ids = torch.zeros(4, dtype=torch.int64)
    for f in (lambda: iso.clip_grads([t], 1.0), lambda: iso.embedding(t, ids), lambda: iso.embedding_backward(ids, t, 9),
              lambda: iso.token_logprobs(t, ids), lambda: iso.gated_ffn(t, t, t),
              lambda: iso.gated_ffn_backward(t, t, t, t)):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(ValueError):
        iso.clip_grads([], 1.0)


# the results and the other tensors lie 400 bytes (100 float32) and 14 bytes (7 bfloat16) long
@pytest.mark.parametrize("src,dst", [
    ([A, A], [A, A]), ([A, B], [C, C]), ([A, B], [C, C + 396]), ([A, B], [C + 12, C]), ([A, B], [B, C]),
    ([A, A + 200], [A, D]), ([A, B], [C, A + 396]),
])
def test_clip_refuses_a_result_over_another_tensor(src, dst):
    refused(ALIAS, iso.isoloco_clip_grads, *changed(CLIP, src=src, dst=dst, norm=E))


def test_clip_finds_the_long_range_before_short_ones():
    # tensor 0 reaches over 1 and 2, which lie apart from each other
    refused(ALIAS, iso.isoloco_clip_grads, [A, B, C], [D, D + 1000, D + 2000], [1000, 4, 4], [0, 0, 0], 1.0, E, WS, BIG)
    refused(ALIAS, iso.isoloco_clip_grads, [A, B, C], [D, E, A + 2000], [1000, 4, 4], [0, 0, 0], 1.0, F, WS, BIG)


def test_workspace_overlaps_are_refused():
    refused(ALIAS, iso.isoloco_clip_grads, *changed(CLIP, norm=WS + 64))
    # (two rows of 50000: split, so that a workspace is needed)
    long = dict(LOGPROB, ld=50000, rows=2, vocab=50000)
    for change in (dict(targets=WS), dict(lse=WS + 8), dict(index=WS + 64), dict(logits=WS)):
        refused(ALIAS, iso.isoloco_token_logprobs, *changed(long, **change))


def test_launches_past_32_bits_of_threads_are_refused():
    refused(-7, iso.isoloco_embedding, *changed(EMBED, n=1 << 26, dim=64, table=A, ids=1 << 40, out=1 << 41))
    refused(-7, iso.isoloco_token_logprobs, *changed(
        LOGPROB, rows=1 << 26, ld=1, vocab=1, top_k=0, targets=1 << 40, logprob=1 << 41, entropy=1 << 42, lse=1 << 43))
    refused(-7, iso.isoloco_token_logprobs_backward, *changed(
        LOGPROB_GRAD, rows=1 << 24, ld=1, ld_d=1, vocab=1, targets=1 << 40, lse=1 << 41, entropy=1 << 42,
        dlogprob=1 << 43, dentropy=1 << 44, dlogits=1 << 45))
