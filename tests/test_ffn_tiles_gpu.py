"""Every kernel instance of the gated block's tile products against the formulas in 64 bits
(on the GPU: plain float64 products), with both activations."""
import pytest

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

from _ffn_cases import CASES  # noqa: E402
from test_operators_gpu import BF16, F32, ROUND, U32, ffn_inputs, ffn_reference, gen, iso, randn  # noqa: E402,F401


def close(got, want, bound, name):
    far = ((got.double() - want).abs() - bound).max().item()
    assert torch.isfinite(got).all() and far <= 0, "%s off by %g more than the bound" % (name, far)


@pytest.mark.parametrize("act", ["silu", "gelu"])
@pytest.mark.parametrize("f32,tokens,dim,hidden", [c[:4] for c in CASES])
def test_instance(iso, f32, tokens, dim, hidden, act):  # noqa: F811
    """The bounds are those of a sum of n float32 terms, of the activations' slopes (|act'| <=
    1.13, |act''| <= 0.8) and of the roundings of da, du (bfloat16) and of the results."""
    dtype = F32 if f32 else BF16
    x, wg, wu, dh = (t.cuda() for t in ffn_inputs(tokens, dim, hidden, dtype, 21))
    g, u, a, da, eg, eu, ea = ffn_reference(x, wg, wu, act)
    want = a * u
    close(iso.gated_ffn(x, wg, wu, act=act), want,
          ea * u.abs() + a.abs() * eu + ea * eu + ROUND[dtype] * want.abs() + 1e-37, "out")
    X, G, W, D = (t.double() for t in (x, wg, wu, dh))
    dg, du = D * u * da, D * a
    rnd = 4 * U32 if f32 else ROUND[dtype]
    edg = D.abs() * ((da.abs() + 1e-6) * eu + u.abs() * (0.8 * eg + 16 * U32) + 0.8 * eg * eu) + rnd * dg.abs()
    edu = D.abs() * ea + rnd * du.abs()
    del g, u, a, da, eg, eu, ea
    nk, nt = (2 * hidden + 8) * U32, (tokens + 8) * U32
    grads = iso.gated_ffn_backward(x, wg, wu, dh, act=act)
    for name, got, want, bound in (
            ("dx", grads[0], dg @ G + du @ W,
             edg @ G.abs() + edu @ W.abs() + nk * (dg.abs() @ G.abs() + du.abs() @ W.abs())),
            ("dw_gate", grads[1], dg.T @ X, edg.T @ X.abs() + nt * (dg.abs().T @ X.abs())),
            ("dw_up", grads[2], du.T @ X, edu.T @ X.abs() + nt * (du.abs().T @ X.abs()))):
        close(got, want, 1.01 * bound + ROUND[dtype] * want.abs() + 1e-37, name)
        # random errors: far below the bound's worst case
        assert ((got.double() - want).norm() / want.norm()).item() <= (2.0 ** -20 if f32 else 2.0 ** -8)
    # one of the products alone: the same bits
    assert torch.equal(iso.gated_ffn_backward(x, wg, wu, dh, act=act, need_dw=False)[0], grads[0])
    only = iso.gated_ffn_backward(x, wg, wu, dh, act=act, need_dx=False)
    assert torch.equal(only[1], grads[1]) and torch.equal(only[2], grads[2])
