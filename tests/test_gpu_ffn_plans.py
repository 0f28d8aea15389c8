"""GPU parity of the gated feed-forward block at shapes that take every kernel and every dealing of its tiles, against fp64 on the GPU
with the element bounds of oracle/gated_ffn.py (tolerances as in test_gpu_gated_ffn.py)."""
import math

import pytest
import torch

import paper_2505_23725_amd as mlc
import synth_inputs as S
from ffn_shapes import PLAN_SHAPES
from oracle.gated_ffn import U

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16
FRO = 6e-3
GUARD = 512


def _reference(x, wg, wu, wd, dy, act):
    """name -> (value, bound), in fp64."""
    x, wg, wu, wd, dy = (v.double() for v in (x, wg, wu, wd, dy))
    g, u = x @ wg.t(), x @ wu.t()
    if act == "silu":
        s = torch.sigmoid(g)
        a, da = g * s, s + g * s * (1 - s)
    else:
        c, k = math.sqrt(2 / math.pi), 0.044715
        s = torch.sigmoid(2 * c * (g + k * g ** 3))
        a, da = g * s, s + 2 * c * g * s * (1 - s) * (1 + 3 * k * g * g)
    h = a * u
    dh = dy @ wd
    dg, du = dh * u * da, dh * a
    eg, eu = 2 * U * dg.abs(), 2 * U * du.abs()
    out = {"y": (h @ wd.t(), U * (h.abs() @ wd.t().abs())),
           "dx": (dg @ wg + du @ wu, eg @ wg.abs() + eu @ wu.abs()),
           "dwg": (dg.t() @ x, eg.t() @ x.abs()), "dwu": (du.t() @ x, eu.t() @ x.abs()),
           "dwd": (dy.t() @ h, U * (dy.t().abs() @ h.abs()))}
    return {k: (v, b + U * v.abs()) for k, (v, b) in out.items()}


@pytest.mark.parametrize("act", ["silu", "gelu_tanh"])
@pytest.mark.parametrize("t,d,f", PLAN_SHAPES)
def test_forward_and_backward(t, d, f, act):
    guards = []

    def between(shape, value=None):
        """A tensor between two runs of NaN."""
        n = math.prod(shape)
        flat = torch.full((n + 2 * GUARD,), float("nan"), dtype=BF, device=DEV)
        guards.append(flat)
        inner = flat[GUARD:GUARD + n].view(shape)
        if value is not None:
            inner.copy_(value)
        return inner

    def work(backward):
        """A work space of exactly the size asked for, of bits that are NaN."""
        n = mlc.muloco_gated_ffn_workspace_bytes(t, d, f, backward)
        flat = torch.full((n + 4096,), 255, dtype=torch.uint8, device=DEV)
        return flat[n:], flat[:n] if n else None
    x, wg, wu, wd, dy = (between(s, S.normal(s, std, 5, i, dtype=BF, device=DEV)) for i, (s, std) in enumerate(
        (((t, d), 1.0), ((f, d), d ** -0.5), ((f, d), d ** -0.5), ((d, f), f ** -0.5), ((t, d), 1.0))))
    y, hidden, gate, up = between((t, d)), between((t, f)), between((t, f)), between((t, f))
    grads = [between((t, d)), between((f, d)), between((f, d)), between((d, f))]
    behind, ws = work(False)
    behind_back, ws_back = work(True)
    mlc.muloco_gated_ffn(x, wg, wu, wd, y, hidden, ws, act=act, gate=gate, up=up)
    mlc.muloco_gated_ffn_backward(dy, x, wg, wu, wd, gate, up, hidden, *grads, ws_back, act=act)
    for flat in guards:
        assert torch.isnan(flat[:GUARD]).all() and torch.isnan(flat[-GUARD:]).all(), "something was written outside a result"
    assert (behind == 255).all() and (behind_back == 255).all(), "something was written behind a work space"
    for (k, (ref, bound)), got in zip(_reference(x, wg, wu, wd, dy, act).items(), [y, *grads]):
        off = got.double() - ref
        assert torch.isfinite(off).all(), k
        over = (off.abs() - 1.02 * bound - 1e-5 * bound.max()).max().item()
        assert over <= 0, f"{k}: {over:.3g} beyond an element's bound"
        assert ref.numel() < 1000 or (off.norm() / ref.norm()).item() <= FRO, (k, (off.norm() / ref.norm()).item())
