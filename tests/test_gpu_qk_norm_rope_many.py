"""GPU parity of the q/k norm at sizes that take its other kernels: several heads a lane group in every width and type, the
element-by-element form with more tokens than there are partial rows, and as many heads as there may be; against fp64 on the GPU.

Tolerances as in test_gpu_qk_norm_rope.py, held row by row, so that no row can hide among many."""
import pytest
import torch

import paper_2505_23725_amd as mlc
import synth_inputs as S
from helpers import EW_TOL

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _reference(dy, x, gain, offset, cos, sin, eps, inter):
    """y, dx and the gain's gradient in fp64; cos, sin: [tokens, rot / 2]."""
    x, dy, w, c, s = x.double(), dy.double(), gain.double() + offset, cos.double()[:, None], sin.double()[:, None]
    rot = 2 * cos.shape[1]

    def turn(v, s):
        out = v.clone()
        a, b = (v[..., 0:rot:2], v[..., 1:rot:2]) if inter else (v[..., :rot // 2], v[..., rot // 2:rot])
        ya, yb = a * c - b * s, b * c + a * s
        if inter:
            out[..., 0:rot:2], out[..., 1:rot:2] = ya, yb
        else:
            out[..., :rot // 2], out[..., rot // 2:rot] = ya, yb
        return out
    r = (x.square().mean(-1, keepdim=True) + eps).rsqrt()
    dn = turn(dy, -s)
    d = dn * w
    return turn(x * r * w, s), r * (d - x * r.square() * (d * x).mean(-1, keepdim=True)), (dn * x * r).sum((0, 1))


def _rows_close(got, ref, what):
    off = (got.double() - ref).abs()
    if got.dtype == torch.float32:
        norm = ref.norm(dim=-1)
        bad = off.norm(dim=-1) > EW_TOL * norm.clamp(min=norm.mean().item())
    else:          # a correct rounding of a value that close: half a unit of the 8 bits
        half = torch.ldexp(torch.ones_like(ref), torch.frexp(ref)[1] - 9)
        bad = (off > half + EW_TOL * ref.abs().clamp(min=ref.square().mean().sqrt().item())).any(-1)
    assert not bad.any(), (what, bad.nonzero()[:4].tolist())


@pytest.mark.parametrize("dim,rot,inter,dtype,tokens,hq,hk", [
    (64, 64, False, torch.float32, 22001, 7, 3), (24, 16, True, torch.bfloat16, 22001, 7, 3),
    (128, 64, True, torch.float32, 11003, 7, 3), (120, 120, False, torch.bfloat16, 11003, 6, 2),
    (256, 256, False, torch.bfloat16, 5501, 7, 3), (200, 104, True, torch.float32, 5501, 9, 1),
    (512, 512, True, torch.bfloat16, 2801, 7, 3), (384, 128, False, torch.float32, 2801, 7, 3),
    (64, 64, False, torch.bfloat16, 33001, 7, 0), (128, 128, False, torch.bfloat16, 3, 1024, 1024),
    # element by element
    (20, 12, False, torch.bfloat16, 7001, 7, 3), (122, 116, True, torch.float32, 3501, 7, 3),
    (250, 250, False, torch.bfloat16, 1801, 7, 3), (510, 508, True, torch.float32, 901, 7, 3), (126, 126, False, torch.float32, 40001, 2, 1)])
@pytest.mark.parametrize("offset", [0.0, 1.0])
def test_forward_and_backward(dim, rot, inter, dtype, tokens, hq, hk, offset):
    new = lambda shape, i, dt=dtype: S.normal(shape, 1.0, 9, i, dtype=dt, device=DEV)  # noqa: E731
    q, k, dq, dk = (new((tokens, h, dim), i) for i, h in enumerate((hq, hk, hq, hk)))
    wq, wk = new((dim,), 4, torch.float32) * 0.3, new((dim,), 5, torch.float32) * 0.3
    rows = 500
    angle = torch.arange(rows, device=DEV)[:, None] * 1e4 ** (-torch.arange(rot // 2, device=DEV) / (rot // 2))
    cos, sin = angle.cos().contiguous(), angle.sin().contiguous()
    pos = torch.randint(0, rows, (tokens,), generator=torch.Generator(device=DEV).manual_seed(1), device=DEV)
    nan = lambda t: torch.full_like(t, float("nan"))  # noqa: E731
    y, dx, dw = (nan(q), nan(k)), (nan(q), nan(k)), (nan(wq), nan(wk))
    hp = mlc.QKNormRopeHParams(eps=1e-5, gain_offset=offset, interleaved=inter)
    ws = torch.full((mlc.muloco_qk_norm_rope_workspace_bytes(dim),), 255, dtype=torch.uint8, device=DEV)
    mlc.muloco_qk_norm_rope(q, k, wq, wk, cos, sin, pos, *y, hp)
    mlc.muloco_qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, *dx, *dw, ws, hp)
    for i, (x, w, dy, what) in enumerate(((q, wq, dq, "q"), (k, wk, dk, "k"))):
        if x.shape[1] == 0:
            assert not dw[i].any()
            continue
        ry, rx, rw = _reference(dy, x, w, offset, cos[pos], sin[pos], 1e-5, inter)
        _rows_close(y[i], ry, what)
        _rows_close(dx[i], rx, "d" + what)
        assert (dw[i].double() - rw).norm() <= EW_TOL * rw.norm(), what


def test_squares_beyond_the_range():
    """(as the header states it; the largest whose squares still fit are normed as any others)"""
    x = torch.full((2, 2, 64), 1e18, device=DEV)
    x[1] = 1e30
    one, none, pos = torch.ones(64, device=DEV), torch.empty(0, 0, device=DEV), torch.zeros(2, dtype=torch.int64, device=DEV)
    y, k = torch.empty_like(x), torch.empty(2, 0, 64, device=DEV)
    mlc.muloco_qk_norm_rope(x, k, one, one, none, none, pos, y, k)
    assert torch.allclose(y[0], torch.ones_like(y[0]), rtol=1e-6) and not y[1].any()
