"""The training operators on tensors of more than 2^31 elements: what lies behind the range of 32-bit offsets is as right as the rest."""
import numpy as np
import pytest
import torch

import paper_2505_23725_amd as mlc
import synth_inputs as S
import test_gpu_ffn_plans as ffn
from helpers import EW_TOL, assert_stored_close, to_f64
from oracle import adamw8
from test_gpu_qk_norm_rope_many import _reference, _rows_close

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF = torch.bfloat16


def test_adamw8():
    n = (1 << 31) + 3 * 8192 + 77
    param = torch.full((n,), 0.5, dtype=BF, device=DEV)
    grad = torch.full((n,), 1e-3, dtype=BF, device=DEV)
    m8, v8, scales = mlc.adamw8_state(param)
    kw = dict(lr=3e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1)
    # blocks at the front, on both sides of 2^31 and at the end have their own numbers
    size, refs = 2048, []
    for i, at in enumerate((0, (1 << 31) - size, 1 << 31, n - n % 256 - size)):
        to = min(at + size, n) if i < 3 else n
        param[at:to] = S.normal((to - at,), 0.02, 8, i, dtype=BF).to(DEV)
        grad[at:to] = S.normal((to - at,), 1e-3, 8, 10 + i, dtype=BF).to(DEV)
        m8[at:to] = torch.randint(0, 121, (to - at,), generator=torch.Generator().manual_seed(i), dtype=torch.uint8).to(DEV)
        v8[at:to] = torch.randint(150, 249, (to - at,), generator=torch.Generator().manual_seed(9 + i), dtype=torch.uint8).to(DEV)
        blocks = slice(at // 256, (to + 255) // 256)
        scales[blocks] = torch.rand(blocks.stop - blocks.start, 2, generator=torch.Generator().manual_seed(i)).to(DEV) * 1e-3
        s = scales[blocks].cpu().numpy()
        args = to_f64(param[at:to]), to_f64(grad[at:to]), m8[at:to].cpu().numpy(), v8[at:to].cpu().numpy(), s[:, 0].copy(), s[:, 1].copy()
        refs.append((slice(at, to), blocks, adamw8.step(*args, **kw)))
    tensor = (param, grad, m8, v8, scales)
    mlc.muloco_adamw8_step([tensor], mlc.AdamWHParams(**kw))
    for where, blocks, (new, rm, rv, sm, sv, _, _) in refs:
        assert np.array_equal(scales[blocks].cpu().numpy(), np.stack([sm, sv], 1))
        assert np.array_equal(m8[where].cpu().numpy(), rm) and np.array_equal(v8[where].cpu().numpy(), rv)
        assert_stored_close(param[where].cpu(), new, "parameters")
    # every other element is as any other
    rest = torch.ones(n, dtype=torch.bool, device=DEV)
    for where, blocks, _ in refs:
        rest[blocks.start * 256:min(blocks.stop * 256, n)] = False
    mid = n // 2
    for t in (param, m8, v8):
        assert (t.eq(t[mid]) | ~rest).all()
    m, v = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    mlc.muloco_adamw8_values([tensor], [m], [v])
    for where, _, (_, rm, rv, sm, sv, _, _) in refs:
        assert np.array_equal(m[where].cpu().numpy(), adamw8.decode_m(rm, sm)) and np.array_equal(v[where].cpu().numpy(), adamw8.decode_v(rv, sv))


def test_qk_norm_rope():
    """Slices of a fused projection whose rows pass 2^31 elements, and 2^32 bytes, apart from their start."""
    tokens, hq, hk, dim = 70000, 6, 2, 64
    fused = torch.empty(tokens, 512, dim, dtype=BF, device=DEV)
    assert fused.numel() > 1 << 31
    q, k = fused[:, 500:506], fused[:, 506:508]
    for i, t in enumerate((q, k)):
        t.copy_(S.normal(t.shape, 1.0, 2, i, dtype=BF, device=DEV))
    dq, dk = (S.normal(t.shape, 1.0, 2, 2 + i, dtype=BF, device=DEV) for i, t in enumerate((q, k)))
    wq, wk = S.normal((dim,), 0.3, 2, 5, device=DEV), S.normal((dim,), 0.3, 2, 6, device=DEV)
    angle = torch.arange(300, device=DEV)[:, None] * 1e4 ** (-torch.arange(dim // 2, device=DEV) / (dim // 2))
    cos, sin, pos = angle.cos().contiguous(), angle.sin().contiguous(), torch.arange(tokens, device=DEV) % 300
    want = [_reference(dy, x, w, 0.0, cos[pos], sin[pos], 1e-6, False) for dy, x, w in ((dq, q, wq), (dk, k, wk))]
    grads, gains = torch.empty_like(fused), [torch.empty(dim, device=DEV) for _ in range(2)]
    ws = torch.empty(mlc.muloco_qk_norm_rope_workspace_bytes(dim), dtype=torch.uint8, device=DEV)
    outs = grads[:, 500:506], grads[:, 506:508]
    mlc.muloco_qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, *outs, *gains, ws)
    mlc.muloco_qk_norm_rope(q, k, wq, wk, cos, sin, pos, q, k)
    for got, dx, dw, (y, rx, rw), what in zip((q, k), outs, gains, want, "qk"):
        _rows_close(got, y, what)
        _rows_close(dx, rx, "d" + what)
        assert (dw.double() - rw).norm() <= EW_TOL * rw.norm()


def test_gated_ffn():
    tokens, d, f = 390001, 64, 5632
    assert tokens * f > 1 << 31
    x, wg, wu, wd, dy = [S.normal(s, std, 4, i, dtype=BF, device=DEV) for i, (s, std) in enumerate(
        (((tokens, d), 1.0), ((f, d), d ** -0.5), ((f, d), d ** -0.5), ((d, f), f ** -0.5), ((tokens, d), 1.0)))]
    for factors in (BF, torch.float32):
        new = lambda *s, dt=BF: torch.full(s, float("nan"), dtype=dt, device=DEV)  # noqa: E731
        y, hidden, gate, up = new(tokens, d), new(tokens, f), new(tokens, f, dt=factors), new(tokens, f, dt=factors)
        grads = [new(tokens, d), new(f, d), new(f, d), new(d, f)]
        ws = torch.empty(max(mlc.muloco_gated_ffn_workspace_bytes(tokens, d, f, b) for b in (False, True)), dtype=torch.uint8, device=DEV)
        mlc.muloco_gated_ffn(x, wg, wu, wd, y, hidden, ws, gate=gate, up=up)
        mlc.muloco_gated_ffn_backward(dy, x, wg, wu, wd, gate, up, hidden, *grads, ws)
        del gate, up, hidden, ws
        sums, step = {}, 30000
        for at in range(0, tokens, step):
            rows = slice(at, min(at + step, tokens))
            ref = ffn._reference(x[rows], wg, wu, wd, dy[rows], "silu")
            for k, got in (("y", y[rows]), ("dx", grads[0][rows])):
                off = got.double() - ref[k][0]
                assert torch.isfinite(off).all(), k
                assert (off.norm(dim=1) <= 3 * ffn.FRO * ref[k][0].norm(dim=1)).all(), (k, at)
                assert off.norm() <= ffn.FRO * ref[k][0].norm(), (k, at)
            for k in ("dwg", "dwu", "dwd"):
                sums[k] = sums.get(k, 0) + ref[k][0]
            del ref
        for k, got in zip(("dwg", "dwu", "dwd"), grads[1:]):
            assert (got.double() - sums[k]).norm() <= ffn.FRO * sums[k].norm(), k
