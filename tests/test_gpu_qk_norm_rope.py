"""GPU parity: muloco_qk_norm_rope and its backward call against the fp64 oracle.

Tolerances: everything is fp32 arithmetic on the stored inputs, rounded once.  A sum over a head of up to 512 squares and a
reciprocal root are within 1e-6 of exact, so fp32 outputs agree to EW_TOL (relative Frobenius) and bf16 ones are correct
roundings of such values (assert_stored_close); gains' gradients are fp32 sums, EW_TOL."""
import numpy as np
import pytest
import torch

import paper_2505_23725_amd as mlc
import synth_inputs as S
from oracle import qk_norm_rope as oracle
from helpers import assert_fp32_close, assert_stored_close, to_f64

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _tables(rows, half):
    a = torch.arange(rows, dtype=torch.float64)[:, None] * 1e4 ** (-torch.arange(half, dtype=torch.float64) / max(1, half))
    return a.cos().float(), a.sin().float()


def _case(tokens, hq, hk, dim, rot, dtype, gain_dtype=torch.float32, seed=1, rows=50):
    q, k = S.normal((tokens, hq, dim), 1.0, seed, 0, dtype=dtype), S.normal((tokens, hk, dim), 2.0, seed, 1, dtype=dtype)
    dq, dk = S.normal((tokens, hq, dim), 1.0, seed, 2, dtype=dtype), S.normal((tokens, hk, dim), 1.0, seed, 3, dtype=dtype)
    wq, wk = S.normal((dim,), 0.3, seed, 4, dtype=gain_dtype), S.normal((dim,), 0.3, seed, 5, dtype=gain_dtype)
    cos, sin = _tables(rows, rot // 2)
    pos = torch.randint(0, rows, (tokens,), generator=torch.Generator().manual_seed(seed))
    return q, k, dq, dk, wq, wk, cos, sin, pos


def _check(got, ref, dtype, what):
    (assert_fp32_close if dtype == torch.float32 else assert_stored_close)(got.cpu(), ref, what)


CASES = [
    # tokens, q heads, k heads, dim, rot, interleaved, dtype, gain dtype, offset
    (1, 1, 1, 128, 128, False, torch.bfloat16, torch.float32, 0.0),
    (5, 4, 2, 128, 128, False, torch.bfloat16, torch.bfloat16, 1.0),
    (5, 4, 2, 128, 128, True, torch.float32, torch.float32, 1.0),
    (7, 3, 1, 64, 64, False, torch.float32, torch.bfloat16, 0.0),
    (3, 5, 3, 96, 32, False, torch.bfloat16, torch.float32, 1.0),        # part of a head turned
    (3, 5, 3, 80, 16, True, torch.bfloat16, torch.float32, 0.0),
    (4, 2, 1, 256, 256, False, torch.bfloat16, torch.float32, 1.0),
    (4, 2, 1, 512, 64, True, torch.float32, torch.float32, 1.0),
    (3, 2, 2, 8, 8, False, torch.float32, torch.float32, 0.0),
    (3, 2, 2, 2, 2, False, torch.float32, torch.float32, 0.0),           # element by element from here on
    (6, 3, 2, 20, 12, False, torch.bfloat16, torch.float32, 1.0),
    (6, 3, 2, 122, 116, True, torch.float32, torch.float32, 0.0),
    (3, 2, 1, 264, 44, False, torch.bfloat16, torch.float32, 1.0),
    (3, 2, 1, 510, 510, False, torch.float32, torch.float32, 0.0),
    (4, 2, 2, 64, 0, False, torch.bfloat16, torch.float32, 0.0),         # the norm alone
    (130, 9, 3, 64, 64, False, torch.bfloat16, torch.float32, 0.0),
]


@pytest.mark.parametrize("tokens,hq,hk,dim,rot,inter,dtype,gd,offset", CASES)
def test_forward_and_backward_match_oracle(tokens, hq, hk, dim, rot, inter, dtype, gd, offset):
    q, k, dq, dk, wq, wk, cos, sin, pos = _case(tokens, hq, hk, dim, rot, dtype, gd)
    hp = mlc.QKNormRopeHParams(eps=1e-5, gain_offset=offset, interleaved=inter)
    d = [x.to(DEV) for x in (q, k, wq, wk, cos, sin, pos)]
    qo, ko = torch.empty_like(d[0]), torch.empty_like(d[1])
    mlc.muloco_qk_norm_rope(*d, qo, ko, hp)
    gq, gk = torch.empty_like(d[0]), torch.empty_like(d[1])
    gwq, gwk = torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
    ws = torch.empty(mlc.muloco_qk_norm_rope_workspace_bytes(dim), dtype=torch.uint8, device=DEV)
    mlc.muloco_qk_norm_rope_backward(dq.to(DEV), dk.to(DEV), *d, gq, gk, gwq, gwk, ws, hp)
    torch.cuda.synchronize()
    for x, w, dy, y, gx, gw, what in ((q, wq, dq, qo, gq, gwq, "q"), (k, wk, dk, ko, gk, gwk, "k")):
        args = (to_f64(x), to_f64(w), offset, to_f64(cos), to_f64(sin), pos.tolist(), 1e-5, inter)
        _check(y, oracle.forward(*args), dtype, what)
        rx, rw = oracle.backward(to_f64(dy), *args)
        _check(gx, rx, dtype, "d" + what)
        assert_fp32_close(gw.cpu(), rw, "gradient of the gain of " + what)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_slices_orders_and_in_place(dtype):
    """Slices of a fused projection, heads-first order, a shared head (stride 0), int32 positions, outputs on the inputs: the
    same bits as contiguous tensors."""
    q, k, dq, dk, wq, wk, cos, sin, pos = _case(37, 6, 2, 64, 64, dtype)
    dev = [x.to(DEV) for x in (wq, wk, cos, sin)]
    fused = torch.zeros(37, 3, 11, 64, dtype=dtype, device=DEV)[:, 1]
    fused[:, :6], fused[:, 6:8] = q.to(DEV), k.to(DEV)
    qo, ko = torch.empty(37, 6, 64, dtype=dtype, device=DEV), torch.empty(37, 2, 64, dtype=dtype, device=DEV)
    mlc.muloco_qk_norm_rope(q.to(DEV), k.to(DEV), *dev, pos.to(DEV), qo, ko)
    first = torch.empty(6, 37, 64, dtype=dtype, device=DEV)
    ko2 = torch.empty_like(ko)
    mlc.muloco_qk_norm_rope(fused[:, :6], fused[:, 6:8], *dev, pos.to(DEV).int(), first.transpose(0, 1), ko2)
    assert torch.equal(first.transpose(0, 1), qo) and torch.equal(ko2, ko)
    before = fused.clone()
    mlc.muloco_qk_norm_rope(fused[:, :6], fused[:, 6:8], *dev, pos.to(DEV), fused[:, :6], fused[:, 6:8])
    assert torch.equal(fused[:, :6], qo) and torch.equal(fused[:, 6:8], ko) and torch.equal(fused[:, 8:], before[:, 8:])
    one = q[:, :1].to(DEV)
    mlc.muloco_qk_norm_rope(one.expand(37, 6, 64), k.to(DEV), *dev, pos.to(DEV), qo, ko)
    assert all(torch.equal(qo[:, 0], qo[:, h]) for h in range(6))
    # odd element offsets: rows that start on no vector's boundary
    flat = torch.zeros(37 * 6 * 66 + 1, dtype=dtype, device=DEV)
    odd = flat[1:].view(37, 6, 66)[..., :64]
    odd.copy_(q)
    qo2 = torch.empty(37, 6, 65, dtype=dtype, device=DEV)[..., :64]
    mlc.muloco_qk_norm_rope(odd, k.to(DEV), *dev, pos.to(DEV), qo2, ko2)
    mlc.muloco_qk_norm_rope(q.to(DEV), k.to(DEV), *dev, pos.to(DEV), qo, ko)
    assert torch.equal(qo2, qo) and torch.equal(ko2, ko)


def test_many_tokens_take_several_heads_and_repeat_bit_for_bit():
    """Enough rows that a group takes four heads (7 and 3: runs that are not full), and more than there are partial rows."""
    dim, n = 64, 30000
    q, k, dq, dk, wq, wk, cos, sin, pos = [x.to(DEV) for x in _case(n, 7, 3, dim, dim, torch.bfloat16, rows=4000)]
    out = []
    ws = torch.empty(mlc.muloco_qk_norm_rope_workspace_bytes(dim), dtype=torch.uint8, device=DEV)
    for _ in range(2):
        o = [torch.empty_like(q), torch.empty_like(k), torch.empty_like(q), torch.empty_like(k),
             torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)]
        mlc.muloco_qk_norm_rope(q, k, wq, wk, cos, sin, pos, o[0], o[1])
        mlc.muloco_qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, *o[2:], ws)
        out.append(o)
    assert all(torch.equal(a, b) for a, b in zip(*out))
    pick = torch.tensor([0, 1, 17, 14999, n - 1])
    for x, w, dy, y, gx in ((q, wq, dq, out[0][0], out[0][2]), (k, wk, dk, out[0][1], out[0][3])):
        args = (to_f64(x[pick]), to_f64(w), 0.0, to_f64(cos), to_f64(sin), pos[pick].tolist(), 1e-6, False)
        assert_stored_close(y[pick].cpu(), oracle.forward(*args), "y")
        assert_stored_close(gx[pick].cpu(), oracle.backward(to_f64(dy[pick]), *args)[0], "dx")
    # gains' gradients: the sums over all tokens in fp64, vectorised
    for x, dy, gw in ((q, dq, out[0][4]), (k, dk, out[0][5])):
        x, dy, c, s = x.double(), dy.double(), cos[pos].double()[:, None], sin[pos].double()[:, None]
        r = (x.square().mean(-1, keepdim=True) + 1e-6).rsqrt()
        a, b = dy.split(dim // 2, -1)
        dn = torch.cat([a * c + b * s, b * c - a * s], -1)
        assert_fp32_close(gw.cpu(), to_f64((dn * x * r).sum((0, 1))), "gradient of the gain")


def test_positions_outside_the_tables_read_nothing():
    q, k, dq, dk, wq, wk, cos, sin, pos = [x.to(DEV) for x in _case(4, 2, 1, 64, 64, torch.float32)]
    pos[1], pos[2] = 50, -1
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    mlc.muloco_qk_norm_rope(q, k, wq, wk, cos, sin, pos, qo, ko)
    for y in (qo, ko):
        assert torch.isnan(y[1:3]).all() and torch.isfinite(y[[0, 3]]).all()


def test_a_head_of_zeros_and_one_that_is_not_finite():
    q, k, dq, dk, wq, wk, cos, sin, pos = [x.to(DEV) for x in _case(3, 2, 1, 64, 64, torch.float32)]
    q[0, 0] = 0.0
    q[1, 1, 5] = float("inf")
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    mlc.muloco_qk_norm_rope(q, k, wq, wk, cos, sin, pos, qo, ko)
    assert torch.all(qo[0, 0] == 0) and not torch.isfinite(qo[1, 1]).all()
    assert torch.isfinite(qo[1, 0]).all() and torch.isfinite(qo[2]).all() and torch.isfinite(ko).all()


def test_no_tokens():
    q, k, dq, dk, wq, wk, cos, sin, pos = [x.to(DEV) for x in _case(0, 2, 1, 64, 64, torch.bfloat16)]
    ws = torch.empty(mlc.muloco_qk_norm_rope_workspace_bytes(64), dtype=torch.uint8, device=DEV)
    mlc.muloco_qk_norm_rope(q, k, wq, wk, cos, sin, pos, torch.empty_like(q), torch.empty_like(k))
    gq, gk = torch.full((64,), 3.0, device=DEV), torch.full((64,), 3.0, device=DEV)
    mlc.muloco_qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, torch.empty_like(q), torch.empty_like(k), gq, gk, ws)
    torch.cuda.synchronize()
    assert not gq.any() and not gk.any()


def test_refusals():
    q, k, dq, dk, wq, wk, cos, sin, pos = [x.to(DEV) for x in _case(4, 2, 1, 64, 64, torch.float32)]
    qo, ko = torch.zeros_like(q), torch.zeros_like(k)
    call = lambda *a: mlc.muloco_qk_norm_rope(*a)  # noqa: E731
    with pytest.raises(ValueError):
        call(q, k[:3], wq, wk, cos, sin, pos, qo, ko)
    with pytest.raises(TypeError):
        call(q, k.bfloat16(), wq, wk, cos, sin, pos, qo, ko)
    with pytest.raises(TypeError):
        call(q, k, wq, wk, cos, sin, pos, qo.bfloat16(), ko)
    with pytest.raises(ValueError):
        call(q, k, wq[:32], wk, cos, sin, pos, qo, ko)
    with pytest.raises(ValueError):
        call(q, k, wq, wk, cos, sin.double(), pos, qo, ko)
    with pytest.raises(ValueError):
        call(q, k, wq, wk, cos, sin, pos[:3], qo, ko)
    with pytest.raises(ValueError):
        call(q, k, wq, wk, cos, sin, pos.float(), qo, ko)
    with pytest.raises(ValueError):
        call(q, k, wq, wk, cos, sin, pos, qo[:, :1].expand(4, 2, 64), ko)       # outputs on one another
    with pytest.raises(ValueError):
        call(q.transpose(1, 2).contiguous().transpose(1, 2), k, wq, wk, cos, sin, pos, qo, ko)
    with pytest.raises(mlc.MulocoError):
        call(q, k, wq, wk, cos.repeat(1, 2), sin.repeat(1, 2), pos, qo, ko)     # more to turn than a head has
    ws = torch.empty(1024, dtype=torch.uint8, device=DEV)
    with pytest.raises(mlc.MulocoError):
        mlc.muloco_qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, torch.empty_like(q), torch.empty_like(k),
                                         torch.empty(64, device=DEV), torch.empty(64, device=DEV), ws)
    assert not qo.any() and not ko.any()


@pytest.mark.parametrize("dim,rot", [(64, 64), (20, 12)])
def test_tables_without_rows_are_not_read(dim, rot):
    """No position lies in tables of no rows (whose address is NULL): every output and gradient is NaN, as for any other position
    outside."""
    q, k, dq, dk, wq, wk, cos, sin, pos = [x.to(DEV) for x in _case(5, 3, 2, dim, rot, torch.bfloat16)]
    cos, sin = cos[:0].contiguous(), sin[:0].contiguous()
    assert cos.data_ptr() == 0 and cos.shape == (0, rot // 2)
    out = [torch.zeros_like(x) for x in (q, k, q, k)]
    gains = [torch.zeros(dim, device=DEV) for _ in range(2)]
    ws = torch.empty(mlc.muloco_qk_norm_rope_workspace_bytes(dim), dtype=torch.uint8, device=DEV)
    mlc.muloco_qk_norm_rope(q, k, wq, wk, cos, sin, pos, *out[:2])
    mlc.muloco_qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, *out[2:], *gains, ws)
    assert all(torch.isnan(x).all() for x in out + gains)


@pytest.mark.parametrize("dim,rows", [(64, 0), (20, 0), (64, 3)])
def test_the_norm_alone_needs_no_positions(dim, rows):
    """Nothing to turn: whatever the tables' rows and the positions are, the results are those of rotation by nothing."""
    q, k, dq, dk, wq, wk, _, _, pos = [x.to(DEV) for x in _case(5, 3, 2, dim, 0, torch.float32)]
    ws = torch.empty(mlc.muloco_qk_norm_rope_workspace_bytes(dim), dtype=torch.uint8, device=DEV)

    def both(empty, positions):
        out = [torch.zeros_like(x) for x in (q, k, q, k)] + [torch.zeros(dim, device=DEV) for _ in range(2)]
        mlc.muloco_qk_norm_rope(q, k, wq, wk, empty, empty, positions, *out[:2])
        mlc.muloco_qk_norm_rope_backward(dq, dk, q, k, wq, wk, empty, empty, positions, *out[2:], ws)
        return out
    got = both(torch.empty(rows, 0, device=DEV), pos + 100)
    args = (to_f64(wq), 0.0, np.zeros((50, 0)), np.zeros((50, 0)), pos.tolist(), 1e-6, False)
    assert_fp32_close(got[0].cpu(), oracle.forward(to_f64(q), *args), "q")
    rx, rw = oracle.backward(to_f64(dq), to_f64(q), *args)
    assert_fp32_close(got[2].cpu(), rx, "dq")
    assert_fp32_close(got[4].cpu(), rw, "gradient of the gain of q")
    inside = both(torch.empty(50, 0, device=DEV), pos)
    assert all(torch.equal(a, b) for a, b in zip(got, inside))


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("dim,rot", [(64, 32), (64, 0), (22, 10)])
def test_elements_that_are_passed_on_stay_by_themselves(dim, rot, interleaved):
    """What is not finite in one element that is not turned shows in that element alone: a gain there, and a gradient in the sums of
    the gains' gradients (the head's own gradient has a mean over all of it)."""
    q, k, dq, dk, wq, wk, cos, sin, pos = [x.to(DEV) for x in _case(4, 2, 1, dim, rot, torch.float32)]
    ws = torch.empty(mlc.muloco_qk_norm_rope_workspace_bytes(dim), dtype=torch.uint8, device=DEV)
    hp = mlc.QKNormRopeHParams(interleaved=interleaved)
    for at in (rot, rot + 3, dim - 1):
        rest = [i for i in range(dim) if i != at]
        for bad in (float("inf"), float("nan")):
            w = wq.clone()
            w[at] = bad
            out, clean = [torch.empty_like(q) for _ in range(2)], torch.empty_like(k)
            mlc.muloco_qk_norm_rope(q, k, w, wk, cos, sin, pos, out[0], clean, hp)
            mlc.muloco_qk_norm_rope(q, k, wq, wk, cos, sin, pos, out[1], clean, hp)
            assert not torch.isfinite(out[0][..., at]).any() and torch.equal(out[0][..., rest], out[1][..., rest]), at
            dy = dq.clone()
            dy[1, 1, at] = bad
            grads = [[torch.empty_like(q), torch.empty_like(k), torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)] for _ in range(2)]
            mlc.muloco_qk_norm_rope_backward(dy, dk, q, k, wq, wk, cos, sin, pos, *grads[0], ws, hp)
            mlc.muloco_qk_norm_rope_backward(dq, dk, q, k, wq, wk, cos, sin, pos, *grads[1], ws, hp)
            assert not torch.isfinite(grads[0][2][at]) and torch.equal(grads[0][2][rest], grads[1][2][rest]), at
