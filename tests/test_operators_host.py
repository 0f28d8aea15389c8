"""CPU-only checks of the operators' C entry points: bad arguments are refused before the GPU is touched (none of these calls
enqueues work), work-space sizes, and the binding's structures against the header's."""
import ctypes as C
import os
import shutil
import subprocess

import pytest

import paper_2505_23725_amd as mlc
from paper_2505_23725_amd import binding as B

NULL, SHAPE, DTYPE, WORKSPACE, ARG = -1, -2, -3, -4, -5
P = 0x1000          # an address that nothing reads: every call here is refused first


def _adamw8(n=1, hp=None, dither=0, **change):
    g = dict(count=512, param=P, param_dtype=0, grad=P, grad_dtype=1, exp_avg=P, exp_avg_sq=P, scales=P)
    g.update(change)
    h = dict(lr=1e-3, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.0, bias_correction=0, step=1)
    h.update(hp or {})
    arr = (B._AdamW8Group * 1)(B._AdamW8Group(*g.values()))
    return mlc.library().muloco_adamw8_step(arr, n, C.byref(B._AdamWHParams(*h.values())), dither, 0, None)


@pytest.mark.parametrize("want,args", [
    (0, dict(n=0)), (ARG, dict(n=-1)), (ARG, dict(dither=2)), (ARG, dict(hp=dict(lr=-1.0))), (ARG, dict(hp=dict(beta1=1.0))),
    (ARG, dict(hp=dict(beta2=float("nan")))), (ARG, dict(hp=dict(bias_correction=1, step=0))), (NULL, dict(param=None)),
    (NULL, dict(grad=None)), (NULL, dict(exp_avg=None)), (NULL, dict(exp_avg_sq=None)), (NULL, dict(scales=None)),
    (DTYPE, dict(param_dtype=2)), (DTYPE, dict(grad_dtype=-1)), (SHAPE, dict(count=0)), (SHAPE, dict(count=1 << 41)),
    (ARG, dict(scales=P + 2)), (ARG, dict(param=P + 2)), (ARG, dict(grad=P + 1))])
def test_adamw8_step(want, args):
    assert _adamw8(**args) == want


def test_adamw8_values():
    lib = mlc.library()
    arr = (B._AdamW8Group * 1)(B._AdamW8Group(512, None, 0, None, 0, P, P, P))
    ptr = lambda x: (C.c_void_p * 1)(x)  # noqa: E731
    assert lib.muloco_adamw8_values(arr, 0, ptr(P), ptr(P), None) == 0
    assert lib.muloco_adamw8_values(arr, 1, None, ptr(P), None) == NULL
    assert lib.muloco_adamw8_values(arr, 1, ptr(None), ptr(P), None) == NULL
    assert lib.muloco_adamw8_values(arr, 1, ptr(P), ptr(P + 2), None) == ARG
    arr[0].scales = None
    assert lib.muloco_adamw8_values(arr, 1, ptr(P), ptr(P), None) == NULL


def _qk(back=False, change=None, heads=None, **kw):
    d = dict(tokens=4, q_heads=2, k_heads=1, head_dim=64, rot_dim=64, dtype=1, q_gain=P, k_gain=P, gain_dtype=0, cos=P, sin=P,
             table_rows=8, positions=P, positions_32bit=0, eps=1e-6, gain_offset=0.0, interleaved=0)
    d.update(change or {})
    desc = B._QKNormRope(*d.values())
    h = {k: [P, 192, 64] for k in ("q", "k", "q_out", "k_out", "dq_out", "dk_out", "dq", "dk")}
    for k, v in (heads or {}).items():
        h[k] = v
    h = {k: None if v is None else C.byref(B._Heads(*v)) for k, v in h.items()}
    lib = mlc.library()
    if not back:
        return lib.muloco_qk_norm_rope(C.byref(desc), h["q"], h["k"], h["q_out"], h["k_out"], None)
    a = dict(dq_gain=P, dk_gain=P, ws=P, size=1 << 30)
    a.update(kw)
    return lib.muloco_qk_norm_rope_backward(C.byref(desc), h["dq_out"], h["dk_out"], h["q"], h["k"], h["dq"], h["dk"], a["dq_gain"],
                                            a["dk_gain"], a["ws"], a["size"], None)


BAD_QK = [
    (SHAPE, dict(change=dict(tokens=-1))), (SHAPE, dict(change=dict(q_heads=0))), (SHAPE, dict(change=dict(k_heads=-1))),
    (SHAPE, dict(change=dict(q_heads=2000))), (SHAPE, dict(change=dict(head_dim=63))), (SHAPE, dict(change=dict(head_dim=514))),
    (SHAPE, dict(change=dict(rot_dim=66))), (SHAPE, dict(change=dict(rot_dim=3))), (DTYPE, dict(change=dict(dtype=2))),
    (DTYPE, dict(change=dict(gain_dtype=7))), (ARG, dict(change=dict(eps=-1.0))), (ARG, dict(change=dict(eps=float("nan")))),
    (ARG, dict(change=dict(gain_offset=float("nan")))), (ARG, dict(change=dict(interleaved=2))), (ARG, dict(change=dict(table_rows=-1))),
    (ARG, dict(change=dict(positions_32bit=3))), (NULL, dict(change=dict(q_gain=None))), (NULL, dict(change=dict(k_gain=None))),
    (NULL, dict(change=dict(cos=None))), (NULL, dict(change=dict(positions=None))), (ARG, dict(change=dict(positions=P + 4))),
    (ARG, dict(change=dict(cos=P + 2))), (NULL, dict(heads=dict(q=None))), (NULL, dict(heads=dict(k=[None, 64, 64]))),
    (ARG, dict(heads=dict(q=[P + 1, 192, 64]))), (ARG, dict(heads=dict(q=[P, -192, 64])))]


@pytest.mark.parametrize("want,args", BAD_QK + [(ARG, dict(heads=dict(q_out=[P, 192, 63]))), (ARG, dict(heads=dict(k_out=[P, 0, 64]))),
                                                 (0, dict(change=dict(tokens=0)))])
def test_qk_norm_rope(want, args):
    assert _qk(**args) == want


@pytest.mark.parametrize("want,args", BAD_QK + [(ARG, dict(heads=dict(dq=[P, 192, 63]))), (NULL, dict(dq_gain=None)), (NULL, dict(dk_gain=None)),
                                                 (ARG, dict(dq_gain=P + 2)), (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(ws=P + 16)),
                                                 (WORKSPACE, dict(size=100))])
def test_qk_norm_rope_backward(want, args):
    assert _qk(back=True, **args) == want


def test_workspaces():
    assert mlc.muloco_qk_norm_rope_workspace_bytes(128) > 0
    assert mlc.muloco_qk_norm_rope_workspace_bytes(127) == mlc.muloco_qk_norm_rope_workspace_bytes(1024) == 0
    size = mlc.muloco_gated_ffn_workspace_bytes
    assert size(1, 2048, 5632) == 0                                      # the weights are streamed: nothing to put down
    assert size(100, 100, 64) == size(-1, 64, 64) == size(1, 64, 0) == 0      # refused shapes
    t, d, f = 16384, 2048, 5632
    assert 4 * t * f <= size(t, d, f, True) <= 4 * t * f + (64 << 20)      # dg and du, and at most a round of partial tiles
    assert size(0, 64, 64, True) >= 0


def _ffn(back=False, tokens=4, d=64, f=72, act=0, ws=P, size=1 << 30, **change):
    a = dict(x=P, w_gate=P, w_up=P, w_down=P, gate=P, up=P, hidden=P, y=P, dy=P, dx=P, dw_gate=P, dw_up=P, dw_down=P)
    a.update(change)
    desc = B._GatedFFN(tokens, d, f, act, a["x"], a["w_gate"], a["w_up"], a["w_down"])
    lib = mlc.library()
    if not back:
        return lib.muloco_gated_ffn(C.byref(desc), a["gate"], a["up"], a["hidden"], a["y"], ws, size, None)
    return lib.muloco_gated_ffn_backward(C.byref(desc), a["gate"], a["up"], a["hidden"], a["dy"], a["dx"], a["dw_gate"], a["dw_up"],
                                         a["dw_down"], ws, size, None)


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("want,args", [
    (SHAPE, dict(tokens=-1)), (SHAPE, dict(d=60)), (SHAPE, dict(f=4)), (SHAPE, dict(d=1 << 22)), (ARG, dict(act=2)), (NULL, dict(x=None)),
    (NULL, dict(w_gate=None)), (NULL, dict(w_down=None)), (NULL, dict(hidden=None)), (ARG, dict(x=P + 2)), (ARG, dict(w_up=P + 8)),
    (ARG, dict(hidden=P + 8)), (NULL, dict(gate=None)), (NULL, dict(up=None))])
def test_gated_ffn(want, args, back):
    assert _ffn(back, **args) == want


@pytest.mark.parametrize("want,args", [(NULL, dict(dy=None)), (NULL, dict(dx=None)), (NULL, dict(dw_down=None)), (ARG, dict(dw_up=P + 4)),
                                        (WORKSPACE, dict(ws=None)), (WORKSPACE, dict(size=16)), (WORKSPACE, dict(ws=P + 16))])
def test_gated_ffn_backward(want, args):
    assert _ffn(True, **args) == want


def test_no_tokens_forward_is_nothing_to_do():
    assert _ffn(tokens=0, x=None, hidden=None, y=None, gate=None, up=None, ws=None, size=0) == 0


STRUCTS = {"mlc_adamw8_group": B._AdamW8Group, "mlc_heads": B._Heads, "mlc_qk_norm_rope": B._QKNormRope, "mlc_gated_ffn": B._GatedFFN}


@pytest.mark.skipif(shutil.which("gcc") is None, reason="no C compiler")
def test_structures_match_the_header(tmp_path):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    lines = ["#include <stddef.h>", "#include <stdio.h>", '#include "muloco.h"', "int main(void) {"]
    for name, st in STRUCTS.items():
        lines.append(f'  printf("{name} size %zu\\n", sizeof({name}));')
        lines += [f'  printf("{name} {f[0]} %zu\\n", offsetof({name}, {f[0]}));' for f in st._fields_]
    lines += ['  printf("block %d\\n", MLC_ADAMW8_BLOCK);', '  printf("act %d %d\\n", MLC_ACT_SILU, MLC_ACT_GELU_TANH);', "  return 0;", "}"]
    (tmp_path / "s.c").write_text("\n".join(lines))
    subprocess.run(["gcc", "-std=c99", "-pedantic", "-Werror", "-Wall", "-I", os.path.join(root, "include"), str(tmp_path / "s.c"), "-o",
                    str(tmp_path / "s")], check=True)
    for line in subprocess.run([str(tmp_path / "s")], capture_output=True, text=True, check=True).stdout.splitlines():
        w = line.split()
        if w[0] == "block":
            assert int(w[1]) == mlc.ADAMW8_BLOCK
        elif w[0] == "act":
            assert [int(x) for x in w[1:]] == [mlc.ACTIVATIONS["silu"], mlc.ACTIVATIONS["gelu_tanh"]]
        elif w[1] == "size":
            assert C.sizeof(STRUCTS[w[0]]) == int(w[2]), line
        else:
            assert getattr(STRUCTS[w[0]], w[1]).offset == int(w[2]), line


@pytest.mark.parametrize("back", [False, True])
def test_tables_without_rows_may_be_null(back):
    """(refused for what comes behind the tables: an odd address of a bf16 tensor)"""
    heads = dict(heads={"dq_out" if back else "q": [P + 1, 192, 64]})
    assert _qk(back, change=dict(table_rows=0, cos=None, sin=None), **heads) == ARG
    assert _qk(back, change=dict(cos=None, sin=None), **heads) == NULL


@pytest.mark.parametrize("back", [False, True])
def test_positions_are_not_needed_where_nothing_is_turned(back):
    heads = dict(heads={"dq_out" if back else "q": [P + 1, 192, 64]})
    assert _qk(back, change=dict(rot_dim=0, positions=None, cos=None, sin=None), **heads) == ARG
    assert _qk(back, change=dict(positions=None), **heads) == NULL


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("tokens,heads,token_stride,head_stride,fine", [
    (4, 2, 64, 64, False),            # head 1 of a token is head 0 of the next
    (4, 2, 127, 64, False), (4, 2, 128, 64, True), (4, 2, 128, 65, False), (4, 2, 129, 65, True), (4, 2, 64, 255, False), (4, 2, 64, 256, True),
    (4, 3, 0, 1 << 20, False), (1, 3, 0, 64, True), (1, 3, 0, 63, False), (4, 1, 64, 0, True), (4, 1, 63, 0, False), (1, 1, 0, 0, True),
    (2, 2, 1 << 62, 1 << 62, False), (1 << 40, 2, 1 << 62, 64, True), (1 << 40, 2, 64, 1 << 46, True), (1 << 40, 2, 64, (1 << 46) - 1, False),
    (1 << 40, 2, 1 << 61, 1 << 62, False)])
def test_heads_of_an_output_may_not_overlap(tokens, heads, token_stride, head_stride, fine, back):
    """(what is fine goes on to the next tensor, which is missing)"""
    first, second = ("dq", "dk") if back else ("q_out", "k_out")
    got = _qk(back, change=dict(tokens=tokens, q_heads=heads), heads={first: [P, token_stride, head_stride], second: None})
    assert got == (NULL if fine else ARG)


@pytest.mark.parametrize("back", [False, True])
def test_type_of_the_factors(back):
    lib, ws = mlc.library(), [P, 1 << 30, None]
    for flag, x, want in ((2, P, ARG), (-1, P, ARG), (1, None, NULL), (0, None, NULL)):
        desc = B._GatedFFN(4, 64, 72, 0, x, P, P, P, flag)
        got = lib.muloco_gated_ffn_backward(C.byref(desc), *[P] * 8, *ws) if back else lib.muloco_gated_ffn(C.byref(desc), *[P] * 4, *ws)
        assert got == want, (flag, x)
