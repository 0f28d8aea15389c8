"""The example that runs the training operators together: it learns, and its gradients are those of plain fp32 torch."""
import importlib.util
import math
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
spec = importlib.util.spec_from_file_location("train_layer", os.path.join(ROOT, "examples", "train_layer.py"))
layer = importlib.util.module_from_spec(spec)
spec.loader.exec_module(layer)


def test_it_learns():
    losses = layer.train(steps=30, log=lambda s: None)
    # the next token is certain: from about log(128) down by more than half
    assert losses[0] > 0.8 * math.log(128) and losses[-1] < 0.5 * losses[0], (losses[0], losses[-1])


def test_gradients_against_plain_torch(monkeypatch):
    """The same layer with both operators in elementary fp32 operations.  bf16 activations pass through a few roundings
    of 1.7e-3 (rms) each on either side: 3e-2 holds six of them on both."""
    dev, dim = "cuda:0", 64
    p = layer.init(64, 128, 264, dim, dev)
    half = dim // 2
    angle = torch.arange(16, device=dev)[:, None] * 1e4 ** (-torch.arange(half, device=dev) / half)
    tables = angle.cos().contiguous(), angle.sin().contiguous()
    tokens = torch.randint(0, 64, (5, 17), generator=torch.Generator().manual_seed(3)).to(dev)
    loss = layer.loss_of(p, tokens, tables, dim)
    grads = dict(zip(p, torch.autograd.grad(loss, list(p.values()))))

    def qk(q, k, qg, kg, cos, sin, pos, hp):
        def one(x, w):
            x = x.float()
            n = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + hp.eps) * w
            a, b = n.split(half, -1)
            c, s = cos[pos][:, None], sin[pos][:, None]
            return torch.cat([a * c - b * s, b * c + a * s], -1).to(torch.bfloat16)
        return one(q, qg), one(k, kg)

    def ffn(x, wg, wu, wd, act):
        x, wg, wu, wd = (v.float() for v in (x, wg, wu, wd))
        return ((torch.nn.functional.silu(x @ wg.t()) * (x @ wu.t())) @ wd.t()).to(torch.bfloat16)
    monkeypatch.setattr(layer, "QKNormRope", type("Q", (), {"apply": staticmethod(qk)}))
    monkeypatch.setattr(layer, "GatedFFN", type("F", (), {"apply": staticmethod(ffn)}))
    ref = layer.loss_of(p, tokens, tables, dim)
    refs = dict(zip(p, torch.autograd.grad(ref, list(p.values()))))
    assert abs(loss.item() - ref.item()) < 1e-2
    for k in p:
        err = ((grads[k].float() - refs[k].float()).norm() / refs[k].float().norm()).item()
        assert err < 3e-2, (k, err)


def test_workers_are_one_model_after_an_outer_step(monkeypatch):
    """Each worker goes its own way on its own data, in every parameter, until the outer step, and both learn."""
    replicas, losses, met = [], [], []
    init, loss_of, outer = layer.init, layer.loss_of, layer.mlc.muloco_outer_step

    def kept(*args):
        replicas.append(init(*args))
        return replicas[-1]

    def noted(*args):
        loss = loss_of(*args)
        losses.append(loss.item())
        return loss

    def joined(groups, hp):
        assert not any(torch.equal(replicas[0][k], replicas[1][k]) for k in replicas[0])
        outer(groups, hp)
        assert [k for k in replicas[0] if not torch.equal(replicas[0][k], replicas[1][k])] == []
        met.append(len(losses) // 2)
    monkeypatch.setattr(layer, "init", kept)
    monkeypatch.setattr(layer, "loss_of", noted)
    monkeypatch.setattr(layer.mlc, "muloco_outer_step", joined)
    layer.train(steps=30, log=lambda s: None)
    assert met == [10, 20, 30] and len(losses) == 60
    for rank in (0, 1):
        assert losses[rank] > 0.8 * math.log(128) and losses[58 + rank] < 0.5 * losses[rank], (rank, losses[rank], losses[58 + rank])
