"""One transformer layer trained with this library: the q/k norm with rotary positions and the gated feed-forward block make
the gradients, Muon steps the matrices, AdamW with 8-bit states the embedding and the gains, and every few steps the DiLoCo outer
step brings two resident workers together: all their parameters are the same after it.

    python examples/train_layer.py [--steps 40] [--width 256] [--hidden 704] [--tokens 512]

The task is synthetic: sequences in which every token is a fixed permutation of the one before it.  Attention itself and the
plain projections are torch's.
"""
import argparse
import math
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch  # noqa: E402

import paper_2505_23725_amd as mlc  # noqa: E402

BF = torch.bfloat16


class QKNormRope(torch.autograd.Function):
    """q, k [tokens, heads, head_dim]; gains float32."""

    @staticmethod
    def forward(ctx, q, k, q_gain, k_gain, cos, sin, positions, hp):
        out = torch.empty(q.shape, dtype=q.dtype, device=q.device), torch.empty(k.shape, dtype=k.dtype, device=k.device)
        mlc.muloco_qk_norm_rope(q, k, q_gain, k_gain, cos, sin, positions, *out, hp)
        ctx.save_for_backward(q, k, q_gain, k_gain, cos, sin, positions)
        ctx.hp = hp
        return out

    @staticmethod
    def backward(ctx, dq_out, dk_out):
        q, k, q_gain, k_gain, cos, sin, positions = ctx.saved_tensors
        dq, dk = torch.empty(q.shape, dtype=q.dtype, device=q.device), torch.empty(k.shape, dtype=k.dtype, device=k.device)
        dqg, dkg = torch.empty_like(q_gain), torch.empty_like(k_gain)
        ws = torch.empty(mlc.muloco_qk_norm_rope_workspace_bytes(q.shape[2]), dtype=torch.uint8, device=q.device)
        mlc.muloco_qk_norm_rope_backward(dq_out.contiguous(), dk_out.contiguous(), q, k, q_gain, k_gain, cos, sin, positions,
                                         dq, dk, dqg, dkg, ws, ctx.hp)
        return dq, dk, dqg, dkg, None, None, None, None


class GatedFFN(torch.autograd.Function):
    """x [tokens, d] and the three matrices, bf16."""

    @staticmethod
    def forward(ctx, x, w_gate, w_up, w_down, act):
        t, d, f = x.shape[0], x.shape[1], w_gate.shape[0]
        new = lambda *s: torch.empty(s, dtype=BF, device=x.device)  # noqa: E731
        y, hidden, gate, up = new(t, d), new(t, f), new(t, f), new(t, f)
        ws = torch.empty(max(1, mlc.muloco_gated_ffn_workspace_bytes(t, d, f)), dtype=torch.uint8, device=x.device)
        mlc.muloco_gated_ffn(x, w_gate, w_up, w_down, y, hidden, ws, act=act, gate=gate, up=up)
        ctx.save_for_backward(x, w_gate, w_up, w_down, gate, up, hidden)
        ctx.act = act
        return y

    @staticmethod
    def backward(ctx, dy):
        x, w_gate, w_up, w_down, gate, up, hidden = ctx.saved_tensors
        grads = [torch.empty_like(v) for v in (x, w_gate, w_up, w_down)]
        ws = torch.empty(max(1, mlc.muloco_gated_ffn_workspace_bytes(*x.shape, w_gate.shape[0], True)), dtype=torch.uint8, device=x.device)
        mlc.muloco_gated_ffn_backward(dy.contiguous(), x, w_gate, w_up, w_down, gate, up, hidden, *grads, ws, act=ctx.act)
        return (*grads, None)


MATRICES = ("w_q", "w_k", "w_v", "w_o", "w_gate", "w_up", "w_down")       # Muon's; the rest is AdamW's


def init(vocab, d, f, head_dim, device):
    g = torch.Generator(device=device).manual_seed(0)
    new = lambda *s: (torch.randn(s, generator=g, device=device) * s[-1] ** -0.5).to(BF)  # noqa: E731
    p = {"embedding": new(vocab, d) * math.sqrt(d), "q_gain": torch.ones(head_dim, device=device), "k_gain": torch.ones(head_dim, device=device),
         "w_q": new(d, d), "w_k": new(d, d), "w_v": new(d, d), "w_o": new(d, d), "w_gate": new(f, d), "w_up": new(f, d), "w_down": new(d, f)}
    return {k: v.requires_grad_() for k, v in p.items()}


def norm(x):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6)).to(BF)


def loss_of(p, tokens, tables, head_dim):
    """tokens [sequences, length + 1]; mean cross entropy of each next token."""
    n, length = tokens.shape[0], tokens.shape[1] - 1
    d = p["embedding"].shape[1]
    heads = d // head_dim
    x = p["embedding"][tokens[:, :-1]].reshape(n * length, d)
    h = norm(x)
    q, k, v = ((h @ p[w].t()).view(n * length, heads, head_dim) for w in ("w_q", "w_k", "w_v"))
    positions = torch.arange(length, device=x.device).repeat(n)
    q, k = QKNormRope.apply(q, k, p["q_gain"], p["k_gain"], *tables, positions, mlc.QKNormRopeHParams())
    # attention in fp32, one product a sequence and head
    split = lambda z: z.view(n, length, heads, head_dim).transpose(1, 2).float()  # noqa: E731
    scores = (split(q) @ split(k).transpose(-1, -2).contiguous()) / math.sqrt(head_dim)
    mask = torch.ones(length, length, dtype=torch.bool, device=x.device).triu(1)
    a = scores.masked_fill(mask, float("-inf")).softmax(-1) @ split(v)
    x = x + a.transpose(1, 2).reshape(n * length, d).to(BF) @ p["w_o"].t()
    x = x + GatedFFN.apply(norm(x), p["w_gate"], p["w_up"], p["w_down"], "silu")
    logits = (norm(x) @ p["embedding"].t()).float() / math.sqrt(d)
    return torch.nn.functional.cross_entropy(logits, tokens[:, 1:].reshape(-1))


def train(steps=40, width=256, hidden=704, tokens=512, vocab=128, head_dim=64, every=10, workers=2, device="cuda:0", log=print):
    """Returns the losses of worker 0, step by step."""
    half, length = head_dim // 2, 32
    angle = torch.arange(length, device=device)[:, None] * 1e4 ** (-torch.arange(half, device=device) / half)
    tables = angle.cos().contiguous(), angle.sin().contiguous()
    replicas = [init(vocab, width, hidden, head_dim, device) for _ in range(workers)]
    flat = lambda v: v.detach().view(-1, v.shape[-1])  # noqa: E731  (gains are matrices of one row to the outer step)
    shared = {k: flat(v).float().clone() for k, v in replicas[0].items()}          # the global copy and its momentum
    outer = {k: torch.zeros_like(v) for k, v in shared.items()}
    momenta = [{k: torch.zeros_like(shared[k]) for k in MATRICES} for _ in replicas]
    states = [{k: mlc.adamw8_state(v) for k, v in p.items() if k not in MATRICES} for p in replicas]
    muon = mlc.MuonHParams(eta=2e-2, weight_decay=0.0, beta=0.9)
    order = torch.randperm(vocab, generator=torch.Generator().manual_seed(1)).to(device)
    draw = torch.Generator(device=device).manual_seed(2)
    work, losses = None, []
    for step in range(1, steps + 1):
        for rank, p in enumerate(replicas):
            seq = [torch.randint(0, vocab, (tokens // length,), generator=draw, device=device)]
            for _ in range(length):
                seq.append(order[seq[-1]])
            loss = loss_of(p, torch.stack(seq, 1), tables, head_dim)
            grads = dict(zip(p, torch.autograd.grad(loss, list(p.values()))))
            with torch.no_grad():
                groups = [mlc.InnerGroup(p[k].detach(), grads[k].contiguous(), momenta[rank][k], math.sqrt(p[k].shape[1] / p[k].shape[0]))
                          for k in MATRICES]
                if work is None:
                    work = torch.empty(mlc.muloco_inner_workspace_bytes(groups), dtype=torch.uint8, device=device)
                mlc.muloco_inner_step(groups, muon, work)
                mlc.muloco_adamw8_step([(p[k].detach(), grads[k].contiguous(), *s) for k, s in states[rank].items()],
                                       mlc.AdamWHParams(lr=3e-3, beta2=0.99, bias_correction=True, step=step), seed=step * workers + rank)
            if rank == 0:
                losses.append(loss.detach())
        if step % every == 0:
            mlc.muloco_outer_step([mlc.OuterGroup([flat(p[k]) for p in replicas], shared[k], outer[k]) for k in shared],
                                  mlc.OuterHParams(K=workers, eta_out=0.7, mu=0.6))
            log(f"step {step}: loss {losses[-1].item():.4f}")
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    ap = argparse.ArgumentParser()
    for name, default in (("steps", 40), ("width", 256), ("hidden", 704), ("tokens", 512)):
        ap.add_argument("--" + name, type=int, default=default)
    train(**vars(ap.parse_args()))
