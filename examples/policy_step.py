"""A model that learns from its own answers: sampling, scoring, loss, backward, clipping and update, with the library's
calls for each.

The model is one adapted projection with a 4-bit base weight, beside its input, under a frozen 4-bit LM head:
    x = embedding[token],  h = x + x W^T + s (x A^T) B^T,  p(next) = softmax(h E^T)
Every round
    lora_decode_q4        samples 16 answers token by token (the projection, then the head, 16 tokens a call)
    lora_linear_fwd_q4    the projection of all their tokens at once, su kept for the backward
    lora_ce_fwd_bwd       the tokens' -log p, and its gradient by the hidden states
    lora_policy_fwd_bwd   the clipped policy loss against the sampled probabilities, with the reference model's
    (or lora_pref_fwd_bwd the loss of better against worse answers)
    lora_linear_bwd_q4    dA and dB
    lora_clip_grads       their clipping to a global norm
and A and B take a step.  An answer's reward is the share of its tokens among the first 64 of the vocabulary.

    python examples/policy_step.py [--loss policy|pref] [--rounds N]
"""
from __future__ import annotations

import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2606_19528_gb300 import lora  # noqa: E402

D, V, RANK, SCALE = 256, 512, 16, 2.0  # hidden size, vocabulary, adapter
SEQS, LENGTH, END = 16, 24, V - 1      # answers of a round, their longest, the token that ends one
WANTED = 64


def quantized(n, k, g):
    """A random [n, k] weight in 4-bit form, and the bf16 matrix that it stands for."""
    s = torch.empty(n, k // 64, device="cuda").uniform_(0.25, 0.41, generator=g) * k**-0.5
    params = torch.stack([s, -7.5 * s], dim=-1).to(torch.bfloat16)
    codes = torch.randint(0, 256, (n, k // 2), generator=g, device="cuda", dtype=torch.uint8)
    shift = torch.tensor([0, 16], device="cuda")[None, :] + 4 * torch.arange(4, device="cuda")[:, None]
    q = (codes.view(torch.int32)[:, :, None, None] >> shift) & 15  # [n, k / 8, 4, 2]
    p = params.float()
    dense = p[:, :, :1] * q.reshape(n, k // 64, 64).float() + p[:, :, 1:]
    return codes, params, dense.to(torch.bfloat16).view(n, k)


def workspace(size):
    return torch.empty(max(size, 256), dtype=torch.uint8, device="cuda")


class Model:
    def __init__(self, seed=0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.g = g
        self.embedding = torch.randn(V, D, generator=g, device="cuda").to(torch.bfloat16)
        self.codes, self.params, _ = quantized(D, D, g)
        self.head_codes, self.head_params, self.head = quantized(V, D, g)
        self.Wq = lora.make_q4(self.codes, self.params)
        # the adapter in fp32, and what the kernels read; B = 0: the model starts as its reference
        self.A32 = torch.empty(RANK, D, device="cuda").uniform_(-1, 1, generator=g) * D**-0.5
        self.B32 = torch.zeros(D, RANK, device="cuda")
        self.A, self.B = self.A32.to(torch.bfloat16), self.B32.to(torch.bfloat16)

        bf16 = dict(dtype=torch.bfloat16, device="cuda")
        self.x1, self.y1 = torch.empty(SEQS, D, **bf16), torch.empty(SEQS, D, **bf16)
        self.h1, self.logits = torch.empty(SEQS, D, **bf16), torch.empty(SEQS, V, **bf16)
        # the descriptors of a call made again on the same buffers are made once
        self.layer = lora.make_projs([lora.make_proj(lora.make_shape(SEQS, D, D, RANK, SCALE), x=self.x1, A=self.A,
                                                     B=self.B, y=self.y1, Wq=self.Wq)])
        self.lm_head = lora.make_projs([lora.make_proj(lora.make_shape(SEQS, D, V, 0, 0.0), x=self.h1, y=self.logits,
                                                       Wq=lora.make_q4(self.head_codes, self.head_params))])
        self.decode_ws = workspace(max(lora.lora_decode_workspace_size(self.layer),
                                       lora.lora_decode_workspace_size(self.lm_head)))

    def sample(self):
        """Answers [SEQS, LENGTH] with the tokens that led to each, -log p of each, and which tokens count."""
        ws = self.decode_ws
        before = torch.empty(SEQS, LENGTH, dtype=torch.int64, device="cuda")
        after, nll = torch.empty_like(before), torch.empty(SEQS, LENGTH, device="cuda")
        mask = torch.empty(SEQS, LENGTH, dtype=torch.uint8, device="cuda")
        token = torch.randint(0, V - 1, (SEQS,), generator=self.g, device="cuda")
        alive = torch.ones(SEQS, dtype=torch.uint8, device="cuda")
        for t in range(LENGTH):
            self.x1.copy_(self.embedding[token])
            lora.lora_decode_q4(self.layer, ws, ws.numel())
            torch.add(self.x1, self.y1, out=self.h1)
            lora.lora_decode_q4(self.lm_head, ws, ws.numel())
            logp = torch.log_softmax(self.logits.float(), dim=1)
            before[:, t] = token
            token = torch.multinomial(logp.exp(), 1, generator=self.g)[:, 0]
            after[:, t], nll[:, t], mask[:, t] = token, -logp.gather(1, token[:, None])[:, 0], alive
            alive = alive * (token != END).to(torch.uint8)
        return before, after, nll.view(-1), mask.view(-1)

    def score(self, before, after, mask, rank):
        """nll [T] and d nll / d h [T, D] of all tokens under the model (rank 0: its reference), with x and su."""
        T = before.numel()
        x = self.embedding[before.reshape(-1)]
        y, su = torch.empty_like(x), torch.empty(T, RANK, dtype=torch.bfloat16, device="cuda")
        shape = lora.make_shape(T, D, D, rank, SCALE if rank else 0.0)
        ws = workspace(lora.lora_workspace_size(shape, lora.LORA_FWD_BWD))
        lora.lora_linear_fwd_q4(shape, x, self.Wq, self.A if rank else None, self.B if rank else None, y,
                                su if rank else None, ws, ws.numel())
        h, dh = x + y, torch.empty_like(x)
        nll, loss = torch.empty(T, device="cuda"), torch.empty(1, device="cuda")
        targets = after.reshape(-1).int()
        ce = lora.make_ce_args(T, D, V, h, self.head, targets, loss, mask=mask, token_loss=nll, dh=dh)
        ce_ws = workspace(lora.lora_ce_workspace_size(ce))
        lora.lora_ce_fwd_bwd(ce, ce_ws, ce_ws.numel())
        return nll, dh, x, su

    def update(self, x, su, dh, rate, max_norm):
        """One step of gradient descent on A and B; the gradients' norm before clipping."""
        shape = lora.make_shape(x.shape[0], D, D, RANK, SCALE)
        dA, dB = torch.empty_like(self.A32), torch.empty_like(self.B32)
        ws = workspace(lora.lora_workspace_size(shape, lora.LORA_FWD_BWD))
        lora.lora_linear_bwd_q4(shape, dh, x, self.Wq, self.A, self.B, su, None, dA, dB, ws, ws.numel())
        grads = lora.make_grads([(dA, dA), (dB, dB)])
        norm = torch.empty(1, device="cuda")
        ws = workspace(lora.lora_clip_workspace_size(grads))
        lora.lora_clip_grads(grads, max_norm, norm, None, ws, ws.numel())
        self.A32.sub_(dA, alpha=rate)
        self.B32.sub_(dB, alpha=rate)
        self.A.copy_(self.A32)
        self.B.copy_(self.B32)
        return norm


def learn(model, kind="policy", rate=0.3, max_norm=0.5, steps=2):
    """One round: 16 answers, and `steps` updates from them.  Returns what it measured."""
    before, after, old_nll, mask = model.sample()
    T = before.numel()
    m = mask.view(SEQS, LENGTH).float()
    reward = ((after < WANTED).float() * m).sum(1) / m.sum(1)
    ref_nll = model.score(before, after, mask, 0)[0]
    if kind == "pref":  # the best against the worst answer, the second best against the second worst, ..
        order = reward.argsort(descending=True)
        order = torch.stack([order[:SEQS // 2], order.flip(0)[:SEQS // 2]], dim=1).view(-1)
        before, after = before[order], after[order]
        mask, old_nll, ref_nll = (t.view(SEQS, LENGTH)[order].reshape(-1) for t in (mask, old_nll, ref_nll))
    wanted = (after < WANTED).float().reshape(-1)  # a token's own reward: an answer's is their mean
    advantage = (wanted - reward.mean()) / 0.5
    offsets = (torch.arange(SEQS + 1, device="cuda") * LENGTH).int()
    loss, stats = torch.empty(1, device="cuda"), torch.zeros(2, device="cuda")
    losses, drift = [], None
    for _ in range(steps):
        nll, dh, x, su = model.score(before, after, mask, RANK)
        if drift is None:  # the two forwards of one model
            drift = ((nll - old_nll).abs() * mask).max().item()
        if kind == "policy":
            args = lora.make_policy_args(T, SEQS, D, offsets, nll, old_nll, advantage, loss, ref_nll=ref_nll, mask=mask,
                                         clip_low=0.2, clip_high=0.28, beta=0.02, reduction=lora.LORA_MEAN_TOKENS,
                                         advantage_per_token=True, dh_nll=dh, dh=dh, stats=stats)
            ws = workspace(lora.lora_policy_workspace_size(args))
            lora.lora_policy_fwd_bwd(args, ws, ws.numel())
        else:
            args = lora.make_pref_args(T, SEQS // 2, D, offsets, nll, loss, ref_nll=ref_nll, mask=mask, beta=0.1,
                                       dh_nll=dh, dh=dh)
            ws = workspace(lora.lora_pref_workspace_size(args))
            lora.lora_pref_fwd_bwd(args, ws, ws.numel())
        norm = model.update(x, su, dh, rate, max_norm)
        losses.append(loss.item())
    if lora.lora_read_status() != lora.LORA_OK:
        raise RuntimeError("a call's offsets or a bounded wait failed")
    return {"reward": reward.mean().item(), "losses": losses, "kl": stats[0].item(), "clipped": stats[1].item(),
            "norm": norm.item(), "drift": drift}


def main():
    p = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    p.add_argument("--loss", choices=["policy", "pref"], default="policy")
    p.add_argument("--rounds", type=int, default=40)
    a = p.parse_args()
    model = Model()
    for i in range(a.rounds):
        r = learn(model, a.loss)
        print(f"round {i:3d}  reward {r['reward']:.3f}  loss {r['losses'][0]:+.4f} -> {r['losses'][-1]:+.4f}  "
              f"kl {r['kl']:.4f}  clipped {r['clipped']:.3f}  norm {r['norm']:.3f}", flush=True)


if __name__ == "__main__":
    main()
