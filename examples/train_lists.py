"""A training loop over a model's many tensors: gradient accumulation, the norm test, clipping and AdamW with the calls on lists.

A small language model in bfloat16 learns synthetic text (every token follows from the one before, mostly).  Per step, J workers, here one
after the other, take M micro-batches each, whose size follows the batch size:

    normtest_accumulate      a micro-batch's bf16 gradients are added to the worker's fp32 row, 1/M each
    normtest_step            mean gradient, norm-test statistic and next batch size of the J rows
    normtest_grad_norm       global norm of the mean gradient and the clipping factor
    normtest_adamw_tensors   clipped AdamW on the fp32 weights, tensor by tensor, and the model's bf16 weights beside them

Run: python examples/train_lists.py [steps]
"""
from __future__ import annotations

import os
import sys

import torch
from torch import nn

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2412_21124_amd import binding as B  # noqa: E402

VOCAB, WIDTH, WORKERS, MICRO_STEPS, MICRO_BATCH = 512, 128, 4, 2, 64
MAX_NORM, ETA, B_MAX = 0.75, 0.06, 4096


def model(device) -> nn.Module:
    return nn.Sequential(nn.Embedding(VOCAB, WIDTH), nn.Linear(WIDTH, 4 * WIDTH), nn.GELU(), nn.LayerNorm(4 * WIDTH),
                         nn.Linear(4 * WIDTH, WIDTH), nn.GELU(), nn.Linear(WIDTH, VOCAB)).to(device=device, dtype=torch.bfloat16)


def text(n, gen, device):
    """(tokens, next tokens): the successor of a token is fixed, but one in eight is drawn."""
    x = torch.randint(VOCAB, (n,), device=device, generator=gen)
    noise = torch.randint(VOCAB, (n,), device=device, generator=gen)
    keep = torch.rand(n, device=device, generator=gen) > 0.125
    return x, torch.where(keep, (x * 7 + 3) % VOCAB, noise)


class Trainer:
    """What a program keeps from step to step: the model, fp32 weights and moments, the workers' rows, and a list for each."""

    def __init__(self, device="cuda:0", seed=0):
        torch.manual_seed(seed)
        self.device = torch.device(device)
        self.gen = torch.Generator(device=self.device).manual_seed(seed)
        self.net = model(self.device)
        self.params = list(self.net.parameters())
        for p in self.params:
            p.grad = torch.zeros_like(p)   # of the list below: zeroed, never replaced
        sizes = [p.numel() for p in self.params]
        d = sum(sizes)
        self.rows = torch.zeros(WORKERS, (d + 63) // 64 * 64, device=self.device)
        self.d, self.mean = d, torch.zeros(d, device=self.device)

        def tensors(flat):
            return [x.view(p.shape) for x, p in zip(flat[:d].split(sizes), self.params)]
        self.w = [p.detach().float() for p in self.params]
        self.m, self.v = [torch.zeros_like(w) for w in self.w], [torch.zeros_like(w) for w in self.w]
        self.grads = B.make_tensor_list([p.grad for p in self.params])
        alike = lambda ts: B.make_tensor_list(ts, like=self.grads)   # noqa: E731
        self.row_lists = [alike(tensors(row)) for row in self.rows]
        self.mean_list = alike(tensors(self.mean))
        self.w_list, self.m_list, self.v_list = alike(self.w), alike(self.m), alike(self.v)
        self.copy_list = alike([p.detach() for p in self.params])
        self.norms = B.make_norms(self.grads)
        self.b_k, self.k = WORKERS * MICRO_STEPS * MICRO_BATCH, 0

    def backward(self) -> torch.Tensor:
        x, y = text(self.b_k // (WORKERS * MICRO_STEPS), self.gen, self.device)
        loss = nn.functional.cross_entropy(self.net(x).float(), y)
        loss.backward()
        return loss.detach()

    def step(self) -> dict:
        self.k += 1
        losses = []
        for row in self.row_lists:
            for micro in range(MICRO_STEPS):
                torch._foreach_zero_([p.grad for p in self.params])
                losses.append(self.backward())
                B.normtest_accumulate(row, self.grads, beta=0.0 if micro == 0 else 1.0, scale=1.0 / MICRO_STEPS)
        hyper = B.make_hyper(lr=2e-3, weight_decay=0.01, eta=ETA, step=self.k, b_k=self.b_k, b_max=B_MAX, round_to=WORKERS * MICRO_STEPS,
                             flags=B.NT_DO_STATS | B.NT_WRITE_GBAR)
        result = B.normtest_step(self.rows, None, None, None, hyper, d=self.d, gbar_out=self.mean)
        B.normtest_grad_norm(self.mean_list, self.norms, max_norm=MAX_NORM)
        B.normtest_adamw_tensors(self.mean_list, self.w_list, self.m_list, self.v_list, hyper, norms=self.norms, copy=self.copy_list,
                                 skip_nonfinite=True)
        # one synchronisation a step; a program that tests every few steps needs none in between
        r, n = B.read_result(result), B.read_norms(self.norms)[0]
        self.b_k = r.next_b
        return {"loss": float(torch.stack(losses).mean()), "norm": n.norm, "clipped": bool(n.clipped), "T": r.T, "next_b": r.next_b,
                "gbar_sq": r.gbar_sq}


def main(steps: int = 40) -> list:
    trainer = Trainer()
    history = []
    for k in range(steps):
        history.append(trainer.step())
        if k % 10 == 0 or k == steps - 1:
            print("step %3d  loss %.3f  norm %.3f%s  T %.1f  next batch size %d" % (
                k + 1, history[-1]["loss"], history[-1]["norm"], " (clipped)" if history[-1]["clipped"] else "", history[-1]["T"], history[-1]["next_b"]))
    return history


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 40)
