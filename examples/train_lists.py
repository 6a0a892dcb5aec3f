"""A training loop over a model's many tensors: gradient accumulation, the norm test, clipping and AdamW with the calls on lists.

A small language model in bfloat16 learns synthetic text (every token follows from the one before, mostly).  Per step, J workers, here one
after the other, take M micro-batches each, whose size follows the batch size:

    normtest_accumulate      a micro-batch's bf16 gradients are added to the worker's fp32 row, 1/M each
    normtest_step            mean gradient, norm-test statistic and next batch size of the J rows
    normtest_grad_norm       global norm of the mean gradient and the clipping factor
    normtest_adamw_tensors   clipped AdamW on the fp32 weights, tensor by tensor, and the model's bf16 weights beside them

With --mx the model's layers are low-precision ones: an RMS norm that adds the residual and leaves 8-bit codes (normtest_rms_norm), weights in 4 bits,
quantised anew after every update (normtest_mx_quantize), products of the two (normtest_mx_matmul), and gradients rounded to 8 bits without bias, in both
directions, for the two products of the way back.

Run: python examples/train_lists.py [steps] [--mx]
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


class Linear4(nn.Module):
    """A linear layer whose weight is multiplied in 4 bits: its codes, and its transpose's for the way back."""

    def __init__(self, width, out, device):
        super().__init__()
        self.weight = nn.Parameter(torch.randn(out, width, device=device).mul_(width ** -0.5).to(torch.bfloat16))
        self.forth, self.back = B.make_mx(out, width, B.NT_MX_E2M1, device), B.make_mx(width, out, B.NT_MX_E2M1, device)
        self.requantize()

    def requantize(self):
        B.normtest_mx_quantize(self.weight.detach(), self.forth, self.back)

    def forward(self, x):
        return _Linear.apply(x, self.weight, self)


class NormLinear4(Linear4):
    """The layer behind an RMS norm of x + residual.  Returns its output and that sum."""

    def __init__(self, width, out, device):
        super().__init__(width, out, device)
        self.gain = nn.Parameter(torch.ones(width, device=device))

    def forward(self, x, residual=None):
        return _NormLinear.apply(x, residual, self.gain, self.weight, self)


def _both_ways(x, noise=None):
    """8-bit codes of x (tokens x width) and of its transpose."""
    codes, turned = (B.make_mx(*shape, B.NT_MX_E4M3, x.device) for shape in (x.shape, x.shape[::-1]))
    B.normtest_mx_quantize(x, codes, turned, fit=noise is not None, noise=noise)
    return codes, turned


def _gradients(d, turned, layer):
    """Of the input and of the weight, from the output's, rounded without bias."""
    d, d_turned = _both_ways(d.contiguous(), torch.randint(256, d.shape, dtype=torch.uint8, device=d.device))
    return B.normtest_mx_matmul(d, layer.back), B.normtest_mx_matmul(d_turned, turned)


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, layer):
        codes, ctx.turned = _both_ways(x)
        ctx.layer = layer
        return B.normtest_mx_matmul(codes, layer.forth)

    @staticmethod
    def backward(ctx, d):
        return *_gradients(d, ctx.turned, ctx.layer), None


class _NormLinear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, residual, gain, weight, layer):
        total, y, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(x.shape[0], device=x.device)
        codes, ctx.turned = (B.make_mx(*shape, B.NT_MX_E4M3, x.device) for shape in (x.shape, x.shape[::-1]))
        B.normtest_rms_norm(x, gain, y, residual=residual, sum_out=total, out_mx=codes, rstd=rstd)
        B.normtest_mx_quantize(y, None, ctx.turned)
        ctx.layer, ctx.added = layer, residual is not None
        ctx.save_for_backward(total, gain, rstd)
        return B.normtest_mx_matmul(codes, layer.forth), total

    @staticmethod
    def backward(ctx, d, dsum):
        total, gain, rstd = ctx.saved_tensors
        dy, dweight = _gradients(d, ctx.turned, ctx.layer)
        dgain = torch.empty_like(gain)
        B.normtest_rms_norm_backward(dy, total, gain, rstd, dy, dsum=dsum.contiguous(), dweight=dgain)
        return dy, dy if ctx.added else None, dgain, dweight, None


class LowPrecision(nn.Module):
    def __init__(self, device):
        super().__init__()
        self.embed = nn.Embedding(VOCAB, WIDTH).to(device=device, dtype=torch.bfloat16)
        self.up, self.down = NormLinear4(WIDTH, 4 * WIDTH, device), Linear4(4 * WIDTH, WIDTH, device)
        self.head = NormLinear4(WIDTH, VOCAB, device)

    def forward(self, tokens):
        x, kept = self.up(self.embed(tokens))
        return self.head(self.down(nn.functional.gelu(x)), kept)[0]


def text(n, gen, device):
    """(tokens, next tokens): the successor of a token is fixed, but one in eight is drawn."""
    x = torch.randint(VOCAB, (n,), device=device, generator=gen)
    noise = torch.randint(VOCAB, (n,), device=device, generator=gen)
    keep = torch.rand(n, device=device, generator=gen) > 0.125
    return x, torch.where(keep, (x * 7 + 3) % VOCAB, noise)


class Trainer:
    """What a program keeps from step to step: the model, fp32 weights and moments, the workers' rows, and a list for each."""

    def __init__(self, device="cuda:0", seed=0, mx=False):
        torch.manual_seed(seed)
        self.device = torch.device(device)
        self.gen = torch.Generator(device=self.device).manual_seed(seed)
        self.net = LowPrecision(self.device) if mx else model(self.device)
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
        for layer in self.net.modules():
            if isinstance(layer, Linear4):
                layer.requantize()
        # one synchronisation a step; a program that tests every few steps needs none in between
        r, n = B.read_result(result), B.read_norms(self.norms)[0]
        self.b_k = r.next_b
        return {"loss": float(torch.stack(losses).mean()), "norm": n.norm, "clipped": bool(n.clipped), "T": r.T, "next_b": r.next_b,
                "gbar_sq": r.gbar_sq}


def main(steps: int = 40, mx: bool = False) -> list:
    trainer = Trainer(mx=mx)
    history = []
    for k in range(steps):
        history.append(trainer.step())
        if k % 10 == 0 or k == steps - 1:
            print("step %3d  loss %.3f  norm %.3f%s  T %.1f  next batch size %d" % (
                k + 1, history[-1]["loss"], history[-1]["norm"], " (clipped)" if history[-1]["clipped"] else "", history[-1]["T"], history[-1]["next_b"]))
    return history


if __name__ == "__main__":
    given = [a for a in sys.argv[1:] if a != "--mx"]
    main(int(given[0]) if given else 40, "--mx" in sys.argv[1:])
