"""A small decoder trained with the whole optimizer path, as a pre-training program would use it:

* the weight matrices of the layers are TSR blocks (BF16 gradients, cores in a small subspace);
* the token embedding and the output head are dense parameters with 8-bit AdamW states, stochastically rounded, FP32 masters
  and the BF16 image that the model computes with;
* the normalisation weights are dense parameters with FP32 states and without weight decay;
* one global gradient norm over all of them clips the step: its factor goes to the dense step as a device scalar and, the core
  projection being linear, onto the cores;
* half-way the dense states are written out as FP32 moments and read back, as a checkpoint would.

    python examples/pretrain_small.py [steps]
"""
import math
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2602_08007_b200 as tsr  # noqa: E402

VOCAB, HIDDEN, FFN, LAYERS, HEADS, LENGTH, BATCH, RANK = 512, 256, 688, 2, 4, 64, 16, 32
SHAPES = [(HIDDEN, HIDDEN)] * 4 + [(FFN, HIDDEN)] * 2 + [(HIDDEN, FFN)]   # q, k, v, o, gate, up, down: weights are (out, in)


class Rotary:
    def __init__(self, device):
        freq = 1.0 / 10000 ** (torch.arange(0, HIDDEN // HEADS, 2, device=device) / (HIDDEN // HEADS))
        angle = torch.arange(LENGTH, device=device)[:, None] * freq[None, :]
        self.cos, self.sin = angle.cos(), angle.sin()

    def __call__(self, x):   # batch, heads, length, head size
        a, b = x.float().chunk(2, dim=-1)
        return torch.cat([a * self.cos - b * self.sin, a * self.sin + b * self.cos], dim=-1).to(x.dtype)


def norm(x, w):
    return (x.float() * torch.rsqrt(x.float().square().mean(-1, keepdim=True) + 1e-6) * w).to(x.dtype)


def logits_of(tokens, embed, mats, norms, head, rotary):
    x = embed[tokens]
    mask = torch.full((LENGTH, LENGTH), -math.inf, device=x.device).triu(1)
    for layer in range(LAYERS):
        q, k, v, o, gate, up, down = mats[layer * 7:layer * 7 + 7]
        h = norm(x, norms[2 * layer])
        split = lambda t: t.view(t.shape[0], LENGTH, HEADS, HIDDEN // HEADS).transpose(1, 2)  # noqa: E731
        a = rotary(split(h @ q.t())) @ rotary(split(h @ k.t())).transpose(-1, -2)
        a = torch.softmax(a.float() / math.sqrt(HIDDEN // HEADS) + mask, dim=-1).to(x.dtype) @ split(h @ v.t())
        x = x + a.transpose(1, 2).reshape(x.shape) @ o.t()
        h = norm(x, norms[2 * layer + 1])
        x = x + (torch.nn.functional.silu(h @ gate.t()) * (h @ up.t())) @ down.t()
    return (norm(x, norms[-1]) @ head.t()).float()


def batches(device, seed):
    """Synthetic text: from every token one of four others follows, the first most often."""
    gen = torch.Generator(device="cpu").manual_seed(seed)
    after = torch.randint(VOCAB, (VOCAB, 4), generator=gen)
    odds = torch.tensor([0.7, 0.15, 0.1, 0.05])
    while True:
        t = torch.empty(BATCH, LENGTH + 1, dtype=torch.int64)
        t[:, 0] = torch.randint(VOCAB, (BATCH,), generator=gen)
        for i in range(LENGTH):
            t[:, i + 1] = after[t[:, i], torch.multinomial(odds, BATCH, replacement=True, generator=gen)]
        yield t.to(device)


def train(steps=60, seed=0, lr=3e-3, max_norm=1.0, log=None):
    """Returns the losses and the gradient norms of all steps."""
    device = torch.device("cuda")
    torch.manual_seed(seed)
    blocks = [dict(m=m, n=n, r=RANK, p=8, q=1, K=20) for m, n in SHAPES * LAYERS]
    plan = tsr.Plan(blocks, g_dtype=torch.bfloat16)
    for W in plan.W:
        W.normal_(0, 0.02)

    params = [torch.empty(VOCAB, HIDDEN, device=device).normal_(0, 0.02) for _ in range(2)] + [torch.ones(HIDDEN, device=device) for _ in range(2 * LAYERS + 1)]
    grads = [torch.zeros_like(p, dtype=torch.bfloat16 if p.dim() == 2 else torch.float32) for p in params]
    images = [p.bfloat16() if p.dim() == 2 else None for p in params]
    dense = tsr.DensePlan(params, grads, images=images, norm_only=plan.G, wd_mult=[1.0 if p.dim() == 2 else 0.0 for p in params],
                          state_dtype=[torch.float8_e4m3fn if p.dim() == 2 else torch.float32 for p in params])
    rotary, data = Rotary(device), batches(device, seed + 1)
    losses, norms = [], []
    for t in range(1, steps + 1):
        tokens = next(data)
        mats = [W.bfloat16().requires_grad_() for W in plan.W]
        leaves = [(image if image is not None else p).detach().requires_grad_() for p, image in zip(params, images)]
        out = logits_of(tokens[:, :-1], leaves[0], mats, leaves[2:], leaves[1], rotary)
        loss = torch.nn.functional.cross_entropy(out.reshape(-1, VOCAB), tokens[:, 1:].reshape(-1))
        loss.backward()
        for G, w in zip(plan.G + grads, mats + leaves):
            G.copy_(w.grad)

        hyper = tsr.make_hyper(t, lr=lr * min(1.0, t / 10), beta2=0.99, weight_decay=0.01)
        clip = dense.grad_norm(max_norm)                  # (norm, factor) on the device; no host read
        if t == 1:
            plan.init_subspace(seed=seed)
        elif t % 20 == 0:
            plan.rsvd_refresh(seed=seed + t)
        plan.project_core()
        torch._foreach_mul_(plan.C, clip[1])              # U^T (f G) V = f C
        plan.adam_core_step(hyper)
        plan.backproject_apply(hyper)
        dense.step(hyper, grad_scale=clip[1:], rounding=tsr.TSR_ROUND_STOCHASTIC, seed=seed)

        losses.append(loss.detach())
        norms.append(clip[0].clone())
        if t == steps // 2:                               # to FP32 moments and back
            saved = tsr.DensePlan(None, None, states=[tuple(torch.zeros(p.numel(), device=device) for _ in range(2)) for p in params])
            kept = tsr.DensePlan(None, None, states=dense.states)
            saved.copy_state(kept)
            kept.copy_state(saved)
        if log:
            log("step %3d  loss %.4f  gradient norm %.3f" % (t, float(losses[-1]), float(norms[-1])))
    assert all(s == tsr.TSR_OK for s in plan.poll_status())
    return torch.stack(losses).tolist(), torch.stack(norms).tolist()


if __name__ == "__main__":
    train(int(sys.argv[1]) if len(sys.argv) > 1 else 60, log=print)
