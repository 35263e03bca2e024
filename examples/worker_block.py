"""N data-parallel workers' training steps on one GPU with a model of residual feed-forward blocks, all in the library's calls.

    h = dropout(sqrt(dim) * E[ids])                                      adasum_embedding_forward, adasum_dropout
    y = norm(h) w_0                                                      adasum_residual_norm
    per block:  a = gelu(y w1^T + b1)                                    adasum_fp8_pack, adasum_fp8_linear, adasum_checkpoint_save
                h = h + gate * dropout(norm(a w2^T + b2) w_post)         the same, adasum_residual_norm
                y = norm(h) w_next                                       (the same call)
    logits = y wo^T, cross entropy to the next token

Products take their operands in 8 bits: weights are packed once per step for all workers and both directions,
activations and gradients as they come.  Inputs of linear layers and of the activation are kept in 8 bits for the
gradients of the weights (adasum_checkpoint_*).  The dropouts' masks are computed again on the way back: `seed` is one number
per worker and step on the GPU, the place in the model tells the masks of a step apart.  Every gradient is written into
the worker's fused buffer; the buffers are combined with the N-way Adasum operator, tensor by tensor.

Run it with:  python examples/worker_block.py [--workers N] [--steps K]
"""
import argparse
import math
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2006_02924_b200 import binding as ad  # noqa: E402

EPS = 1e-5


class Model:
    """Shared fp32 parameters, as views of one flat buffer, and their places in a fused gradient buffer."""

    def __init__(self, vocab=997, dim=256, hidden=1024, blocks=2, seed=0, device="cuda"):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        self.dim, self.hidden, self.vocab, self.blocks = dim, hidden, vocab, blocks
        self.shapes = {"embedding": (vocab, dim), "norm0": (dim,)}
        for i in range(blocks):
            self.shapes |= {f"w1.{i}": (hidden, dim), f"b1.{i}": (hidden,), f"w2.{i}": (dim, hidden), f"b2.{i}": (dim,),
                            f"post.{i}": (dim,), f"gate.{i}": (dim,), f"norm{i + 1}": (dim,)}
        self.shapes["wo"] = (vocab, dim)
        self.names = list(self.shapes)
        self.offsets = [0]
        for name in self.names:
            self.offsets.append(self.offsets[-1] + math.prod(self.shapes[name]))
        self.flat = torch.empty(self.offsets[-1], device=device).normal_(generator=gen)
        for name in self.names:
            p = self.view(self.flat, name)
            if name.startswith(("norm", "post", "gate")):
                p.mul_(0.1).add_(0.5 if name.startswith("gate") else 1.0)
            else:
                p.mul_(0.0 if name.startswith("b") else 1 / math.sqrt(self.shapes[name][-1]))

    def view(self, flat, name):
        """Tensor `name` inside a flat buffer of the model's size."""
        i = self.names.index(name)
        return flat[self.offsets[i]:self.offsets[i + 1]].view(self.shapes[name])

    def __getitem__(self, name):
        return self.view(self.flat, name)

    def pack(self):
        """The weight matrices in 8 bits: once per step, for all workers and both directions."""
        return {name: ad.adasum_fp8_pack_weight(self[name]) for name in self.names if name[0] == "w"}


def _linear(packed, x, w, bias=None):
    rows, features = x.shape
    outputs = packed[w][1]
    return ad.adasum_fp8_linear(ad.adasum_fp8_pack(x), packed[w][0], rows, features, outputs, bias=bias, out_dtype=x.dtype)


def _linear_grad(packed, dy, w, features):
    rows, outputs = dy.shape
    return ad.adasum_fp8_linear_grad(ad.adasum_fp8_pack(dy), packed[w][0], rows, features, outputs, out_dtype=dy.dtype)


def worker_gradients(model, packed, ids, targets, grads, seed, p=0.1, scale=1.0, dtype=torch.bfloat16):
    """One worker's forward and backward on `ids`; writes scale * gradient into the fused buffer `grads` and returns the
    loss.  `packed`: the weights of model.pack()."""
    packed = {name: (w, model.shapes[name][0]) for name, w in packed.items()}
    dim, hidden = model.dim, model.hidden

    def grad(name):
        return model.view(grads, name)

    def keep(x, activation="none"):
        return ad.adasum_checkpoint_save(x, activation, want_out=activation != "none")

    x = ad.adasum_embedding_forward(model["embedding"], ids, scale=math.sqrt(dim), out_dtype=dtype)
    h = ad.adasum_dropout(x, p, seed, site=0, out=x)
    _, y, stats = ad.adasum_residual_norm(None, h, pre_weight=model["norm0"], eps=EPS, out_dtype=dtype, want_h=False)
    joints, kept = [(None, h, stats, dict(pre_weight=model["norm0"], eps=EPS))], []
    for i in range(model.blocks):
        _, kept_y = keep(y)
        a, kept_u = keep(_linear(packed, y, f"w1.{i}", model[f"b1.{i}"].to(dtype)), "gelu")
        _, kept_a = keep(a)
        f = _linear(packed, a, f"w2.{i}", model[f"b2.{i}"].to(dtype))
        joint = dict(post_norm="rms", post_weight=model[f"post.{i}"], pre_weight=model[f"norm{i + 1}"], eps=EPS,
                     gate=model[f"gate.{i}"], dropout=p, seed=seed, site=i + 1)
        h, y, stats = ad.adasum_residual_norm(f, h, **joint)
        joints.append((f, h, stats, joint))
        kept.append((kept_y, kept_u, kept_a))
    _, kept_out = keep(y)
    logits = _linear(packed, y, "wo").float()

    log_p = torch.log_softmax(logits, dim=1)
    loss = -log_p.gather(1, targets[:, None]).mean()
    d_logits = log_p.exp_()
    d_logits.scatter_add_(1, targets[:, None], torch.full_like(targets, -1, dtype=torch.float32)[:, None])
    d_logits = d_logits.div_(ids.numel()).to(dtype)

    ad.adasum_checkpoint_weight_grad(kept_out, d_logits, grad_weight=grad("wo"), scale=scale)
    dy, dh = _linear_grad(packed, d_logits, "wo", dim), None
    for i in reversed(range(model.blocks)):
        f, h, stats, joint = joints[i + 1]
        kept_y, kept_u, kept_a = kept[i]
        df, dh = ad.adasum_residual_norm_grad(f, h, stats, dy, dh, grad_post_weight=grad(f"post.{i}"),
                                              grad_pre_weight=grad(f"norm{i + 1}"), grad_gate=grad(f"gate.{i}"),
                                              scale=scale, gate_scale=scale, **joint)
        ad.adasum_checkpoint_weight_grad(kept_a, df, grad_weight=grad(f"w2.{i}"), grad_bias=grad(f"b2.{i}"), scale=scale)
        du = ad.adasum_checkpoint_act_grad(kept_u, _linear_grad(packed, df, f"w2.{i}", hidden), "gelu")
        ad.adasum_checkpoint_weight_grad(kept_y, du, grad_weight=grad(f"w1.{i}"), grad_bias=grad(f"b1.{i}"), scale=scale)
        dy = _linear_grad(packed, du, f"w1.{i}", dim)
    _, h, stats, joint = joints[0]
    _, dh = ad.adasum_residual_norm_grad(None, h, stats, dy, dh, want_x=False, grad_pre_weight=grad("norm0"), scale=scale, **joint)
    dx = ad.adasum_dropout(dh, p, seed, site=0, out=dh)
    ad.adasum_embedding_grad(dx, ids, grad_table=grad("embedding"), scale=scale * math.sqrt(dim))
    return loss


def train(workers=4, steps=20, tokens=512, lr=0.5, grad_dtype=torch.float32, seed=0):
    """`steps` optimizer steps of `workers` workers on a fixed synthetic text; returns the mean loss of each step."""
    model = Model(seed=seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1)
    follows = torch.randperm(model.vocab, generator=gen, device="cuda")    # the text's rule: each token has one successor
    total = model.flat.numel()
    grads = [torch.empty(total, dtype=grad_dtype, device="cuda") for _ in range(workers)]
    workspace = torch.empty(ad.adasum_workspace_bytes(total, len(model.names), workers, grad_dtype), dtype=torch.uint8, device="cuda")
    update = torch.empty(total, device="cuda")
    seeds = torch.arange(workers, device="cuda")                           # the workers' masks
    losses = []
    for _ in range(steps):
        packed, step_losses = model.pack(), []
        for worker in range(workers):
            ids = torch.randint(0, model.vocab, (tokens,), generator=gen, device="cuda")
            step_losses.append(worker_gradients(model, packed, ids, follows[ids], grads[worker], seeds[worker:worker + 1]))
        ad.adasum_reduce(grads, model.offsets, out=update, workspace=workspace)
        model.flat.sub_(update, alpha=lr)
        seeds.add_(workers)
        losses.append(torch.stack(step_losses).mean())
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--workers", type=int, default=4)
    parser.add_argument("--steps", type=int, default=20)
    args = parser.parse_args()
    for step, loss in enumerate(train(args.workers, args.steps)):
        print(f"step {step:3d}  loss {loss:.4f}")
