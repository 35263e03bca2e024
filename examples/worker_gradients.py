"""One optimizer step of N data-parallel workers on one GPU, from token ids to the combined update.

Every worker runs forward and backward of a small language model on its own microbatch.  Its activations are
kept in 8 bits (a quarter of the fp32, half of the bf16 memory), its gradients are written straight into its
fused buffer, and the N buffers are combined with the N-way Adasum operator, tensor by tensor:

    x  = sqrt(dim) * E[ids]                       adasum_embedding_forward
    h  = x w1^T + b1                              kept: x (for w1), h (for the activation)
    a  = gelu(h)                                  adasum_checkpoint_save, which also keeps h; kept: a (for w2)
    logits = a w2^T + b2, cross entropy to the next token
    dw2, db2 from kept a;  dh = da * gelu'(kept h);  dw1, db1 from kept x;  dE by sorted tokens

The matrix products of the forward pass and of the input gradients are torch's; no gradient goes through
autograd.  Run it with:  python examples/worker_gradients.py [--workers N] [--steps K]
"""
import argparse
import math
import os
import sys

import torch

if __name__ == "__main__":
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

from paper_2006_02924_b200 import binding as ad  # noqa: E402

NAMES = ("embedding", "w1", "b1", "w2", "b2")


class Model:
    """Shared fp32 parameters, as views of one flat buffer, and their places in a fused gradient buffer."""

    def __init__(self, vocab=997, dim=256, hidden=1024, seed=0, device="cuda"):
        gen = torch.Generator(device=device)
        gen.manual_seed(seed)
        shapes = {"embedding": (vocab, dim), "w1": (hidden, dim), "b1": (hidden,), "w2": (vocab, hidden), "b2": (vocab,)}
        self.dim, self.shapes, self.offsets = dim, shapes, [0]
        for name in NAMES:
            self.offsets.append(self.offsets[-1] + math.prod(shapes[name]))
        self.flat = torch.empty(self.offsets[-1], device=device).normal_(generator=gen)
        for name, size in (("embedding", 1 / math.sqrt(dim)), ("w1", 1 / math.sqrt(dim)), ("b1", 0.0),
                           ("w2", 1 / math.sqrt(hidden)), ("b2", 0.0)):
            self.view(self.flat, name).mul_(size)

    def view(self, flat, name):
        """Tensor `name` inside a flat buffer of the model's size."""
        i = NAMES.index(name)
        return flat[self.offsets[i]:self.offsets[i + 1]].view(self.shapes[name])


def worker_gradients(model, ids, targets, grads, scale=1.0, dtype=torch.bfloat16):
    """One worker's forward and backward on `ids`; writes scale * gradient into the fused buffer `grads` and
    returns the loss.  The activations held between the passes are the three checkpoints."""
    def param(name):
        return model.view(model.flat, name)

    w1, w2 = param("w1").to(dtype), param("w2").to(dtype)
    x = ad.adasum_embedding_forward(param("embedding"), ids, scale=math.sqrt(model.dim), out_dtype=dtype)
    h = torch.addmm(param("b1").to(dtype), x, w1.t())
    _, kept_x = ad.adasum_checkpoint_save(x, want_out=False)
    a, kept_h = ad.adasum_checkpoint_save(h, "gelu")
    _, kept_a = ad.adasum_checkpoint_save(a, want_out=False)
    logits = torch.addmm(param("b2").to(dtype), a, w2.t()).float()
    del x, h, a

    log_p = torch.log_softmax(logits, dim=1)
    loss = -log_p.gather(1, targets[:, None]).mean()
    d_logits = log_p.exp_()
    d_logits.scatter_add_(1, targets[:, None], torch.full_like(targets, -1, dtype=torch.float32)[:, None])
    d_logits = d_logits.div_(ids.numel()).to(dtype)

    ad.adasum_checkpoint_weight_grad(kept_a, d_logits, grad_weight=model.view(grads, "w2"),
                                     grad_bias=model.view(grads, "b2"), scale=scale)
    d_h = ad.adasum_checkpoint_act_grad(kept_h, d_logits @ w2, "gelu")
    ad.adasum_checkpoint_weight_grad(kept_x, d_h, grad_weight=model.view(grads, "w1"),
                                     grad_bias=model.view(grads, "b1"), scale=scale)
    ad.adasum_embedding_grad(d_h @ w1, ids, grad_table=model.view(grads, "embedding"),
                             scale=scale * math.sqrt(model.dim))
    return loss


def train(workers=4, steps=20, tokens=512, lr=0.5, grad_dtype=torch.float32, seed=0):
    """`steps` optimizer steps of `workers` workers on a fixed synthetic text; returns the mean loss of each step."""
    model = Model(seed=seed)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed + 1)
    vocab = model.shapes["embedding"][0]
    follows = torch.randperm(vocab, generator=gen, device="cuda")       # the text's rule: each token has one successor
    grads = [torch.empty(model.flat.numel(), dtype=grad_dtype, device="cuda") for _ in range(workers)]
    total, tensors = model.flat.numel(), len(NAMES)
    workspace = torch.empty(ad.adasum_workspace_bytes(total, tensors, workers, grad_dtype), dtype=torch.uint8, device="cuda")
    update = torch.empty(total, device="cuda")
    losses = []
    for _ in range(steps):
        step_losses = []
        for worker in range(workers):
            ids = torch.randint(0, vocab, (tokens,), generator=gen, device="cuda")
            step_losses.append(worker_gradients(model, ids, follows[ids], grads[worker]))
        ad.adasum_reduce(grads, model.offsets, out=update, workspace=workspace)
        model.flat.sub_(update, alpha=lr)
        losses.append(torch.stack(step_losses).mean())
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    parser = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    parser.add_argument("--workers", type=int, default=4)
    parser.add_argument("--steps", type=int, default=20)
    args = parser.parse_args()
    for step, loss in enumerate(train(args.workers, args.steps)):
        print(f"step {step:3d}  loss {loss:.4f}")
