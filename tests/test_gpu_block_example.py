"""The operators around the linear layers together: a worker's gradients against autograd, and steps with the reduce."""
import math
import os
import sys

import pytest
import torch

pytestmark = pytest.mark.gpu

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


def _want(model, ids, targets, seed, p, scale):
    """The gradients of the same model in 64 bits, with the same masks, nothing in 8 bits."""
    from paper_2006_02924_b200 import binding as ad

    q = {n: model[n].double().requires_grad_() for n in model.names}

    def mask(site):
        ones = torch.ones(ids.numel(), model.dim, device="cuda")
        return ad.adasum_dropout(ones, p, seed, site=site).double()

    def norm(x):
        return x * torch.rsqrt(x.square().mean(1, keepdim=True) + 1e-5)

    h = mask(0) * q["embedding"][ids] * math.sqrt(model.dim)
    y = norm(h) * q["norm0"]
    for i in range(model.blocks):
        a = torch.nn.functional.gelu(y @ q[f"w1.{i}"].t() + q[f"b1.{i}"])
        f = a @ q[f"w2.{i}"].t() + q[f"b2.{i}"]
        h = h + q[f"gate.{i}"] * mask(i + 1) * (norm(f) * q[f"post.{i}"])
        y = norm(h) * q[f"norm{i + 1}"]
    loss = torch.nn.functional.cross_entropy(y @ q["wo"].t(), targets)
    loss.backward()
    return loss.item(), {n: scale * q[n].grad for n in model.names}


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_against_autograd(dtype):
    import worker_block as ex

    model = ex.Model(vocab=301, dim=96, hidden=200, blocks=2, seed=3)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    ids = torch.randint(0, 301, (2000,), generator=gen, device="cuda")
    targets = torch.randint(0, 301, (2000,), generator=gen, device="cuda")
    seed = torch.tensor([12345], device="cuda")
    grads = torch.full((model.flat.numel(),), 7.0, device="cuda")
    loss = ex.worker_gradients(model, model.pack(), ids, targets, grads, seed, scale=0.5, dtype=dtype)
    want_loss, want = _want(model, ids, targets, seed, 0.1, 0.5)
    assert abs(loss.item() - want_loss) < 0.02 * want_loss
    for name in model.names:
        g, w = model.view(grads, name).double(), want[name]
        off = ((g - w).norm() / w.norm()).item()
        # An e4m3 code is off by at most 2^-4 of its value: between 0 and 1/16, uniformly, over a significand between 1 and
        # 2, which is a root mean square of 0.025; a product of two such matrices is off by 0.036 of its norm where
        # errors are independent.  A gradient here has at most nine products on its way (five forward, four back) and four
        # factors kept in 8 bits (0.014 each): sqrt(9 * 0.036^2 + 4 * 0.014^2) = 0.11 for gains of one.  The norms and the
        # activation's curvature let forward errors count more than once: a factor of two is left for them.
        assert off < 0.22, (name, off)


@pytest.mark.parametrize("grad_dtype", [torch.float32, torch.bfloat16])
def test_training_steps_run(grad_dtype):
    import worker_block as ex

    losses = ex.train(workers=3, steps=4, tokens=300, grad_dtype=grad_dtype)
    assert len(losses) == 4 and all(math.isfinite(x) for x in losses)


def test_the_same_step_twice_and_captured():
    """A step is the same from run to run, and a captured one follows its seed."""
    import worker_block as ex

    model = ex.Model(vocab=200, dim=64, hidden=128, blocks=1, seed=5)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(6)
    ids = torch.randint(0, 200, (333,), generator=gen, device="cuda")
    seed, packed = torch.tensor([1], device="cuda"), model.pack()
    out = [torch.empty(model.flat.numel(), device="cuda") for _ in range(3)]
    for grads in out[:2]:
        ex.worker_gradients(model, packed, ids, ids, grads, seed)
    assert torch.equal(out[0], out[1])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        ex.worker_gradients(model, packed, ids, ids, out[2], seed)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out[2], out[0])
    seed.fill_(2)
    graph.replay()
    ex.worker_gradients(model, packed, ids, ids, out[1], seed)
    torch.cuda.synchronize()
    assert torch.equal(out[2], out[1]) and not torch.equal(out[2], out[0])
