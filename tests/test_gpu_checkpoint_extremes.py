"""Activations and their gradients where a kept value is far outside the range that the functions change in, and
where a group is kept as NaN."""
import pytest
import torch

from operator_reference import TORCH

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
LARGE = {"f32": [1e4, 1e9, 1e13, 1.2e13, 2e13, 1e15, 6e18, 1e20, 1e30, 3.4028234e38],
         "f16": [1e4, 3e4, 65504.0],
         "bf16": [1e4, 1e9, 1e13, 1.2e13, 2e13, 1e15, 6e18, 1e20, 1e30, 3.38e38]}


@pytest.fixture(scope="module")
def b():
    from paper_2006_02924_b200 import binding

    return binding


def _large(dtype, pad):
    """One large value per group of 32, and where they are; `pad` more columns cut off again (unaligned rows)."""
    values = torch.tensor(LARGE[dtype] + [-v for v in LARGE[dtype]], device="cuda")
    at = 32 * torch.arange(values.numel(), device="cuda") + 5
    x = torch.zeros(3, 32 * values.numel() + pad, dtype=TORCH[dtype], device="cuda")
    x[1, at] = values.to(TORCH[dtype])
    x[1, at + 9] = 1.0                       # far below the step: its code is 0
    return x[:, :32 * values.numel()], at


@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("name", ACTS)
def test_large_values(b, name, dtype, pad):
    """From |x| = 1e4 on the slope is 1 or 0, and y is x or 0, to fp32 precision (the tails are below exp(-1e4)):
    exact equality, at every magnitude that the type holds."""
    x, at = _large(dtype, pad)
    y, kept = b.adasum_checkpoint_save(x, name)
    positive = (x[1, at] > 0) | (name == "none")
    assert torch.equal(y[1, at], torch.where(positive, x[1, at], 0))
    values = b.adasum_checkpoint_load(kept, *x.shape)
    assert torch.isfinite(values).all() and torch.equal(values[1, at] > 0, x[1, at] > 0)
    dy = torch.full_like(x, 3.0)
    got = b.adasum_checkpoint_act_grad(kept, dy, name)
    assert torch.isfinite(got).all()
    assert torch.equal(got[1, at], torch.where(positive, dy[1, at], 0))


@pytest.mark.parametrize("pad", [0, 3])
@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("name", ["relu", "gelu", "gelu_tanh", "silu"])
def test_a_group_kept_as_nan_has_no_gradient(b, name, dtype, pad):
    """The values of such a group are not known, so neither is the slope: NaN, whichever activation, so that an
    overflow on the way forward shows in the gradients.  Its neighbours are not touched."""
    x = torch.ones(4, 96 + pad, dtype=TORCH[dtype], device="cuda")
    x[0, 40], x[1, 3], x[2, 95] = float("inf"), float("nan"), -float("inf")
    x[3] = -1.0
    x = x[:, :96]
    bad = torch.zeros(4, 96, dtype=torch.bool, device="cuda")
    bad[0, 32:64], bad[1, :32], bad[2, 64:] = True, True, True
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    dy = torch.full_like(x, 2.0)
    dy[:, 7] = 0.0
    got = b.adasum_checkpoint_act_grad(kept, dy, name)
    assert torch.equal(torch.isnan(got), bad)
    if name == "relu":
        assert torch.equal(got[~bad], torch.where(x > 0, dy, 0)[~bad])


def test_fp32_tanh_gelu_slope_is_as_near_as_torch_arithmetic(b):
    """Against 64 bits, the fp32 slope is no further off (in the norm) than the same formula in fp32 torch operations."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(21)
    x = torch.randn(610, 1024, generator=gen, device="cuda")
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    at = b.adasum_checkpoint_load(kept, 610, 1024)

    def slope(v):
        k = (2 / torch.pi) ** 0.5
        t = torch.tanh(k * (v + 0.044715 * v * v * v))
        return 0.5 * (1 + t) + 0.5 * v * (1 - t * t) * k * (1 + 3 * 0.044715 * v * v)

    want = slope(at.double())
    got = b.adasum_checkpoint_act_grad(kept, torch.ones_like(x), "gelu_tanh")
    assert (got.double() - want).norm() <= (slope(at).double() - want).norm()
