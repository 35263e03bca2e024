"""Activations kept in 8 bits: codes bit by bit, activations and their slopes in 64 bits."""
import numpy as np
import pytest
import torch

from operator_reference import (TINY, TORCH, UNIT, act, act_error, act_slope, assert_close, keep, kept_values,
                                      pack, to64)

pytestmark = pytest.mark.gpu

ACTS = ["none", "relu", "gelu", "gelu_tanh", "silu"]
SIZES = [(1, 1, 0, 0), (1, 32, 0, 0), (3, 31, 0, 0), (2, 33, 7, 1), (37, 1000, 24, 0), (61, 1023, 1, 0), (5, 4096, 0, 0),
         (257, 64, 8, 0), (130, 8, 0, 4)]


@pytest.fixture(scope="module")
def b():
    from paper_2006_02924_b200 import binding

    return binding


def _x(seed, rows, cols, dtype, pad=0, shift=0):
    """Values of every size that a group can meet: columns from 2^-12 to 2^7, some zeros, whole groups of zeros."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    flat = torch.randn(rows * (cols + pad) + shift, generator=gen, device="cuda")
    x = flat[shift:].view(rows, cols + pad)
    x *= torch.exp2(torch.randint(-12, 5, (1, cols + pad), generator=gen, device="cuda").float())
    x[torch.rand(rows, cols + pad, generator=gen, device="cuda") < 0.1] = 0.0
    if rows > 2:
        x[2] = 0.0
    return flat.to(TORCH[dtype])[shift:].view(rows, cols + pad)[:, :cols]


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,shift", SIZES)
@pytest.mark.parametrize("name", ACTS)
def test_save_and_load(b, dtype, rows, cols, pad, shift, name):
    x = _x(5, rows, cols, dtype, pad, shift)
    guard = torch.full((b.adasum_checkpoint_bytes(rows, cols) + 16,), 99, dtype=torch.uint8, device="cuda")
    y, kept = b.adasum_checkpoint_save(x, name, checkpoint=guard)
    x64 = to64(x)
    codes, steps = keep(x64)
    size = b.adasum_checkpoint_bytes(rows, cols)
    assert np.array_equal(kept[:size].cpu().numpy(), pack(codes, steps))
    assert torch.all(guard[size:] == 99)
    want = act(x64, name)
    assert_close(to64(y), want, (UNIT[dtype] + act_error(x64, name, dtype)) * np.abs(want) + TINY[dtype]
                 + 2.0**-125 * (1 + np.abs(x64)))       # underflow of the tail's fp32 factors
    values = kept_values(codes, steps, cols)
    assert np.array_equal(to64(b.adasum_checkpoint_load(kept, rows, cols)), values)
    # exact in the 16-bit types too, where the values came from them
    out = torch.full((rows, cols + pad), 5.0, dtype=TORCH[dtype], device="cuda")
    b.adasum_checkpoint_load(kept, rows, cols, out=out[:, :cols])
    if dtype != "f16":
        assert np.array_equal(to64(out[:, :cols]), values)
    assert torch.all(out[:, cols:] == 5.0)
    # in place
    z = x.clone() if pad == 0 else x
    b.adasum_checkpoint_save(z, name, out=z)
    assert torch.equal(z, y)


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,shift", SIZES)
@pytest.mark.parametrize("name", ACTS)
def test_act_grad(b, dtype, rows, cols, pad, shift, name):
    x = _x(6, rows, cols, dtype)
    dy = _x(7, rows, cols, dtype, pad, shift)
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    got = b.adasum_checkpoint_act_grad(kept, dy, name)
    values = kept_values(*keep(to64(x)), cols)
    slope, size = act_slope(values, name)
    want = to64(dy) * slope
    # the terms' errors times |dy|, two more fp32 operations, one rounding to the type
    bound = np.abs(to64(dy)) * (act_error(values, name, dtype) + 2.0**-22) * size
    assert_close(to64(got), want, bound + UNIT[dtype] * 1.001 * (np.abs(want) + bound) + TINY[dtype]
                 + 2.0**-125 * (1 + np.abs(values)) * (1 + np.abs(to64(dy))))
    b.adasum_checkpoint_act_grad(kept, dy, name, grad_in=dy)
    assert torch.equal(got, dy)


@pytest.mark.parametrize("name", ACTS)
def test_act_grad_against_differences(b, name):
    """Central differences of the forward formula in 64 bits, step 2^-10: their own error is h^2 / 6 times the third
    derivative (below 2 for all of these), under 4e-7; relu only away from its corner."""
    x = torch.linspace(-6, 6, 4000, device="cuda").view(10, 400)
    if name == "relu":
        x[x.abs() < 0.1] = 1.0
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    at = to64(b.adasum_checkpoint_load(kept, 10, 400))
    if name == "relu":
        at = np.where(np.abs(at) < 2.0**-9, 1.0, at)
    h = 2.0**-10
    want = (act(at + h, name) - act(at - h, name)) / (2 * h)
    got = to64(b.adasum_checkpoint_act_grad(kept, torch.ones_like(x), name))
    assert_close(got, want, 4e-7 + act_error(at, name, "f32") * (1 + np.abs(at)) + 2.0**-22)


def test_groups_at_the_ends_of_the_range(b):
    big, small = float(np.finfo(np.float32).max), 2.0**-149
    x = torch.zeros(9, 40, device="cuda")
    x[0, :32] = torch.linspace(-big, big, 32, device="cuda")     # the span overflows: Inf and NaN among these
    x[1, 0], x[1, 1] = big, small
    x[2, :4] = torch.tensor([small, -small, 2.0**-126, 2.0**-120], device="cuda")
    x[3, 5] = float("inf")
    x[4, 6] = float("nan")
    x[5, 35] = -float("inf")                                    # the filled-up group
    x[6, :6] = torch.tensor([127.5, 126.5, 127.499, -127.5, 63.5, -128 + 2.0**-9], device="cuda")   # ties, the limit
    x[7, :3] = torch.tensor([1.0, 0.5 + 2.0**-8, 1.5 * 2.0**-7], device="cuda")
    x[8] = 1.0
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    codes, steps = keep(to64(x))
    assert np.array_equal(kept.cpu().numpy(), pack(codes, steps))
    got = to64(b.adasum_checkpoint_load(kept, 9, 40))
    want = kept_values(codes, steps, 40)
    assert np.array_equal(np.isnan(got), np.isnan(want)) and np.isnan(want).sum() == 3 * 32 + 8
    assert np.array_equal(np.nan_to_num(got), np.nan_to_num(want))
    slope = to64(b.adasum_checkpoint_act_grad(kept, torch.ones_like(x), "silu"))
    assert np.array_equal(np.isnan(slope), np.isnan(want))


def test_largest_values(b):
    x = torch.linspace(-1, 1, 64, device="cuda").view(1, 64) * float(np.finfo(np.float32).max)
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    codes, steps = keep(to64(x))
    assert np.array_equal(kept.cpu().numpy(), pack(codes, steps)) and np.all(steps == 127 + 121)
    assert np.array_equal(to64(b.adasum_checkpoint_load(kept, 1, 64)), kept_values(codes, steps, 64))


def test_fp16_and_bf16_ranges(b):
    for dtype, top in ((torch.float16, 65504.0), (torch.bfloat16, 3.38e38)):
        x = torch.full((2, 64), top, dtype=dtype, device="cuda")
        x[1] = torch.finfo(dtype).tiny * 2.0**-3                  # a subnormal
        _, kept = b.adasum_checkpoint_save(x, want_out=False)
        values = kept_values(*keep(to64(x)), 64)
        got = b.adasum_checkpoint_load(kept, 2, 64, dtype=dtype)
        assert np.array_equal(to64(got), values)


def test_error_of_a_kept_value(b):
    x = _x(8, 500, 320, "f32")
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    off = (b.adasum_checkpoint_load(kept, 500, 320) - x).abs().view(500, 10, 32)
    top = x.abs().view(500, 10, 32).amax(dim=2, keepdim=True)
    assert torch.all(off <= top / 64)
    assert torch.all(off[x.view(500, 10, 32).abs() < 0.99 * top] <= (top / 128).expand_as(off)[x.view(500, 10, 32).abs() < 0.99 * top])


def test_no_rows(b):
    x = torch.empty(0, 40, device="cuda")
    y, kept = b.adasum_checkpoint_save(x, "gelu")
    assert y.shape == (0, 40) and kept.numel() == 0
    assert b.adasum_checkpoint_load(kept, 0, 40).shape == (0, 40)
    assert b.adasum_checkpoint_act_grad(kept, x, "gelu").shape == (0, 40)


def test_large_matrix(b):
    """More than 2^32 values: indexes pass 32 bits in every kernel."""
    rows, cols = (1 << 17) + 1, 1 << 15
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-1] = 3.0
    x[-2, 100] = -1.0
    y, kept = b.adasum_checkpoint_save(x, "relu", out=x)
    assert torch.all(y[-1] == 3.0) and torch.all(y[-2] == 0.0)
    tail = kept[(rows - 2) * cols:(rows - 1) * cols].view(torch.int8)
    assert tail[100] == -64 and tail.float().abs().sum() == 64
    del x
    out = b.adasum_checkpoint_act_grad(kept, y, "relu", grad_in=y)
    assert torch.all(out[-1] == 3.0) and torch.all(out[:5] == 0)
    b.adasum_checkpoint_load(kept, rows, cols, out=out)
    assert torch.all(out[-1] == 3.0) and out[-2, 100] == -1.0


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("name", ACTS)
def test_activation_of_inf_and_nan(b, dtype, name):
    x = torch.ones(3, 40, dtype=TORCH[dtype], device="cuda")
    x[0, 1], x[1, 38], x[2, 0] = float("inf"), float("nan"), -float("inf")
    y, kept = b.adasum_checkpoint_save(x, name)
    assert y[0, 1] == float("inf") and torch.isnan(y[1, 38])
    if name in ("none", "relu"):
        assert y[2, 0] == (0 if name == "relu" else -float("inf"))
    assert torch.isfinite(y).sum() >= 120 - 3
    values = b.adasum_checkpoint_load(kept, 3, 40)
    bad = torch.zeros(3, 40, dtype=torch.bool, device="cuda")
    bad[0, :32], bad[1, 32:], bad[2, :32] = True, True, True
    assert torch.equal(torch.isnan(values), bad)
    slope = b.adasum_checkpoint_act_grad(kept, torch.ones_like(x), name)
    if name not in ("none", "relu"):                 # their slope is 1 or 0 whatever the value
        assert torch.equal(torch.isnan(slope), bad)
