"""Gradients of a linear layer from kept activations against products in 64 bits."""
import numpy as np
import pytest
import torch

from operator_reference import TINY, TORCH, UNIT, assert_close, keep, kept_values, to64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2006_02924_b200 import binding

    return binding


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _normal(gen, rows, cols, dtype, pad=0, shift=0):
    flat = torch.randn(rows * (cols + pad) + shift, generator=gen, device="cuda")
    return flat.to(TORCH[dtype])[shift:].view(rows, cols + pad)[:, :cols]


def _want(dy, values, scale):
    """Gradients and the error bound of an fp32 sum in which every addition may truncate (2^-23 of the sum of
    magnitudes per term)."""
    unit = (dy.shape[0] + 2) * 2.0**-23 * abs(scale)
    return (dy.T @ values * scale, unit * (np.abs(dy).T @ np.abs(values)),
            dy.sum(0) * scale, unit * np.abs(dy).sum(0))


@pytest.mark.parametrize("in_type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,features,outputs,pad,shift,out_type", [
    (1, 1, 1, 0, 0, "f32"), (1, 32, 8, 0, 0, "f16"), (2, 33, 9, 3, 1, "f32"), (63, 128, 256, 0, 0, "bf16"),
    (64, 256, 256, 0, 0, "f32"), (65, 257, 255, 1, 0, "f32"), (333, 1000, 257, 3, 0, "f32"),
    (1025, 96, 64, 8, 0, "f32"), (700, 520, 300, 4, 1, "f16"), (2048, 130, 1030, 0, 0, "f32"),
    (511, 1, 700, 0, 0, "f32"), (300, 640, 1, 7, 0, "bf16"), (5000, 64, 40, 0, 0, "f32")])
def test_weight_grad(b, in_type, rows, features, outputs, pad, shift, out_type):
    gen = _gen(11)
    x = _normal(gen, rows, features, in_type)
    dy = _normal(gen, rows, outputs, in_type, pad, shift)
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    values = kept_values(*keep(to64(x)), features)
    scale = float(np.float32(0.3))
    flat = torch.full((outputs * features + outputs + 20,), 3.0, dtype=TORCH[out_type], device="cuda")
    at = 5 if shift else 8
    dw, db = flat[at:at + outputs * features], flat[at + outputs * features + 1:at + outputs * features + 1 + outputs]
    b.adasum_checkpoint_weight_grad(kept, dy, features=features, grad_weight=dw, grad_bias=db, scale=scale)
    w, w_err, c, c_err = _want(to64(dy), values, scale)
    u = UNIT[out_type] * 1.001
    assert_close(to64(dw).reshape(outputs, features), w, w_err + u * (np.abs(w) + w_err) + TINY[out_type], "weight")
    assert_close(to64(db), c, c_err + u * (np.abs(c) + c_err) + TINY[out_type], "bias")
    # normwise: at most 16 truncated additions of 16 terms each build a sum before it is rounded into fp32, each
    # off by up to 2^-23 of it
    assert np.linalg.norm(to64(dw) - w.reshape(-1)) <= (2e-6 + u) * np.linalg.norm(w) + TINY[out_type] * np.sqrt(w.size)
    spare = torch.cat((flat[:at], flat[at + outputs * features:at + outputs * features + 1], flat[at + outputs * features + 1 + outputs:]))
    assert torch.all(spare == 3.0), "written outside"
    # again, without the bias: the same bits
    again, none = b.adasum_checkpoint_weight_grad(kept, dy, features=features, grad_dtype=TORCH[out_type], scale=scale)
    assert none is None and torch.equal(again.reshape(-1), dw)
    base = torch.randn(outputs, features, generator=gen, device="cuda").to(TORCH[out_type])
    base_b = torch.randn(outputs, generator=gen, device="cuda").to(TORCH[out_type])
    total, total_b = base.clone(), base_b.clone()
    b.adasum_checkpoint_weight_grad(kept, dy, grad_weight=total, grad_bias=total_b, scale=scale, accumulate=True)
    u += 2.0**-24
    assert_close(to64(total), to64(base) + w, w_err + u * (np.abs(to64(base) + w) + w_err) + TINY[out_type], "weight")
    assert_close(to64(total_b), to64(base_b) + c, c_err + u * (np.abs(to64(base_b) + c) + c_err) + TINY[out_type], "bias")


def test_products_are_exact(b):
    """Values kept without loss and small integer gradients: every product and sum is a whole number below 2^24."""
    gen = _gen(12)
    x = torch.randint(-127, 128, (600, 192), generator=gen, device="cuda").float()
    x[:, ::32] = 64.0 + torch.randint(0, 64, (600, 6), generator=gen, device="cuda").float()      # step 1
    dy = torch.randint(-60, 61, (600, 136), generator=gen, device="cuda").float()
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    for dtype in TORCH.values():
        dw, db = b.adasum_checkpoint_weight_grad(kept, dy.to(dtype), features=192, want_bias=True)
        assert torch.equal(dw.double(), dy.double().t() @ x.double())
        assert torch.equal(db.double(), dy.double().sum(0))


def test_fp32_gradients_keep_their_24_bits(b):
    """One row: every gradient is one product, so it must be right to fp32 rounding."""
    gen = _gen(13)
    x = torch.randn(1, 96, generator=gen, device="cuda")
    dy = torch.randn(1, 72, generator=gen, device="cuda") * torch.exp2(torch.randint(-90, 90, (1, 72), generator=gen, device="cuda").float())
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    dw, db = b.adasum_checkpoint_weight_grad(kept, dy, features=96, want_bias=True)
    values = kept_values(*keep(to64(x)), 96)
    want = to64(dy).T @ values
    assert_close(to64(dw), want, 4 * 2.0**-23 * np.abs(want))
    assert_close(to64(db), to64(dy)[0], 4 * 2.0**-23 * np.abs(to64(dy)[0]))


def test_nan_and_inf_stay_in_their_rows_and_columns(b):
    for dtype in TORCH.values():
        x = torch.ones(70, 96, device="cuda")
        x[69, 40] = float("nan")                                  # kept as NaN: features 32 .. 63
        dy = torch.ones(70, 80, device="cuda")
        dy[0, 3] = float("inf")
        dy[5, 7] = float("nan")
        _, kept = b.adasum_checkpoint_save(x, want_out=False)
        dw, db = b.adasum_checkpoint_weight_grad(kept, dy.to(dtype), features=96, want_bias=True)
        bad = torch.zeros(80, 96, dtype=torch.bool, device="cuda")
        bad[:, 32:64] = True
        bad[3] = True
        bad[7] = True
        assert torch.equal(~torch.isfinite(dw), bad)
        assert torch.isinf(dw[3, 0]) and torch.isnan(dw[7, 0]) and torch.isnan(dw[0, 40])
        assert torch.isinf(db[3]) and torch.isnan(db[7]) and torch.isfinite(db).sum() == 78


def test_no_rows_and_no_features(b):
    kept = torch.empty(0, dtype=torch.uint8, device="cuda")
    dw, db = torch.ones(6, 40, device="cuda"), torch.ones(6, device="cuda")
    empty = torch.empty(0, 6, device="cuda")
    b.adasum_checkpoint_weight_grad(kept, empty, grad_weight=dw, grad_bias=db, accumulate=True)
    assert torch.all(dw == 1) and torch.all(db == 1)
    b.adasum_checkpoint_weight_grad(kept, empty, grad_weight=dw, grad_bias=db)
    assert torch.all(dw == 0) and torch.all(db == 0)
    dy = torch.ones(5, 6, device="cuda")
    _, db = b.adasum_checkpoint_weight_grad(kept, dy, grad_weight=torch.empty(6, 0, device="cuda"), want_bias=True)
    assert torch.all(db == 5)


def test_gradient_is_the_adjoint(b):
    """Differences of y = x w^T in the direction v against the gradient: <x v^T, dy> = <v, dw>."""
    gen = _gen(14)
    x = torch.randn(300, 160, generator=gen, device="cuda")
    dy = torch.randn(300, 72, generator=gen, device="cuda")
    v = torch.randn(72, 160, generator=gen, device="cuda").double()
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    dw, _ = b.adasum_checkpoint_weight_grad(kept, dy, features=160)
    at = b.adasum_checkpoint_load(kept, 300, 160).double()
    left, right = (at @ v.t() * dy.double()).sum(), (v * dw.double()).sum()
    size = (at.abs() @ v.t().abs() * dy.double().abs()).sum()
    assert abs(left - right) <= 302 * 2.0**-23 * size


def test_other_stream_and_graph(b):
    gen = _gen(15)
    x, dy = _normal(gen, 400, 200, "bf16"), _normal(gen, 400, 120, "bf16")
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    want, want_b = b.adasum_checkpoint_weight_grad(kept, dy, features=200, want_bias=True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got, got_b = b.adasum_checkpoint_weight_grad(kept, dy, features=200, want_bias=True, stream=side)
    side.synchronize()
    assert torch.equal(got, want) and torch.equal(got_b, want_b)
    ws = torch.empty(b.adasum_checkpoint_weight_grad_workspace_bytes(400, 200, 120, "bf16"), dtype=torch.uint8, device="cuda")
    dw = torch.zeros(120, 200, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.adasum_checkpoint_weight_grad(kept, dy, grad_weight=dw, workspace=ws)
    ws.random_(0, 255)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(dw, want)


def test_status_and_refusals(b):
    x, dy = torch.ones(130, 64, device="cuda"), torch.ones(130, 24, device="cuda")
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    ws = torch.empty(b.adasum_checkpoint_weight_grad_workspace_bytes(130, 64, 24, "f32"), dtype=torch.uint8, device="cuda")
    b.adasum_checkpoint_weight_grad(kept, dy, features=64, workspace=ws)
    assert b.adasum_checkpoint_weight_grad_status(130, 64, 24, "f32", ws) == 0
    with pytest.raises(b.AdasumError, match="WORKSPACE"):
        b.adasum_checkpoint_weight_grad(kept, dy, features=64, workspace=ws[:1024])
    with pytest.raises(b.AdasumError, match="DTYPE"):
        b.adasum_checkpoint_weight_grad(kept, dy.double(), features=64)
    with pytest.raises(ValueError):
        b.adasum_checkpoint_weight_grad(kept, dy, features=256)                  # the checkpoint is too small
    with pytest.raises(ValueError):
        b.adasum_checkpoint_weight_grad(kept, dy, grad_weight=torch.empty(64, 24, device="cuda"))
    with pytest.raises(ValueError):
        b.adasum_checkpoint_weight_grad(kept, dy.t(), features=64)
    with pytest.raises(TypeError):
        b.adasum_checkpoint_weight_grad(kept.float(), dy, features=64)
    with pytest.raises(ValueError):
        b.adasum_checkpoint_weight_grad(kept, dy, features=64, accumulate=True)  # onto nothing


def test_large_offsets(b):
    """Codes beyond 2^32 bytes: only the last rows hold anything."""
    rows, features = (1 << 20) + 70, 4160
    kept = torch.zeros(b.adasum_checkpoint_bytes(rows, features), dtype=torch.uint8, device="cuda")
    kept[rows * features:] = 127                                                 # step 1
    kept[(rows - 3) * features:rows * features] = 5
    dy = torch.zeros(rows, 8, dtype=torch.bfloat16, device="cuda")
    dy[-2:] = 1.0
    dw, db = b.adasum_checkpoint_weight_grad(kept, dy, features=features, want_bias=True)
    assert torch.all(dw == 10.0) and torch.all(db == 2.0)
