"""Refusals and sizes of the calls around a residual block's linear layers, without a GPU: the pointers are made-up device
addresses, so every check below must fail before any CUDA call."""
import numpy as np
import pytest
import torch

import residual_reference as ref

F32, F16, BF16, F64 = 0, 1, 2, 3
A, B, C, D, W = 0x10000000, 0x20000000, 0x30000000, 0x50000000, 0x40000000      # far apart, 256-byte aligned
BIG = 1 << 40


@pytest.fixture(scope="module")
def b():
    from paper_2006_02924_b200 import build

    build.build()
    from paper_2006_02924_b200 import binding

    return binding


def test_the_reference_generator_gives_the_published_answers():
    ones = 0xffffffff
    assert ref.philox((ones, ones), (ones,) * 4) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    keep, factor = ref.kept(5, 20, 0.5, (7 << 32) + 5, 3)
    words = ref.philox((5, 7), (4 * 3 + 2, 0, 3, 0))
    assert factor == 2.0 and keep[4, 17] == ((words[0] >> 16) >= 32768)


def test_dropout_refusals(b):
    def call(x=A, stride=40, rows=3, features=40, dtype=BF16, r=B, r_stride=40, p=0.5, seed=D, out=C, out_stride=40):
        return b.adasum_status_string(b.raw().adasum_dropout(x, stride, rows, features, dtype, r, r_stride, p, seed, 7, out,
                                                             out_stride, None))

    assert call(dtype=F64) == call(dtype=-1) == "ADASUM_ERR_DTYPE"
    assert call(x=None) == call(out=None) == call(seed=None) == "ADASUM_ERR_NULL"
    assert call(p=-0.1) == call(p=1.1) == call(p=float("nan")) == call(seed=D + 4) == "ADASUM_ERR_ARG"
    assert call(rows=-1) == call(features=1 << 31) == call(stride=39) == call(r_stride=2) == call(out_stride=0) == "ADASUM_ERR_ARG"
    assert call(x=A + 1) == call(r=B + 1) == call(out=C + 1) == "ADASUM_ERR_ARG"
    assert call(out=A + 16) == call(out=B + 16) == call(out=A, out_stride=48) == call(out=D) == "ADASUM_ERR_ARG"
    assert call(rows=0) == call(features=0) == call(rows=0, x=None, out=None) == "ADASUM_OK"
    assert b.adasum_last_error() == ""


def _block(b, rows=6, features=40, dtype=BF16, stream=BF16, param=F32, gate_dtype=BF16, post=1, pre=2, post_w=None, post_b=None,
           pre_w=None, pre_b=None, gate=None, gate_stride=40, per_gate=2, eps=1e-5, p=0.0, seed=None):
    return b._RESIDUAL_NORM.pack(rows, features, dtype, stream, param, gate_dtype, post, pre, post_w or 0, post_b or 0, pre_w or 0,
                                 pre_b or 0, gate or 0, gate_stride, per_gate, eps, 1.0, 1.0, p, 0, seed or 0)


P = 0x60000000          # vectors: P + k * 0x10000


def test_residual_norm_refusals(b):
    def call(x=A, x_stride=40, r=B, r_stride=40, h=C, h_stride=40, y=D, y_stride=40, stats=W, **block):
        return b.adasum_status_string(b.raw().adasum_residual_norm(_block(b, **block), x, x_stride, r, r_stride, h, h_stride, y,
                                                                   y_stride, stats, None))

    assert b.adasum_status_string(b.raw().adasum_residual_norm(None, A, 40, B, 40, C, 40, D, 40, W, None)) == "ADASUM_ERR_NULL"
    assert call(dtype=F64) == call(stream=F64) == call(param=F64) == call(gate_dtype=9) == call(stream=F16) == "ADASUM_ERR_DTYPE"
    assert call(post=3) == call(pre=-1) == call(eps=-1.0) == call(eps=float("nan")) == "ADASUM_ERR_ARG"
    assert call(rows=-1) == call(features=-8) == call(features=32769) == "ADASUM_ERR_ARG"
    assert call(x=None, r=None) == call(h=None, pre=0) == call(y=None) == call(p=0.5) == "ADASUM_ERR_NULL"
    assert call(x_stride=39) == call(r_stride=39) == call(h_stride=39) == call(y_stride=39) == call(stats=W + 2) == "ADASUM_ERR_ARG"
    assert call(x=A + 1) == call(r=B + 1) == call(h=C + 1) == call(y=D + 1) == call(pre_w=P + 2) == "ADASUM_ERR_ARG"
    assert call(gate=P, per_gate=0) == call(gate=P + 1) == call(gate=P, gate_stride=39) == "ADASUM_ERR_ARG"
    assert call(h=A) == call(y=B) == call(h=D) == call(stats=A) == call(h=B + 80) == call(y=A + 80) == "ADASUM_ERR_ARG"
    assert call(h=B, h_stride=48) == call(y=A, y_stride=48) == call(pre_w=C) == call(gate=D) == call(p=0.5, seed=W) == "ADASUM_ERR_ARG"
    assert call(rows=0) == call(features=0) == call(rows=0, x=None, r=None) == "ADASUM_OK"


def test_residual_norm_grad_refusals(b):
    E, F, G = 0x70000000, 0x80000000, 0x90000000

    def call(x=A, h=B, dy=C, dh=D, stats=E, dx=F, dr=G, strides=(40,) * 6, post_g=P, post_gb=None, pre_g=None, pre_gb=None, gate_g=None,
             dtype=F32, gate_dtype=F32, accumulate=0, ws=W, ws_bytes=BIG, **block):
        s = strides
        grads = b._RESIDUAL_NORM_GRADS.pack(x or 0, h or 0, dy or 0, dh or 0, stats or 0, s[0], s[1], s[2], s[3], dx or 0, dr or 0, s[4], s[5],
                                            post_g or 0, post_gb or 0, pre_g or 0, pre_gb or 0, gate_g or 0, dtype, gate_dtype, 1.0, 1.0,
                                            accumulate)
        return b.adasum_status_string(b.raw().adasum_residual_norm_grad(_block(b, **block), grads, ws, ws_bytes, None))

    assert b.adasum_status_string(b.raw().adasum_residual_norm_grad(_block(b), None, W, BIG, None)) == "ADASUM_ERR_NULL"
    assert call(dtype=F64) == call(gate_dtype=F64) == "ADASUM_ERR_DTYPE"
    assert call(dy=None, dh=None) == call(x=None) == call(h=None) == call(stats=None) == "ADASUM_ERR_NULL"
    assert call(x=None, dx=None) == call(x=None, post=0, post_g=None, gate=P + 0x10000, gate_g=P) == "ADASUM_ERR_NULL"
    assert call(gate_g=P + 0x10000) == call(post=0) == call(pre=0, dy=None, pre_g=P + 0x10000) == call(pre=0) == "ADASUM_ERR_ARG"
    for i in range(6):
        assert call(strides=tuple(39 if i == k else 40 for k in range(6))) == "ADASUM_ERR_ARG"
    assert call(x=A + 1) == call(dx=F + 1) == call(post_g=P + 2) == call(stats=E + 1) == "ADASUM_ERR_ARG"
    assert call(ws=None) == call(ws_bytes=1000) == "ADASUM_ERR_WORKSPACE"
    assert call(ws=W + 16) == call(ws=A) == call(ws=P) == call(dx=G) == call(dx=A) == call(dr=B) == call(dx=C + 16) == "ADASUM_ERR_ARG"
    assert call(dr=C) == call(dx=D) == call(dx=C, strides=(40, 40, 40, 40, 48, 40)) == call(pre_g=P) == call(post_g=F) == "ADASUM_ERR_ARG"
    assert call(features=0) == call(rows=0, accumulate=1) == "ADASUM_OK"


def test_residual_norm_workspace(b):
    ws = b.adasum_residual_norm_grad_workspace_bytes
    assert 0 < ws(1) <= ws(8) <= ws(1024) < ws(1024, gate=True) < 16 << 20
    assert ws(1000) == ws(1000) and ws(32769) == ws(-1) == 0
    # the sums of 296 blocks, five vectors each
    assert ws(4096) >= 296 * 5 * 4096 * 4


def test_fp8_refusals(b):
    def pack(x=A, stride=40, rows=3, columns=40, dtype=BF16, out=C, weight=False):
        f = b.raw().adasum_fp8_pack_weight if weight else b.raw().adasum_fp8_pack
        return b.adasum_status_string(f(x, stride, rows, columns, dtype, out, None))

    def unpack(packed=C, rows=3, columns=40, out=A, stride=40, dtype=BF16):
        return b.adasum_status_string(b.raw().adasum_fp8_unpack(packed, rows, columns, out, stride, dtype, None))

    for weight in (False, True):
        assert pack(dtype=F64, weight=weight) == "ADASUM_ERR_DTYPE"
        assert pack(x=None, weight=weight) == pack(out=None, weight=weight) == "ADASUM_ERR_NULL"
        assert pack(rows=-1, weight=weight) == pack(columns=1 << 31, weight=weight) == pack(stride=39, weight=weight) == "ADASUM_ERR_ARG"
        assert pack(out=C + 8, weight=weight) == pack(x=A + 1, weight=weight) == pack(out=A, weight=weight) == "ADASUM_ERR_ARG"
        assert pack(rows=0, weight=weight) == pack(columns=0, weight=weight) == "ADASUM_OK"
    assert unpack(dtype=F64) == "ADASUM_ERR_DTYPE" and unpack(packed=None) == unpack(out=None) == "ADASUM_ERR_NULL"
    assert unpack(packed=C + 4) == unpack(stride=39) == unpack(out=C) == unpack(rows=1 << 31) == "ADASUM_ERR_ARG"
    assert unpack(rows=0) == unpack(columns=0) == "ADASUM_OK"
    for rows, columns in ((1, 1), (128, 128), (129, 129), (0, 5), (5, 0), (300, 1000)):
        assert b.adasum_fp8_bytes(rows, columns) == b._fp8_size(rows, columns)
    assert b.adasum_fp8_bytes(300, 1000) == 300 * 1024 + 3 * 8 * 512 and b.adasum_fp8_bytes(-1, 5) == 0


def test_fp8_linear_refusals(b):
    def call(x=A, w=B, rows=50, features=40, outputs=24, bias=P, bias_dtype=F32, y=C, stride=None, dtype=BF16, ws=W, ws_bytes=BIG, grad=False):
        stride = stride if stride is not None else (features if grad else outputs)
        if grad:
            code = b.raw().adasum_fp8_linear_grad(x, w, rows, features, outputs, y, stride, dtype, ws, ws_bytes, None)
        else:
            code = b.raw().adasum_fp8_linear(x, w, rows, features, outputs, bias, bias_dtype, y, stride, dtype, ws, ws_bytes, None)
        return b.adasum_status_string(code)

    for grad in (False, True):
        assert call(dtype=F64, grad=grad) == "ADASUM_ERR_DTYPE"
        assert call(x=None, grad=grad) == call(w=None, grad=grad) == call(y=None, grad=grad) == "ADASUM_ERR_NULL"
        assert call(rows=-1, grad=grad) == call(features=1 << 31, grad=grad) == call(outputs=-3, grad=grad) == "ADASUM_ERR_ARG"
        assert call(x=A + 8, grad=grad) == call(w=B + 4, grad=grad) == call(y=C + 1, grad=grad) == call(stride=23, grad=grad) == "ADASUM_ERR_ARG"
        assert call(ws=None, grad=grad) == call(ws_bytes=1000, grad=grad) == "ADASUM_ERR_WORKSPACE"
        assert call(ws=W + 128, grad=grad) == call(y=A, grad=grad) == call(y=B, grad=grad) == call(y=W, grad=grad) == call(ws=A, grad=grad) == "ADASUM_ERR_ARG"
        assert call(rows=0, grad=grad) == "ADASUM_OK"
        assert call(rows=1 << 30, features=1 << 30, outputs=1 << 30, bias=None, grad=grad) == "ADASUM_ERR_ARG"
    assert call(outputs=0, stride=0) == call(features=0, grad=True, stride=0) == "ADASUM_OK"
    assert call(bias_dtype=F64) == "ADASUM_ERR_DTYPE" and call(bias=P + 2) == call(bias=C) == call(bias=W) == "ADASUM_ERR_ARG"
    ws = b.adasum_fp8_linear_workspace_bytes
    assert ws(-1, 8, 8) == ws(8, 1 << 31, 8) == 0 and ws(0, 8, 8) > 0
    for features, outputs in ((1, 1), (1000, 257), (4096, 1024)):
        sizes = [ws(n, features, outputs) for n in range(0, 3000, 7)]
        assert all(x <= y for x, y in zip(sizes, sizes[1:]))
    test = b.raw().adasum_fp8_linear_selftest
    for hand_over in (0, 3, 4, 7):
        assert b.adasum_status_string(test(A, B, 50, 40, 24, C, 24, BF16, W, BIG, None, hand_over)) == "ADASUM_ERR_ARG"
    assert b.adasum_status_string(test(None, B, 50, 40, 24, C, 24, BF16, W, BIG, None, 1)) == "ADASUM_ERR_NULL"
    assert b.adasum_status_string(b.raw().adasum_fp8_linear_status(None, None)) == "ADASUM_ERR_NULL"


def test_binding_refusals(b):
    """What the Python wrappers refuse before they call the library; no tensor here is on a GPU."""
    x, packed = torch.zeros(4, 40), torch.zeros(4000, dtype=torch.uint8)
    with pytest.raises(TypeError):
        b.adasum_dropout(x, 0.5, torch.zeros(1, dtype=torch.int64))
    with pytest.raises(TypeError):
        b.adasum_residual_norm(x, x)
    with pytest.raises(ValueError):
        b.adasum_residual_norm(None, None)
    with pytest.raises(TypeError):
        b.adasum_residual_norm_grad(x, x, torch.zeros(4, 4), x, x)
    with pytest.raises(ValueError):
        b.adasum_residual_norm_grad(x, x, torch.zeros(4, 4), None, None)
    for f in (b.adasum_fp8_pack, b.adasum_fp8_pack_weight):
        with pytest.raises(TypeError):
            f(x)
    with pytest.raises(TypeError):
        b.adasum_fp8_unpack(packed, 4, 40)
    with pytest.raises(TypeError):
        b.adasum_fp8_linear(packed, packed, 4, 40, 24)
    with pytest.raises(TypeError):
        b.adasum_fp8_linear_grad(packed, packed, 4, 40, 24)


def test_reference_rounding_to_eight_bits():
    """The tests' own e4m3: every code is a fixed point, ties go to even, the largest magnitude decides the step."""
    one = np.full((1, 1), 127, np.uint8)
    values = np.array([ref.fp8_values(np.full((1, 128), c, np.uint8), one, 1)[0, 0] for c in range(127)])
    assert values[1] == 2.0**-9 and values[8] == 2.0**-6 and values[126] == 448 and np.all(np.diff(values) > 0)
    x = np.stack((values, np.full(127, 448.0)), axis=1)
    codes, steps = ref.fp8_pack(x)
    assert np.array_equal(codes[:, 0], np.arange(127)) and np.all(steps == 127)
    codes, _ = ref.fp8_pack(np.stack(((values[1:] + values[:-1]) / 2, np.full(126, 448.0)), axis=1))
    assert np.all(codes[:, 0] % 2 == 0)


@pytest.mark.parametrize("per_gate", [7, 1 << 31, (1 << 63) - 6, (1 << 63) - 1])
def test_a_gate_for_more_rows_than_there_are(b, per_gate):
    """A gate whose row serves any number of rows is one row: it and its gradient are checked for overlaps as such."""
    gate = dict(gate=P, per_gate=per_gate)
    forward = b.raw().adasum_residual_norm
    for h in (P, P - 80, P + 79 - 79 % 16):
        code = forward(_block(b, **gate), A, 40, B, 40, h, 40, D, 40, W, None)
        assert b.adasum_status_string(code) == "ADASUM_ERR_ARG"
    E, F, G = 0x70000000, 0x80000000, 0x90000000
    for into in (F, G, A, W, P):
        grads = b._RESIDUAL_NORM_GRADS.pack(A, B, C, D, E, 40, 40, 40, 40, F, G, 40, 40, 0, 0, 0, 0, into, F32, F32, 1.0, 1.0, 0)
        code = b.raw().adasum_residual_norm_grad(_block(b, **gate), grads, W, BIG, None)
        assert b.adasum_status_string(code) == "ADASUM_ERR_ARG"


class _OnDevice:
    """Stands in for a contiguous tensor of a GPU that this machine need not have."""
    is_cuda = True

    def __init__(self, device, shape, dtype=torch.float32):
        self.device, self.shape, self.dtype = torch.device("cuda", device), torch.Size(shape), dtype

    def get_device(self):
        return self.device.index

    def dim(self):
        return len(self.shape)

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return self.dtype.itemsize

    def stride(self):
        return tuple(torch.Size(self.shape[i + 1:]).numel() for i in range(len(self.shape)))

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return 0x10000000


@pytest.fixture
def current(monkeypatch):
    """The current device as torch.cuda.device makes it, without a GPU; the handle of its current stream tells it."""
    now = [0]

    class Guard:
        def __init__(self, device):
            self.index = device.index if isinstance(device, torch.device) else device

        def __enter__(self):
            self.before, now[0] = now[0], self.index

        def __exit__(self, *_):
            now[0] = self.before

    monkeypatch.setattr(torch.cuda, "device", Guard)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *_: type("Stream", (), {"cuda_stream": 1000 + now[0]}))
    return now


def test_status_and_self_test_calls_run_on_their_tensors_device(b, monkeypatch, current):
    """With GPU 0 current and everything on GPU 1, the library is called with GPU 1 current, on its current stream."""
    seen = []

    def library(*args):
        seen.append((current[0], [a for a in args if a in (1000, 1001)]))
        return 0

    for name in ("adasum_device_status", "adasum_checkpoint_weight_grad_status", "adasum_checkpoint_weight_grad_selftest",
                 "adasum_fp8_linear_status", "adasum_fp8_linear_selftest"):
        monkeypatch.setattr(b._lib, name, library)
    ws, u8 = _OnDevice(1, (1 << 20,), torch.uint8), torch.uint8
    assert b.adasum_device_status(100, 1, 2, "f32", ws) == 0
    assert b.adasum_checkpoint_weight_grad_status(4, 40, 24, "f32", ws) == 0
    b.adasum_checkpoint_weight_grad_selftest("landed", _OnDevice(1, (4 * 66,), u8), _OnDevice(1, (4, 24)), _OnDevice(1, (24, 40)), None, ws)
    assert b.adasum_fp8_linear_status(ws) == 0
    x8, w8 = _OnDevice(1, (b._fp8_size(4, 40),), u8), _OnDevice(1, (b._fp8_size(24, 40),), u8)
    b.adasum_fp8_linear_selftest("landed", x8, w8, 4, 40, 24, _OnDevice(1, (4, 24)), ws)
    assert seen == [(1, [1001])] * 5 and current[0] == 0
    with pytest.raises(ValueError):
        b.adasum_fp8_linear_selftest("landed", x8, w8, 4, 40, 24, _OnDevice(1, (4, 24)), _OnDevice(0, (1 << 20,), u8))
    with pytest.raises(ValueError):
        b.adasum_checkpoint_weight_grad_selftest("landed", _OnDevice(1, (4 * 66,), u8), _OnDevice(1, (4, 24)), _OnDevice(0, (24, 40)), None, ws)


def test_status_of_what_is_no_workspace(b, monkeypatch, current):
    """The library reads the words of all blocks: a buffer that has no room for them is refused."""
    monkeypatch.setattr(b._lib, "adasum_fp8_linear_status", lambda *_: 0)
    smallest = b.adasum_fp8_linear_workspace_bytes(1, 0, 1)
    assert b.adasum_fp8_linear_status(_OnDevice(1, (smallest,), torch.uint8)) == 0
    assert b.adasum_fp8_linear_status(_OnDevice(1, (smallest // 4,), torch.int32)) == 0
    for size in (0, 256, smallest - 1):
        with pytest.raises(ValueError):
            b.adasum_fp8_linear_status(_OnDevice(1, (size,), torch.uint8))
