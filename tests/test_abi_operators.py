"""Refusals and sizes of the calls that produce a worker's gradients, without a GPU: the pointers are made-up
device addresses, so every check below must fail before any CUDA call."""
import numpy as np
import pytest
import torch

F32, F16, BF16, F64 = 0, 1, 2, 3
A, B, C, W = 0x10000000, 0x20000000, 0x30000000, 0x40000000      # far apart, 256-byte aligned
BIG = 1 << 40


@pytest.fixture(scope="module")
def b():
    from paper_2006_02924_b200 import build

    build.build()
    from paper_2006_02924_b200 import binding

    return binding


def _status(b, code):
    return b.adasum_status_string(code)


def test_checkpoint_bytes(b):
    assert b.adasum_checkpoint_bytes(0, 40) == 0 and b.adasum_checkpoint_bytes(3, 0) == 0
    assert b.adasum_checkpoint_bytes(1, 1) == 33
    assert b.adasum_checkpoint_bytes(37, 1000) == 37 * 1024 + 37 * 32
    assert b.adasum_checkpoint_bytes(-1, 5) == 0 and b.adasum_checkpoint_bytes(5, 1 << 31) == 0
    for rows, features in ((1, 1), (5, 31), (5, 32), (5, 33), (7, 4096)):
        assert b._checkpoint_size(rows, features) == b.adasum_checkpoint_bytes(rows, features)


def test_workspace_bytes(b):
    ws = b.adasum_embedding_grad_workspace_bytes
    assert 0 < ws(0, 5, 8) <= ws(1, 5, 8) <= ws(1000, 5, 8) <= ws(1000, 5, 800)
    assert ws(1000, 5, 8) >= 2 * 1000 * 8                  # the sorted list and the sort's other half
    assert ws(-1, 5, 8) == ws(1, -5, 8) == ws(1, 5, (1 << 22) + 1) == 0
    wg = b.adasum_checkpoint_weight_grad_workspace_bytes
    assert 0 < wg(0, 8, 8, "bf16") <= wg(64, 8, 8, "bf16") <= wg(100000, 1024, 1024, "bf16")
    assert wg(5000, 8, 24, "f32") >= wg(5000, 8, 24, "f16") + 2 * 5000 * 24 * 2     # three planes instead of one
    assert wg(-1, 8, 8, "bf16") == wg(8, 8, 8, "f64") == wg(8, 1 << 31, 8, "bf16") == 0
    assert wg(1 << 30, 1 << 30, 1 << 30, "bf16") == 0      # more steps than the product can count


def test_embedding_forward_refusals(b):
    def call(table=A, stride=8, rows=10, dim=8, dtype=F32, tokens=B, width=8, n=4, out=C, out_stride=8, out_dtype=F32):
        return _status(b, b.raw().adasum_embedding_forward(table, stride, rows, dim, dtype, tokens, width, n, 1.0, out,
                                                           out_stride, out_dtype, None))

    assert call(dtype=F64) == call(out_dtype=F64) == call(dtype=9) == "ADASUM_ERR_DTYPE"
    assert call(table=None) == call(tokens=None) == call(out=None) == "ADASUM_ERR_NULL"
    assert call(n=-1) == call(rows=-1) == call(dim=-1) == call(dim=(1 << 22) + 1) == call(n=1 << 31) == "ADASUM_ERR_ARG"
    assert call(width=2) == call(tokens=B + 4) == call(table=A + 2) == call(out=C + 2) == "ADASUM_ERR_ARG"
    assert call(stride=7) == call(out_stride=7) == "ADASUM_ERR_ARG"
    assert "stride" in b.adasum_last_error()
    assert call(out=A + 32) == call(out=B) == "ADASUM_ERR_ARG"
    assert call(n=0) == call(dim=0) == "ADASUM_OK" and b.adasum_last_error() == ""
    assert call(n=0, tokens=None, out=None) == "ADASUM_OK"


def test_embedding_grad_refusals(b):
    def call(grad=A, stride=8, dtype=F32, tokens=B, width=8, n=4, table=C, rows=10, dim=8, out_dtype=F32, accumulate=0,
             ws=W, ws_bytes=BIG):
        return _status(b, b.raw().adasum_embedding_grad(grad, stride, dtype, tokens, width, n, 1.0, table, rows, dim,
                                                        out_dtype, accumulate, ws, ws_bytes, None))

    assert call(dtype=F64) == call(out_dtype=F64) == "ADASUM_ERR_DTYPE"
    assert call(grad=None) == call(tokens=None) == call(table=None) == "ADASUM_ERR_NULL"
    assert call(n=-1) == call(rows=1 << 31) == call(dim=-8) == call(width=1) == "ADASUM_ERR_ARG"
    assert call(grad=A + 1) == call(table=C + 2) == call(stride=3) == "ADASUM_ERR_ARG"
    assert call(ws=None) == call(ws_bytes=100) == "ADASUM_ERR_WORKSPACE"
    assert call(ws=W + 16) == "ADASUM_ERR_ARG"
    assert call(table=A) == call(table=B) == call(table=W) == call(ws=A) == call(ws=B) == "ADASUM_ERR_ARG"
    assert call(rows=0) == call(dim=0) == call(n=0, accumulate=1) == "ADASUM_OK"


def test_checkpoint_refusals(b):
    def save(x=A, stride=40, rows=3, features=40, dtype=BF16, act=2, y=B, y_stride=40, kept=C):
        return _status(b, b.raw().adasum_checkpoint_save(x, stride, rows, features, dtype, act, y, y_stride, kept, None))

    def load(kept=C, rows=3, features=40, out=A, stride=40, dtype=BF16):
        return _status(b, b.raw().adasum_checkpoint_load(kept, rows, features, out, stride, dtype, None))

    def grad(kept=C, rows=3, features=40, act=2, dy=A, stride=40, dtype=BF16, dx=B, dx_stride=40):
        return _status(b, b.raw().adasum_checkpoint_act_grad(kept, rows, features, act, dy, stride, dtype, dx, dx_stride,
                                                             None))

    assert save(dtype=F64) == load(dtype=F64) == grad(dtype=F64) == "ADASUM_ERR_DTYPE"
    assert save(act=5) == save(act=-1) == grad(act=7) == "ADASUM_ERR_ARG"
    assert save(x=None) == save(kept=None) == load(out=None) == load(kept=None) == "ADASUM_ERR_NULL"
    assert grad(dy=None) == grad(dx=None) == grad(kept=None) == "ADASUM_ERR_NULL"
    assert save(kept=C + 8) == load(kept=C + 4) == grad(kept=C + 1) == "ADASUM_ERR_ARG"
    assert save(stride=39) == save(y_stride=39) == load(stride=1) == grad(stride=39) == grad(dx_stride=0) == "ADASUM_ERR_ARG"
    assert save(x=A + 1) == load(out=A + 1) == grad(dx=B + 1) == "ADASUM_ERR_ARG"
    assert save(rows=-1) == load(features=-1) == grad(rows=1 << 31) == "ADASUM_ERR_ARG"
    assert save(y=A + 2) == save(y=A, y_stride=48) == save(kept=A) == save(kept=B) == "ADASUM_ERR_ARG"
    assert load(out=C) == grad(dx=A + 2) == grad(dx=C) == grad(dx=A, dx_stride=41) == "ADASUM_ERR_ARG"
    assert save(rows=0) == load(features=0) == grad(rows=0) == save(features=0, kept=None, x=None) == "ADASUM_OK"


def test_weight_grad_refusals(b):
    def call(kept=A, rows=50, features=40, dy=B, stride=24, outputs=24, dtype=BF16, dw=C, db=C + 0x100000, out_dtype=F32,
             accumulate=0, ws=W, ws_bytes=BIG):
        return _status(b, b.raw().adasum_checkpoint_weight_grad(kept, rows, features, dy, stride, outputs, dtype, 1.0, dw,
                                                                db, out_dtype, accumulate, ws, ws_bytes, None))

    assert call(dtype=F64) == call(out_dtype=F64) == call(dtype=-1) == "ADASUM_ERR_DTYPE"
    assert call(kept=None) == call(dy=None) == call(dw=None) == "ADASUM_ERR_NULL"
    assert call(rows=-1) == call(features=1 << 31) == call(outputs=-3) == "ADASUM_ERR_ARG"
    assert call(kept=A + 8) == call(dy=B + 1) == call(dw=C + 2) == call(db=C + 0x100002) == "ADASUM_ERR_ARG"
    assert call(stride=23) == "ADASUM_ERR_ARG"
    assert call(ws=None) == call(ws_bytes=1000) == "ADASUM_ERR_WORKSPACE"
    assert call(ws=W + 128) == "ADASUM_ERR_ARG"
    assert call(dw=A) == call(dw=B) == call(db=B) == call(db=C) == call(ws=A) == call(ws=C) == "ADASUM_ERR_ARG"
    assert call(outputs=0) == call(features=0, db=None) == call(rows=0, accumulate=1) == "ADASUM_OK"
    assert call(rows=1 << 30, features=1 << 30, outputs=1 << 30, stride=1 << 30, db=None) == "ADASUM_ERR_ARG"
    status = b.raw().adasum_checkpoint_weight_grad_status
    assert _status(b, status(50, 40, 24, BF16, None, None)) == "ADASUM_ERR_NULL"
    assert _status(b, status(50, 40, 24, F64, W, None)) == "ADASUM_ERR_DTYPE"
    assert _status(b, status(-50, 40, 24, BF16, W, None)) == "ADASUM_ERR_ARG"


def test_binding_refusals(b):
    """What the Python wrappers refuse before they call the library; no tensor here is on a GPU."""
    x = torch.zeros(4, 40)
    with pytest.raises(TypeError):
        b.adasum_checkpoint_save(x)
    with pytest.raises(TypeError):
        b.adasum_embedding_forward(x, torch.zeros(3, dtype=torch.int64))
    with pytest.raises(TypeError):
        b.adasum_embedding_grad(x, torch.zeros(4), 5)
    with pytest.raises(TypeError):
        b.adasum_checkpoint_load(torch.zeros(200, dtype=torch.uint8), 4, 40)
    with pytest.raises(TypeError):
        b.adasum_checkpoint_act_grad(torch.zeros(200, dtype=torch.uint8), x, "gelu")
    with pytest.raises(TypeError):
        b.adasum_checkpoint_weight_grad(torch.zeros(200, dtype=torch.uint8), x, features=40)
    with pytest.raises(TypeError):
        b._operator_dtype(torch.int32)


def _runs(begin, end, chains):
    """The order in which a pair of blocks walks its units (a model of the kernel's cursor): the beginning of a cut-off
    last tile, the end of a cut-off first one (or a run inside one tile), then whole tiles."""
    inside = end // chains == begin // chains
    first_whole = end if inside else -(-begin // chains) * chains
    parts = [(max(begin, end // chains * chains), end) if not inside else (end, end),
             (begin, min(end, first_whole))]
    whole = min(end, first_whole)
    parts.append((whole, max(whole, end // chains * chains)))
    return parts


def test_units_of_the_weight_gradient_are_covered_once():
    """Every unit of every tile belongs to exactly one pair, and a pair has at most one cut-off share that is not its
    first tile's (what the two partial-sum slots per pair rely on)."""
    rng = np.random.default_rng(3)
    for _ in range(500):
        chains, tiles = int(rng.integers(1, 12)), int(rng.integers(1, 30))
        units = chains * tiles
        pairs = int(rng.integers(1, min(units, 74) + 1))
        seen = []
        for p in range(pairs):
            begin, end = p * units // pairs, (p + 1) * units // pairs
            for part, (lo, hi) in enumerate(_runs(begin, end, chains)):
                seen += range(lo, hi)
                if part == 2 and lo < hi:
                    assert lo % chains == 0 and hi % chains == 0
                if part == 0 and lo < hi:
                    assert lo % chains == 0 and lo // chains != begin // chains
                if part == 1 and lo < hi:
                    assert (hi - 1) // chains == lo // chains == begin // chains
            for u in range(begin, end):
                assert ((u + 1) * pairs - 1) // units == p          # the join's inverse of the split
        assert sorted(seen) == list(range(units))


def test_a_workspace_for_a_long_list_does_for_a_shorter_one():
    """The last batch of an epoch uses the workspace of the others: sizes never fall as a count rises."""
    from paper_2006_02924_b200 import binding as b

    for dim in (1, 203, 1024):
        sizes = [b.adasum_embedding_grad_workspace_bytes(n, 5, dim) for n in range(5000)]
        assert all(x <= y for x, y in zip(sizes, sizes[1:])), dim
        more = [b.adasum_embedding_grad_workspace_bytes(n, 5, dim) for n in (4999, 6144, 6145, 8192, 100000, 1 << 30)]
        assert sizes[-1] <= more[0] and all(x <= y for x, y in zip(more, more[1:]))
    for dtype in ("f32", "f16", "bf16"):
        for features, outputs in ((1, 1), (1000, 257), (4096, 1024)):
            sizes = [b.adasum_checkpoint_weight_grad_workspace_bytes(n, features, outputs, dtype) for n in range(0, 6000, 7)]
            assert all(x <= y for x, y in zip(sizes, sizes[1:]))


def test_weight_grad_selftest_refusals(b):
    def call(hand_over, kept=A, ws=W):
        return _status(b, b.raw().adasum_checkpoint_weight_grad_selftest(kept, 50, 40, B, 24, 24, BF16, 1.0, C, C + 0x100000,
                                                                         F32, 0, ws, BIG, None, hand_over))

    assert call(0) == call(7) == call(-1) == "ADASUM_ERR_ARG" and "hand-over" in b.adasum_last_error()
    assert call(1, kept=None) == "ADASUM_ERR_NULL"
    assert call(6, ws=None) == "ADASUM_ERR_WORKSPACE"


def test_every_call_is_reached_through_the_package(b):
    import paper_2006_02924_b200 as package

    calls = [name for name in dir(b) if name.startswith("adasum_") and callable(getattr(b, name))]
    assert "adasum_checkpoint_weight_grad_status" in calls and len(calls) > 25
    for name in calls:
        assert getattr(package, name) is getattr(b, name)
