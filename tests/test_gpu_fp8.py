"""Packed 8-bit matrices and their products against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import residual_reference as ref
from operator_reference import TINY, TORCH, UNIT, assert_close, to64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2006_02924_b200 import binding

    return binding


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _matrix(gen, rows, cols, dtype, pad=0, shift=0, size=1.0):
    flat = torch.randn(rows * (cols + pad) + shift, generator=gen, device="cuda") * size
    return flat.to(TORCH[dtype])[shift:].view(rows, cols + pad)[:, :cols]


def _codes_and_steps(packed, rows, cols):
    wide, up = -(-cols // 128), -(-rows // 128)
    p = packed.cpu().numpy()
    steps = p[rows * wide * 128:].reshape(up, wide, 32, 4, 4)
    return p[:rows * wide * 128].reshape(rows, wide * 128), steps


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,shift", [(1, 1, 0, 0), (1, 128, 0, 0), (3, 129, 2, 1), (37, 1000, 0, 0), (130, 257, 7, 0),
                                                 (257, 384, 0, 0), (128, 72, 8, 0), (1000, 40, 0, 1)])
def test_pack(b, dtype, rows, cols, pad, shift):
    gen = _gen(1)
    x = _matrix(gen, rows, cols, dtype, pad, shift)
    if dtype != "f16":       # the whole range, subnormals included
        x = x * torch.exp2(torch.randint(-140, 120, (rows, 1), generator=gen, device="cuda").double()).to(x.dtype)
    if rows > 2:
        x[1] = 0
        x[2, 0] = 448.0 * 2.0**-3 if cols > 1 else 1.0
    for weight, pack in ((False, b.adasum_fp8_pack), (True, b.adasum_fp8_pack_weight)):
        codes, steps = ref.fp8_pack(to64(x), weight)
        size = b.adasum_fp8_bytes(rows, cols)
        spare = torch.full((size + 64,), 0x5a, dtype=torch.uint8, device="cuda")
        packed = pack(x, packed=spare[:size])
        assert (spare[size:] == 0x5a).all()
        got, got_steps = _codes_and_steps(packed, rows, cols)
        assert np.array_equal(got, codes)
        want = ref.fp8_buffer(codes, steps)[codes.size:].reshape(got_steps.shape)
        row = np.arange(got_steps.shape[0])[:, None, None] * 128 + np.arange(32)[:, None] + 32 * np.arange(4)
        inside = np.broadcast_to((row < rows)[:, None, :, :, None], got_steps.shape)
        assert np.array_equal(got_steps[inside], want[inside])
        if weight:
            assert (got_steps == got_steps[:, :, :1, :1, :1]).all()
        values = ref.fp8_values(codes, steps, cols)
        assert np.array_equal(to64(b.adasum_fp8_unpack(packed, rows, cols)), values)
        for out_type in ("f16", "bf16"):
            out = torch.full((rows, cols + 3), 9.0, dtype=TORCH[out_type], device="cuda")
            b.adasum_fp8_unpack(packed, rows, cols, out=out[:, :cols])
            assert torch.equal(out[:, :cols], torch.from_numpy(values).cuda().to(torch.float32).to(TORCH[out_type])) and (out[:, cols:] == 9.0).all()


def test_every_code_and_tie(b):
    """All magnitudes between neighbouring codes' midpoints, midpoints themselves to even, steps at their borders."""
    one = np.full((1, 1), 127, np.uint8)
    values = np.array([ref.fp8_values(np.full((1, 128), c, np.uint8), one, 1)[0, 0] for c in range(127)])
    mid = (values[1:] + values[:-1]) / 2
    x = np.zeros((4 * 126, 8))
    x[:, 0] = np.concatenate((mid, np.nextafter(mid, 0), np.nextafter(mid, 1e9), -mid)).astype(np.float32)
    x[:, 1] = 448.0                                          # step 1
    got = to64(b.adasum_fp8_unpack(b.adasum_fp8_pack(torch.from_numpy(x).float().cuda()), x.shape[0], 8))
    want = ref.fp8_values(*ref.fp8_pack(x.astype(np.float32).astype(np.float64)), 8)
    assert np.array_equal(got, want)
    top = torch.tensor([[448.0], [np.nextafter(np.float32(448), np.float32(449))], [3.4e38], [1e-45], [2.0**-126 * 448]], device="cuda")
    _, steps = _codes_and_steps(b.adasum_fp8_pack(top), 5, 1)
    # 448 * 2^119 = 2.98e38 is below 3.4e38, so its step is 2^120
    assert [int(steps[0, 0, r, 0, 0]) for r in range(5)] == [127, 128, 127 + 120, 1, 1]


def test_blocks_that_are_not_numbers(b):
    for dtype in TORCH.values():
        x = torch.ones(140, 300, device="cuda", dtype=dtype)
        x[3, 130], x[139, 299] = float("nan"), float("-inf")
        v = b.adasum_fp8_unpack(b.adasum_fp8_pack(x), 140, 300)
        bad = torch.zeros(140, 300, dtype=torch.bool, device="cuda")
        bad[3, 128:256] = bad[139, 256:] = True
        assert torch.equal(torch.isnan(v), bad) and (v[~bad] == 1).all()
        v = b.adasum_fp8_unpack(b.adasum_fp8_pack_weight(x), 140, 300)
        bad[:128, 128:256] = bad[128:, 256:] = True
        assert torch.equal(torch.isnan(v), bad) and (v[~bad] == 1).all()
        # in products: the rows (columns) whose sums meet such a block
        w = torch.randn(96, 300, device="cuda").to(dtype)
        y = b.adasum_fp8_linear(b.adasum_fp8_pack(x), b.adasum_fp8_pack_weight(w), 140, 300, 96)
        assert torch.isnan(y).all(1).nonzero().flatten().tolist() == [3, 139] and torch.isnan(y).sum() == 2 * 96
        y = b.adasum_fp8_linear(b.adasum_fp8_pack(w), b.adasum_fp8_pack_weight(x), 96, 300, 140)
        assert torch.isnan(y).all(0).all()                   # both row blocks of the weight hold one
        dx = b.adasum_fp8_linear_grad(b.adasum_fp8_pack(w[:, :140].contiguous()), b.adasum_fp8_pack_weight(x), 96, 300, 140)
        assert torch.isnan(dx).any(0).nonzero().flatten().tolist() == list(range(128, 300))


SHAPES = [  # rows, features, outputs
    (1, 1, 1), (1, 1024, 4096), (2, 130, 7), (37, 1024, 4096), (64, 128, 256), (65, 129, 257), (128, 1000, 300), (129, 260, 120),
    (192, 256, 256), (193, 384, 512), (240, 256, 256), (384, 640, 256), (576, 300, 300), (333, 1000, 257), (480, 2048, 130), (700, 64, 1030), (1000, 5000, 200), (300, 40, 9000),
    (17, 16500, 33), (2049, 1024, 1024), (5, 8200, 8200)]


def _product(a, w):
    """The product and what truncating additions of all its terms may be off, in 64 bits on the GPU."""
    a, w = (torch.from_numpy(v).cuda() for v in (a, w))
    return to64(a @ w), to64((a.abs() @ w.abs()) * ((a.shape[1] + 2) * 2.0**-23))


@pytest.mark.parametrize("rows,features,outputs", SHAPES)
@pytest.mark.parametrize("out_type", ["f32", "f16", "bf16"])
def test_linear(b, rows, features, outputs, out_type):
    gen = _gen(2)
    x, w = _matrix(gen, rows, features, "bf16"), _matrix(gen, outputs, features, "f32", size=features**-0.5)
    # rows and blocks of very different sizes, so that a step byte in the wrong place shows
    x = x * torch.exp2(torch.randint(-2, 3, (rows, -(-features // 128)), generator=gen, device="cuda")).repeat_interleave(128, 1)[:, :features].bfloat16()
    w = w * torch.exp2(torch.randint(-2, 3, (-(-outputs // 128), -(-features // 128)), generator=gen, device="cuda").float()
                       ).repeat_interleave(128, 0)[:outputs].repeat_interleave(128, 1)[:, :features]
    bias = torch.randn(outputs, generator=gen, device="cuda").to(TORCH[out_type])
    px, pw = b.adasum_fp8_pack(x.contiguous()), b.adasum_fp8_pack_weight(w.contiguous())
    vx, vw = ref.fp8_values(*ref.fp8_pack(to64(x)), features), ref.fp8_values(*ref.fp8_pack(to64(w), True), features)
    want, err = _product(vx, vw.T.copy())
    u = UNIT[out_type] * 1.001
    spare = torch.full((rows + 2, outputs + 5), 3.0, dtype=TORCH[out_type], device="cuda")
    y = spare[1:1 + rows, 2:2 + outputs]
    ws = torch.empty(b.adasum_fp8_linear_workspace_bytes(rows, features, outputs), dtype=torch.uint8, device="cuda")
    b.adasum_fp8_linear(px, pw, rows, features, outputs, bias=bias, out=y, workspace=ws)
    assert b.adasum_fp8_linear_status(ws) == 0
    full = want + to64(bias)
    assert_close(to64(y), full, err + (u + 2.0**-24) * (np.abs(full) + err) + TINY[out_type], "y")
    outside = torch.ones_like(spare, dtype=torch.bool)
    outside[1:1 + rows, 2:2 + outputs] = False
    assert (spare[outside] == 3.0).all(), "written outside"
    plain = b.adasum_fp8_linear(px, pw, rows, features, outputs, out_dtype=TORCH[out_type])
    assert_close(to64(plain), want, err + u * (np.abs(want) + err) + TINY[out_type], "y without bias")
    # normwise: 32 truncated additions build a sum before it is rounded into fp32, each off by up to 2^-23 of it
    assert np.linalg.norm(to64(plain) - want) <= (4e-6 + u) * np.linalg.norm(want) + TINY[out_type] * np.sqrt(want.size)
    assert torch.equal(plain, b.adasum_fp8_linear(px, pw, rows, features, outputs, out_dtype=TORCH[out_type]))


@pytest.mark.parametrize("rows,features,outputs", SHAPES)
@pytest.mark.parametrize("out_type", ["f32", "f16", "bf16"])
def test_linear_grad(b, rows, features, outputs, out_type):
    gen = _gen(3)
    dy, w = _matrix(gen, rows, outputs, "bf16"), _matrix(gen, outputs, features, "f32", size=outputs**-0.5)
    dy = dy * torch.exp2(torch.randint(-2, 3, (rows, -(-outputs // 128)), generator=gen, device="cuda")).repeat_interleave(128, 1)[:, :outputs].bfloat16()
    w = w * torch.exp2(torch.randint(-2, 3, (-(-outputs // 128), -(-features // 128)), generator=gen, device="cuda").float()
                       ).repeat_interleave(128, 0)[:outputs].repeat_interleave(128, 1)[:, :features]
    pdy, pw = b.adasum_fp8_pack(dy.contiguous()), b.adasum_fp8_pack_weight(w.contiguous())
    vdy, vw = ref.fp8_values(*ref.fp8_pack(to64(dy)), outputs), ref.fp8_values(*ref.fp8_pack(to64(w), True), features)
    want, err = _product(vdy, vw)
    u = UNIT[out_type] * 1.001
    spare = torch.full((rows + 2, features + 5), 3.0, dtype=TORCH[out_type], device="cuda")
    dx = spare[1:1 + rows, 1:1 + features]
    b.adasum_fp8_linear_grad(pdy, pw, rows, features, outputs, out=dx)
    assert_close(to64(dx), want, err + u * (np.abs(want) + err) + TINY[out_type], "dx")
    outside = torch.ones_like(spare, dtype=torch.bool)
    outside[1:1 + rows, 1:1 + features] = False
    assert (spare[outside] == 3.0).all(), "written outside"
    again = b.adasum_fp8_linear_grad(pdy, pw, rows, features, outputs, out_dtype=TORCH[out_type])
    assert torch.equal(again, dx)
    assert np.linalg.norm(to64(dx) - want) <= (4e-6 + u) * np.linalg.norm(want) + TINY[out_type] * np.sqrt(want.size)


def test_products_are_exact(b):
    """Small whole numbers: every product and sum is a whole number below 2^24, exact in any order."""
    gen = _gen(4)
    x = torch.randint(-15, 16, (600, 700), generator=gen, device="cuda").float()
    w = torch.randint(-15, 16, (400, 700), generator=gen, device="cuda").float()
    x[:, ::128], w[:, ::128] = 448.0, 448.0                  # steps of 1
    px, pw = b.adasum_fp8_pack(x), b.adasum_fp8_pack_weight(w)
    assert torch.equal(b.adasum_fp8_linear(px, pw, 600, 700, 400, out_dtype=torch.float32).double(), x.double() @ w.double().t())
    dy = torch.randint(-15, 16, (600, 400), generator=gen, device="cuda").float()
    dy[:, ::128] = 448.0
    assert torch.equal(b.adasum_fp8_linear_grad(b.adasum_fp8_pack(dy), pw, 600, 700, 400, out_dtype=torch.float32).double(),
                       dy.double() @ w.double())


def test_gradient_against_differences(b):
    """sum(dy y(x)) along a direction: the product is linear in the packed values, so differences of the values are exact."""
    gen = _gen(5)
    rows, features, outputs = 150, 300, 200
    x, v, w, dy = (_matrix(gen, *s, "f32") for s in ((rows, features), (rows, features), (outputs, features), (rows, outputs)))
    pw, pdy = b.adasum_fp8_pack_weight(w), b.adasum_fp8_pack(dy)
    dx = to64(b.adasum_fp8_linear_grad(pdy, pw, rows, features, outputs, out_dtype=torch.float32))
    vdy = to64(b.adasum_fp8_unpack(pdy, rows, outputs))
    y, at = [], []
    for s in (0.5, -0.5):
        p = b.adasum_fp8_pack(x + s * v)
        at.append(to64(b.adasum_fp8_unpack(p, rows, features)))
        y.append(to64(b.adasum_fp8_linear(p, pw, rows, features, outputs, out_dtype=torch.float32)))
    diff, want = (vdy * (y[0] - y[1])).sum(), (dx * (at[0] - at[1])).sum()
    size = np.linalg.norm(vdy) * max(np.linalg.norm(t) for t in y) + np.linalg.norm(dx) * np.linalg.norm(at[0])
    assert abs(diff - want) <= 4e-6 * 2 * size


def test_nothing_to_sum_and_nothing_to_write(b):
    empty = torch.empty(0, dtype=torch.uint8, device="cuda")
    bias = torch.arange(40, device="cuda", dtype=torch.float32)
    y = b.adasum_fp8_linear(empty, empty, 5, 0, 40, bias=bias)
    assert torch.equal(y, bias.bfloat16().expand(5, 40))
    assert not torch.any(b.adasum_fp8_linear_grad(empty, empty, 5, 40, 0))
    w = b.adasum_fp8_pack_weight(torch.ones(40, 30, device="cuda"))
    assert b.adasum_fp8_linear(empty, w, 0, 30, 40).shape == (0, 40)
    x = b.adasum_fp8_pack(torch.ones(4, 30, device="cuda"))
    assert b.adasum_fp8_linear(x, empty, 4, 30, 0).shape == (4, 0)


def test_long_offsets(b):
    """Codes, step bytes and results beyond 2^31 bytes."""
    rows, features, outputs = 1 << 21, 1100, 1100
    if torch.cuda.mem_get_info()[0] < 24 << 30:
        pytest.skip("not enough memory")
    gen = _gen(6)
    w = torch.randn(outputs, features, generator=gen, device="cuda")
    pw = b.adasum_fp8_pack_weight(w)
    x = torch.zeros(rows, features, dtype=torch.bfloat16, device="cuda")
    tail = torch.randn(300, features, generator=gen, device="cuda").bfloat16()
    x[-300:] = tail
    px = b.adasum_fp8_pack(x)
    y = b.adasum_fp8_linear(px, pw, rows, features, outputs)
    small = b.adasum_fp8_linear(b.adasum_fp8_pack(tail), pw, 300, features, outputs)
    assert torch.equal(y[-300:], small) and not torch.any(y[:-300])
    del y
    assert torch.equal(b.adasum_fp8_unpack(px, rows, features, dtype=torch.bfloat16)[-300:], b.adasum_fp8_unpack(b.adasum_fp8_pack(tail), 300, features, dtype=torch.bfloat16))


def test_captured_products_on_two_streams(b):
    gen = _gen(7)
    sizes = [(500, 3000, 300), (40, 4096, 1024)]             # one of them joins parts of tiles
    data, want, got, graphs, workspaces, streams = [], [], [], [], [], [torch.cuda.Stream() for _ in sizes]
    for rows, features, outputs in sizes:
        x, w = _matrix(gen, rows, features, "bf16"), b.adasum_fp8_pack_weight(_matrix(gen, outputs, features, "f32"))
        data.append((x, w))
        want.append(b.adasum_fp8_linear(b.adasum_fp8_pack(x), w, rows, features, outputs))
    for (rows, features, outputs), (x, w), s in zip(sizes, data, streams):
        ws = torch.empty(b.adasum_fp8_linear_workspace_bytes(rows, features, outputs), dtype=torch.uint8, device="cuda")
        workspaces.append(ws)                                # they live as long as the graphs
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            got.append(b.adasum_fp8_linear(b.adasum_fp8_pack(x), w, rows, features, outputs, workspace=ws))
        graphs.append(g)
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    for w, g in zip(want, got):
        assert torch.equal(w, g)


# More sums per pair of blocks than tensor memory holds, and more steps than shared memory, so that every kind of
# hand-over is waited for.
@pytest.mark.parametrize("rows", [40, 128, 384])
@pytest.mark.parametrize("hand_over", ["landed", "multiplied", "formed", "taken"])
def test_a_wait_that_runs_out(b, hand_over, rows):
    features, outputs = 128 * 8 * 4 * 74, 24
    gen = _gen(8)
    px, pw = b.adasum_fp8_pack(_matrix(gen, rows, features, "bf16")), b.adasum_fp8_pack_weight(_matrix(gen, outputs, features, "bf16"))
    ws = torch.empty(b.adasum_fp8_linear_workspace_bytes(rows, features, outputs), dtype=torch.uint8, device="cuda")
    y = torch.zeros(rows, outputs, device="cuda")

    def good():
        b.adasum_fp8_linear(px, pw, rows, features, outputs, out=y, workspace=ws)
        assert b.adasum_fp8_linear_status(ws) == 0
        return y.clone()

    want = good()
    assert torch.isfinite(want).all()
    b.adasum_fp8_linear_selftest(hand_over, px, pw, rows, features, outputs, y, ws)
    assert b.adasum_fp8_linear_status(ws) == 7
    assert "bounded wait" in b.adasum_last_error()
    if hand_over in ("landed", "formed"):           # they fail in the first sum
        assert torch.isnan(y).all()
    assert torch.equal(good(), want)


# Five to eight steps and several tiles of the same rows for every pair of blocks: the weights stay in shared memory.  Runs that
# begin and end inside a row of tiles, ragged edges.
STAYING = [(3700, 1024, 4096, "bf16"), (3701, 1000, 4001, "f32"), (3900, 700, 3900, "f16"), (3800, 600, 4000, "f32"),
           (19150, 640, 700, "bf16")]


@pytest.mark.parametrize("rows,depth,wide,out_type", STAYING)
def test_weights_that_stay(b, rows, depth, wide, out_type):
    test_linear(b, rows, depth, wide, out_type)


@pytest.mark.parametrize("rows,depth,wide,out_type", STAYING)
def test_weights_that_stay_on_the_way_back(b, rows, depth, wide, out_type):
    test_linear_grad(b, rows, wide, depth, out_type)


@pytest.mark.parametrize("hand_over", ["landed", "multiplied", "formed", "taken"])
def test_a_wait_that_runs_out_where_weights_stay(b, hand_over):
    rows, features, outputs = 3700, 700, 4096
    gen = _gen(9)
    px, pw = b.adasum_fp8_pack(_matrix(gen, rows, features, "bf16")), b.adasum_fp8_pack_weight(_matrix(gen, outputs, features, "bf16"))
    ws = torch.empty(b.adasum_fp8_linear_workspace_bytes(rows, features, outputs), dtype=torch.uint8, device="cuda")
    y = torch.zeros(rows, outputs, device="cuda")
    b.adasum_fp8_linear(px, pw, rows, features, outputs, out=y, workspace=ws)
    assert b.adasum_fp8_linear_status(ws) == 0
    want = y.clone()
    assert torch.isfinite(want).all()
    b.adasum_fp8_linear_selftest(hand_over, px, pw, rows, features, outputs, y, ws)
    assert b.adasum_fp8_linear_status(ws) == 7
    if hand_over in ("landed", "formed"):
        assert torch.isnan(y).all()
    b.adasum_fp8_linear(px, pw, rows, features, outputs, out=y, workspace=ws)
    assert b.adasum_fp8_linear_status(ws) == 0 and torch.equal(y, want)


def test_calls_from_two_threads(b):
    """Threads with streams and workspaces of their own, whose calls overlap on the host and on the GPU."""
    from concurrent.futures import ThreadPoolExecutor

    jobs = []
    for seed, (rows, features, outputs) in enumerate([(300, 1024, 1000), (3700, 700, 4096), (70, 2000, 640), (1000, 1024, 4096)]):
        gen = _gen(seed)
        px, pw = b.adasum_fp8_pack(_matrix(gen, rows, features, "bf16")), b.adasum_fp8_pack_weight(_matrix(gen, outputs, features, "f32"))
        want = b.adasum_fp8_linear(px, pw, rows, features, outputs)
        norm = b.adasum_residual_norm(None, want, pre_norm="layer")[1]
        jobs.append((px, pw, rows, features, outputs, want, norm))
    torch.cuda.synchronize()

    def work(order):
        stream = torch.cuda.Stream()
        same = []
        with torch.cuda.stream(stream):
            for _ in range(10):
                for i in order:
                    px, pw, rows, features, outputs, want, norm = jobs[i]
                    y = b.adasum_fp8_linear(px, pw, rows, features, outputs)
                    z = b.adasum_residual_norm(None, y, pre_norm="layer")[1]
                    same += [(y == want).all(), (z == norm).all()]
        stream.synchronize()
        return all(bool(s) for s in same)

    with ThreadPoolExecutor(2) as pool:
        assert all(pool.map(work, [(0, 1, 2, 3), (3, 1, 0, 2)]))


# Every pair of blocks has more steps than shared memory has stages and more than two sums, so no kind of hand-over that never
# completes lets a pair finish: (rows, features, outputs) of tiles of 64, 128 and 192 tokens that are cut, and of whole ones
# whose weights stay.
@pytest.mark.parametrize("rows,features,outputs", [(40, 128 * 8 * 4 * 74, 24), (128, 128 * 8 * 4 * 74, 24), (384, 128 * 8 * 4 * 74, 24),
                                                   (3700, 700, 4096)])
@pytest.mark.parametrize("hand_over", ["landed", "multiplied", "formed", "taken"])
def test_nothing_of_an_unfinished_product_is_left(b, hand_over, rows, features, outputs):
    """NaN everywhere, whatever the result and the workspace held."""
    gen = _gen(10)
    px, pw = b.adasum_fp8_pack(_matrix(gen, rows, features, "bf16")), b.adasum_fp8_pack_weight(_matrix(gen, outputs, features, "bf16"))
    ws = torch.empty(b.adasum_fp8_linear_workspace_bytes(rows, features, outputs), dtype=torch.uint8, device="cuda")
    for dtype in (torch.float32, torch.bfloat16):
        y = torch.full((rows, outputs), 123.0, dtype=dtype, device="cuda")
        b.adasum_fp8_linear(px, pw, rows, features, outputs, out=torch.empty_like(y), workspace=ws)    # sums of a finished one
        b.adasum_fp8_linear_selftest(hand_over, px, pw, rows, features, outputs, y, ws)
        assert b.adasum_fp8_linear_status(ws) == 7
        assert torch.isnan(y).all()
