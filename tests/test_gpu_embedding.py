"""Token embedding and its gradient against plain sums in 64 bits."""
import numpy as np
import pytest
import torch

from operator_reference import TINY, TORCH, UNIT, assert_close, embedding_grad, to64

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def b():
    from paper_2006_02924_b200 import binding

    return binding


def _matrix(gen, rows, cols, dtype, pad=0, shift=0, size=1.0):
    """rows x cols of a wider buffer whose first element is `shift` elements past a 16-byte boundary."""
    flat = torch.randn(rows * (cols + pad) + shift, generator=gen, device="cuda") * size
    return flat.to(TORCH[dtype])[shift:].view(rows, cols + pad)[:, :cols]


def _ids(gen, n, num_rows, index, kind):
    if kind == "one":
        ids = torch.full((n,), num_rows - 1, device="cuda")
    elif kind == "none":
        ids = torch.full((n,), -1, device="cuda")
    elif kind == "uneven":        # a few rows take nearly everything, some tokens are outside on either side
        u = torch.rand(n, generator=gen, device="cuda")
        ids = (num_rows * u**6).long()
        ids = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.1, -5, ids)
        ids = torch.where(torch.rand(n, generator=gen, device="cuda") < 0.1, num_rows, ids)
    else:
        ids = torch.randint(0, num_rows, (n,), generator=gen, device="cuda")
    return ids.to(torch.int32 if index == 32 else torch.int64)


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


@pytest.mark.parametrize("table_type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("out_type", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("n,num_rows,dim,pad,shift,index", [
    (1, 7, 1, 0, 0, 64), (1, 1000, 1024, 0, 0, 64), (33, 5, 8, 8, 0, 32), (129, 300, 203, 5, 1, 64),
    (700, 2, 64, 0, 3, 32), (257, 1009, 136, 8, 0, 64), (5, 3, 9, 0, 0, 64)])
def test_forward(b, table_type, out_type, n, num_rows, dim, pad, shift, index):
    gen = _gen(1)
    table = _matrix(gen, num_rows, dim, table_type, pad, shift)
    ids = _ids(gen, n, num_rows, index, "uneven")
    out = torch.full((n, dim + pad), 7.0, dtype=TORCH[out_type], device="cuda")
    got = b.adasum_embedding_forward(table, ids, scale=0.37, out=out[:, :dim])
    i = ids.cpu().numpy().astype(np.int64)
    ok = (i >= 0) & (i < num_rows)
    scale = float(np.float32(0.37))
    want = np.where(ok[:, None], to64(table)[np.where(ok, i, 0)] * scale, 0.0)
    # one fp32 product, one rounding to the type
    assert_close(to64(got), want, (UNIT[out_type] + 2.0**-24) * 1.001 * np.abs(want) + TINY[out_type])
    assert torch.all(out[:, dim:] == 7.0), "columns beyond the row were written"


def test_forward_large_offsets(b):
    """Rows whose element offset passes 2^32."""
    table = torch.empty((1 << 22) + 3, 1024, dtype=torch.bfloat16, device="cuda")
    rows = torch.tensor([0, 1 << 22, (1 << 22) + 2, 77], device="cuda")
    table[rows] = torch.arange(4, device="cuda", dtype=torch.bfloat16)[:, None] + 1
    got = b.adasum_embedding_forward(table, rows, scale=2.0)
    assert torch.equal(got, (torch.arange(4, device="cuda", dtype=torch.bfloat16)[:, None] + 1).expand(4, 1024) * 2)


@pytest.mark.parametrize("kind", ["uniform", "uneven", "one", "none"])
@pytest.mark.parametrize("n,num_rows,dim,pad,shift,in_type,out_type,index", [
    (1, 1, 1, 0, 0, "f32", "f32", 64),
    (1, 30522, 16, 0, 0, "bf16", "f32", 64),
    (31, 255, 40, 0, 0, "f16", "bf16", 32),        # one pass of the sort and all its keys
    (32, 256, 40, 8, 0, "bf16", "bf16", 32),       # the key for "outside" needs a second byte
    (33, 65535, 8, 0, 0, "f32", "f16", 64),
    (65, 65536, 8, 0, 0, "bf16", "f32", 64),
    (999, 1009, 203, 5, 1, "f32", "f32", 32),
    (1000, 3, 129, 0, 1, "bf16", "f16", 64),
    (8193, 50, 64, 0, 0, "f16", "f16", 64),
    (20011, 2000, 24, 8, 0, "bf16", "f32", 32),    # longer tiles
    (16384, 2, 136, 0, 0, "f16", "f32", 64),
])
def test_grad(b, kind, n, num_rows, dim, pad, shift, in_type, out_type, index):
    gen = _gen(2)
    dy = _matrix(gen, n, dim, in_type, pad, shift)
    ids = _ids(gen, n, num_rows, index, kind)
    scale = float(np.float32(1.7))
    # the destination is a piece of a fused buffer, at an odd place
    flat = torch.full((num_rows * dim + 12,), 3.0, dtype=TORCH[out_type], device="cuda")
    place = 5 if shift else 8
    table = flat[place:place + num_rows * dim]
    b.adasum_embedding_grad(dy, ids, num_rows=num_rows, grad_table=table, scale=scale)
    want, bound = embedding_grad(to64(dy), ids.cpu().numpy().astype(np.int64), num_rows, scale)
    got = to64(table).reshape(num_rows, dim)
    assert_close(got, want, bound + (UNIT[out_type] * 1.001) * (np.abs(want) + bound) + TINY[out_type])
    assert torch.all(flat[:place] == 3.0) and torch.all(flat[place + num_rows * dim:] == 3.0), "written outside"
    # the same bits again, and the accumulating form on top of known values
    again = b.adasum_embedding_grad(dy, ids, num_rows=num_rows, grad_dtype=TORCH[out_type], scale=scale)
    assert torch.equal(again.reshape(-1), table)
    base = torch.randn(num_rows, dim, generator=gen, device="cuda").to(TORCH[out_type])
    total = base.clone()
    b.adasum_embedding_grad(dy, ids, grad_table=total, scale=scale, accumulate=True)
    want2 = to64(base) + want
    assert_close(to64(total), want2, bound + (UNIT[out_type] + 2.0**-24) * 1.001 * (np.abs(want2) + bound) + TINY[out_type])


def test_grad_of_no_tokens(b):
    table = torch.ones(5, 7, device="cuda")
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    dy = torch.empty(0, 7, device="cuda")
    b.adasum_embedding_grad(dy, none, grad_table=table, accumulate=True)
    assert torch.all(table == 1)
    b.adasum_embedding_grad(dy, none, grad_table=table)
    assert torch.all(table == 0)
    assert b.adasum_embedding_forward(table, none).shape == (0, 7)


def test_grad_spreads_nan_and_inf_to_their_rows_only(b):
    dy = torch.ones(100, 32, device="cuda")
    dy[3, 4], dy[50, 0] = float("nan"), float("inf")
    ids = torch.arange(100, device="cuda") % 7
    ids[60] = -1
    dy[60] = float("nan")                  # padding: never read into a sum
    got = b.adasum_embedding_grad(dy, ids, num_rows=8)
    bad = ~torch.isfinite(got)
    assert bad.sum() == 2 and bad[3, 4] and torch.isinf(got[1, 0]) and torch.all(got[7] == 0)


def test_gradient_is_the_adjoint(b):
    """Differences of the lookup in the direction d against the gradient: <lookup(W + d) - lookup(W), dy> = <d, dW>."""
    gen = _gen(3)
    w = torch.randint(-8, 8, (37, 24), generator=gen, device="cuda").float()
    d = torch.randint(-8, 8, (37, 24), generator=gen, device="cuda").float()
    dy = torch.randint(-8, 8, (500, 24), generator=gen, device="cuda").float()
    ids = torch.randint(-2, 39, (500,), generator=gen, device="cuda")
    left = ((b.adasum_embedding_forward(w + d, ids, 0.5) - b.adasum_embedding_forward(w, ids, 0.5)).double() * dy).sum()
    right = (b.adasum_embedding_grad(dy, ids, 37, scale=0.5).double() * d).sum()
    assert left == right                   # small integers: every sum is exact


def test_other_stream_and_graph(b):
    gen = _gen(4)
    dy = _matrix(gen, 300, 64, "bf16")
    ids = _ids(gen, 300, 40, 64, "uniform")
    want = b.adasum_embedding_grad(dy, ids, 40)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = b.adasum_embedding_grad(dy, ids, 40, stream=side)
    looked = b.adasum_embedding_forward(got, ids, stream=side)
    side.synchronize()
    assert torch.equal(got, want)
    table = torch.zeros(40, 64, device="cuda")
    ws = torch.empty(b.adasum_embedding_grad_workspace_bytes(300, 40, 64), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(looked)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.adasum_embedding_grad(dy, ids, grad_table=table, workspace=ws)
        b.adasum_embedding_forward(table, ids, out=out)
    ws.random_(0, 255)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(table, want) and torch.equal(out, looked)


def test_grad_large_offsets(b):
    """Gradients beyond 2^31 elements, more tokens than the sort keeps in registers."""
    n = (1 << 21) + 9
    dy = torch.zeros(n, 1024, dtype=torch.bfloat16, device="cuda")
    dy[-5:] = 1.0
    ids = (torch.arange(n, device="cuda") % 300).to(torch.int32)
    got = b.adasum_embedding_grad(dy, ids, 301)
    want = torch.zeros(301, 1024, device="cuda")
    want[ids[-5:].long()] = 1.0
    assert torch.equal(got, want)


@pytest.mark.parametrize("lengths", [[8, 8, 8, 8], [1, 15, 16, 17, 31, 32, 33, 47, 48, 49], [16, 16, 32, 64, 1, 1, 7],
                                     [7, 1, 9, 24, 25, 3], [2000, 5, 40, 33]])
@pytest.mark.parametrize("extra", [0, 1, 2100])
def test_runs_at_the_tiles_ends(b, lengths, extra):
    """Runs of equal tokens that start, end and go on at every place of the sorted list's tiles (8 or 16 entries),
    followed by tokens outside the table."""
    ids = torch.cat([torch.full((c,), 3 * i) for i, c in enumerate(lengths)] + [torch.full((extra,), -7)])
    gen = _gen(6)
    ids = ids[torch.randperm(ids.numel())].cuda()
    dy = torch.randint(-9, 10, (ids.numel(), 40), generator=gen, device="cuda").float()
    got = b.adasum_embedding_grad(dy, ids, 3 * len(lengths))
    want, _ = embedding_grad(to64(dy), ids.cpu().numpy(), 3 * len(lengths), 1.0)
    assert np.array_equal(to64(got), want)          # whole numbers: exact


def test_refusals(b):
    table, ids = torch.ones(5, 8, device="cuda"), torch.zeros(3, dtype=torch.int64, device="cuda")
    with pytest.raises(b.AdasumError, match="DTYPE"):
        b.adasum_embedding_forward(table.double(), ids)
    with pytest.raises(ValueError):
        b.adasum_embedding_forward(table.t(), ids)
    with pytest.raises(TypeError):
        b.adasum_embedding_forward(table, ids.float())
    with pytest.raises(ValueError):
        b.adasum_embedding_forward(table, ids, out=torch.empty(3, 9, device="cuda"))
    dy = torch.ones(3, 8, device="cuda")
    with pytest.raises(ValueError):
        b.adasum_embedding_grad(dy, ids[:2], 5)
    with pytest.raises(ValueError):
        b.adasum_embedding_grad(dy, ids, grad_table=torch.empty(8, 5, device="cuda"))
    with pytest.raises(ValueError):
        b.adasum_embedding_grad(dy, ids)
    with pytest.raises(b.AdasumError, match="WORKSPACE"):
        b.adasum_embedding_grad(dy, ids, 5, workspace=torch.empty(64, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("accumulate", [False, True])
@pytest.mark.parametrize("n", [2047, 2048, 4736, 4737, 6144, 6145])
@pytest.mark.parametrize("num_rows,dim", [(30522, 300), (997, 20)])
def test_lists_around_a_change_of_method(b, n, num_rows, dim, accumulate):
    """The same sums, whichever way the tokens were brought into order and however long the tiles are: small whole
    numbers, so that every association gives the same."""
    gen = _gen(31)
    ids = _ids(gen, n, num_rows, 64, "uneven")
    dy = torch.randint(-8, 9, (n, dim), generator=gen, device="cuda").float()
    old = torch.randint(-8, 9, (num_rows, dim), generator=gen, device="cuda").float()
    want = old.clone() if accumulate else torch.zeros_like(old)
    inside = (ids >= 0) & (ids < num_rows)
    want.index_add_(0, ids[inside], dy[inside] * 2)
    workspace = torch.empty(b.adasum_embedding_grad_workspace_bytes(6145, num_rows, dim), dtype=torch.uint8, device="cuda")
    got = b.adasum_embedding_grad(dy, ids, grad_table=old.clone(), scale=2.0, accumulate=accumulate, workspace=workspace)
    assert torch.equal(got, want)
