"""Dropout from the counter-based generator against its definition."""
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


def _seed(value):
    return torch.tensor([value], dtype=torch.int64, device="cuda")


def _matrix(seed, rows, cols, dtype, pad=0, shift=0):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    flat = torch.randn(rows * (cols + pad) + shift, generator=gen, device="cuda")
    return flat.to(TORCH[dtype])[shift:].view(rows, cols + pad)[:, :cols]


SEED, SITE = -0x123456789abcdef, (7 << 40) + 12345


@pytest.mark.parametrize("dtype", ["f32", "f16", "bf16"])
@pytest.mark.parametrize("rows,cols,pad,shift,p,residual", [
    (1, 1, 0, 0, 0.5, False), (1, 8, 0, 0, 0.1, True), (3, 7, 2, 1, 0.5, True), (5, 32, 0, 0, 0.25, False),
    (2, 33, 3, 0, 0.1, True), (61, 1023, 1, 0, 0.1, False), (130, 1024, 0, 0, 0.1, True), (1000, 24, 8, 0, 0.9, False),
    (7, 8192, 0, 0, 1e-5, True), (37, 100, 0, 0, 1.0, True), (37, 104, 0, 0, 0.0, True), (9, 64, 0, 0, 0.99, False)])
def test_dropout(b, dtype, rows, cols, pad, shift, p, residual):
    x = _matrix(1, rows, cols, dtype, pad, shift)
    r = _matrix(2, rows, cols, dtype, pad, shift) if residual else None
    spare = torch.full((rows * (cols + pad) + shift + 8,), 3.0, dtype=TORCH[dtype], device="cuda")
    out = spare[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols]
    seed = _seed(SEED)
    b.adasum_dropout(x, p, seed, site=SITE, residual=r, out=out)
    mask = ref.kept(rows, cols, p, SEED & (2**64 - 1), SITE)
    branch = ref.dropped(to64(x), mask)
    want = branch + (to64(r) if residual else 0.0)
    # the factor, its product, the sum, the stored value: one rounding each
    bound = 2 * ref.U * np.abs(branch) + ref.U * np.abs(want)
    bound = bound + UNIT[dtype] * (np.abs(want) + bound) + TINY[dtype]
    assert_close(to64(out), want, bound)
    # nothing else is written
    full = torch.full_like(spare, 3.0)
    full[shift:shift + rows * (cols + pad)].view(rows, cols + pad)[:, :cols] = out
    assert torch.equal(spare, full)
    # in place, and on its own allocation
    assert torch.equal(b.adasum_dropout(x, p, seed, site=SITE, residual=r), out)
    again = x.clone()
    assert torch.equal(b.adasum_dropout(again, p, seed, site=SITE, residual=r, out=again), out)
    if residual:
        again = r.clone()
        assert torch.equal(b.adasum_dropout(x, p, seed, site=SITE, residual=again, out=again), out)


def test_generator_by_hand(b):
    """The published generator, one counter at a time, and its published answer for all-ones inputs."""
    assert ref.philox((M := 0xffffffff, M), (M, M, M, M)) == [0x408f276d, 0x41c83b0e, 0xa20bc7c6, 0x6d5451fd]
    assert ref.philox((0, 0), (0, 0, 0, 0)) == [0x6627e8d5, 0xe169c58d, 0xbc57ac4c, 0x9b00dbd8]
    seed, site = 0x0123456789abcdef, (5 << 32) + 9
    out = b.adasum_dropout(torch.ones(3, 20, device="cuda"), 0.5, _seed(seed), site=site).cpu().numpy()
    for row in range(3):
        for col in range(20):
            words = ref.philox((seed & M, seed >> 32), (row * 3 + col // 8, 0, site & M, site >> 32))
            bits = words[col % 8 // 2] >> (16 * (col % 2)) & 0xffff
            assert out[row, col] == (2.0 if bits >= 32768 else 0.0)


def test_dropped_elements_are_zero_whatever_they_hold(b):
    x = torch.full((64, 40), float("nan"), device="cuda")
    x[::2] = float("inf")
    for dtype in TORCH.values():
        out = b.adasum_dropout(x.to(dtype), 0.5, _seed(3))
        keep, _ = ref.kept(64, 40, 0.5, 3, 0)
        assert np.array_equal(torch.isfinite(out).cpu().numpy(), ~keep) and torch.all(out[torch.isfinite(out)] == 0)
        assert not torch.any(b.adasum_dropout(x.to(dtype), 1.0, _seed(3)))


def test_rate_and_expectation(b):
    """2^24 draws: rate within five standard deviations, seeds and sites independent."""
    n = 1 << 24
    ones = torch.ones(4096, 4096, device="cuda")
    a = b.adasum_dropout(ones, 0.1, _seed(11), site=0)
    q = 6554 / 65536
    rate = (a == 0).double().mean().item()
    assert abs(rate - q) < 5 * (q * (1 - q) / n) ** 0.5
    # the mean's factor is exact for the rate used, not for p
    assert abs(a.double().mean().item() - 1) < 5 * (q / (1 - q) / n) ** 0.5
    for other in (b.adasum_dropout(ones, 0.1, _seed(12), site=0), b.adasum_dropout(ones, 0.1, _seed(11), site=1)):
        both = ((a == 0) & (other == 0)).double().mean().item()
        assert abs(both - q * q) < 5 * (q * q / n) ** 0.5
    # neighbours in a vector, a row apart
    for x, y in ((a[:, :-1], a[:, 1:]), (a[:-1], a[1:])):
        assert abs(((x == 0) & (y == 0)).double().mean().item() - q * q) < 5 * (q * q / n) ** 0.5


def test_gradient_against_differences(b):
    """Dropout is linear for a given mask: d sum(g * out) / dx is the same call on g."""
    x, g = _matrix(5, 50, 70, "f32"), _matrix(6, 50, 70, "f32")
    seed = _seed(9)
    dx = to64(b.adasum_dropout(g, 0.3, seed, site=4))
    for k in range(5):
        v = _matrix(10 + k, 50, 70, "f32")
        plus, minus = (to64(b.adasum_dropout(x + s * v, 0.3, seed, site=4)) for s in (1.0, -1.0))
        diff, size = ((plus - minus) / 2 * to64(g)), np.abs(to64(g)) * (np.abs(plus) + np.abs(minus) + np.abs(to64(v)))
        # x +- v and the outputs are rounded
        assert abs(diff.sum() - (dx * to64(v)).sum()) <= 8 * ref.U * size.sum()


def test_masks_change_inside_a_captured_graph(b):
    x = torch.ones(128, 256, device="cuda", dtype=torch.bfloat16)
    seed, out = _seed(1), torch.empty_like(x)
    b.adasum_dropout(x, 0.5, seed, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.adasum_dropout(x, 0.5, seed, out=out)
    for value in (1, 2, -5):
        seed.fill_(value)
        graph.replay()
        keep, _ = ref.kept(128, 256, 0.5, value & (2**64 - 1), 0)
        assert np.array_equal((out != 0).cpu().numpy(), keep)


def test_another_stream(b):
    x = _matrix(3, 300, 500, "f32")
    want = b.adasum_dropout(x, 0.2, _seed(4))
    side = torch.cuda.Stream()
    seed = _seed(4)
    torch.cuda.synchronize()
    got = b.adasum_dropout(x, 0.2, seed, stream=side)
    side.synchronize()
    assert torch.equal(got, want)


def test_offsets_beyond_32_bits(b):
    """More than 2^32 elements: the last rows are right, and differ from those whose vector numbers agree in 32 bits."""
    rows, cols = 65600, 65544
    free = torch.cuda.mem_get_info()[0]
    if free < 3 * rows * cols * 2:
        pytest.skip("not enough memory")
    x = torch.ones(rows, cols, dtype=torch.bfloat16, device="cuda")
    out = b.adasum_dropout(x, 0.5, _seed(21), site=3, out=x)
    for row in (0, 32768, rows - 1):
        keep, _ = ref.kept(1, cols, 0.5, 21, 3, first_row=row)
        assert np.array_equal((out[row] != 0).cpu().numpy(), keep[0])


def test_nothing_to_do(b):
    assert b.adasum_dropout(torch.empty(0, 5, device="cuda"), 0.5, _seed(1)).shape == (0, 5)
    assert b.adasum_dropout(torch.empty(5, 0, device="cuda"), 0.5, _seed(1)).shape == (5, 0)
    x = torch.randn(5, 9, device="cuda")
    assert torch.equal(b.adasum_dropout(x, 0.0, None), x)
    assert torch.equal(b.adasum_dropout(x, 2.0**-18, _seed(1)), x)
