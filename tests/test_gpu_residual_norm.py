"""The joint between two residual blocks and its gradients against the formulas in 64 bits."""
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


SEED, SITE = 0x7edcba9876543210, 77
EPS = float(np.float32(1e-5))


def _seed(value=SEED):
    return torch.tensor([value], dtype=torch.int64, device="cuda")


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _matrix(gen, rows, cols, dtype, pad=0, shift=0, size=1.0, mean=0.0):
    flat = torch.randn(rows * (cols + pad) + shift, generator=gen, device="cuda") * size + mean
    return flat.to(TORCH[dtype])[shift:].view(rows, cols + pad)[:, :cols]


# rows, features, dtype, stream, params, post, pre, rows per gate (0: no gate, -1: one for all), p, pad, shift
CASES = [
    (1, 1, "f32", "f32", "f32", "none", "rms", 0, 0.0, 0, 0),
    (1, 5, "f32", "f32", "f32", "layer", "layer", -1, 0.0, 0, 0),
    (3, 7, "bf16", "f32", "bf16", "rms", "layer", 2, 0.25, 1, 1),
    (70, 32, "f16", "f16", "f32", "rms", "rms", 1, 0.0, 0, 0),
    (257, 40, "bf16", "bf16", "bf16", "layer", "rms", 100, 0.1, 8, 0),
    (129, 64, "f32", "f32", "f16", "none", "none", -1, 0.5, 0, 0),
    (37, 100, "f16", "f32", "f16", "none", "layer", 0, 0.1, 0, 0),
    (64, 256, "bf16", "bf16", "f32", "rms", "rms", 8, 0.0, 0, 0),
    (65, 257, "f32", "f32", "f32", "layer", "layer", -1, 0.25, 3, 1),
    (999, 203, "f32", "f32", "f32", "layer", "layer", -1, 0.25, 5, 0),
    (2050, 264, "bf16", "f32", "f32", "layer", "rms", 700, 0.1, 0, 0),
    (33, 1000, "bf16", "bf16", "bf16", "none", "layer", 0, 0.1, 24, 0),
    (1500, 1024, "bf16", "bf16", "f32", "none", "layer", 0, 0.1, 0, 0),
    (5, 2048, "f16", "f16", "f16", "layer", "layer", 3, 0.0, 0, 0),
    (301, 4096, "bf16", "f32", "f32", "rms", "rms", 128, 0.0, 0, 0),
    (3, 4097, "f32", "f32", "f32", "rms", "layer", -1, 0.1, 0, 0),
    (31, 8200, "bf16", "bf16", "f32", "layer", "rms", 10, 0.25, 0, 0),
    (2, 32768, "f32", "f32", "f32", "layer", "layer", 1, 0.1, 0, 0),
    (19, 20001, "f16", "f32", "f32", "rms", "rms", -1, 0.0, 1, 0),
]


class Case:
    def __init__(self, spec, seed=1):
        (self.rows, self.features, self.dtype, self.stream, self.params, post, pre, gate, self.p, self.pad, self.shift) = spec
        gen = _gen(seed)
        m = lambda dtype, **k: _matrix(gen, self.rows, self.features, dtype, self.pad, self.shift, **k)  # noqa: E731
        self.x, self.residual = m(self.dtype, mean=0.3), m(self.stream, size=2.0)
        self.dy, self.dh = m(self.dtype), m(self.stream, size=0.5)
        vec = lambda mean: (torch.randn(self.features, generator=gen, device="cuda") * 0.3 + mean).to(TORCH[self.params])  # noqa: E731
        self.per_gate = max(self.rows, 1) if gate < 0 else gate
        gates = 0 if gate == 0 else -(-self.rows // self.per_gate)
        gate_type = self.dtype if gate > 0 else self.params
        self.call = dict(
            post_norm=post, post_weight=vec(1.0) if post != "none" else None, post_bias=vec(0.0) if post == "layer" else None,
            pre_norm=pre, pre_weight=vec(1.0) if pre != "none" else None, pre_bias=vec(0.1) if pre == "layer" else None,
            eps=EPS, gate=_matrix(gen, gates, self.features, gate_type, 0, 0, 0.3, 0.5) if gates else None,
            rows_per_gate=self.per_gate if gates else None, branch_scale=0.75, residual_scale=-1.25, dropout=self.p,
            seed=_seed() if self.p > 0 else None, site=SITE)
        self.options = {k: to64(v) if torch.is_tensor(v) else v for k, v in self.call.items()}
        for k, fill in (("post_weight", 1.0), ("post_bias", 0.0), ("pre_weight", 1.0), ("pre_bias", 0.0)):
            if self.options[k] is None:
                self.options[k] = fill
        self.mask = ref.kept(self.rows, self.features, self.p, SEED, SITE)


def _close(got, pair, dtype, what):
    want, bound = pair
    assert_close(to64(got), want, 1.1 * bound + UNIT[dtype] * (np.abs(want) + 1.1 * bound) + TINY[dtype], what)


@pytest.mark.parametrize("spec", CASES, ids=lambda s: "-".join(map(str, s)))
def test_forward(b, spec):
    c = Case(spec)
    h, y, stats = b.adasum_residual_norm(c.x, c.residual, **c.call)
    want = ref.joint(to64(c.x), to64(c.residual), c.options, c.mask)
    _close(h, want["h"], c.stream, "h")
    if c.call["pre_norm"] == "none":
        assert y is None
    else:
        _close(y, want["y"], c.dtype, "y")
    for name, at in (("post", 0), ("pre", 2)):
        if name in want:
            mean, dmean, rstd, drstd = want[name]
            if c.call[name + "_norm"] == "layer":
                assert_close(to64(stats[at]), mean, 1.1 * dmean + 2 * ref.U * np.abs(mean) + 1e-37, name + " mean")
            assert_close(to64(stats[at + 1]), rstd, 1.1 * drstd + 2 * ref.U * rstd, name + " rstd")
    # in place, without the statistics: the same bits
    residual = c.residual.clone(memory_format=torch.preserve_format)
    h2, y2, none = b.adasum_residual_norm(c.x, residual, h=residual, want_stats=False, **c.call)
    assert none is None and h2 is residual and torch.equal(h2, h) and (y is None or torch.equal(y2, y))
    if y is not None:
        x = c.x.clone()
        none, y3, _ = b.adasum_residual_norm(x, c.residual, y=x, want_h=False, **c.call)
        assert none is None and torch.equal(y3, y)


def _grads(b, c, h, stats, accumulate=False, scale=1.0, fill=5.0, grad_dtype=torch.float32, **more):
    flat = torch.full((4 * (c.features + 3) + 1,), fill, dtype=grad_dtype, device="cuda")
    places = {}
    for i, name in enumerate(("post_weight", "post_bias", "pre_weight", "pre_bias")):
        if c.call[name] is not None:
            at = 1 + i * (c.features + 3)                    # odd places in a fused buffer
            places["grad_" + name] = flat[at:at + c.features]
    if c.call["gate"] is not None:
        places["grad_gate"] = torch.full(c.call["gate"].shape, fill, dtype=grad_dtype, device="cuda")
    dy = c.dy if c.call["pre_norm"] != "none" else None
    dx, dr = b.adasum_residual_norm_grad(c.x, h, stats, dy, c.dh, accumulate=accumulate, scale=scale, gate_scale=scale / 2,
                                         **places, **c.call, **more)
    written = sum(p.numel() for n, p in places.items() if n != "grad_gate")
    assert (flat == fill).sum().item() >= flat.numel() - written, "written outside"
    return {"x": dx, "residual": dr, **{n[5:]: p for n, p in places.items()}}


@pytest.mark.parametrize("spec", CASES, ids=lambda s: "-".join(map(str, s)))
def test_gradients(b, spec):
    c = Case(spec)
    h, _, stats = b.adasum_residual_norm(c.x, c.residual, **c.call)
    dy = to64(c.dy) if c.call["pre_norm"] != "none" else None
    want = ref.joint_grad(to64(c.x), to64(h), to64(stats), dy, to64(c.dh), c.options, c.mask)
    got = _grads(b, c, h, stats)
    assert set(got) <= set(want) | {"x"}
    for name, t in got.items():
        value, bound = want[name]
        if name == "gate":
            value, bound = value / 2, bound / 2
        if name in ("x", "residual"):
            _close(t, (value, bound), c.dtype if name == "x" else c.stream, name)
        else:
            _close(t, (value, bound + 2 * ref.U * np.abs(value)), "f32", name)
    again = _grads(b, c, h, stats)
    assert all(torch.equal(again[n], got[n]) for n in got), "not the same from run to run"
    # added in another type, half as large
    more = _grads(b, c, h, stats, accumulate=True, scale=0.5, fill=2.0, grad_dtype=torch.bfloat16)
    for name in got:
        if name not in ("x", "residual"):
            value, bound = want[name]
            part = 0.25 if name == "gate" else 0.5
            _close(more[name], (2 + part * value, part * bound + 2 * ref.U * (2 + np.abs(value))), "bf16", name)


@pytest.mark.parametrize("spec", [CASES[i] for i in (2, 8, 10, 15)], ids=lambda s: "-".join(map(str, s)))
def test_gradients_against_differences(b, spec):
    """The gradients of sum(cy y) + sum(ch h) along random directions against central differences of the forward
    formula in 64 bits (fp32 inputs, so that only the kernel's own rounding and that of h as it is kept remain)."""
    spec = spec[:2] + ("f32", "f32", "f32") + spec[5:]
    c = Case(spec)
    h, _, stats = b.adasum_residual_norm(c.x, c.residual, **c.call)
    got = {n: to64(t) * (2 if n == "gate" else 1) for n, t in _grads(b, c, h, stats).items()}
    dy, dh = to64(c.dy), to64(c.dh)
    rng = np.random.default_rng(5)
    base = {"x": to64(c.x), "residual": to64(c.residual), **{n: c.options[n] for n in got if n not in ("x", "residual")}}

    def value(at):
        out = ref.joint(at["x"], at["residual"], {**c.options, **at}, c.mask)
        return (dy * out["y"][0]).sum() + (dh * out["h"][0]).sum()

    for name in got:
        v = rng.standard_normal(base[name].shape)
        step = 1e-5
        plus, minus = (value({**base, name: base[name] + s * step * v}) for s in (1, -1))
        diff, exact = (plus - minus) / (2 * step), (got[name] * v).sum()
        # per element the kernel is off by some dozens of roundings of magnitudes like the gradient's own; the
        # differences by step^2 and by the sums' cancellation (1e-16 of 1e5 values over the step)
        size = np.sqrt((got[name] ** 2).sum() * (v * v).sum())
        assert abs(diff - exact) <= 1e-5 * size + 1e-5 * abs(diff) + 1e-4, (name, diff, exact, size)


WIDEST = [
    (3, 32767, "f32", "f32", "f32", "layer", "layer", -1, 0.1, 1, 1),
    (3, 32768, "bf16", "f32", "bf16", "none", "layer", 0, 0.1, 0, 0),
    (2, 32768, "f16", "f16", "f32", "rms", "rms", 0, 0.0, 0, 0),
    (2, 32761, "bf16", "bf16", "f32", "none", "rms", 1, 0.25, 7, 0),
    (3, 16392, "f32", "f32", "f32", "none", "rms", 0, 0.0, 8, 4),
]


@pytest.mark.parametrize("spec", WIDEST, ids=lambda s: "-".join(map(str, s)))
def test_widest_rows(b, spec):
    """Rows that a cluster of blocks shares, in every form of the kernels."""
    test_forward(b, spec)
    test_gradients(b, spec)


def test_no_rows_on_another_stream(b):
    """The gradient of a gate of no rows is cleared on the call's stream, given as an object or as a handle."""
    x, gate = torch.empty(0, 24, device="cuda"), torch.ones(2, 24, device="cuda")
    _, _, stats = b.adasum_residual_norm(x, x)
    for stream in (torch.cuda.Stream(), torch.cuda.Stream().cuda_stream):
        grad = torch.ones(2, 24, device="cuda")
        torch.cuda.synchronize()
        b.adasum_residual_norm_grad(x, x, stats, x, x, gate=gate, rows_per_gate=5, grad_gate=grad, stream=stream)
        torch.cuda.synchronize()
        assert not torch.any(grad)


def test_only_what_is_wanted(b):
    """Parts of the joint: a norm alone, a residual sum alone, gradients of one side only."""
    gen = _gen(3)
    r, w = _matrix(gen, 40, 136, "f32"), torch.randn(136, generator=gen, device="cuda")
    none, y, stats = b.adasum_residual_norm(None, r, pre_weight=w, eps=EPS, want_h=False)
    want, bound, *_ = ref.norm(to64(r), 0 * to64(r), "rms", EPS, to64(w))
    assert none is None
    _close(y, (want, bound), "f32", "norm alone")
    x = _matrix(gen, 40, 136, "f32")
    h, none, _ = b.adasum_residual_norm(x, r, pre_norm="none", want_stats=False)
    assert none is None and torch.equal(h, x + r)
    h, none, _ = b.adasum_residual_norm(x, None, pre_norm="none", want_stats=False, branch_scale=0.5)
    assert torch.equal(h, 0.5 * x)
    # the norm's gradient alone; no vectors, so no workspace
    dy = _matrix(gen, 40, 136, "f32")
    dx, dr = b.adasum_residual_norm_grad(None, r, stats, dy, None, pre_weight=w, eps=EPS, want_x=False)
    o = dict(post_norm="none", post_weight=1.0, post_bias=0.0, pre_norm="rms", pre_weight=to64(w), pre_bias=0.0, gate=None,
             branch_scale=1.0, residual_scale=1.0, rows_per_gate=None)
    pair = ref.joint_grad(None, to64(r), to64(stats), to64(dy), None, o, None)["residual"]
    assert dx is None
    _close(dr, pair, "f32", "norm's gradient alone")
    # through the residual stream alone: the norm before the next block has no part in it
    gw = torch.full((136,), 9.0, device="cuda")
    dx, dr = b.adasum_residual_norm_grad(None, None, None, None, dy, pre_weight=w, grad_pre_weight=gw, residual_scale=2.0,
                                         branch_scale=3.0)
    assert torch.equal(dr, 2 * dy) and torch.equal(dx, 3 * dy) and not torch.any(gw)
    # in place
    into = dy.clone()
    _, dr2 = b.adasum_residual_norm_grad(None, None, None, None, into, grad_residual=into, residual_scale=2.0, want_x=False)
    assert dr2 is into and torch.equal(into, dr)


def test_rows_that_are_not_numbers_stay_by_themselves(b):
    """Inf and NaN in one row spoil that row and the vectors' gradients, and nothing else; dropped ones nothing at all."""
    gen = _gen(4)
    for features in (24, 520, 5000):
        x, r = _matrix(gen, 9, features, "f32"), _matrix(gen, 9, features, "f32")
        x[4, 3], x[7, 8] = float("nan"), float("inf")
        h, y, stats = b.adasum_residual_norm(x, r, post_norm="rms", pre_norm="layer")
        good = [0, 1, 2, 3, 5, 6, 8]
        assert torch.isfinite(h[good]).all() and torch.isfinite(y[good]).all() and torch.isnan(y[4]).all() and torch.isnan(y[7]).all()
        dx, dr = b.adasum_residual_norm_grad(x, h, stats, r, x[:1].expand(9, features).contiguous(), post_norm="rms", pre_norm="layer")
        assert torch.isfinite(dx[good]).all() and torch.isfinite(dr[good]).all()
        keep, _ = ref.kept(9, features, 0.5, 5, 0)
        x = torch.where(torch.from_numpy(keep).cuda(), 1.0, float("nan"))
        h, y, stats = b.adasum_residual_norm(x, r, dropout=0.5, seed=_seed(5))
        assert torch.isfinite(h).all() and torch.isfinite(y).all()
        # infinite parameters do not reach rows beyond the last (odd numbers of rows, gates that end inside a pair)
        gate, gw = torch.full((3, features), 1.0, device="cuda"), torch.zeros(3, features, device="cuda")
        gate[1] = float("inf")
        b.adasum_residual_norm_grad(r, h, stats, r, r, gate=gate, rows_per_gate=3, grad_gate=gw)
        assert torch.isfinite(gw).all()


def test_large_and_tiny_values(b):
    """A mean far from zero (no cancellation of squares), values near fp32's ends, rows of zeros."""
    gen = _gen(6)
    x = _matrix(gen, 50, 1000, "f32", mean=1000.0)
    none, y, _ = b.adasum_residual_norm(None, x, pre_norm="layer", eps=EPS, want_h=False)
    want, bound, *_ = ref.norm(to64(x), 0 * to64(x), "layer", EPS)
    _close(y, (want, bound), "f32", "far mean")
    for size in (1e-25, 1e15):
        z = x * size
        none, y, stats = b.adasum_residual_norm(None, z, eps=0.0, want_h=False)
        want, bound, *_ = ref.norm(to64(z), 0 * to64(z), "rms", 0.0)
        if size > 1:
            _close(y, (want, bound), "f32", "large")
        else:
            # squares of 1e-22 are 1e-44: multiples of 2^-149, each off by at most 2^-150 = 7e-46, and so is their mean
            # (a sum of subnormals is exact) by once more when it is formed: 1.4e-45 of 1e-44, half of it in the root
            assert_close(to64(stats[3]), 1 / np.sqrt((to64(z) ** 2).mean(1)), 0.08 / np.sqrt((to64(z) ** 2).mean(1)))
    zero = torch.zeros(3, 40, device="cuda")
    h, y, stats = b.adasum_residual_norm(zero, zero, post_norm="layer", pre_norm="rms", eps=EPS)
    assert not torch.any(y) and torch.allclose(stats[1], torch.full_like(stats[1], EPS**-0.5), rtol=1e-6)


def test_rows_behind_the_last_are_left_alone(b):
    buffers = [torch.full((20, 72), 7.0, device="cuda") for _ in range(4)]
    x = torch.randn(13, 72, device="cuda")
    h, y, dx, dr = (t[:13] for t in buffers)
    _, _, stats = b.adasum_residual_norm(x, x, post_norm="layer", pre_norm="rms", h=h, y=y)
    b.adasum_residual_norm_grad(x, h, stats, x, x, post_norm="layer", pre_norm="rms", grad_x=dx, grad_residual=dr)
    for t in buffers:
        assert (t[13:] == 7.0).all() and (t[:13] != 7.0).all()


def test_captured_beside_an_eager_graph_and_on_two_streams(b):
    """Captured calls, each with its own workspace, replayed on two streams at once give what eager calls give."""
    spec = (700, 520, "bf16", "f32", "f32", "rms", "layer", 50, 0.1, 0, 0)
    cases = [Case(spec, seed) for seed in (1, 2)]
    want = []
    for c in cases:
        h, y, stats = b.adasum_residual_norm(c.x, c.residual, **c.call)
        want.append((h, y, stats, _grads(b, c, h, stats)))
    leaf = cases[0].x.float().requires_grad_()               # an eager graph of the same data lives on
    alive = (leaf * 2).sum()
    streams, graphs, got, workspaces = [torch.cuda.Stream() for _ in cases], [], [], []
    for c, s in zip(cases, streams):
        ws = torch.empty(b.adasum_residual_norm_grad_workspace_bytes(520, gate=True), dtype=torch.uint8, device="cuda")
        workspaces.append(ws)                                # they live as long as the graphs
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=s):
            h, y, stats = b.adasum_residual_norm(c.x, c.residual, **c.call)
            got.append((h, y, stats, _grads_only(b, c, h, stats, ws)))
        graphs.append(g)
    for _ in range(3):
        for g, s in zip(graphs, streams):
            with torch.cuda.stream(s):
                g.replay()
    torch.cuda.synchronize()
    alive.backward()
    for (h, y, stats, grads), (h2, y2, stats2, grads2) in zip(want, got):
        assert torch.equal(h, h2) and torch.equal(y, y2)
        for name in grads:
            assert torch.equal(grads[name], grads2[name]), name


def _grads_only(b, c, h, stats, ws):
    places = {"grad_" + n: torch.empty(c.features, device="cuda") for n in ("post_weight", "pre_weight", "pre_bias")}
    places["grad_gate"] = torch.empty(c.call["gate"].shape, device="cuda")
    dx, dr = b.adasum_residual_norm_grad(c.x, h, stats, c.dy, c.dh, workspace=ws, gate_scale=0.5, **places, **c.call)
    return {"x": dx, "residual": dr, **{n[5:]: t for n, t in places.items()}}


def test_no_rows(b):
    x = torch.empty(0, 24, device="cuda")
    h, y, stats = b.adasum_residual_norm(x, x, post_norm="rms")
    assert h.shape == y.shape == (0, 24) and stats.shape == (4, 0)
    gw, gg = torch.ones(24, device="cuda"), torch.ones(1, 24, device="cuda")
    gate = torch.ones(1, 24, device="cuda")
    b.adasum_residual_norm_grad(x, h, stats, x, x, gate=gate, rows_per_gate=5, grad_pre_weight=gw, grad_gate=gg)
    assert not torch.any(gw) and not torch.any(gg)
    gw.fill_(3.0)
    b.adasum_residual_norm_grad(x, h, stats, x, x, grad_pre_weight=gw, accumulate=True)
    assert (gw == 3.0).all()
    empty = torch.empty(4, 0, device="cuda")
    h, y, _ = b.adasum_residual_norm(empty, empty)
    assert h.shape == (4, 0) and y.shape == (4, 0)


@pytest.mark.parametrize("rows,features", [(600, 512), (37, 203), (2000, 64), (20, 8192)])
def test_calls_in_a_row_on_one_stream_read_the_last_statistics(b, rows, features):
    """Forward and gradient calls in turn, each brought in while the last one ends, over one buffer of statistics and with
    other inputs each time: the same bits as calls that wait for one another."""
    gen = _gen(11)
    xs = [_matrix(gen, rows, features, "bf16", size=2.0**i, mean=0.5 * i) for i in range(4)]
    residual, dy, dh = (_matrix(gen, rows, features, "bf16") for _ in range(3))
    seeds = [_seed(5), _seed(6), _seed(7)]
    stats, h, y = torch.empty(4, rows, device="cuda"), torch.empty_like(residual), torch.empty_like(residual)

    def run(times, wait):
        out = [torch.empty(2, rows, features, dtype=torch.bfloat16, device="cuda") for _ in range(times)]
        torch.cuda.synchronize()
        for i, (dx, dr) in enumerate(out):
            call = dict(post_norm="layer", pre_norm="layer", dropout=0.25, seed=seeds[i % 3], site=i)
            b.adasum_residual_norm(xs[i % 4], residual, h=h, y=y, stats=stats, **call)
            if wait:
                torch.cuda.synchronize()
            b.adasum_residual_norm_grad(xs[i % 4], h, stats, dy, dh, grad_x=dx, grad_residual=dr, **call)
            if wait:
                torch.cuda.synchronize()
        torch.cuda.synchronize()
        return out

    want = run(60, True)
    for _ in range(3):
        assert all(torch.equal(x, y) for x, y in zip(run(60, False), want))


# rows, features, dtype: a few lanes, whole vectors, short ones, several warps, a cluster of blocks
ENDS = [(9, 24, "f32"), (50, 1000, "f32"), (33, 203, "f32"), (5, 4096, "bf16"), (3, 20001, "f32"), (2, 32768, "bf16")]


def _check_norm_alone(b, x, kind, eps, dtype, what):
    eps = float(np.float32(eps))
    none, y, stats = b.adasum_residual_norm(None, x, pre_norm=kind, eps=eps, want_h=False)
    want, bound, mean, dmean, rstd, drstd = ref.norm(to64(x), 0 * to64(x), kind, eps)
    _close(y, (want, bound), dtype, f"{what} y")
    if kind == "layer":
        # a rounding below fp32's normal values is off by half their step, 2^-150, once in the mean and once in its sum
        assert_close(to64(stats[2]), mean, 1.1 * dmean + 2 * ref.U * np.abs(mean) + 2.0**-149, f"{what} mean")
    assert_close(to64(stats[3]), rstd, 1.1 * drstd + 2 * ref.U * rstd, f"{what} rstd")
    return stats


@pytest.mark.parametrize("shape", ENDS, ids=lambda s: "-".join(map(str, s)))
@pytest.mark.parametrize("kind", ["rms", "layer"])
@pytest.mark.parametrize("size", [1e-15, 1e-18, 1e-20, 1e-22, 1e-25, 1e-36, 1e18, 1e22, 1e36])
def test_rows_whose_squares_leave_the_range(b, size, kind, shape):
    """Without eps, and with one that fp32 holds as a subnormal: sums of squares that are too small or too large for fp32,
    and (1e36, layer) sums of the values that are too large, give what the formula gives, and so do the gradients."""
    rows, features, dtype = shape
    gen = _gen(12)
    x = (_matrix(gen, rows, features, "f32", mean=3.0 if size > 1 else 0.3).double() * size).to(TORCH[dtype])
    for eps in (0.0, 1e-40):
        stats = _check_norm_alone(b, x, kind, eps, dtype, f"eps {eps}")
    dy = _matrix(gen, rows, features, dtype)
    _, dr = b.adasum_residual_norm_grad(None, x, stats, dy, None, pre_norm=kind, want_x=False)
    o = dict(post_norm="none", pre_norm=kind, pre_weight=1.0, pre_bias=0.0, gate=None, branch_scale=1.0, residual_scale=1.0)
    _close(dr, ref.joint_grad(None, to64(x), to64(stats), to64(dy), None, o, None)["residual"], dtype, "gradient")


@pytest.mark.parametrize("shape", ENDS, ids=lambda s: "-".join(map(str, s)))
def test_rows_of_all_sizes_side_by_side(b, shape):
    """Rows of one warp or block that need no other scale, a larger and a smaller one; a row of zeros without eps is no
    number; one of the smallest subnormals, whose rstd fp32 cannot hold, still has its normalised values."""
    _, features, dtype = shape
    gen = _gen(13)
    sizes = torch.tensor([1.0, 1e-25, 1e25, 1e-22, 0.0, 1e-3, 1e-36, 1e30, 1.0], dtype=torch.float64, device="cuda")
    x = (_matrix(gen, 9, features, "f32").double() * sizes[:, None]).to(TORCH[dtype])
    some = sizes != 0
    for kind in ("rms", "layer"):
        none, y, stats = b.adasum_residual_norm(None, x, pre_norm=kind, eps=0.0, want_h=False)
        assert torch.isnan(y[~some]).all()
        want, bound, *_ = ref.norm(to64(x[some]), 0 * to64(x[some]), kind, 0.0)
        _close(y[some], (want, bound), dtype, kind)
    steps = torch.randint(1, 100, (9, features), generator=gen, device="cuda").double()
    x = (steps * (2.0**-149 if dtype == "f32" else 2.0**-133)).to(TORCH[dtype])
    none, y, stats = b.adasum_residual_norm(None, x, eps=0.0, want_h=False)
    want, bound, *_ = ref.norm(to64(x), 0 * to64(x), "rms", 0.0)
    _close(y, (want, bound), dtype, "subnormal")


@pytest.mark.parametrize("eps", [2.0**-68, 2.0**-66, 2.0**-64, 1e-12])
def test_small_rows_beside_eps(b, eps):
    """Rows from far above eps to far below it."""
    gen = _gen(14)
    for size in (2.0**-20, 2.0**-33, 2.0**-45, 2.0**-52, 2.0**-60, 2.0**-80):
        x = _matrix(gen, 20, 1000, "f32", mean=0.3) * size
        for kind in ("rms", "layer"):
            _check_norm_alone(b, x, kind, eps, "f32", f"{size} {kind}")


@pytest.mark.parametrize("features", [24, 203, 1024, 4096])
def test_small_branches_behind_a_norm(b, features):
    """The norm after the block has the same range as the one before the next."""
    gen = _gen(15)
    for size in (1e-25, 1e-36, 1e25):
        x, r = _matrix(gen, 17, features, "f32", mean=0.3) * size, _matrix(gen, 17, features, "f32")
        for post in ("rms", "layer"):
            h, y, stats = b.adasum_residual_norm(x, r, post_norm=post, pre_norm="rms", eps=0.0)
            o = dict(post_norm=post, post_weight=1.0, post_bias=0.0, pre_norm="rms", pre_weight=1.0, pre_bias=0.0, eps=0.0, gate=None,
                     rows_per_gate=None, branch_scale=1.0, residual_scale=1.0)
            want = ref.joint(to64(x), to64(r), o, (np.ones((17, features), bool), 1.0))
            _close(h, want["h"], "f32", f"{size} {post} h")
            _close(y, want["y"], "f32", f"{size} {post} y")


def test_offsets_beyond_32_bits(b):
    """Rows past element 2^31 of every matrix: the same bits as calls on those rows alone."""
    rows, features, tail = (1 << 21) + 2000, 1024, 3000
    x = torch.empty(rows, features, dtype=torch.bfloat16, device="cuda").normal_(generator=_gen(16))
    weight, gates = torch.rand(features, device="cuda") + 0.5, torch.rand(-(-rows // 1000), features, device="cuda")
    call = dict(post_norm="rms", post_weight=weight, pre_norm="layer", pre_weight=weight, eps=EPS)
    h, y, stats = b.adasum_residual_norm(x, x, gate=gates, rows_per_gate=1000, **call)
    first = rows - tail - rows % 1000                        # a gate row's first
    part, gate = x[first:], gates[first // 1000:].contiguous()
    h2, y2, stats2 = b.adasum_residual_norm(part, part, gate=gate, rows_per_gate=1000, **call)
    assert torch.equal(h[first:], h2) and torch.equal(y[first:], y2) and torch.equal(stats[:, first:], stats2)
    grad_gate, grad_gate2 = torch.empty_like(gates), torch.empty_like(gate)
    dx, dr = b.adasum_residual_norm_grad(x, h, stats, y, x, gate=gates, rows_per_gate=1000, grad_gate=grad_gate, **call)
    dx2, dr2 = b.adasum_residual_norm_grad(part, h2, stats2, y2, part, gate=gate, rows_per_gate=1000, grad_gate=grad_gate2, **call)
    assert torch.equal(dx[first:], dx2) and torch.equal(dr[first:], dr2)
    # a gate row's sum is cut in other places: twice 1000 terms with a rounding each and a few for the parts.  A term is the
    # gradient of h (that of the residual before its rounding to bf16, 2^-8) times the branch behind its norm
    n = part.double() * stats2[1].double()[:, None] * weight.double()
    size = torch.stack([t.sum(0) for t in (dr2.double() * n).abs().split(1000)]) * (1 + 2.0**-7)
    assert ((grad_gate[first // 1000:].double() - grad_gate2.double()).abs() <= 2 * 1010 * ref.U * size).all()
