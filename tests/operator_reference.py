"""Plain forms in 64 bits of the operators that produce a worker's gradients (numpy, from the formulas)."""
import numpy as np
import torch

GROUP = 32
TORCH = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
# half a unit in the last place, relative: the error of one rounding to the type
UNIT = {"f32": 2.0**-24, "f16": 2.0**-11, "bf16": 2.0**-8}
# half the smallest subnormal: the absolute error of one rounding near zero
TINY = {"f32": 2.0**-150, "f16": 2.0**-25, "bf16": 2.0**-134}


def to64(t):
    return t.detach().double().cpu().numpy()


def keep(x):
    """Codes [rows, W] and step exponents [rows, W / 32] (None: the group is kept as NaN) of x, a float64 array."""
    rows, features = x.shape
    width = -(-features // GROUP) * GROUP
    v = np.zeros((rows, width))
    v[:, :features] = x
    v = v.reshape(rows, width // GROUP, GROUP)
    bad = ~np.isfinite(v).all(axis=2)
    v[bad] = 0.0
    top = np.abs(v).max(axis=2)
    exponent = np.frexp(np.where(top > 0, top, 1.0))[1] - 1
    exponent = np.maximum(np.where(top > 0, exponent, -1000) - 6, -126)
    codes = np.clip(np.rint(np.ldexp(v, -exponent[:, :, None])), -127, 127).reshape(rows, width)
    return codes.astype(np.int8), np.where(bad, 255, exponent + 127).astype(np.uint8)


def pack(codes, steps):
    return np.concatenate((codes.view(np.uint8).reshape(-1), steps.reshape(-1)))


def kept_values(codes, steps, features):
    rows, width = codes.shape
    step = np.where(steps == 255, np.nan, np.ldexp(1.0, steps.astype(np.int64) - 127))
    return (codes.reshape(rows, width // GROUP, GROUP) * step[:, :, None]).reshape(rows, width)[:, :features]


def normal_cdf(x):
    # erfc, not 1 + erf: the lower tail to full relative precision
    return torch.erfc(torch.from_numpy(np.ascontiguousarray(x)) * -np.sqrt(0.5)).numpy() / 2


def _tanh_parts(x):
    z = 2 * np.sqrt(2 / np.pi) * (x + 0.044715 * x**3)
    s = 1 / (1 + np.exp(-z))
    return z, s, 1 / (1 + np.exp(z)), 2 * np.sqrt(2 / np.pi) * (1 + 0.134145 * x**2)


@np.errstate(over="ignore", invalid="ignore", under="ignore")
def act(x, name):
    if name == "relu":
        return np.where(x > 0, x, 0.0)
    if name == "gelu":
        return x * normal_cdf(x)
    if name == "gelu_tanh":
        return x * _tanh_parts(x)[1]
    if name == "silu":
        return x / (1 + np.exp(-x))
    return x


@np.errstate(over="ignore", invalid="ignore", under="ignore")
def act_slope(x, name):
    """The slope and the sum of its terms' magnitudes (what rounding errors scale with)."""
    if name == "relu":
        return (x > 0) * 1.0, (x > 0) * 1.0
    if name == "gelu":
        a, b = normal_cdf(x), x * np.exp(-x * x / 2) / np.sqrt(2 * np.pi)
    elif name == "gelu_tanh":
        _, a, rest, dz = _tanh_parts(x)
        b = x * a * rest * dz
    elif name == "silu":
        a = 1 / (1 + np.exp(-x))
        b = x * a / (1 + np.exp(x))
    else:
        return np.ones_like(x), np.ones_like(x)
    return a + b, np.abs(a) + np.abs(b)


@np.errstate(over="ignore")
def act_error(x, name, dtype):
    """Relative error of the terms above in fp32 arithmetic: a few units of the functions (erfcf, expf: 4
    units; the fits and approximations for 16-bit results: 1e-5), and the rounding of the exponent's argument z
    (three operations), which the exponential turns into a relative error of |z| units each."""
    z = {"gelu": x * x / 2, "gelu_tanh": np.abs(_tanh_parts(x)[0]), "silu": np.abs(x)}.get(name, 0.0 * x)
    return (2.0**-20 if dtype == "f32" else 1.5e-5) + 4 * z * 2.0**-24


def embedding_grad(dy, ids, num_rows, scale):
    """The gradient, and per element the error bound of an fp32 sum in any order: (terms + 1) units of the sum of magnitudes."""
    out, size, count = np.zeros((num_rows, dy.shape[1])), np.zeros((num_rows, dy.shape[1])), np.zeros((num_rows, 1))
    ok = (ids >= 0) & (ids < num_rows)
    np.add.at(out, ids[ok], dy[ok])
    np.add.at(size, ids[ok], np.abs(dy[ok]))
    np.add.at(count, ids[ok], 1.0)
    return out * scale, (count + 1) * 2.0**-24 * size * abs(scale)


def assert_close(got, want, bound, what=""):
    assert got.shape == want.shape, (got.shape, want.shape)
    nan = np.isnan(want)
    assert np.array_equal(np.isnan(got), nan), f"{what}: NaN in other places"
    inf = np.isinf(want)
    assert np.array_equal(got[inf], want[inf]), f"{what}: Inf in other places"
    fine = ~nan & ~inf
    off = np.abs(got - want)[fine] - np.broadcast_to(bound, want.shape)[fine]
    assert off.size == 0 or off.max() <= 0, f"{what}: {(off > 0).sum()} of {off.size} values, worst by {off.max():.3e}"
