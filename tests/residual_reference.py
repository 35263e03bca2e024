"""Plain forms in 64 bits of the operators around a residual block's linear layers (numpy, from the formulas), with bounds
of what fp32 arithmetic may be off.  Bounds are first order: U = 2^-24 relative per operation; a sum of F values is
formed by eight additions per thread, five shuffles, up to four more between warps and eight between blocks, less
than SUM = 32 roundings on any value's way."""
import numpy as np

U = 2.0**-24
SUM = 32
# kernel's 1 / sqrt: an approximation (2^-22) with a Newton step (its square, and three roundings)
ROOT = 4 * U
M32 = 0xffffffff


def philox(key, counter):
    """Philox4x32-10 of one counter: four words, in plain integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & M32, (a >> 32) ^ c[3] ^ k[1], a & M32]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return c


def kept(rows, features, p, seed, site, first_row=0):
    """Which elements dropout keeps, and the factor of those; all of them for t = 0."""
    t = int(np.floor(np.float32(p) * 65536 + 0.5))
    if t == 0:
        return np.ones((rows, features), bool), 1.0
    per_row = -(-features // 8)
    n = (np.uint64(first_row * per_row) + np.arange(rows * per_row, dtype=np.uint64))
    u = np.uint64
    c = [n & u(M32), n >> u(32), np.full(n.shape, site & M32, u), np.full(n.shape, site >> 32, u)]
    k = [seed & M32, (seed >> 32) & M32]
    for _ in range(10):
        a, b = c[0] * u(0xD2511F53), c[2] * u(0xCD9E8D57)
        c = [(b >> u(32)) ^ c[1] ^ u(k[0]), b & u(M32), (a >> u(32)) ^ c[3] ^ u(k[1]), a & u(M32)]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    halves = np.stack([w >> u(16 * i) & u(0xffff) for w in c for i in (0, 1)], axis=1)
    keep = halves.reshape(rows, -1)[:, :features] >= t
    return keep, 65536 / (65536 - t) if t < 65536 else 0.0


def dropped(x, mask):
    keep, factor = mask
    return np.where(keep, x * factor, 0.0)


def norm(x, dx, kind, eps, weight=1.0, bias=0.0):
    """(result, its bound, mean, bound, rstd, bound) of a norm of x, known up to dx."""
    zero = np.zeros((x.shape[0], 1))
    m = x.mean(1, keepdims=True) if kind == "layer" else zero
    dm = dx.mean(1, keepdims=True) + SUM * U * np.abs(x).mean(1, keepdims=True) if kind == "layer" else zero
    c = x - m
    dc = dx + dm + U * np.abs(c)
    var = (c * c).mean(1, keepdims=True)
    dvar = (2 * np.abs(c) * dc + dc * dc).mean(1, keepdims=True) + (SUM + 4) * U * (var + eps)
    rstd = 1 / np.sqrt(var + eps)
    rho = 0.5 * dvar / (var + eps) + 0.375 * (dvar / (var + eps)) ** 2 * 2 + ROOT
    u = c * rstd
    du = (dc * rstd) * (1 + rho) + np.abs(u) * (rho + U)
    y = u * weight + bias
    return y, du * np.abs(weight) + U * (np.abs(y) + np.abs(u * weight)), m[:, 0], dm[:, 0], rstd[:, 0], (rho * rstd)[:, 0]


def gates(gate, rows, rows_per_gate):
    return 1.0 if gate is None else gate[np.arange(rows) // rows_per_gate]


def joint(x, residual, o, mask):
    """The forward pass: values and bounds.  o: the call's options, arrays in 64 bits."""
    out = {}
    like = x if x is not None else residual
    branch, d = np.zeros_like(like), np.zeros_like(like)
    if x is not None:
        branch = x
        if o["post_norm"] != "none":
            branch, d, *out["post"] = norm(x, d, o["post_norm"], o["eps"], o["post_weight"], o["post_bias"])
        keep, factor = mask
        d = np.where(keep, d * factor + 2 * U * np.abs(branch * factor), 0.0)
        branch = dropped(branch, mask)
        scale = o["branch_scale"] * gates(o["gate"], x.shape[0], o["rows_per_gate"])
        branch, d = branch * scale, d * np.abs(scale) + 3 * U * np.abs(branch * scale)
    h = branch + (0.0 if residual is None else o["residual_scale"] * residual)
    d = d + U * np.abs(h)
    out["h"] = h, d
    if o["pre_norm"] != "none":
        y, dy, *out["pre"] = norm(h, d, o["pre_norm"], o["eps"], o["pre_weight"], o["pre_bias"])
        out["y"] = y, dy
    return out


def _normalised(x, mean, rstd):
    u = (x - mean) * rstd
    return u, 3 * U * (np.abs(x) + np.abs(mean)) * rstd


def _back(kind, u, du, rstd, v, dv):
    f = u.shape[1]
    s = (u * v).sum(1, keepdims=True) / f
    ds = ((du * np.abs(v) + np.abs(u) * dv) + (SUM + 2) * U * np.abs(u * v)).sum(1, keepdims=True) / f
    t = v.sum(1, keepdims=True) / f if kind == "layer" else 0.0 * s
    dt = (dv + (SUM + 2) * U * np.abs(v)).sum(1, keepdims=True) / f if kind == "layer" else 0.0 * s
    d = rstd * (v - t - u * s)
    return d, rstd * (dv + dt + du * np.abs(s) + np.abs(u) * ds + 5 * U * (np.abs(v) + np.abs(t) + np.abs(u * s)))


def _columns(terms, bound):
    """A sum over the rows: at most as many roundings as rows (and a few)."""
    return terms.sum(0), (bound + (terms.shape[0] + 4) * U * np.abs(terms)).sum(0)


def joint_grad(x, h, stats, grad_y, grad_h, o, mask):
    """Gradients and bounds, from the forward pass's results as they were kept."""
    out = {}
    post_mean, post_rstd, pre_mean, pre_rstd = stats[:, :, None]
    like = grad_y if grad_y is not None else grad_h
    d = np.zeros_like(like) if grad_h is None else grad_h
    e = np.zeros_like(d)
    if grad_y is not None:
        mean = pre_mean if o["pre_norm"] == "layer" else 0 * pre_mean
        u, du = _normalised(h, mean, pre_rstd)
        out["pre_weight"] = _columns(grad_y * u, np.abs(grad_y) * du)
        out["pre_bias"] = _columns(grad_y, 0.0)
        v = grad_y * o["pre_weight"]
        back, eb = _back(o["pre_norm"], u, du, pre_rstd, v, U * np.abs(v))
        d, e = d + back, eb + U * np.abs(d + back)
    out["residual"] = d * o["residual_scale"], abs(o["residual_scale"]) * (e + U * np.abs(d))
    d, e = d * o["branch_scale"], abs(o["branch_scale"]) * (e + U * np.abs(d))
    if x is None:
        return out
    keep, factor = mask
    n, en, u, du = x, 0.0 * x, x, 0.0 * x
    if o["post_norm"] != "none":
        mean = post_mean if o["post_norm"] == "layer" else 0 * post_mean
        u, du = _normalised(x, mean, post_rstd)
        n = u * o["post_weight"] + o["post_bias"]
        en = du * np.abs(o["post_weight"]) + U * (np.abs(n) + np.abs(u * o["post_weight"]))
    if o["gate"] is not None:
        n, en = dropped(n, mask), np.where(keep, factor * (en + 2 * U * np.abs(n)), 0.0)
        terms, bound = d * n, e * np.abs(n) + np.abs(d) * en
        row = np.arange(x.shape[0]) // o["rows_per_gate"]
        parts = [_columns(terms[row == g], bound[row == g]) for g in range(o["gate"].shape[0])]
        out["gate"] = np.stack([p[0] for p in parts]), np.stack([p[1] for p in parts])
        g = gates(o["gate"], x.shape[0], o["rows_per_gate"])
        d, e = d * g, e * np.abs(g) + U * np.abs(d * g)
    d, e = dropped(d, mask), np.where(keep, factor * (e + 2 * U * np.abs(d)), 0.0)
    if o["post_norm"] != "none":
        out["post_weight"] = _columns(d * u, e * np.abs(u) + np.abs(d) * du)
        out["post_bias"] = _columns(d, e)
        v = d * o["post_weight"]
        d, e = _back(o["post_norm"], u, du, post_rstd, v, e * np.abs(o["post_weight"]) + U * np.abs(v))
    out["x"] = d, e
    return out


# ---- packed 8-bit matrices ----------------------------------------------------------------------------

def fp8_pack(x, weight=False):
    """Codes [rows, W] and step bytes [rows, W / 128] of x (float64)."""
    rows, columns = x.shape
    wide, high = -(-columns // 128), 128 if weight else 1
    v = np.zeros((-(-rows // high) * high, wide * 128))
    v[:rows, :columns] = x
    v = v.reshape(-1, high, wide, 128)
    bad = ~np.isfinite(v).all(axis=(1, 3))
    top = np.where(bad, 0.0, np.abs(np.where(np.isfinite(v), v, 0.0)).max(axis=(1, 3)))
    fraction, exponent = np.frexp(top)                       # top = fraction * 2^exponent, fraction in [0.5, 1)
    step = exponent - 9 + (fraction > 0.875)                 # 448 = 0.875 * 2^9
    step = np.maximum(np.where(top > 0, step, -1000), -126)
    scaled = np.where(bad[:, None, :, None], 0.0, np.ldexp(np.where(np.isfinite(v), v, 0.0), -step[:, None, :, None]))
    # four significant bits, at least 2^-9; rint takes ties to even
    place = np.maximum(np.frexp(scaled)[1] - 4, -9)
    value = np.ldexp(np.rint(np.ldexp(scaled, -place)), place)
    magnitude = np.abs(value)
    e = np.maximum(np.frexp(magnitude)[1] - 1, -6)           # of a normal code; subnormals share -6
    mantissa = np.ldexp(magnitude, 3 - e).astype(np.int64)   # 8 .. 15 with the hidden bit, below 8 for subnormals
    codes = np.where(mantissa >= 8, ((e + 7) << 3) + mantissa - 8, mantissa) | (np.signbit(scaled) << 7)
    step_bytes = np.repeat(np.where(bad, 255, step + 127), high, axis=0)[:rows]
    return codes.reshape(v.shape[0] * high, -1)[:rows].astype(np.uint8), step_bytes.astype(np.uint8)


def fp8_values(codes, steps, columns):
    magnitude, sign = (codes & 127).astype(np.int64), np.where(codes >> 7, -1.0, 1.0)
    e, m = magnitude >> 3, magnitude & 7
    v = sign * np.where(e > 0, np.ldexp(8.0 + m, e - 10), np.ldexp(1.0 * m, -9))
    step = np.where(steps == 255, np.nan, np.ldexp(1.0, steps.astype(np.int64) - 127))
    return (v.reshape(codes.shape[0], -1, 128) * step[:, :, None]).reshape(codes.shape)[:, :columns]


def fp8_buffer(codes, steps):
    """The packed bytes; step bytes of rows beyond the matrix are 0."""
    rows, wide = steps.shape
    up = -(-rows // 128)
    full = np.zeros((up * 128, wide), np.uint8)
    full[:rows] = steps
    area = np.zeros((up, wide, 32, 4, 4), np.uint8)
    area[...] = full.reshape(up, 4, 32, wide).transpose(0, 3, 2, 1)[..., None]
    return np.concatenate((codes.reshape(-1), area.reshape(-1)))
