"""Cases of the operators around a linear layer of a worker's residual block, and their plain forms.

Six kinds of pass are covered:

    dropout     out = [residual +] keep * x / (1 - q), the mask formed from (seed, site, row, column) and never stored
    join        h = residual_scale * residual + branch_scale * gate * dropout(post(x)),  y = pre(h)
    join_grad   gradients of x, of the residual, of both norms' weights and biases and of the gate
    pack        a weight matrix in 8 bits: e4m3 codes, a power of two for every 128 x 128 block
    linear      y = x8 w8^T + bias: x packed on the way, with a power of two for 128 neighbouring features of a row
    linear_grad dx = dy8 w8, dy packed the same way, the same packed weights

post and pre are "none", "rms" (x / sqrt(mean(x^2) + eps) * weight) or "layer" ((x - mean) / sqrt(var + eps) *
weight + bias).  Row r takes row r // rows_per_gate of the gate.

Dropout: t = round(65536 p), q = t / 65536.  Eight neighbouring columns of a row share the 128 random bits of
Philox4x32-10 (Salmon et al., "Parallel random numbers: as easy as 1, 2, 3", 2011) with the key (low, high half of
seed) and the counter (low, high half of n; low, high half of site), n = row * ceil(columns / 8) + column // 8.
Column c takes bits 16 (c % 2) .. + 15 of word (c % 8) // 2 and is kept if they are at least t.

Packed matrices hold, with W = 128 * ceil(columns / 128), first rows x W codes, row by row (zeros beyond the
matrix), then for every block of 128 rows and every 128 columns 512 bytes: the step byte (exponent + 127) of row r at
16 * (r % 32) + 4 * (r % 128 // 32), four times.  The step is the smallest power of two, 2^-126 at least, by
which a block's largest magnitude is at most 448; a block with an Inf or NaN has step byte 255 and codes 0.
"""
import math

import numpy as np
import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}
BLOCK = 128


# ---- the cases -------------------------------------------------------------------------------------

def listed():
    return [
        # the hidden states of 32 sequences of 512 on their way into the residual stream
        {"name": "dropout, 16384 x 1024", "kind": "dropout", "rows": 16384, "features": 1024, "type": "bf16",
         "p": 0.1, "residual": True, "slack": 0},
        # the gradient of one short odd sequence in fp32, columns of a wider matrix
        {"name": "dropout, 61 x 1023", "kind": "dropout", "rows": 61, "features": 1023, "type": "f32",
         "p": 0.1, "residual": False, "slack": 1},
        # the end of a layer of 32 sequences of 512: dropout, residual, LayerNorm
        {"name": "join, 16384 x 1024", "kind": "join", "rows": 16384, "features": 1024, "type": "bf16",
         "stream": "bf16", "params": "f32", "post": "none", "pre": "layer", "gate": 0, "p": 0.1, "slack": 0},
        # the next token of one sequence, norms on both sides of the block and a gate per channel: nothing but latency
        {"name": "join, one token", "kind": "join", "rows": 1, "features": 1024, "type": "bf16",
         "stream": "bf16", "params": "bf16", "post": "rms", "pre": "rms", "gate": 1, "p": 0.0, "slack": 0},
        # the first case's way back
        {"name": "join_grad, 16384 x 1024", "kind": "join_grad", "rows": 16384, "features": 1024, "type": "bf16",
         "stream": "bf16", "params": "f32", "post": "none", "pre": "layer", "gate": 0, "p": 0.1, "slack": 0},
        # wide rows, 8 sequences of 512 with a gate each, norms on both sides, residual stream in fp32
        {"name": "join_grad, 4096 x 4096", "kind": "join_grad", "rows": 4096, "features": 4096, "type": "bf16",
         "stream": "f32", "params": "f32", "post": "rms", "pre": "rms", "gate": 512, "p": 0.0, "slack": 0},
        # a small odd model in fp32 with a gate per channel: nothing is a multiple of anything
        {"name": "join_grad, odd sizes", "kind": "join_grad", "rows": 999, "features": 203, "type": "f32",
         "stream": "f32", "params": "f32", "post": "layer", "pre": "layer", "gate": 1, "p": 0.25, "slack": 5},
        # first feed-forward matrix of BERT-Large, once per optimizer step from the fp32 master weights
        {"name": "pack, 4096 x 1024", "kind": "pack", "rows": 4096, "features": 1024, "type": "f32", "slack": 0},
        # the first feed-forward layer of 32 sequences of 512
        {"name": "linear, 16384 tokens", "kind": "linear", "rows": 16384, "features": 1024, "outputs": 4096,
         "type": "bf16", "out": "bf16", "bias": True, "slack": 0},
        # a few odd tokens: the weights' bytes and latency
        {"name": "linear, 37 tokens", "kind": "linear", "rows": 37, "features": 1024, "outputs": 4096,
         "type": "bf16", "out": "bf16", "bias": True, "slack": 0},
        # the first feed-forward layer's way back to its input
        {"name": "linear_grad, 16384 tokens", "kind": "linear_grad", "rows": 16384, "features": 1024, "outputs": 4096,
         "type": "bf16", "out": "bf16", "slack": 0},
        # a small odd layer in fp32
        {"name": "linear_grad, odd sizes", "kind": "linear_grad", "rows": 333, "features": 1000, "outputs": 257,
         "type": "f32", "out": "f32", "slack": 3},
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], spread over its logarithm; every other one a multiple of 8."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if n >= 16 and rng.random() < 0.5:
        n -= n % 8
    return max(low, min(high, n))


def draw(rng):
    kind = rng.choice(["dropout", "join", "join_grad", "pack", "linear", "linear_grad"])
    slack = rng.choice([0, 0, 1, 8, 24])
    types = ["f32", "f16", "bf16"]
    if kind == "pack":
        features = _spread(rng, 1, 8192)
        return {"kind": kind, "rows": min(_spread(rng, 1, 8192), (1 << 24) // features), "features": features,
                "type": rng.choice(types), "slack": slack}
    if kind in ("linear", "linear_grad"):
        features, outputs = _spread(rng, 1, 8192), _spread(rng, 1, 8192)
        rows = min(_spread(rng, 1, 16384), (1 << 36) // (features * outputs), (1 << 26) // max(features, outputs))
        case = {"kind": kind, "rows": rows, "features": features, "outputs": outputs, "type": rng.choice(types),
                "out": rng.choice(types), "slack": slack}
        if kind == "linear":
            case["bias"] = rng.random() < 0.5
        return case
    features = _spread(rng, 1 if kind == "dropout" else 16, 8192)
    rows = min(_spread(rng, 1, 32768), (1 << 24) // features)
    case = {"kind": kind, "rows": rows, "features": features, "type": rng.choice(types), "slack": slack,
            "p": rng.choice([0.0, 0.1, 0.25])}
    if kind == "dropout":
        case["p"] = rng.choice([0.05, 0.1, 0.5])
        case["residual"] = rng.random() < 0.5
        return case
    case["stream"] = rng.choice([case["type"], "f32"])
    case["params"] = rng.choice([case["type"], "f32"])
    case["post"] = rng.choice(["none", "rms", "layer"])
    case["pre"] = rng.choice(["rms", "layer"])
    # no gate, one for all rows, or one for as many rows as a sequence has
    case["gate"] = rng.choice([0, 1, _spread(rng, 2, 2048)])
    return case


def _gate_rows(case):
    return 0 if case["gate"] == 0 else 1 if case["gate"] == 1 else -(-case["rows"] // case["gate"])


def work(case):
    kind, rows, features = case["kind"], case["rows"], case["features"]
    n = rows * features
    if kind == "dropout":
        return {"bytes": n * BYTES[case["type"]] * (3 if case["residual"] else 2), "flops": 2 * n}
    if kind == "pack":
        return {"bytes": n * (BYTES[case["type"]] + 1), "flops": 2 * n}
    if kind in ("linear", "linear_grad"):
        outputs = case["outputs"]
        read, written = (features, outputs) if kind == "linear" else (outputs, features)
        return {"bytes": rows * read * BYTES[case["type"]] + features * outputs + rows * written * BYTES[case["out"]],
                "flops": 2 * n * outputs}
    t, s = BYTES[case["type"]], BYTES[case["stream"]]
    vectors = features * BYTES[case["params"]] * ((case["post"] != "none") + (case["pre"] != "none"))
    gate = _gate_rows(case) * features * t
    if kind == "join":           # x and the residual read, h and y written
        return {"bytes": n * 2 * (t + s) + vectors + gate, "flops": 16 * n}
    # x, h and the gradients of y and h read; the gradients of x and of the residual written
    reads_x = case["post"] != "none" or case["gate"] > 0
    return {"bytes": n * ((3 if reads_x else 2) * t + 3 * s) + 2 * vectors + 2 * gate, "flops": 30 * n}


# ---- inputs ----------------------------------------------------------------------------------------

def _matrix(gen, rows, cols, slack, dtype, size=1.0):
    """Normal values, a few columns much larger than the rest (as activations have them); with slack, the
    first columns of a wider matrix."""
    wide = torch.empty(rows, cols + slack, dtype=torch.float32, device="cuda").normal_(generator=gen)
    loud = torch.rand(cols + slack, generator=gen, device="cuda") < 0.01
    wide.mul_(torch.where(loud, 12.0 * size, size))
    return wide.to(dtype)[:, :cols]


def _gradient_size(case):
    """fp16 gradients are kept multiplied by a scale that holds them inside the type's range."""
    return 1.0 if "f16" in (case["type"], case.get("out"), case.get("stream")) else 0.01


def _vector(gen, n, dtype, mean, size):
    return (torch.empty(n, device="cuda").normal_(generator=gen) * size + mean).to(dtype)


EPS = 1e-5


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind, rows, features, dtype = case["kind"], case["rows"], case["features"], TYPES[case["type"]]
    slack = case["slack"]
    state = {"case": case}
    if kind in ("dropout", "join", "join_grad"):
        # one number per optimizer step on the GPU; the place in the model tells a step's masks apart
        state["seed"] = torch.randint(0, 2**63 - 1, (1,), generator=gen, device="cuda", dtype=torch.int64)
        state["site"] = 5 + (seed & 0xffff)
    if kind == "dropout":
        state["x"] = _matrix(gen, rows, features, slack, dtype)
        state["residual"] = _matrix(gen, rows, features, slack, dtype) if case["residual"] else None
        return state
    if kind == "pack":
        state["x"] = _matrix(gen, rows, features, slack, dtype, 0.03)
        return state
    if kind in ("linear", "linear_grad"):
        outputs = case["outputs"]
        forward = kind == "linear"
        state["w"] = _pack(_matrix(gen, outputs, features, 0, torch.float32, 0.03), True)
        state["x"] = _matrix(gen, rows, features if forward else outputs, slack, dtype,
                             1.0 if forward else _gradient_size(case))
        state["bias"] = _vector(gen, outputs, dtype, 0.0, 0.1) if forward and case["bias"] else None
        return state
    stream, params = TYPES[case["stream"]], TYPES[case["params"]]
    state["x"] = _matrix(gen, rows, features, slack, dtype)
    state["residual"] = _matrix(gen, rows, features, slack, stream)
    for norm in ("post", "pre"):
        state[norm + "_weight"] = _vector(gen, features, params, 1.0, 0.2) if case[norm] != "none" else None
        state[norm + "_bias"] = _vector(gen, features, params, 0.0, 0.2) if case[norm] == "layer" else None
    state["gate"] = _vector(gen, _gate_rows(case) * features, dtype, 0.5, 0.3).view(-1, features) if case["gate"] else None
    state["rows_per_gate"] = rows if case["gate"] == 1 else case["gate"]
    state["branch_scale"], state["residual_scale"] = 0.75, 1.25
    if kind == "join_grad":      # what the forward pass has left
        state["scale"] = 0.5
        out = _join(state)
        wide = torch.zeros(rows, features + slack, dtype=stream, device="cuda")
        wide[:, :features] = out["h"]
        state["h"] = wide[:, :features]
        none = torch.zeros(rows, device="cuda")
        state["stats"] = torch.stack([out.get(k, none) for k in ("post_mean", "post_rstd", "pre_mean", "pre_rstd")])
        state["dy"] = _matrix(gen, rows, features, slack, dtype, _gradient_size(case))
        state["dh"] = _matrix(gen, rows, features, slack, stream, _gradient_size(case))
        del state["residual"]
        # the parameters' places in the worker's fused buffer, and the gate's gradient
        for name in ("post_weight", "post_bias", "pre_weight", "pre_bias"):
            state["d" + name] = None if state[name] is None else torch.zeros(features, device="cuda")
        state["dgate"] = None if state["gate"] is None else torch.zeros(state["gate"].shape, device="cuda")
    return state


# ---- the plain forms -------------------------------------------------------------------------------

M32 = 0xffffffff


def _kept(state, rows, features):
    """keep / (1 - q) of every element, or None without dropout."""
    t = int(round(state["case"]["p"] * 65536))
    if t == 0:
        return None
    per_row = -(-features // 8)
    n = torch.arange(rows * per_row, device="cuda", dtype=torch.int64)
    site = state["site"]
    c0, c1 = n & M32, n >> 32
    c2, c3 = torch.full_like(n, site & M32), torch.full_like(n, site >> 32)
    k0, k1 = state["seed"] & M32, (state["seed"] >> 32) & M32
    for _ in range(10):
        p0, p1 = c0 * 0xD2511F53, c2 * 0xCD9E8D57        # their 64 bits, whatever the sign
        c0, c1, c2, c3 = ((p1 >> 32) & M32) ^ c1 ^ k0, p1 & M32, ((p0 >> 32) & M32) ^ c3 ^ k1, p0 & M32
        k0, k1 = (k0 + 0x9E3779B9) & M32, (k1 + 0xBB67AE85) & M32
    words = torch.stack((c0 & 0xffff, c0 >> 16, c1 & 0xffff, c1 >> 16, c2 & 0xffff, c2 >> 16, c3 & 0xffff, c3 >> 16), dim=1)
    keep = words.view(rows, per_row * 8)[:, :features] >= t
    return torch.where(keep, 65536.0 / (65536 - t), 0.0)


def _dropped(x, kept):
    return x if kept is None else torch.where(kept > 0, x * kept, 0.0)


def _normed(state, x, norm):
    """(mean, rstd, normalised x, the norm's result) in 32 bits."""
    kind = state["case"][norm]
    mean = x.mean(dim=1) if kind == "layer" else None
    centred = x if mean is None else x - mean[:, None]
    rstd = 1.0 / torch.sqrt((centred * centred).mean(dim=1) + EPS)
    hat = centred * rstd[:, None]
    out = hat * state[norm + "_weight"].to(torch.float32)
    if state[norm + "_bias"] is not None:
        out = out + state[norm + "_bias"].to(torch.float32)
    return mean, rstd, hat, out


def _gates(state):
    if state["gate"] is None:
        return None
    row = torch.arange(state["case"]["rows"], device="cuda") // state["rows_per_gate"]
    return state["gate"].to(torch.float32)[row]


def _stats(case, norm, mean, rstd):
    return {norm + "_mean": mean, norm + "_rstd": rstd} if case[norm] == "layer" else {norm + "_rstd": rstd}


def _join(state):
    case = state["case"]
    x, residual = state["x"].to(torch.float32), state["residual"].to(torch.float32)
    out = {}
    branch = x
    if case["post"] != "none":
        mean, rstd, _, branch = _normed(state, x, "post")
        out.update(_stats(case, "post", mean, rstd))
    branch = _dropped(branch, _kept(state, *x.shape)) * state["branch_scale"]
    if state["gate"] is not None:
        branch = branch * _gates(state)
    h = residual * state["residual_scale"] + branch
    mean, rstd, _, y = _normed(state, h, "pre")
    out.update(_stats(case, "pre", mean, rstd))
    return {"h": h.to(TYPES[case["stream"]]), "y": y.to(TYPES[case["type"]]), **out}


def _norm_back(kind, hat, rstd, dhat):
    """The gradient of a norm's input from that of the normalised values."""
    inner = dhat - hat * (dhat * hat).mean(dim=1, keepdim=True)
    if kind == "layer":
        inner = inner - dhat.mean(dim=1, keepdim=True)
    return inner * rstd[:, None]


def _join_grad(state):
    case, scale = state["case"], state["scale"]
    f32 = torch.float32
    x, h, dy = state["x"].to(f32), state["h"].to(f32), state["dy"].to(f32)
    post_mean, post_rstd, pre_mean, pre_rstd = state["stats"]
    out = {}

    def vectors(norm, d, hat):
        if state[norm + "_weight"] is not None:
            out[norm + "_weight"] = state["d" + norm + "_weight"].copy_((d * hat).sum(dim=0) * scale)
        if state[norm + "_bias"] is not None:
            out[norm + "_bias"] = state["d" + norm + "_bias"].copy_(d.sum(dim=0) * scale)

    hat = (h - pre_mean[:, None]) * pre_rstd[:, None] if case["pre"] == "layer" else h * pre_rstd[:, None]
    vectors("pre", dy, hat)
    dh = state["dh"].to(f32) + _norm_back(case["pre"], hat, pre_rstd, dy * state["pre_weight"].to(f32))
    kept = _kept(state, *x.shape)
    branch = dh * state["branch_scale"]
    n, hat = x, x
    if case["post"] != "none":
        hat = (x - post_mean[:, None]) * post_rstd[:, None] if case["post"] == "layer" else x * post_rstd[:, None]
        n = hat * state["post_weight"].to(f32)
        if state["post_bias"] is not None:
            n = n + state["post_bias"].to(f32)
    if state["gate"] is not None:
        gates = state["dgate"].shape[0]
        row = torch.arange(case["rows"], device="cuda") // state["rows_per_gate"]
        sums = torch.zeros(gates, case["features"], device="cuda").index_add_(0, row, branch * _dropped(n, kept))
        out["gate"] = state["dgate"].copy_(sums * scale)
        branch = branch * _gates(state)
    branch = _dropped(branch, kept)
    if case["post"] != "none":
        vectors("post", branch, hat)
        branch = _norm_back(case["post"], hat, post_rstd, branch * state["post_weight"].to(f32))
    return {"x": branch.to(state["x"].dtype), "residual": (dh * state["residual_scale"]).to(state["h"].dtype), **out}


def _blocks(x, shared):
    """x filled up to whole blocks: [row blocks, rows, column blocks, 128], and the step bytes of every row and
    column block; shared: one step for 128 rows."""
    rows, cols = x.shape
    high = BLOCK if shared else 1
    up, wide = -(-rows // high) * high, -(-cols // BLOCK) * BLOCK
    v = torch.zeros(up, wide, dtype=torch.float32, device=x.device)
    v[:rows, :cols] = x
    v = v.view(up // high, high, wide // BLOCK, BLOCK)
    top = v.abs().amax(dim=(1, 3)).view(torch.int32)
    step = ((top >> 23) - 8 + ((top & 0x7fffff) > 0x600000)).clamp_(min=1)
    return v, torch.where((top >> 23) == 255, 255, step)


def _codes(v, step):
    back = ((254 - step).clamp_(min=0) << 23).view(torch.float32)
    scaled = v * back[:, None, :, None]
    return torch.where(step[:, None, :, None] == 255, 0.0, scaled).to(torch.float8_e4m3fn)


def _round8(x, shared):
    """The values that x stands for when packed."""
    v, step = _blocks(x, shared)
    values = _codes(v, step).to(torch.float32) * (step << 23).view(torch.float32)[:, None, :, None]
    return values.reshape(v.shape[0] * v.shape[1], -1)[: x.shape[0], : x.shape[1]]


def _pack(x, shared):
    """The packed matrix, in the layout that the module's docstring gives."""
    rows = x.shape[0]
    v, step = _blocks(x, shared)
    codes = _codes(v, step).view(torch.uint8).reshape(v.shape[0] * v.shape[1], -1)[:rows]
    up = -(-rows // BLOCK) * BLOCK
    per_row = step.repeat_interleave(v.shape[1], dim=0).to(torch.uint8)
    full = torch.full((up, step.shape[1]), 127, dtype=torch.uint8, device=x.device)
    full[: per_row.shape[0]] = per_row
    # [row block, r % 128 // 32, r % 32, column block] -> [row block, column block, r % 32, r % 128 // 32, four times]
    full = full.view(up // BLOCK, 4, 32, -1).permute(0, 3, 2, 1).unsqueeze(-1).expand(-1, -1, -1, -1, 4)
    return torch.cat((codes.reshape(-1), full.reshape(-1)))


def _values8(packed, rows, cols):
    """The values of a packed matrix."""
    wide = -(-cols // BLOCK) * BLOCK
    up = -(-rows // BLOCK) * BLOCK
    codes = packed[: rows * wide].view(torch.float8_e4m3fn).view(rows, wide // BLOCK, BLOCK).to(torch.float32)
    step = packed[rows * wide :].view(up // BLOCK, wide // BLOCK, 32, 4, 4)[..., 0].permute(0, 3, 2, 1)
    step = (step.reshape(up, wide // BLOCK)[:rows].to(torch.int32) << 23).view(torch.float32)
    return (codes * step[:, :, None]).view(rows, wide)[:, :cols]


def _plain(state):
    case = state["case"]
    kind, rows, features = case["kind"], case["rows"], case["features"]
    if kind == "dropout":
        x = state["x"]
        out = _dropped(x.to(torch.float32), _kept(state, rows, features))
        if state["residual"] is not None:
            out = state["residual"].to(torch.float32) + out
        return out.to(x.dtype)
    if kind == "join":
        return _join(state)
    if kind == "join_grad":
        return _join_grad(state)
    if kind == "pack":
        return _round8(state["x"].to(torch.float32), True)
    w = _values8(state["w"], case["outputs"], features)
    x = _round8(state["x"].to(torch.float32), False)
    if kind == "linear_grad":
        return torch.matmul(x, w).to(TYPES[case["out"]])
    y = torch.matmul(x, w.t())
    if state["bias"] is not None:
        y = y + state["bias"].to(torch.float32)
    return y.to(TYPES[case["out"]])


def _own(state):
    from paper_2006_02924_b200 import binding

    case = state["case"]
    kind, rows, features = case["kind"], case["rows"], case["features"]
    if kind == "dropout":
        return binding.adasum_dropout(state["x"], case["p"], state["seed"], site=state["site"], residual=state["residual"])
    if kind == "pack":
        packed = binding.adasum_fp8_pack_weight(state["x"])
        return binding.adasum_fp8_unpack(packed, rows, features)
    if kind == "linear":
        packed = binding.adasum_fp8_pack(state["x"])
        return binding.adasum_fp8_linear(packed, state["w"], rows, features, case["outputs"], bias=state["bias"],
                                         out_dtype=TYPES[case["out"]])
    if kind == "linear_grad":
        packed = binding.adasum_fp8_pack(state["x"])
        return binding.adasum_fp8_linear_grad(packed, state["w"], rows, features, case["outputs"],
                                              out_dtype=TYPES[case["out"]])
    block = dict(post_norm=case["post"], post_weight=state["post_weight"], post_bias=state["post_bias"],
                 pre_norm=case["pre"], pre_weight=state["pre_weight"], pre_bias=state["pre_bias"], eps=EPS,
                 gate=state["gate"], rows_per_gate=state["rows_per_gate"], branch_scale=state["branch_scale"],
                 residual_scale=state["residual_scale"], dropout=case["p"], seed=state["seed"], site=state["site"])
    if kind == "join":
        h, y, stats = binding.adasum_residual_norm(state["x"], state["residual"], **block)
        out = {"h": h, "y": y}
        for i, norm in ((0, "post"), (2, "pre")):
            if case[norm] != "none":
                out.update(_stats(case, norm, stats[i], stats[i + 1]))
        return out
    dx, dresidual = binding.adasum_residual_norm_grad(
        state["x"], state["h"], state["stats"], state["dy"], state["dh"], grad_post_weight=state["dpost_weight"],
        grad_post_bias=state["dpost_bias"], grad_pre_weight=state["dpre_weight"], grad_pre_bias=state["dpre_bias"],
        grad_gate=state["dgate"], scale=state["scale"], gate_scale=state["scale"], **block)
    out = {"x": dx, "residual": dresidual}
    for name in ("post_weight", "post_bias", "pre_weight", "pre_bias", "gate"):
        if state["d" + name] is not None:
            out[name] = state["d" + name]
    return out


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definitions in 64 bits --------------------------------------------------------------------

def _exact_mask(case, state):
    """1 / (1 - q) where an element is kept, else 0, from the generator's definition in 32-bit words (numpy)."""
    rows, features = case["rows"], case["features"]
    limit = int(round(case["p"] * 65536))
    if limit == 0:
        return torch.ones(rows, features, dtype=torch.float64, device="cuda")
    count = rows * ((features + 7) // 8)
    key = int(state["seed"].item()) & (2**64 - 1)
    k = [key & M32, key >> 32]
    n = np.arange(count, dtype=np.uint64)
    c = [(n & np.uint64(M32)).astype(np.uint32), (n >> np.uint64(32)).astype(np.uint32),
         np.full(count, state["site"] & M32, np.uint32), np.full(count, state["site"] >> 32, np.uint32)]

    def product(words, factor):
        wide = words.astype(np.uint64) * np.uint64(factor)
        return (wide >> np.uint64(32)).astype(np.uint32), wide.astype(np.uint32)

    for _ in range(10):
        high0, low0 = product(c[0], 0xD2511F53)
        high1, low1 = product(c[2], 0xCD9E8D57)
        c = [high1 ^ c[1] ^ np.uint32(k[0]), low1, high0 ^ c[3] ^ np.uint32(k[1]), low0]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    halves = np.stack(c, axis=1).view(np.uint16).reshape(rows, -1)[:, :features]
    return torch.from_numpy((halves >= limit) * (65536 / (65536 - limit))).cuda()


def _exact_norm(kind, x):
    """Normalised x with its mean and 1 / deviation."""
    mean = x.sum(dim=1, keepdim=True) / x.shape[1] if kind == "layer" else torch.zeros(x.shape[0], 1, dtype=x.dtype, device=x.device)
    rstd = ((x - mean).square().sum(dim=1, keepdim=True) / x.shape[1] + EPS).rsqrt()
    return (x - mean) * rstd, mean, rstd


def _exact_affine(state, norm, hat):
    bias = state[norm + "_bias"]
    return hat * state[norm + "_weight"].double() + (0 if bias is None else bias.double())


def _exact_gate(state, rows):
    if state["gate"] is None:
        return 1.0
    return state["gate"].double().repeat_interleave(state["rows_per_gate"], dim=0)[:rows]


def _power(e):
    """2^e as doubles."""
    return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)


def _exact_round(x, high):
    """Every value of x to the nearest e4m3 multiple of its block's step, blocks of `high` rows x 128 columns."""
    out = torch.zeros_like(x)
    for at in range(0, x.shape[1], BLOCK):
        part = x[:, at : at + BLOCK]
        top = part.abs().amax(dim=1)
        if high > 1:
            top = torch.cat([p.amax().expand(p.shape[0]) for p in top.split(high)])
        top = top[:, None]
        # the smallest power of two with top <= 448 steps
        exponent = torch.ceil(torch.log2(torch.where(top > 0, top, 2.0**-126) / 448)).clamp(min=-126)
        exponent = torch.where(224 * _power(exponent) >= top, exponent - 1, exponent)
        exponent = torch.where(448 * _power(exponent) < top, exponent + 1, exponent).clamp(min=-126)
        scaled = part * _power(-exponent)
        # four significant bits, down to multiples of 2^-9
        place = torch.where(scaled == 0, -9, torch.frexp(scaled)[1] - 4).clamp(min=-9)
        out[:, at : at + BLOCK] = (scaled * _power(-place)).round() * _power(place) * _power(exponent)
    return out


def exact(case, seed):
    state = prepare(case, seed)
    kind, rows = case["kind"], case["rows"]
    if kind == "dropout":
        out = state["x"].double() * _exact_mask(case, state)
        return out if state["residual"] is None else out + state["residual"].double()
    if kind == "pack":
        return _exact_round(state["x"].double(), BLOCK)
    if kind in ("linear", "linear_grad"):
        x = _exact_round(state["x"].double(), 1)
        w = _values8(state["w"], case["outputs"], case["features"]).double()
        if kind == "linear_grad":
            return torch.einsum("rn,nk->rk", x, w)
        y = torch.einsum("rk,nk->rn", x, w)
        return y if state["bias"] is None else y + state["bias"].double()
    mask, gate = _exact_mask(case, state), _exact_gate(state, rows)
    x, alpha, beta = state["x"].double(), state["branch_scale"], state["residual_scale"]
    if kind == "join":
        out, n = {}, x
        if case["post"] != "none":
            hat, mean, rstd = _exact_norm(case["post"], x)
            out.update(_stats(case, "post", mean[:, 0], rstd[:, 0]))
            n = _exact_affine(state, "post", hat)
        h = beta * state["residual"].double() + alpha * gate * mask * n
        hat, mean, rstd = _exact_norm(case["pre"], h)
        out.update(_stats(case, "pre", mean[:, 0], rstd[:, 0]))
        return {"h": h, "y": _exact_affine(state, "pre", hat), **out}
    # with u = a norm's normalised input, v its gradient: dx = rstd (v - [mean v] - u mean(u v))
    post_mean, post_rstd, pre_mean, pre_rstd = state["stats"].double()[:, :, None]

    def back(norm, u, v, rstd):
        v = v * state[norm + "_weight"].double()
        d = v - u * torch.einsum("rc,rc->r", u, v)[:, None] / v.shape[1]
        return rstd * (d - v.sum(dim=1, keepdim=True) / v.shape[1] if case[norm] == "layer" else d)

    out, scale = {}, state["scale"]
    dy, u = state["dy"].double(), (state["h"].double() - pre_mean) * pre_rstd
    dh = state["dh"].double() + back("pre", u, dy, pre_rstd)
    named = {"pre_weight": torch.einsum("rc,rc->c", dy, u), "pre_bias": torch.einsum("rc->c", dy)}
    u, n = x, x
    if case["post"] != "none":
        u = (x - post_mean) * post_rstd
        n = _exact_affine(state, "post", u)
    if state["gate"] is not None:
        parts = (alpha * dh * mask * n).split(state["rows_per_gate"])
        named["gate"] = torch.stack([p.sum(dim=0) for p in parts])
    dn = alpha * dh * gate * mask
    if case["post"] != "none":
        named["post_weight"], named["post_bias"] = torch.einsum("rc,rc->c", dn, u), torch.einsum("rc->c", dn)
        dn = back("post", u, dn, post_rstd)
    out = {"x": dn, "residual": beta * dh}
    for name in ("post_weight", "post_bias", "pre_weight", "pre_bias", "gate"):
        if state["d" + name] is not None:
            out[name] = named[name] * scale
    return out
