"""Cases of the operators that produce a worker's gradients, and their plain forms.

A worker's backward pass writes its gradients into the fused buffer that the reduce combines.  Four
kinds of pass are covered:

    lookup        y[t] = scale * table[token[t]]                  (no row: zeros)
    lookup_grad   dtable[v] = scale * sum of dy[t] over the tokens t with token[t] = v
    checkpoint    y = act(x) with x kept in 8 bits, and the kept values read back
    act_grad      dx = dy * act'(kept x)
    weight_grad   dw[n, k] = scale * sum_t dy[t, n] * (kept x)[t, k],  dbias[n] = scale * sum_t dy[t, n]

A checkpoint keeps a [rows, features] matrix as one byte per value: groups of 32 features of a row
(the last one filled up with zeros) share a power of two.  With E the exponent of the group's largest
magnitude the step is 2^(E - 6), at least 2^-126, and a code is the value over the step, rounded to the
nearest integer, ties to even, limited to +-127.  The buffer holds all codes (signed bytes), row by row,
then all steps (their exponent + 127), row by row.  A step byte of 255 marks a group with an Inf or NaN:
its codes are zero and it stands for NaN.
"""
import math

import torch

own = False

GROUP = 32
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
BYTES = {"f32": 4, "f16": 2, "bf16": 2}


# ---- the cases -------------------------------------------------------------------------------------

def listed():
    return [
        # the next token of one sequence: nothing but latency
        {"name": "lookup, one token", "kind": "lookup", "tokens": 1, "table": 30522, "dim": 1024,
         "in": "bf16", "out": "bf16", "index": 64, "slack": 0},
        # a phase-2 batch of BERT-Large (64 sequences of 512), fp32 master weights read as bf16
        {"name": "lookup, 64 x 512 tokens", "kind": "lookup", "tokens": 32768, "table": 30522, "dim": 1024,
         "in": "f32", "out": "bf16", "index": 64, "slack": 0},
        # word embeddings of a phase-1 microbatch (36 sequences of 128) into an fp32 fused buffer
        {"name": "lookup_grad, 36 x 128", "kind": "lookup_grad", "tokens": 4608, "table": 30522, "dim": 1024,
         "in": "bf16", "out": "f32", "index": 64, "slack": 0},
        # token-type embeddings: two rows take all the tokens of 32 sequences of 512
        {"name": "lookup_grad, two rows", "kind": "lookup_grad", "tokens": 16384, "table": 2, "dim": 1024,
         "in": "f16", "out": "f16", "index": 32, "slack": 0},
        # a small odd model: nothing is a multiple of anything, rows of a wider matrix
        {"name": "lookup_grad, odd sizes", "kind": "lookup_grad", "tokens": 999, "table": 1009, "dim": 203,
         "in": "f32", "out": "f32", "index": 32, "slack": 5},
        # the feed-forward activations of 32 sequences of 512
        {"name": "checkpoint, 16384 x 4096", "kind": "checkpoint", "rows": 16384, "features": 4096,
         "type": "bf16", "act": "gelu", "slack": 0},
        # a classifier's last activations on a small batch, features that fill no group
        {"name": "checkpoint, 37 x 1000", "kind": "checkpoint", "rows": 37, "features": 1000,
         "type": "f16", "act": "silu", "slack": 24},
        # the same feed-forward activations on the way back
        {"name": "act_grad, 16384 x 4096", "kind": "act_grad", "rows": 16384, "features": 4096,
         "type": "bf16", "act": "gelu", "slack": 0},
        # one short sequence in fp32
        {"name": "act_grad, 61 x 1023", "kind": "act_grad", "rows": 61, "features": 1023,
         "type": "f32", "act": "gelu_tanh", "slack": 1},
        # first feed-forward matrix of BERT-Large, 32 sequences of 512, fp32 fused buffer
        {"name": "weight_grad, 16384 tokens", "kind": "weight_grad", "rows": 16384, "features": 1024, "outputs": 4096,
         "in": "bf16", "out": "f32", "bias": True, "slack": 0},
        # an attention projection of a phase-1 microbatch: few output tiles, a long sum, fp16 throughout
        {"name": "weight_grad, 4608 tokens", "kind": "weight_grad", "rows": 4608, "features": 1024, "outputs": 1024,
         "in": "f16", "out": "f16", "bias": True, "slack": 0},
        # a small odd layer in fp32
        {"name": "weight_grad, odd sizes", "kind": "weight_grad", "rows": 333, "features": 1000, "outputs": 257,
         "in": "f32", "out": "f32", "bias": False, "slack": 3},
    ]


def _spread(rng, low, high):
    """A whole number of [low, high], spread over its logarithm; every other one a multiple of 8."""
    n = int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))
    if n >= 16 and rng.random() < 0.5:
        n -= n % 8
    return max(low, min(high, n))


def draw(rng):
    kind = rng.choice(["lookup", "lookup_grad", "checkpoint", "act_grad", "weight_grad"])
    slack = rng.choice([0, 0, 1, 8, 24])
    types = ["f32", "f16", "bf16"]
    if kind in ("lookup", "lookup_grad"):
        dim = _spread(rng, 1, 2048)
        table = min(_spread(rng, 2, 65536), (1 << 25) // dim)
        tokens = min(_spread(rng, 1, 32768), (1 << 25) // dim)
        return {"kind": kind, "tokens": tokens, "table": table, "dim": dim, "in": rng.choice(types),
                "out": rng.choice(types), "index": rng.choice([32, 64]), "slack": slack}
    if kind in ("checkpoint", "act_grad"):
        features = _spread(rng, 1, 8192)
        rows = min(_spread(rng, 1, 32768), (1 << 26) // features)
        return {"kind": kind, "rows": rows, "features": features, "type": rng.choice(types),
                "act": rng.choice(["relu", "gelu", "gelu_tanh", "silu"]), "slack": slack}
    features, outputs = _spread(rng, 1, 4096), _spread(rng, 1, 4096)
    rows = min(_spread(rng, 1, 16384), (1 << 36) // (features * outputs))
    return {"kind": kind, "rows": rows, "features": features, "outputs": outputs, "in": rng.choice(types),
            "out": rng.choice(types), "bias": rng.random() < 0.5, "slack": slack}


def work(case):
    kind = case["kind"]
    if kind in ("lookup", "lookup_grad"):
        t, d, v = case["tokens"], case["dim"], case["table"]
        index = t * (case["index"] // 8)
        if kind == "lookup":     # every row that is asked for read once
            return {"bytes": index + min(t, v) * d * BYTES[case["in"]] + t * d * BYTES[case["out"]], "flops": t * d}
        return {"bytes": index + t * d * BYTES[case["in"]] + v * d * BYTES[case["out"]], "flops": t * d}
    rows, features = case["rows"], case["features"]
    groups = -(-features // GROUP)
    kept = rows * (features + groups)
    if kind == "checkpoint":     # x read, y and the checkpoint written, the checkpoint read, its values written
        return {"bytes": 3 * rows * features * BYTES[case["type"]] + 2 * kept, "flops": 20 * rows * features}
    if kind == "act_grad":
        return {"bytes": 2 * rows * features * BYTES[case["type"]] + kept, "flops": 20 * rows * features}
    outputs = case["outputs"]
    written = (outputs * features + (outputs if case["bias"] else 0)) * BYTES[case["out"]]
    return {"bytes": kept + rows * outputs * BYTES[case["in"]] + written, "flops": 2 * rows * features * outputs}


# ---- inputs ----------------------------------------------------------------------------------------

def _matrix(gen, rows, cols, slack, dtype, size=1.0):
    """Normal values, a few columns much larger than the rest (as activations have them); with slack, the
    first columns of a wider matrix."""
    wide = torch.empty(rows, cols + slack, dtype=torch.float32, device="cuda").normal_(generator=gen)
    loud = torch.rand(cols + slack, generator=gen, device="cuda") < 0.01
    wide.mul_(torch.where(loud, 12.0 * size, size))
    return wide.to(dtype)[:, :cols]


def _tokens(gen, case):
    """Token ids: frequencies fall off as in text, one in thirty-two is padding (no row)."""
    table, n = case["table"], case["tokens"]
    u = torch.rand(n, generator=gen, device="cuda", dtype=torch.float64)
    rank = (torch.exp(u * math.log(table + 1.0)) - 1.0).to(torch.int64).clamp_(0, table - 1)
    order = torch.randperm(table, generator=gen, device="cuda")
    ids = order[rank]
    none = torch.rand(n, generator=gen, device="cuda") < 1.0 / 32.0
    return torch.where(none, -1, ids).to(torch.int32 if case["index"] == 32 else torch.int64)


def _keep(x):
    """The checkpoint of x, in the layout that the module's docstring gives."""
    rows, features = x.shape
    width = -(-features // GROUP) * GROUP
    v = torch.zeros(rows, width, dtype=torch.float32, device=x.device)
    v[:, :features] = x
    v = v.view(rows, width // GROUP, GROUP)
    top = v.abs().amax(dim=2).view(torch.int32) >> 23
    step = (top - 6).clamp_(min=1)
    step = torch.where(top == 255, 255, step)
    back = ((254 - step).clamp_(min=0) << 23).view(torch.float32)
    codes = torch.round(v * back[:, :, None]).clamp_(-127, 127)
    codes = torch.where(step[:, :, None] == 255, 0.0, codes).to(torch.int8)
    return torch.cat((codes.view(torch.uint8).reshape(-1), step.to(torch.uint8).reshape(-1)))


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    kind = case["kind"]
    state = {"case": case}
    if kind in ("lookup", "lookup_grad"):
        state["tokens"] = _tokens(gen, case)
        state["scale"] = math.sqrt(case["dim"])
        if kind == "lookup":
            state["table"] = _matrix(gen, case["table"], case["dim"], case["slack"], TYPES[case["in"]], 0.02)
        else:
            state["dy"] = _matrix(gen, case["tokens"], case["dim"], case["slack"], TYPES[case["in"]], 0.01)
            # the tensor's place in the worker's fused buffer
            state["dtable"] = torch.zeros(case["table"], case["dim"], dtype=TYPES[case["out"]], device="cuda")
        return state
    rows, features = case["rows"], case["features"]
    if kind == "checkpoint":
        state["x"] = _matrix(gen, rows, features, case["slack"], TYPES[case["type"]])
        return state
    state["kept"] = _keep(_matrix(gen, rows, features, 0, TYPES[case["type"] if kind == "act_grad" else case["in"]]))
    if kind == "act_grad":
        state["dy"] = _matrix(gen, rows, features, case["slack"], TYPES[case["type"]], 0.01)
        return state
    state["dy"] = _matrix(gen, rows, case["outputs"], case["slack"], TYPES[case["in"]], 0.01)
    state["scale"] = 0.5
    state["dw"] = torch.zeros(case["outputs"], features, dtype=TYPES[case["out"]], device="cuda")
    state["db"] = torch.zeros(case["outputs"], dtype=TYPES[case["out"]], device="cuda") if case["bias"] else None
    return state


# ---- the plain forms -------------------------------------------------------------------------------

def _kept_values(kept, rows, features):
    width = -(-features // GROUP) * GROUP
    codes = kept[: rows * width].view(torch.int8).view(rows, width // GROUP, GROUP)
    step = (kept[rows * width :].view(rows, width // GROUP, 1).to(torch.int32) << 23).view(torch.float32)
    return (codes.to(torch.float32) * step).view(rows, width)[:, :features]


def _act(x, act):
    if act == "relu":
        return torch.where(x > 0, x, 0.0 * x)
    if act == "gelu":
        return 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))
    if act == "silu":
        return x / (1.0 + torch.exp(-x))
    return 0.5 * x * (1.0 + torch.tanh(math.sqrt(2.0 / math.pi) * (x + 0.044715 * x * x * x)))


def _act_slope(x, act):
    if act == "relu":
        return (x > 0).to(torch.float32)
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(x * math.sqrt(0.5))) + x * torch.exp(-0.5 * x * x) * (1.0 / math.sqrt(2.0 * math.pi))
    if act == "silu":
        s = 1.0 / (1.0 + torch.exp(-x))
        return s * (1.0 + x * (1.0 - s))
    c = math.sqrt(2.0 / math.pi)
    t = torch.tanh(c * (x + 0.044715 * x * x * x))
    return 0.5 * (1.0 + t) + 0.5 * x * (1.0 - t * t) * c * (1.0 + 3.0 * 0.044715 * x * x)


def _plain(state):
    case = state["case"]
    kind = case["kind"]
    if kind == "lookup":
        ids = state["tokens"].long()
        inside = (ids >= 0) & (ids < case["table"])
        rows = state["table"][torch.where(inside, ids, 0)].to(torch.float32) * state["scale"]
        return torch.where(inside[:, None], rows, 0.0).to(TYPES[case["out"]])
    if kind == "lookup_grad":
        ids = state["tokens"].long()
        inside = (ids >= 0) & (ids < case["table"])
        sums = torch.zeros(case["table"] + 1, case["dim"], dtype=torch.float32, device="cuda")
        sums.index_add_(0, torch.where(inside, ids, case["table"]), state["dy"].to(torch.float32))
        return state["dtable"].copy_(sums[:-1] * state["scale"])
    if kind == "checkpoint":
        x = state["x"]
        y = _act(x.to(torch.float32), case["act"]).to(x.dtype)
        return {"y": y, "kept": _kept_values(_keep(x), *x.shape).to(x.dtype)}
    x = _kept_values(state["kept"], case["rows"], case["features"])
    dy = state["dy"]
    if kind == "act_grad":
        return (dy.to(torch.float32) * _act_slope(x, case["act"])).to(dy.dtype)
    dy = dy.to(torch.float32)
    out = {"dw": state["dw"].copy_(torch.matmul(dy.t(), x) * state["scale"])}
    if case["bias"]:
        out["db"] = state["db"].copy_(dy.sum(dim=0) * state["scale"])
    return out


def _own(state):
    from paper_2006_02924_b200 import binding

    case = state["case"]
    kind = case["kind"]
    if kind == "lookup":
        return binding.adasum_embedding_forward(state["table"], state["tokens"], scale=state["scale"],
                                                out_dtype=TYPES[case["out"]])
    if kind == "lookup_grad":
        return binding.adasum_embedding_grad(state["dy"], state["tokens"], grad_table=state["dtable"],
                                             scale=state["scale"])
    if kind == "checkpoint":
        y, kept = binding.adasum_checkpoint_save(state["x"], activation=case["act"])
        return {"y": y, "kept": binding.adasum_checkpoint_load(kept, case["rows"], case["features"],
                                                               dtype=TYPES[case["type"]])}
    if kind == "act_grad":
        return binding.adasum_checkpoint_act_grad(state["kept"], state["dy"], activation=case["act"])
    binding.adasum_checkpoint_weight_grad(state["kept"], state["dy"], grad_weight=state["dw"], grad_bias=state["db"],
                                          scale=state["scale"])
    return {"dw": state["dw"], "db": state["db"]} if case["bias"] else {"dw": state["dw"]}


def run(state):
    return _own(state) if own else _plain(state)


# ---- the definitions in 64 bits --------------------------------------------------------------------

def _exact_slope(x, act):
    """d act / dx in doubles, from the distribution and logistic functions themselves."""
    if act == "relu":
        return torch.heaviside(x, torch.zeros_like(x))
    if act == "gelu":        # Phi(x) + x phi(x)
        return torch.special.ndtr(x) + x * torch.exp(-x.square() / 2) / math.sqrt(2 * math.pi)
    if act == "silu":
        return torch.sigmoid(x) + x * torch.sigmoid(x) * torch.sigmoid(-x)
    # x * sigmoid(2 u(x)), u = sqrt(2 / pi) (x + 0.044715 x^3)
    a = 2 * math.sqrt(2 / math.pi)
    s = torch.sigmoid(a * (x + 0.044715 * x.pow(3)))
    return s + x * s * (1 - s) * a * (1 + 0.134145 * x.square())


def _exact_act(x, act):
    if act == "relu":
        return x.clamp(min=0)
    if act == "gelu":
        return x * torch.special.ndtr(x)
    if act == "silu":
        return x * torch.sigmoid(x)
    return x * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x.pow(3)))


def exact(case, seed):
    state = prepare(case, seed)
    kind = case["kind"]
    if kind == "lookup":
        ids = state["tokens"].long()
        padded = torch.cat((state["table"].double() * state["scale"], torch.zeros(1, case["dim"], dtype=torch.float64, device="cuda")))
        return padded[torch.where(ids < 0, case["table"], ids)]
    if kind == "lookup_grad":     # sorted by token: differences of the running sums
        ids, order = torch.sort(state["tokens"].long())
        running = torch.zeros(case["tokens"] + 1, case["dim"], dtype=torch.float64, device="cuda")
        running[1:] = torch.cumsum(state["dy"].double()[order], dim=0)
        row = torch.arange(case["table"], device="cuda")
        first, last = torch.searchsorted(ids, row), torch.searchsorted(ids, row, right=True)
        return (running[last] - running[first]) * state["scale"]
    if kind == "checkpoint":
        x = state["x"].double()
        values = torch.empty_like(x)
        for at in range(0, case["features"], GROUP):
            part = x[:, at : at + GROUP]
            top = part.abs().amax(dim=1, keepdim=True)
            exponent = torch.frexp(top)[1] - 1
            exponent = torch.where(top == 0, -120, exponent).clamp(min=-120)
            step = torch.ldexp(torch.ones_like(top), exponent - 6)
            values[:, at : at + GROUP] = (part / step).round().clamp(-127, 127) * step
        return {"y": _exact_act(x, case["act"]), "kept": values}
    rows, features = case["rows"], case["features"]
    groups = -(-features // GROUP)
    codes = state["kept"][: rows * groups * GROUP].view(torch.int8).view(rows, groups * GROUP).double()
    steps = torch.pow(2.0, state["kept"][rows * groups * GROUP :].view(rows, groups).double() - 127)
    x = (codes * steps.repeat_interleave(GROUP, dim=1))[:, :features]
    dy = state["dy"].double()
    if kind == "act_grad":
        return dy * _exact_slope(x, case["act"])
    out = {"dw": torch.einsum("tn,tk->nk", dy, x) * state["scale"]}
    if case["bias"]:
        out["db"] = torch.einsum("tn->n", dy) * state["scale"]
    return out
