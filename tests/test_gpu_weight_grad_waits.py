"""The bounded waits of the weight gradient's product: one that runs out ends the launch, is reported, and leaves the
device and the workspace usable."""
import pytest
import torch

pytestmark = pytest.mark.gpu

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def b():
    from paper_2006_02924_b200 import binding

    return binding


# More sums per pair of blocks than tensor memory holds, and more steps than shared memory, so that every kind of
# hand-over is waited for: a sum takes 512 tokens (fp32: 85), and at most 74 pairs share the list.
@pytest.mark.parametrize("dtype,rows", [("bf16", 4 * 512 * 74), ("f32", 4 * 85 * 74 + 7)])
@pytest.mark.parametrize("hand_over,bias", [("added", True)] + [
    (name, bias) for name in ("landed", "multiplied", "ready", "formed", "taken") for bias in (True, False)])
def test_a_wait_that_runs_out(b, hand_over, bias, dtype, rows):
    features, outputs = 40, 24
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    x = torch.randn(rows, features, generator=gen, device="cuda")
    dy = torch.randn(rows, outputs, generator=gen, device="cuda").to(TYPES[dtype])
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    ws = torch.empty(b.adasum_checkpoint_weight_grad_workspace_bytes(rows, features, outputs, dtype), dtype=torch.uint8,
                     device="cuda")
    dw = torch.zeros(outputs, features, device="cuda")
    db = torch.zeros(outputs, device="cuda") if bias else None

    def good():
        b.adasum_checkpoint_weight_grad(kept, dy, grad_weight=dw, grad_bias=db, workspace=ws)
        assert b.adasum_checkpoint_weight_grad_status(rows, features, outputs, dtype, ws) == 0
        return dw.clone(), None if db is None else db.clone()

    want, want_b = good()
    b.adasum_checkpoint_weight_grad_selftest(hand_over, kept, dy, dw, db, ws)
    assert b.adasum_checkpoint_weight_grad_status(rows, features, outputs, dtype, ws) == 7
    assert "bounded wait" in b.adasum_last_error()
    got, got_b = good()
    assert torch.equal(got, want) and (db is None or torch.equal(got_b, want_b))


@pytest.mark.parametrize("out_type", [torch.float32, torch.float16])
@pytest.mark.parametrize("rows,features,outputs", [(4 * 512 * 74, 40, 24), (520, 3000, 9000)])
@pytest.mark.parametrize("hand_over", ["landed", "ready", "formed"])
def test_an_unfinished_sum_is_no_gradient(b, hand_over, rows, features, outputs, out_type):
    """Nothing of a product whose waits ran out looks like a gradient: NaN everywhere, be the tiles cut among pairs of
    blocks (one tile of many tokens) or written by one pair each (many tiles); these hand-overs fail in the first sum."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(4)
    x = torch.randn(rows, features, generator=gen, device="cuda")
    dy = torch.randn(rows, outputs, generator=gen, device="cuda").bfloat16()
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    ws = torch.empty(b.adasum_checkpoint_weight_grad_workspace_bytes(rows, features, outputs, "bf16"), dtype=torch.uint8,
                     device="cuda")
    dw = torch.zeros(outputs, features, dtype=out_type, device="cuda")
    db = torch.zeros(outputs, dtype=out_type, device="cuda")
    b.adasum_checkpoint_weight_grad_selftest(hand_over, kept, dy, dw, db, ws)
    assert b.adasum_checkpoint_weight_grad_status(rows, features, outputs, "bf16", ws) == 7
    assert torch.isnan(dw).all() and torch.isnan(db).all()
