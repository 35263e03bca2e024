"""How near the weight gradients of fp32 gradients come to 64 bits."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows", [40, 64, 333, 1000, 5000])
def test_no_further_off_than_an_fp32_product(rows):
    """In the norm, no further from 64 bits than torch's fp32 product of the same matrices."""
    from paper_2006_02924_b200 import binding as b

    gen = torch.Generator(device="cuda")
    gen.manual_seed(41)
    x = torch.randn(rows, 512, generator=gen, device="cuda")
    dy = torch.randn(rows, 384, generator=gen, device="cuda")
    _, kept = b.adasum_checkpoint_save(x, want_out=False)
    at = b.adasum_checkpoint_load(kept, rows, 512)
    want = dy.double().t() @ at.double()
    got, _ = b.adasum_checkpoint_weight_grad(kept, dy, features=512)
    assert not torch.backends.cuda.matmul.allow_tf32
    assert (got.double() - want).norm() <= ((dy.t() @ at).double() - want).norm()
