"""Layer norm of tensors without rows, whichever dimension is empty."""
import pytest
import torch

from paper_2505_01068_amd import binding as B

SHAPES = [(0, 24), (3, 0, 8), (0, 3, 8), (2, 3, 0, 8), (2, 0, 3, 8), (0, 0, 8)]


@pytest.mark.parametrize("shape", SHAPES)
def test_no_rows_whatever_the_strides(shape):
    x = torch.empty(shape)
    assert B._rows("t", "x", x, shape[-1], torch.float32) == (0, shape[-1])
    assert B._rows("t", "x", x, shape[-1], torch.float32, 0) == (0, shape[-1])
    with pytest.raises(ValueError, match="4 are needed"):
        B._rows("t", "x", x, shape[-1], torch.float32, 4)


@pytest.mark.gpu
@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_norm_and_gradients_without_rows(shape, dtype):
    d, x = shape[-1], torch.empty(shape, dtype=dtype, device="cuda")
    assert B.im_layernorm_fwd(x).shape == shape
    stat = torch.empty(shape[:-1], device="cuda")
    assert B.im_layernorm_fwd(x, mean=stat, rstd=stat).shape == shape
    dg, db = (torch.full((d,), 3.0, device="cuda") for _ in range(2))
    B.im_layernorm_bwd(x, None, stat, stat, x, dx=torch.empty_like(x), dgamma=dg, dbeta=db)
    assert torch.all(dg == 0) and torch.all(db == 0)
