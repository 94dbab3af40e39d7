"""Layer norm refuses statistics and gradients that are not aligned to their elements, before anything touches a GPU."""
import pytest

from paper_2505_01068_amd import binding as B
from tests.test_layer_ops_host import NORM, NORM_BWD, ODD, P, err


@pytest.mark.parametrize("name", ["mean", "rstd"])
def test_forward(name):
    a = {**NORM, "mean": P, "rstd": P, name: ODD}
    assert B.lib().im_layernorm_fwd(*a.values(), None) == -1 and "mean or rstd is not aligned" in err()


@pytest.mark.parametrize("name", ["mean", "rstd", "dgamma", "dbeta"])
def test_backward(name):
    a = {**NORM_BWD, name: ODD}
    assert B.lib().im_layernorm_bwd(*a.values(), None) == -1 and "is not aligned" in err()
