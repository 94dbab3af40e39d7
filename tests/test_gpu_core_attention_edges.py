"""im_core_attention_fwd / im_core_attention_bwd at the ends of what they accept, against the fp64 definition within its elementwise bounds."""
import pytest
import torch

from paper_2505_01068_amd import binding as B
from tests.test_gpu_core_attention import Case, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("cap,scale,gain", [
    (1000.0, 0.01, 40.0), (1000.0, 1.0 / 128, 40.0), (1000.0, 1e-3, 40.0), (1000.0, 1e-5, 40.0), (1000.0, 1e-8, 1e6), (1000.0, 1e-36, 1.0), (1000.0, 1e-40, 1.0),
    (1000.0, 1e-44, 1.0), (0.01, 1e-44, 1.0), (0.01, 2000.0, 1e-7), (0.01, 2000.0, 1.0), (0.01, 1e6, 1e-10), (0.01, 1e20, 1.0), (0.01, 3e38, 1.0), (1000.0, 3e38, 1.0)])
def test_any_scale_under_a_cap(dtype, cap, scale, gain):
    """scale / cap from 1e-47 to 3e40, raw scores of some hundreds where the cap's argument is small: lse of one or two keys shows each score."""
    print("core scale", dtype, cap, scale, gain, flush=True)
    for k_len in ((1, 2), (40, 30)):
        case = Case(dtype, 2, (33, 20), k_len, 2, 1, 16, 0b1111, cap=cap, gain=gain, seed=11)
        case.scale = float(torch.tensor(scale))
        case.core = B.make_core(2, case.q_len, k_len, 2, 1, 16, 0b1111, scale, dtype, cap=cap)
        check(case)
