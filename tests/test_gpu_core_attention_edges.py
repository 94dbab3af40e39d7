"""im_core_attention_fwd / im_core_attention_bwd at the ends of what they accept, against the fp64 definition within its elementwise bounds."""
import pytest
import torch

import oracle
from paper_2505_01068_amd import binding as B
from tests.test_gpu_core_attention import Case, check

pytestmark = pytest.mark.gpu
IEM = oracle.IM_IEM


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


HIDDEN = [dict(), dict(cap=5.0, bias=True)]


def partly_hidden(dtype, dh, few, **rules):
    """Queries that see nothing and keys that nobody sees, in tiles that other rows see in part."""
    case = Case(dtype, 2 if few else 8, (40, 70, 20), (40, 70, 20), 4 if few else 24, 2 if few else 24, dh, IEM, docs=2, pad="valid_len", seed=5, **rules)
    case.rules["valid_len"] = torch.tensor([[40, 50, 20], [40, 30, 7]], dtype=torch.int32, device="cuda").repeat(case.batch // 2, 1)
    case.rules["q_doc"][:, 45:60] = 9
    return case


def same(got, want, what):
    for n, t in want.items():
        assert torch.equal(got[n], t), (n, what)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dh,few", [(16, True), (64, True), (64, False), (128, False)])
@pytest.mark.parametrize("rules", range(len(HIDDEN)))
def test_a_query_that_sees_nothing_may_hold_anything(dtype, dh, few, rules):
    """Its own gradient is 0 and no other result changes a bit, whatever it and its output's gradient hold."""
    print("core blind", dtype, dh, few, HIDDEN[rules], flush=True)
    case = partly_hidden(dtype, dh, few, **HIDDEN[rules])
    good = {n: t.clone() for n, t in check(case).items()}
    blind = torch.from_numpy(~case.seen().any(2)).cuda()
    assert blind.any() and torch.all(good["dq"][blind] == 0)
    for name in ("d_o", "q"):
        for bad in (float("nan"), float("inf"), 3e38):
            tensor = getattr(case, name)
            keep = tensor.clone()
            tensor[blind] = bad
            out = case.run()
            tensor.copy_(keep)
            same(out, good, (name, bad))


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("dh,few", [(16, True), (64, True), (64, False), (128, False)])
@pytest.mark.parametrize("rules", range(len(HIDDEN)))
def test_a_key_that_nobody_sees_may_hold_the_largest_numbers(dtype, dh, few, rules):
    """Products with it overflow although its values are finite: no result changes a bit."""
    print("core large", dtype, dh, few, HIDDEN[rules], flush=True)
    case = partly_hidden(dtype, dh, few, **HIDDEN[rules])
    good = {n: t.clone() for n, t in check(case).items()}
    nobody = torch.from_numpy(~case.seen().any(1)).cuda()
    assert nobody.any()
    sign = torch.randn(case.k.shape, generator=torch.Generator().manual_seed(8)).sign().cuda()
    for tensor in (case.k, case.v):
        for bad in (torch.full_like(sign, 3e38), 3e38 * sign):
            keep = tensor.clone()
            tensor[nobody] = bad[nobody].to(tensor.dtype)
            out = case.run()
            tensor.copy_(keep)
            same(out, good, "k" if tensor is case.k else "v")


@pytest.mark.parametrize("dh,few", [(16, True), (64, True), (64, False), (128, False)])
@pytest.mark.parametrize("rules", [dict(), dict(cap=5.0), dict(cap=5.0, bias=True)])
def test_a_bf16_row_depends_on_what_it_sees_alone(dh, few, rules):
    """In training too: neither the numbers at masked keys nor the scores of other rows of its tile change a bit of a row's results."""
    print("core alone", dh, few, rules, flush=True)
    case = partly_hidden("bf16", dh, few, **rules)
    good = {n: t.clone() for n, t in check(case).items()}
    nobody = torch.from_numpy(~case.seen().any(1)).cuda()
    keep = case.k.clone()
    case.k[nobody] = 50.0
    out = case.run()
    case.k = keep
    same(out, good, "masked keys")
    # every fourth query's scores grow late in the stream: the references of its neighbours' wave are looked at again
    case.q[:, ::4] *= 8.0
    out = case.run()
    others = torch.arange(130, device="cuda") % 4 > 0
    for n in ("o", "dq"):
        assert torch.equal(out[n][:, others], good[n][:, others]), n
    assert torch.equal(out["lse"][:, :, others], good["lse"][:, :, others])


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("scale", [1e38, 2.4e38, 3.4e38])
def test_scores_of_zero_under_the_largest_scales(dtype, scale):
    """Without a cap: queries of zeros see the mean of their values."""
    print("core largest scale", dtype, scale, flush=True)
    case = Case(dtype, 2, (33, 20), (40, 30), 2, 1, 16, 0b1111, seed=12)
    case.scale = float(torch.tensor(scale))
    case.core = B.make_core(2, case.q_len, case.k_len, 2, 1, 16, 0b1111, scale, dtype)
    case.q.zero_()
    case.d_o.zero_()   # (dq is scale times what rounding leaves of dS: nothing to hold it to)
    check(case)
