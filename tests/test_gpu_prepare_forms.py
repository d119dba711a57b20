"""Gradients of prepared projections where some are not asked for: the others keep their bits."""
import pytest
import torch

from test_gpu_prepare import Case, backward

pytestmark = pytest.mark.gpu

NAMES = ("dq_weight", "dq_bias", "dk_weight", "dk_bias")


@pytest.fixture(scope="module")
def rv():
    from paper_2609_23286_amd import rv as _rv
    _rv.init()
    return _rv


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("wanted", [(), ("dq_weight",), ("dk_bias",), ("dq_bias", "dk_weight"), NAMES], ids=str)
@pytest.mark.parametrize("values", [False, True])
def test_some_gradients(rv, dtype, wanted, values):
    x = Case(rv, 301, 5, 3, dtype=dtype, fused=True)
    want = backward(rv, x)
    dq, dk, dv = (torch.full_like(t, 7.0) for t in (x.q, x.k, x.v))
    sums = {n: torch.full((64,), 7.0, device="cuda") for n in wanted}
    rv.prepare_qkv_bwd(x.prep, x.q, x.k, x.pos, x.dQ, x.dK, x.dV if values else None, dq, dk, dv if values else None, **sums)
    assert torch.equal(dq, want["dq"]) and torch.equal(dk, want["dk"])
    assert torch.equal(dv, want["dv"]) if values else bool((dv == 7).all())
    for n in wanted:
        assert torch.equal(sums[n], want[n]), n
