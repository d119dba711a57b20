"""Refusals of the calls around a frame's attention on the GPU: nothing is enqueued, nothing changes."""
import pytest
import torch

pytestmark = pytest.mark.gpu

D = 64


@pytest.fixture(scope="module")
def rv():
    from paper_2609_23286_amd import rv as _rv
    _rv.init()
    return _rv


def test_a_sequence_too_large_for_a_launch_is_refused_before_the_others_are_launched(rv):
    """16,384 tokens of 1024 query heads on one are 131,072 query tiles: over 2043 pages they fit, over 2044 they do not."""
    rows, tokens, Hq = 2043 * 64 + 1, 16384, 1024
    pool = rv.Pool(1, 2100, 60, rows)
    seqs = [pool.open() for _ in range(55)]  # more than a launch takes: the large one is not in the first
    K = torch.zeros(3 + rows, 1, D, dtype=torch.bfloat16, device="cuda")
    pool.append([seqs[0], seqs[-1]], K, K, [3, rows])
    n_tokens = [1] * 54 + [tokens]
    Q = torch.zeros(sum(n_tokens), Hq, D, dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(Q, 7.0)
    lse = torch.full((Q.shape[0] * Hq,), 7.0, device="cuda")
    with pytest.raises(rv.RVError, match=f"sequence {seqs[-1]}: too many tokens over too many rows") as e:
        rv.attend_seqs(Q, None, None, pool, seqs, n_tokens, out, lse)
    assert e.value.status == rv.RV_ERR_INVALID
    torch.cuda.synchronize()
    assert bool((out == 7).all()) and bool((lse == 7).all())
