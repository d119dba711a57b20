"""Refusals of the calls around a frame's attention on the GPU: nothing is enqueued, nothing changes."""
import ctypes

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


def test_tensors_of_another_type_of_the_same_size_are_refused(rv):
    """float16 where bf16 is read or written, whole numbers where fp32 is: their bits would be taken for numbers."""
    H, N = 2, 6
    pool = rv.Pool(H, 8, 4, 200)
    s = pool.open()
    frame = torch.zeros(N, H, D, dtype=torch.bfloat16, device="cuda")
    pool.append([s], frame, frame, [N])
    half, lse = frame.half(), torch.zeros(H * N, device="cuda")
    ints = torch.zeros(H * N, dtype=torch.int32, device="cuda")
    prep = rv.QKVPrep(H, H, norm="rms", axes=0)
    x, hx = frame.view(N, H * D), half.view(N, H * D)
    mem = rv.Memory(H, reserve_tokens=16, max_tokens=16)
    four, four_half = frame[None], half[None]
    stats, int_stats = lse.view(1, H, N), ints.view(1, H, N)
    idx, float_idx = ints.view(1, H, N)[..., :1].contiguous(), stats[..., :1].contiguous()
    grid = (1, N, 0, 1)

    def swapped(args, i, other):
        return [other if j == i else a for j, a in enumerate(args)]

    calls = []
    fwd = (x, x, x, None, *(torch.empty_like(frame) for _ in range(3)))
    for i, name in ((0, "q"), (1, "k"), (2, "v")):
        calls.append((lambda i=i: rv.prepare_qkv(prep, *swapped(fwd, i, hx)), name))
        calls.append((lambda i=i: rv.stage_qkv(prep, *swapped((x, x, x, None, torch.empty_like(frame)), i, hx), mem), name))
    for i, name in ((4, "Q"), (5, "K"), (6, "V")):
        calls.append((lambda i=i: rv.prepare_qkv(prep, *swapped(fwd, i, half)), name))
    calls.append((lambda: rv.stage_qkv(prep, x, x, x, None, half, mem), "Q"))
    bwd = (x, x, None, frame, frame, frame, x.clone(), x.clone(), x.clone(), torch.zeros(D, device="cuda"), None, None, None)
    for i, name in ((0, "q"), (1, "k"), (6, "dq"), (7, "dk"), (8, "dv")):
        calls.append((lambda i=i: rv.prepare_qkv_bwd(prep, *swapped(bwd, i, hx)), name))
    for i, name in ((3, "dQ"), (4, "dK"), (5, "dV")):
        calls.append((lambda i=i: rv.prepare_qkv_bwd(prep, *swapped(bwd, i, half)), name))
    calls.append((lambda: rv.prepare_qkv_bwd(prep, *swapped(bwd, 9, torch.zeros(D, dtype=torch.int32, device="cuda"))), "dq_weight"))
    calls.append((lambda: pool.append([s], half, frame, [N]), "K"))
    calls.append((lambda: pool.append([s], frame, half, [N]), "V"))
    calls.append((lambda: pool.gather([s], half, None, [N]), "K"))
    calls.append((lambda: pool.gather([s], None, half, [N]), "V"))
    calls.append((lambda: pool.compact([s], torch.zeros(H, device="cuda"), [1]), "keep"))
    att = (frame, frame, frame, pool, [s], [N], torch.empty_like(frame), lse)
    for i, name in ((0, "Q"), (1, "K"), (2, "V"), (6, "out")):
        calls.append((lambda i=i: rv.attend_seqs(*swapped(att, i, half)), name))
    calls.append((lambda: rv.attend_seqs(*swapped(att, 7, ints)), "lse"))
    adm = (four, four, four, stats, grid, 1, pool, [s], torch.empty_like(stats), idx)
    for i, name, other in ((0, "Q", four_half), (1, "K", four_half), (2, "V", four_half), (3, "lse", int_stats),
                           (8, "saliency_out", int_stats), (9, "idx_out", float_idx)):
        calls.append((lambda i=i, other=other: rv.admit_seqs(*swapped(adm, i, other)), name))
    for n, (call, name) in enumerate(calls):
        with pytest.raises((TypeError, ValueError), match=rf"^{name}: .*(float16|int32|float32)"):
            call()
            pytest.fail(f"call {n} ({name}) was made")
    assert pool.len(s) == N and mem.len == 0
    bits = frame.view(torch.uint16)  # bf16's bits are taken still
    rv.attend_seqs(bits, bits, bits, pool, [s], [N], torch.empty_like(frame).view(torch.int16), lse)
    rv.prepare_qkv(prep, x, x, x, None, *(bits.clone() for _ in range(3)))
    pool.append([s], bits, bits, [N])
    assert pool.len(s) == 2 * N


def test_rows_past_what_a_call_moves_are_refused(rv):
    """2^28 rows x heads of one sequence; the refusal comes before any page is looked for."""
    pool = rv.Pool(1024, 4, 2, 1 << 20)
    s = pool.open()
    seqs, rows = (ctypes.c_int * 1)(s), (ctypes.c_int * 1)((1 << 18) + 1)
    L, at = rv.lib(), ctypes.c_void_p(4096)
    assert L.rv_pool_append(pool.handle, 1, seqs, at, at, rows, None) == rv.RV_ERR_INVALID
    assert b"too many rows for one call" in L.rv_last_error()
    keep, first = (ctypes.c_int64 * 1)((1 << 18) + 1), (ctypes.c_int64 * 1)(0)
    assert L.rv_pool_compact(pool.handle, 1, seqs, first, keep, at, None) == rv.RV_ERR_INVALID
    assert b"too many rows for one call" in L.rv_last_error()
    rows[0] = (1 << 20) + 1
    assert L.rv_pool_append(pool.handle, 1, seqs, at, at, rows, None) == rv.RV_ERR_CAPACITY
    assert pool.len(s) == 0 and pool.free_pages == 4
