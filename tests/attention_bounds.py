"""How far an attention output may be from its definition in 64 bits, element by element and as a whole.

What attend_seqs rounds: each probability to bf16 (2^-8 of it at most) for the value product, and the output to bf16.
Sums, statistics and partial results are fp32.  So with p the probabilities and o = p v,
  |err| <= 2^-8 |o| + (2^-8 + 2^-11) sum_j p_j |v_j|:
2^-11 covers fp32's share of the sums' size: up to 5000 additions of a chain (3.0e-4), a logit's 64 products and its
scaling (|z| < 30: below 1e-4), and the products of two of these roundings.
Where the values are drawn independently of the logits with mean zero, the probabilities' roundings do not add up:
  E err^2 = sum_j (p_j d_j)^2 E v^2 <= 2^-16 E o^2,
and with the output's own rounding the whole error is below sqrt(2) 2^-8 = 0.0055 of the output's size; RMS_BOUND leaves
8 % for sums over finitely many elements (both roundings' typical size is 0.0016)."""
import torch

RMS_BOUND = 0.006


def check_rows(got, z, v, random_values=True):
    """got [n, D] against softmax(z) v for logits z [n, m] and values v [m, D], in 64 bits."""
    p = torch.softmax(z, 1)
    ref = p @ v
    err = (got - ref).abs()
    over = err - 2.0 ** -8 * ref.abs() - (2.0 ** -8 + 2.0 ** -11) * (p @ v.abs())
    assert float(over.max()) <= 0, f"an element is past its bound by {float(over.max())}"
    if random_values:
        rms = float(err.norm() / ref.norm())
        assert rms <= RMS_BOUND, f"relative error {rms}"
