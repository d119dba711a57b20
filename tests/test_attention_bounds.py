"""The bounds of attention_bounds accept the kernel's arithmetic, and reject outputs that are wrong in small parts."""
import pytest
import torch

from attention_bounds import check_rows

D = 64


def case(rows, tokens, seed=0):
    g = torch.Generator().manual_seed(seed)
    q, k, v = (torch.randn(n, D, generator=g).bfloat16().double() for n in (tokens, rows, rows))
    return q @ k.t() / 8, v


def rounded(z, v):
    """The output with the roundings that the kernel makes."""
    e = torch.exp(z - z.amax(1, keepdim=True))
    return (e.bfloat16().double() @ v / e.sum(1, keepdim=True)).bfloat16().double()


@pytest.mark.parametrize("rows,tokens", [(1, 1), (65, 3), (2100, 1), (2100, 40), (52000, 1), (52000, 5)])
def test_the_kernels_roundings_pass(rows, tokens):
    for seed in range(3):
        z, v = case(rows, tokens, seed)
        check_rows(rounded(z, v), z, v)
        check_rows(rounded(z * 0, v), z * 0, v)  # equal weights, rounded the same way


@pytest.mark.parametrize("rows,tokens", [(2100, 1), (2100, 40), (52000, 1), (52000, 5)])
def test_wrong_outputs_are_rejected(rows, tokens):
    z, v = case(rows, tokens)
    page, other = slice(640, 704), slice(1280, 1344)
    dropped, swapped, turned = v.clone(), v.clone(), v.clone()
    dropped[page] = 0
    swapped[page], swapped[other] = v[other], v[page]
    turned[page] = v[page].roll(8, 1)  # a piece of 16 bytes off
    for wrong in (torch.zeros(tokens, D).double(), rounded(z, dropped), rounded(z, swapped), rounded(z, turned)):
        with pytest.raises(AssertionError):
            check_rows(wrong, z, v)
