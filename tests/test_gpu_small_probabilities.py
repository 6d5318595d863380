"""Attention over contexts in which many keys of little weight stand beside one of much weight."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}     # half a step of the last place, relative


@pytest.fixture(scope="module")
def spec():
    from paper_2404_19124_b200 import build
    build.build()
    from paper_2404_19124_b200 import binding
    return binding


def tolerance(dtype, n, want):
    """Of a result whose values are 0 and 1: the probabilities and the result are rounded to `dtype` (half a step each); in fp16 the
    first are held relative to the greatest times 2^7, in whose subnormal range a step is 2^-24, so that each is off by 2^-25 2^-7 at
    most; the products of 16 keys at a time are added in fp32, with an error of 2^-23 of what is there at most, the sums of 64 keys
    with 2^-24.  Beside that 2^-17: arguments of up to 25 in base 2 are off by 2^-20 twice and 2^-19.4 (times ln 2), the joining
    kernel's exponential of such by 13 units of the last place, log-sum-exps, exponentials and the division by less than 2^-20."""
    small = n * 2.0 ** -32 if dtype == torch.float16 else 0.0
    return want * (2 * HALF[dtype] + n / 16 * 2.0 ** -23 + (n / 64 + 64) * 2.0 ** -24 + 2.0 ** -17) * 1.01 + small + 2.0 ** -25


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("n", [1000, 16001, 131071])
@pytest.mark.parametrize("where", [0.0, 0.5, 1.0])
@pytest.mark.parametrize("B,T,Hq,Hkv", [(1, 1, 1, 1), (1, 3, 8, 2), (1, 40, 4, 1), (32, 1, 8, 8)])
def test_many_small_probabilities_keep_their_weight(spec, B, T, Hq, Hkv, where, n, dtype):
    """One key whose score is 17.40625 above those of n others: e^-17.4 is below half of fp16's least number.  (32 sequences of
    the same cache: enough that no other thread block shares their keys.)"""
    D, page = 64, 16
    pages = (n + page) // page + 1
    table = torch.randperm(pages, device="cuda").to(torch.int32).repeat(B, 1)
    q, k = torch.zeros(B, T, Hq, D, dtype=dtype, device="cuda"), torch.zeros(B, T, Hkv, D, dtype=dtype, device="cuda")
    q[..., 0], q[..., 1] = 4.0, 1.0
    k_cache, v_cache = (torch.zeros(pages, page, Hkv, D, dtype=dtype, device="cuda") for _ in range(2))
    top = min(int(where * n), n)                       # n + 1 keys in the cache, this one the great one
    at, offset = int(table[0, top // page]), top % page
    k_cache[at, offset, :, 0], k_cache[at, offset, :, 1] = 4.34375, 0.03125
    v_cache[..., 0] = 1.0                              # column 0: every key, 1: all but the great one, 2: the great one
    v_cache[..., 1] = 1.0
    v_cache[at, offset, :, 1], v_cache[at, offset, :, 2] = 0.0, 1.0
    mask = torch.zeros(B, T, (T + 31) // 32, dtype=torch.int32, device="cuda")        # the tree itself is not seen
    lse = torch.empty(B, T, Hq, device="cuda")
    lens = torch.tensor([n + 1] * B, dtype=torch.int32, device="cuda")
    out = spec.spec_tree_attention(q, k, torch.ones_like(k), k_cache, v_cache, table, lens, mask=mask, scale=1.0, lse=lse)
    p = math.exp(-17.40625)
    total = 1 + n * p
    for column, want in enumerate((1.0, n * p / total, 1 / total)):
        got = out[..., column].double()
        assert ((got - want).abs() <= tolerance(dtype, n, want)).all(), (column, got.flatten()[:3].tolist(), want)
    assert (out[..., 3:] == 0).all()
    assert (lse.double() - (17.40625 + math.log(total))).abs().max() <= 17.4 * 2.0 ** -21 + (n / 64 + 64) * 2.0 ** -24 + 2.0 ** -17
