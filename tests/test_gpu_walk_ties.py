"""Equal maxima on the walk: the first index wins, whichever threads and vectors hold them and wherever a row begins."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

BLOCK, THREADS = 4096, 256            # tokens that go to a CTA in turn, threads that share them


@pytest.fixture(scope="module")
def spec():
    from paper_2404_19124_b200 import build
    build.build()
    from paper_2404_19124_b200 import binding
    return binding


def winners(spec, logits, **given):
    """Arg-max of the roots of B trees of one node."""
    B = logits.shape[0]
    z = lambda value: torch.full((B, 1), value, dtype=torch.int32, device="cuda")
    return spec.spec_verify_tree(z(5), z(-1), z(1)[:, 0].clone(), logits, n=0, **given)[2].cpu().numpy()


def pairs(V, skew, per):
    """(low, high): low among the last tokens of a block, which the thread looks at that counts the block's turn, high in the vectors
    of that thread in later turns, for clusters of 1 to 8 CTAs; and pairs at random."""
    rng, blocks, out = np.random.default_rng(V + skew), (V + BLOCK - 1) // BLOCK, set()
    for ctas in (1, 2, 4, 8):
        for rank in {0, ctas - 1}:
            turns = (blocks - rank + ctas - 1) // ctas
            for turn in range(turns - 1):
                for later in {turn + 1, turns - 1}:
                    begin = (later * ctas + rank) * BLOCK
                    for k in range(BLOCK // per // THREADS):
                        for e in {0, per - 1, int(rng.integers(0, per))}:
                            high = begin - skew + (turn + k * THREADS) * per + e
                            low = (turn * ctas + rank) * BLOCK + BLOCK - 1 - int(rng.integers(0, max(skew, 1)))
                            if begin <= high < V:
                                out.add((low, high))
    for _ in range(64):
        out.add(tuple(sorted(rng.choice(V, 2, replace=False).tolist())))
    return sorted(out)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("V", [9001, 50257, 128259])
@pytest.mark.parametrize("B", [1, 64, 300])           # clusters of 8 to 1 CTAs
def test_the_first_of_two_equal_maxima(spec, B, V, dtype):
    per = 16 // torch.empty(0, dtype=dtype).element_size()
    stride = (V + 2 * per) // per * per
    for skew in range(per):
        at = pairs(V, skew, per)
        if B == 1:
            at = at[::max(1, len(at) // 12)]
        for first in range(0, len(at), B):
            some = at[first:first + B]
            some = some + some[:1] * (B - len(some))
            low, high = (torch.tensor(x, device="cuda") for x in zip(*some))
            logits = torch.zeros(B * stride + per, dtype=dtype, device="cuda")[skew:skew + B * stride].view(B, 1, stride)[..., :V]
            assert logits.data_ptr() % 16 == skew * logits.element_size()
            row = torch.arange(B, device="cuda")
            logits[row, 0, low] = 2.0
            logits[row, 0, high] = 2.0
            got = winners(spec, logits)
            assert np.array_equal(got, low.cpu().numpy()), (skew, [(s, int(g)) for s, g in zip(some, got) if g != s[0]][:5])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("value", [float("-inf"), float("nan"), 0.0])
def test_the_first_of_the_allowed_tokens_where_all_are_equal(spec, dtype, value):
    """A row of one value (NaN counts as minus infinity) of which two tokens are allowed."""
    V, B = 50257, 64
    per = 16 // torch.empty(0, dtype=dtype).element_size()
    stride, words = (V + 2 * per) // per * per, (V + 31) // 32
    for skew in range(per):
        at = pairs(V, skew, per)
        at = at[::max(1, len(at) // B)][:B]
        at = at + at[:1] * (B - len(at))
        allow = np.zeros((B, 1, words * 32), np.uint64)
        for b, two in enumerate(at):
            allow[b, 0, list(two)] = 1
        bits = (allow.reshape(B, 1, words, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32).view(np.int32)
        logits = torch.full((B * stride + per,), value, dtype=dtype, device="cuda")[skew:skew + B * stride]
        got = winners(spec, logits.view(B, 1, stride)[..., :V], allow=torch.from_numpy(bits).cuda())
        assert got.tolist() == [low for low, _ in at], skew
