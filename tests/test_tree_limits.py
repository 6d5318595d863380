"""The documented limits of the walk's constraints: refused just outside (on the host, before any device is touched), served just
inside (on the GPU)."""
import numpy as np
import pytest
import torch

import tree_reference as ref

P = 4096          # an address that is never read: every call on it is refused first
# (penalties, biases): vocabularies up to which any lists fit, for any T and for small trees; list entries for V = 2^20
LIMITS = {(True, False): (327680, 393216, 640, 12000), (False, True): (327680, 393216, 640, 12000), (True, True): (196608, 262144, 768, 9000)}
MANY = 1 << 20


@pytest.fixture(scope="module")
def spec():
    from paper_2404_19124_b200 import build
    build.build()
    from paper_2404_19124_b200 import binding
    return binding


def refused(b, V, T, max_hist, max_bias, n=0):
    args = b._TREE_VERIFY.pack(0, 1, T, V, n, max_hist, max_bias, *[P] * 3, P, T * V, V, *([P] * 6 if max_hist else [0] * 6),
                               *([P] * 3 if max_bias else [0] * 3), 0, *[P] * 4)
    return b._lib.spec_verify_tree(args, None) == b.SPEC_ERR_SHAPE


@pytest.mark.parametrize("penalties,biases", LIMITS)
def test_lists_that_do_not_fit(spec, penalties, biases):
    most, most_small, small, _ = LIMITS[penalties, biases]
    hist, bias = MANY * penalties, MANY * biases
    assert refused(spec, most + 1, 1024, hist, bias) and refused(spec, most_small + 1, 1, hist, bias)
    assert refused(spec, most_small, small + 1, hist, bias)
    entries = {(True, True): 9420}.get((penalties, biases), 12850)      # the last that fit: 9416 and 12842
    assert refused(spec, 1 << 20, 1024, entries * penalties, 1 if biases and penalties else entries * biases)


@pytest.mark.gpu
@pytest.mark.parametrize("where", ["any tree", "small trees", "large vocabulary"])
@pytest.mark.parametrize("penalties,biases", LIMITS)
def test_lists_that_fit(spec, penalties, biases, where):
    most, most_small, small, entries = LIMITS[penalties, biases]
    V, T, length = {"any tree": (most, 1024, MANY), "small trees": (most_small, small, MANY),
                    "large vocabulary": (1 << 20, 1024, entries)}[where]
    n = 1
    max_bias = length - n if not penalties else 300 if biases else 0
    max_hist = length - max_bias - n if penalties else 0
    rng = np.random.default_rng(V + T + max_bias)
    logits = (rng.normal(0, 2, V) * 8).round() / 8
    hist = rng.integers(0, V, (1, max(max_hist, 1)))
    bias_tok, bias_val = rng.integers(0, V, (1, max(max_bias, 1))), rng.normal(0, 4, (1, max(max_bias, 1))).astype(np.float32)
    if penalties:
        hist[0, :50] = np.argsort(-logits)[:50]                          # tokens that matter
    freq, pres = np.array([0.5], np.float32), np.array([0.25], np.float32)
    tok, parent = np.full((1, T), 3, np.int32), np.full((1, T), -1, np.int32)
    g = lambda a, dtype: torch.from_numpy(np.ascontiguousarray(a)).to(dtype).cuda()
    given, host = {}, {}
    if penalties:
        given = dict(hist_tok=g(hist, torch.int32), hist_len=g([max_hist], torch.int32), frequency=g(freq, torch.float32),
                     presence=g(pres, torch.float32))
        host = dict(hist=hist.tolist(), freq=freq, pres=pres)
    if biases:
        given.update(bias_tok=g(bias_tok, torch.int32), bias_val=g(bias_val, torch.float32))
        host["bias"] = [list(zip(bias_tok[0].tolist(), bias_val[0].astype(float).tolist()))]
    x = g(logits, torch.float32)[None, None].expand(1, T, V)
    got = spec.spec_verify_tree(g(tok, torch.int32), g(parent, torch.int32), g([1], torch.int32), x, n=n, **given)
    want = ref.walk(tok, parent, [1], np.broadcast_to(logits, (1, T, V)), n, **host)
    assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(got, want))
