"""Candidates to tree, block tables and slots, the greedy walk and the copy of accepted keys and values, against plain
implementations on the host."""
import numpy as np
import pytest
import torch

import tree_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def spec():
    from paper_2404_19124_b200 import build
    build.build()
    from paper_2404_19124_b200 import binding
    return binding


def gpu(a, dtype=None):
    t = torch.from_numpy(np.ascontiguousarray(a))
    return (t if dtype is None else t.to(dtype)).cuda()


def equal(got, want):
    for g, w in zip(got, want):
        assert np.array_equal(g.cpu().numpy(), w), (g.cpu().numpy(), w)


# ---- spec_tree_plan ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("B,K,n,T,vocab,short", [
    (1, 1, 1, 1, 50, 0.0), (1, 1, 1, 2, 50, 0.0), (2, 1, 5, 6, 9, 0.0), (3, 5, 3, 16, 4, 0.0), (5, 32, 3, 97, 6, 0.3),
    (2, 64, 4, 257, 3, 0.1), (2, 64, 4, 33, 100, 0.0), (70, 7, 2, 15, 2, 0.5), (1, 1024, 8, 1024, 4, 0.0),
    (1, 4096, 2, 1024, 60, 0.1), (2, 2, 64, 129, 2, 0.0), (1, 4096, 1, 32, 40, 0.0), (3, 33, 3, 64, 2, 1.0)])
def test_plan(spec, B, K, n, T, vocab, short):
    rng = np.random.default_rng(K * 100 + n)
    cand = ref.random_candidates(rng, B, K, n, vocab, short=short)
    last, lens = rng.integers(0, vocab, B).astype(np.int32), rng.integers(0, 2 ** 30, B).astype(np.int32)
    tree = spec.spec_tree_plan(gpu(cand), gpu(last), gpu(lens), T)
    equal(tree, ref.plan(cand, last, lens, T))


def test_plan_takes_any_token_and_writes_into_given_tensors(spec):
    cand = np.array([[[2 ** 31 - 1, 0], [2 ** 31 - 1, 2 ** 31 - 1], [0, 0], [-5, 3], [2 ** 31 - 1, -1]]], np.int32)
    out = spec.SpecTree(*(torch.full(s, 77, dtype=torch.int32, device="cuda") for s in
                          ((1, 7), (1, 7), (1, 7), (1, 7, 1), (1, 5, 3), (1,))))
    tree = spec.spec_tree_plan(gpu(cand), gpu([9], torch.int32), gpu([4], torch.int32), 7, tree=out)
    assert all(a is b for a, b in zip(tree, out))
    equal(tree, ref.plan(cand, [9], [4], 7))


# ---- spec_page_tables ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("B,page,max_new,uniform,max_len,spare,slack", [
    (1, 16, 5, True, 100, 9, 4), (64, 16, 5, True, 3000, 0, 2), (3, 1, 7, False, 40, 5, 3), (7, 24, 300, False, 200, 0, 1),
    (33, 64, 4096, False, 1, 3, 0), (2500, 16, 3, True, 90, 1, 2), (1, 128, 1, True, 127, 0, 0), (5, 8, 1, False, 8, 2, 1),
    (40, 16, 200, False, 100, -100, 0), (1500, 4, 9, False, 30, -700, -1)])
def test_page_tables(spec, B, page, max_new, uniform, max_len, spare, slack):
    rng = np.random.default_rng(B + page)
    lens = rng.integers(0, max_len + 1, B).astype(np.int32)
    new = None if uniform else rng.integers(0, max_new + 1, B).astype(np.int32)
    held = ((lens + page - 1) // page + rng.integers(0, 2, B)).astype(np.int32)
    want = (lens + (max_new if uniform else new) + page - 1) // page
    width = max(int(max(want.max(), held.max())) + slack, int(held.max()))
    free = max(int(np.maximum(want - held, 0).sum()) + spare, 1)
    order = rng.permutation(int(held.sum()) + free).astype(np.int32)
    table, at = np.full((B, width), -1, np.int32), 0
    for b in range(B):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
    stack = order[at:]
    w_slots, w_table, w_held, w_count, short = ref.page_tables(lens, new, table, held, stack, len(stack), page, max_new)
    assert short or spare >= 0
    for in_place in (False, True):
        wide = torch.full((B, width + 3), -7, dtype=torch.int32, device="cuda")      # rows further apart than they are long
        t = wide[:, :width]
        t.copy_(gpu(table))
        g_held, g_count, err = gpu(held), gpu([len(stack)], torch.int32), torch.zeros(64, dtype=torch.int32, device="cuda")
        outs = {} if in_place else dict(n_pages_out=torch.zeros_like(g_held), free_count_out=torch.zeros_like(g_count))
        slots = spec.spec_page_tables(gpu(lens), None if uniform else gpu(new), t, g_held, gpu(stack), g_count, page,
                                      max_new=max_new, err_workspace=err, **outs)
        equal((slots, t, outs.get("n_pages_out", g_held), outs.get("free_count_out", g_count)),
              (w_slots, w_table, w_held, np.array([w_count], np.int32)))
        assert (wide[:, width:] == -7).all()
        if not in_place:
            equal((g_held, g_count), (held, np.array([len(stack)], np.int32)))
        assert spec.spec_poll_error(err) == (spec.SPEC_ERR_PAGES if short else spec.SPEC_OK)


@pytest.mark.parametrize("change", ["len", "new_low", "new_high", "held_low", "held_high", "count_low", "count_high", "page"])
def test_page_tables_clamp_what_is_out_of_range(spec, change):
    lens, new, held, count = [20, 5], [3, 2], [2, 1], [4]
    table = np.array([[3, 4, -1, -1], [5, -1, -1, -1]], np.int32)
    stack, ok = np.array([10, 11, 12, 13], np.int32), dict(lens=[20, 5], new=[3, 2], held=[2, 1], count=4)
    if change == "len": lens, ok["lens"] = [-3, 5], [0, 5]
    if change == "new_low": new, ok["new"] = [3, -2 ** 31], [3, 0]
    if change == "new_high": new, ok["new"] = [3, 900], [3, 4]
    if change == "held_low": held, ok["held"] = [2, -1], [2, 0]
    if change == "held_high": held, ok["held"] = [2, 9], [2, 4]
    if change == "count_low": count, ok["count"] = [-5], 0
    if change == "count_high": count, ok["count"] = [500], 4
    if change == "page": table[0, 1] = -9
    lists = (np.array(ok["lens"]), np.array(ok["new"]), table, np.array(ok["held"], np.int32))
    slots, _, w_held, w_count, _ = ref.page_tables(*lists, stack, ok["count"], 16, 4)
    err, t, h, c = torch.zeros(1, dtype=torch.int32, device="cuda"), gpu(table), gpu(held, torch.int32), gpu(count, torch.int32)
    got = spec.spec_page_tables(gpu(lens, torch.int32), gpu(new, torch.int32), t, h, gpu(stack), c, 16, max_new=4,
                                err_workspace=err)
    slots[slots < 0] = -1
    equal((got, h, c), (slots, w_held, np.array([w_count], np.int32)))
    assert spec.spec_poll_error(err) == spec.SPEC_ERR_INDEX_RANGE


# ---- spec_verify_tree ----------------------------------------------------------------------------------------------
def _walk_case(rng, B, K, n, T, V, dtype, agree=0.8):
    """Trees and logits that agree with them for a while; ties and values that penalties reorder among them."""
    cand = ref.random_candidates(rng, B, K, n, V)
    tok, _, parent, _, _, nodes = ref.plan(cand, rng.integers(0, V, B), np.zeros(B, int), T)
    logits = (rng.normal(0, 2, (B, T, V)) * 8).round() / 8          # many exact ties
    for b in range(B):
        for i in range(1, nodes[b]):
            if rng.random() < agree:
                logits[b, parent[b, i], tok[b, i]] = 12.0 + rng.integers(0, 3)
    return tok, parent, nodes, torch.from_numpy(logits).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("B,K,n,T,V", [(1, 1, 1, 2, 1), (2, 3, 2, 7, 7), (5, 8, 4, 20, 1000), (3, 16, 3, 49, 32003), (40, 4, 2, 9, 515),
                                       (2, 2, 0, 1, 4099), (1, 600, 1, 601, 128256), (2, 5, 64, 200, 333)])
def test_walk_without_constraints(spec, B, K, n, T, V, dtype):
    rng = np.random.default_rng(V + n)
    tok, parent, nodes, logits = _walk_case(rng, B, K, max(n, 1), T, V, dtype)
    want = ref.walk(tok, parent, nodes, logits.double().numpy(), n)
    equal(spec.spec_verify_tree(gpu(tok), gpu(parent), gpu(nodes), logits.cuda(), n=n), want)
    # rows further apart than they are long, at every alignment
    wide = torch.full((B, T + 1, V + 13), float("nan"), dtype=dtype, device="cuda")
    for start in range(1, 9, 3):
        view = wide[:, :T, start:start + V]
        view.copy_(logits)
        equal(spec.spec_verify_tree(gpu(tok), gpu(parent), gpu(nodes), view, n=n), want)


def _constraints(rng, B, T, V, tok, hist_max, bias_max):
    size = rng.integers(0, hist_max + 1, B)
    size[0] = hist_max
    hist = rng.integers(0, V, (B, hist_max))
    hist[:, ::3] = rng.choice(tok.reshape(-1), hist[:, ::3].shape)      # tokens that matter, some of them often
    hist[:, 1::7] = rng.choice([-1, V, 2 ** 31 - 1, -2 ** 31], hist[:, 1::7].shape)
    prompt = rng.integers(0, hist_max + 2, B)
    f = dict(rep=rng.uniform(0.7, 1.6, B).astype(np.float32), freq=rng.uniform(-0.4, 0.9, B).astype(np.float32),
             pres=rng.uniform(-0.4, 0.9, B).astype(np.float32))
    bias_len = rng.integers(0, bias_max + 1, B)
    bias_len[0] = bias_max
    bias_tok = rng.choice(tok.reshape(-1), (B, bias_max))
    bias_tok[:, ::2] = rng.integers(-1, V + 1, bias_tok[:, ::2].shape)
    bias_val = rng.normal(0, 4, (B, bias_max)).astype(np.float32)
    allow = rng.random((B, T, V)) < 0.7
    allow[0, 0] = True
    allow[B - 1, :] &= rng.random((T, 1)) < 0.7                       # rows that allow nothing
    words = np.zeros((B, T, (V + 31) // 32 * 32), np.uint64)
    words[:, :, :V] = allow
    words[:, :, V:] = rng.integers(0, 2, words[:, :, V:].shape)       # bits behind the vocabulary do not count
    words = (words.reshape(B, T, -1, 32) << np.arange(32, dtype=np.uint64)).sum(-1).astype(np.uint32).view(np.int32)
    host = dict(hist=[hist[b, :size[b]].tolist() for b in range(B)], prompt=prompt, **f, allow=allow,
                bias=[list(zip(bias_tok[b, :bias_len[b]].tolist(), bias_val[b, :bias_len[b]].astype(float).tolist()))
                      for b in range(B)])
    dev = dict(hist_tok=gpu(hist, torch.int32), hist_len=gpu(size, torch.int32), prompt_len=gpu(prompt, torch.int32),
               repetition=gpu(f["rep"]), frequency=gpu(f["freq"]), presence=gpu(f["pres"]), bias_tok=gpu(bias_tok, torch.int32),
               bias_val=gpu(bias_val), bias_len=gpu(bias_len, torch.int32), allow=gpu(words))
    return host, dev


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
@pytest.mark.parametrize("B,K,n,T,V,hist_max,bias_max", [(2, 3, 2, 7, 7, 5, 3), (6, 8, 4, 30, 1000, 300, 20),
                                                         (3, 16, 3, 40, 32003, 2000, 64), (2, 4, 3, 13, 300007, 900, 30),
                                                         (2, 4, 3, 13, 50000, 30000, 5), (1, 4, 3, 13, 262144, 20000, 300),
                                                         (150, 3, 2, 7, 9000, 40, 3)])
def test_walk_with_constraints(spec, B, K, n, T, V, hist_max, bias_max, dtype):
    rng = np.random.default_rng(V + hist_max)
    tok, parent, nodes, logits = _walk_case(rng, B, K, n, T, V, dtype)
    host, dev = _constraints(rng, B, T, V, tok, hist_max, bias_max)
    x = logits.double().numpy()
    call = lambda **given: spec.spec_verify_tree(gpu(tok), gpu(parent), gpu(nodes), logits.cuda(), n=n, **given)
    hist = ("hist_tok", "hist_len", "prompt_len", "repetition", "frequency", "presence")
    bias = ("bias_tok", "bias_val", "bias_len")
    pick = lambda *names: {k: dev[k] for k in names}
    h = {k: host[k] for k in ("hist", "prompt", "rep", "freq", "pres")}
    equal(call(**dev), ref.walk(tok, parent, nodes, x, n, **host))
    equal(call(**pick(*hist)), ref.walk(tok, parent, nodes, x, n, **h))
    equal(call(**pick(*bias)), ref.walk(tok, parent, nodes, x, n, bias=host["bias"]))
    equal(call(**pick("allow")), ref.walk(tok, parent, nodes, x, n, allow=host["allow"]))
    equal(call(**pick("hist_tok", "hist_len", "repetition")), ref.walk(tok, parent, nodes, x, n, hist=h["hist"], rep=h["rep"]))
    equal(call(**pick("hist_tok", "hist_len", "presence")), ref.walk(tok, parent, nodes, x, n, hist=h["hist"], pres=h["pres"]))


def test_equal_tokens_and_many_of_them(spec):
    """A history of one token, of two in turn, and biases that name one token again and again: the last one counts."""
    V, H = 70000, 5000
    tok, parent, nodes = np.array([[3, 60000], [3, 60000]], np.int32), np.array([[-1, 0]] * 2, np.int32), np.array([2, 2], np.int32)
    logits = np.zeros((2, 2, V), np.float32)
    logits[:, :, 60000], logits[:, :, 5], logits[:, :, 69999] = 900.0, 500.0, 300.0
    hist = np.stack([np.full(H, 60000), np.where(np.arange(H) % 2, 60000, 5)]).astype(np.int32)
    f = np.array([0.125, 0.125], np.float32)
    bias_tok, bias_val = np.full((2, 600), 69999, np.int32), np.tile(np.arange(600, dtype=np.float32), (2, 1))
    got = spec.spec_verify_tree(gpu(tok), gpu(parent), gpu(nodes), gpu(logits), n=1, hist_tok=gpu(hist),
                                hist_len=gpu([H, H], torch.int32), frequency=gpu(f), bias_tok=gpu(bias_tok), bias_val=gpu(bias_val))
    want = ref.walk(tok, parent, nodes, logits.astype(np.float64), 1, hist=hist.tolist(), freq=f,
                    bias=[list(zip(a.tolist(), b.tolist())) for a, b in zip(bias_tok, bias_val)])
    # sequence 0: 900 - 5000 / 8 = 275 < 500; sequence 1: 900 - 312.5 = 587.5, 500 - 312.5; and 300 + 599 = 899 is above them all
    equal(got, want)
    assert got[2].tolist() == [69999, 69999]


def test_penalties_count_the_tokens_taken_on_the_walk(spec):
    """A chain of one token: every step makes it less likely, until another one wins."""
    V, n = 100, 6
    tok, parent = np.full((1, n + 1), 5, np.int32), np.arange(-1, n, dtype=np.int32)[None]
    logits = torch.zeros(1, n + 1, V)
    logits[..., 5], logits[..., 9] = 10.0, 7.5
    f = lambda x: gpu([x], torch.float32)
    got = spec.spec_verify_tree(gpu(tok), gpu(parent), gpu([n + 1], torch.int32), logits.cuda(), n=n,
                                hist_tok=gpu([[5]], torch.int32), hist_len=gpu([1], torch.int32), frequency=f(0.5))
    # 10 - 0.5 c > 7.5 for c = 1 .. 4; at c = 5 the lower index wins the tie, at c = 6 token 9 does
    assert [int(t) for t in got[:3]] == [5, 5, 9] and got[3].tolist() == [[0, 1, 2, 3, 4, 5, -1]]


def test_walk_edges(spec):
    nan, inf = float("nan"), float("inf")
    tok, parent = np.array([[0, 1, 1, 2]] * 7, np.int32), np.array([[-1, 0, 0, 1]] * 7, np.int32)
    logits = torch.zeros(7, 4, 5)
    logits[0, 0, 1] = 1.0                     # two children carry token 1: the lower one; then all equal: token 0
    logits[1, 0] = nan                        # nothing but NaN: token 0
    logits[2, 0] = torch.tensor([nan, -inf, nan, -inf, -inf])
    logits[3, 0] = torch.tensor([nan, inf, inf, nan, 3.0])
    logits[4, 0, 1], logits[4, 1, 2] = 2.0, 2.0
    logits[5, 0, 1], logits[5, 1, 2] = 2.0, 2.0
    nodes = np.array([4, 4, 4, 4, 4, 3, 0], np.int32)       # 5: node 3 is not in use; 6: empty
    got = spec.spec_verify_tree(gpu(tok), gpu(parent), gpu(nodes), logits.cuda(), n=2)
    equal(got, ref.walk(tok, parent, nodes, logits.double().numpy(), 2))
    assert got[0].tolist() == [1, 0, 0, 1, 2, 1, 0] and got[2].tolist() == [0, 0, 0, 0, 0, 2, -1]
    over = nodes.copy()
    over[4], over[6] = 2 ** 30, -5            # more nodes than rows, fewer than none
    equal(spec.spec_verify_tree(gpu(tok), gpu(parent), gpu(over), logits.cuda(), n=2), [g.cpu().numpy() for g in got])


def test_allowed_minus_infinity_wins_over_disallowed_tokens(spec):
    logits = torch.full((1, 1, 40), float("-inf"), device="cuda")
    logits[0, 0, 3] = 1.0
    allow = torch.zeros(1, 1, 2, dtype=torch.int32, device="cuda")
    z = lambda x: gpu([x], torch.int32)
    run = lambda: spec.spec_verify_tree(z([0]), z([-1]), z(1), logits, n=0, allow=allow)
    assert int(run()[2]) == -1
    allow[0, 0, 1] = 1 << 4
    assert int(run()[2]) == 36
    allow[0, 0, 0] = 1 << 2 | 1 << 5
    assert int(run()[2]) == 2


# ---- spec_kv_commit ------------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.int16])
@pytest.mark.parametrize("L,B,T,n,H,D,page,layout", [(1, 1, 1, 0, 1, 8, 1, "nhd"), (3, 5, 9, 3, 2, 64, 16, "hnd"),
                                                     (2, 33, 40, 11, 5, 72, 24, "nhd"), (40, 2, 7, 4, 3, 128, 8, "hnd")])
def test_kv_commit(spec, L, B, T, n, H, D, page, layout, dtype):
    rng = np.random.default_rng(L * B)
    accept = rng.integers(-1, min(n, T - 1) + 1, B).astype(np.int32)
    accept[0] = min(n, T - 1)
    path = np.stack([np.concatenate([[0], np.sort(rng.permutation(T - 1)[:n] + 1), np.full(n, -1)])[:n + 1] for _ in range(B)])
    pages = (B * (n + 1) + page - 1) // page + 2
    slots = rng.permutation(pages * page)[:B * (n + 1)].reshape(B, n + 1)
    lens = rng.integers(0, 1000, B).astype(np.int32)
    make = lambda *s: torch.from_numpy(rng.integers(-2 ** 15, 2 ** 15, s).astype(np.int16)).cuda().view(dtype)
    # trees as slices of one projection [L, B, T, 3, H, D], caches in either order
    kv = make(L, B, T, 3, H, D)
    k, v = kv[:, :, :, 1], kv[:, :, :, 2]
    caches = [make(L, pages, H, page, D).transpose(2, 3) if layout == "hnd" else make(L, pages, page, H, D) for _ in range(2)]
    want = [c.contiguous().view(torch.int16).cpu().numpy() for c in caches]
    for w, src in zip(want, (k, v)):
        rows = src.contiguous().view(torch.int16).cpu().numpy()
        for b in range(B):
            for j in range(accept[b] + 1):
                w[:, slots[b, j] // page, slots[b, j] % page] = rows[:, b, path[b, j]]
    err, new_len = torch.zeros(1, dtype=torch.int32, device="cuda"), gpu(lens)
    spec.spec_kv_commit(k, v, *caches, gpu(path, torch.int32), gpu(accept), gpu(slots, torch.int64), new_len, new_len=new_len,
                        err_workspace=err)
    for c, w in zip(caches, want):
        assert np.array_equal(c.contiguous().view(torch.int16).cpu().numpy(), w)
    assert np.array_equal(new_len.cpu().numpy(), lens + accept + 1) and spec.spec_poll_error(err) == 0


def test_kv_commit_skips_what_is_out_of_range(spec):
    L, B, T, n, H, D, page, pages = 2, 6, 3, 2, 1, 16, 4, 5
    k = torch.arange(L * B * T * H * D, dtype=torch.int16, device="cuda").reshape(L, B, T, H, D)
    caches = [torch.full((L, pages, page, H, D), -1, dtype=torch.int16, device="cuda") for _ in range(2)]
    path = np.array([[0, 1, 2], [0, -1, 2], [0, 3, 2], [0, 1, 2], [0, 1, 2], [0, 1, 2]])
    slots = np.array([[0, 1, 2], [3, 4, 5], [6, 7, 8], [9, -1, 10], [11, 12, 20], [13, 14, 2 ** 40]])
    accept = np.array([9, 2, 2, 2, 2, 2])                              # 9: as many as there are
    lens, err = np.zeros(B), torch.zeros(1, dtype=torch.int32, device="cuda")
    new_len = torch.zeros(B, dtype=torch.int32, device="cuda")
    spec.spec_kv_commit(k, k, *caches, gpu(path, torch.int32), gpu(accept, torch.int32), gpu(slots, torch.int64),
                        gpu(lens, torch.int32), new_len=new_len, err_workspace=err)
    want = np.full((L, pages * page, H, D), -1, np.int16)
    for b in range(B):
        for j in range(3):
            if 0 <= path[b, j] < T and 0 <= slots[b, j] < pages * page:
                want[:, slots[b, j]] = k[:, b, path[b, j]].cpu().numpy()
    for c in caches:
        assert np.array_equal(c.cpu().numpy().reshape(want.shape), want)
    assert new_len.tolist() == [3] * B and spec.spec_poll_error(err) == spec.SPEC_ERR_INDEX_RANGE


def test_an_idle_row_of_the_batch_is_left_as_it_is(spec):
    B, T, n, V = 3, 2, 1, 40
    tok, parent, nodes = gpu([[1, 2]] * B, torch.int32), gpu([[-1, 0]] * B, torch.int32), gpu([2, 0, 1], torch.int32)
    logits = torch.zeros(B, T, V, device="cuda")
    logits[:, 0, 2] = logits[:, 1, 7] = 1
    accept, last, nxt, path = spec.spec_verify_tree(tok, parent, nodes, logits, n)
    assert accept.tolist() == [1, 0, 0] and path.tolist() == [[0, 1], [-1, -1], [0, -1]] and nxt.tolist() == [7, -1, 2]
    lens, held, count = gpu([3, 5, 4], torch.int32), gpu([1, 2, 1], torch.int32), gpu([5], torch.int32)
    table = gpu([[0, -1], [1, 2], [3, -1]], torch.int32)
    slots = spec.spec_page_tables(lens, gpu([2, 0, 2], torch.int32), table, held, gpu([4, 5, 6, 7, 8], torch.int32), count, 4, n + 1)
    assert slots.tolist() == [[3, 32], [-1, -1], [28, 29]]
    k = torch.arange(B * T * 8, dtype=torch.float16, device="cuda").reshape(1, B, T, 1, 8)
    caches = [torch.full((1, 9, 4, 1, 8), -1, dtype=torch.float16, device="cuda") for _ in range(2)]
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    spec.spec_kv_commit(k, k, *caches, path, accept, slots, lens, new_len=lens, err_workspace=err)
    want = torch.full((36, 8), -1, dtype=torch.float16, device="cuda")
    want[3], want[32], want[28] = k[0, 0, 0, 0], k[0, 0, 1, 0], k[0, 2, 0, 0]
    assert all(torch.equal(c.view(36, 8), want) for c in caches)
    assert lens.tolist() == [5, 5, 5] and spec.spec_poll_error(err) == 0


# ---- marshalling ---------------------------------------------------------------------------------------------------
def test_both_ways_of_marshalling_give_the_same(spec, monkeypatch):
    if spec._pycall is None:
        pytest.skip("built without the interpreter's headers")
    rng = np.random.default_rng(3)
    B, K, n, T, V = 3, 6, 3, 14, 700
    cand = ref.random_candidates(rng, B, K, n, V)
    last, lens = rng.integers(0, V, B).astype(np.int32), np.array([7, 0, 300], np.int32)
    logits = torch.from_numpy(rng.normal(0, 2, (B, T, V))).to(torch.float16).cuda()
    hist = gpu(rng.integers(0, V, (B, 50)), torch.int32)
    kv = torch.from_numpy(rng.normal(0, 1, (2, B, T, 3, 2, 64))).to(torch.bfloat16).cuda()
    q = torch.from_numpy(rng.normal(0, 1, (B, T, 4, 64))).to(torch.bfloat16).cuda()

    def run():
        words = lambda *s, dtype=torch.int32: torch.zeros(s, dtype=dtype, device="cuda")
        tree = spec.SpecTree(words(B, T), words(B, T), words(B, T), words(B, T, 1), words(B, K, n + 1), words(B))
        spec.spec_tree_plan(gpu(cand), gpu(last), gpu(lens), T, tree=tree)
        table, held, count = words(B, 30), words(B), gpu([90], torch.int32)
        slots = words(B, n + 1, dtype=torch.int64)
        free = torch.arange(90, dtype=torch.int32, device="cuda")
        spec.spec_page_tables(gpu(lens), None, table, held, free, count, 16, slots=slots)
        caches = torch.ones(2, 2, 90, 16, 2, 64, dtype=torch.bfloat16, device="cuda")
        out, lse = torch.zeros_like(q), torch.zeros(B, T, 4, device="cuda")
        ws = words(spec.spec_tree_attention_workspace_bytes(B, T, 4, 2, 64), dtype=torch.uint8)
        spec.spec_tree_attention(q, kv[0, :, :, 0], kv[0, :, :, 1], caches[0, 0], caches[1, 0], table, gpu(lens), mask=tree.mask,
                                 n_nodes=tree.n_nodes, out=out, lse=lse, workspace=ws)
        outs = words(B), words(B), words(B), words(B, n + 1)
        spec.spec_verify_tree(tree.tok, tree.parent, tree.n_nodes, logits, hist_tok=hist, hist_len=gpu([50, 3, 0], torch.int32),
                              frequency=gpu([0.5, 0.1, 0.2], torch.float32), accept_len=outs[0], last_node=outs[1],
                              next_tok=outs[2], path=outs[3])
        new_len = words(B)
        spec.spec_kv_commit(kv[..., 1, :, :], kv[..., 2, :, :], caches[0], caches[1], outs[3], outs[0], slots, gpu(lens),
                            new_len=new_len)
        return (*tree, table, held, count, slots, out, lse, *outs, caches, new_len)

    calls = []
    for name in ("tree_plan", "page_tables", "tree_attention", "verify_tree", "kv_commit"):
        real = getattr(spec._pycall, name)
        monkeypatch.setattr(spec._pycall, name, lambda *a, _r=real, _n=name: calls.append((_n, _r(*a))) or calls[-1][1])
    fast = run()
    assert [c[0] for c in calls] == ["tree_plan", "page_tables", "tree_attention", "verify_tree", "kv_commit"]
    assert all(status == spec.SPEC_OK for _, status in calls)
    monkeypatch.setattr(spec, "_pycall", None)
    for a, b in zip(fast, run()):
        assert torch.equal(a, b)


def test_marshalling_leaves_what_is_wrong_to_the_checks(spec):
    z = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt, device="cuda")
    h = torch.bfloat16
    tree = spec.SpecTree(z(1, 4), z(1, 4), z(1, 4), z(1, 4, 1), z(1, 2, 4), z(1))
    good = (z(1, 2, 3), z(1), z(1), 4)
    spec.spec_tree_plan(*good, tree=tree)
    for bad in (tree._replace(tok=z(1, 5)), tree._replace(mask=z(1, 4)), tree._replace(n_nodes=z(1).cpu()),
                tree._replace(parent=z(4, 1).T[:, ::1].expand(1, 4)[:, [0, 1, 2, 3]].long())):
        with pytest.raises(ValueError):
            spec.spec_tree_plan(*good, tree=bad)
    for slots in (z(1, 3), z(2, 3, dt=torch.int64)):
        with pytest.raises(ValueError):
            spec.spec_page_tables(z(1), None, z(1, 4), z(1), z(8), z(1), 16, slots=slots)
    with pytest.raises(ValueError):
        spec.spec_page_tables(z(2), None, z(1, 4).expand(2, 4), z(2), z(8), z(1), 16, slots=z(2, 3, dt=torch.int64))
    outs = dict(accept_len=z(1), last_node=z(1), next_tok=z(1), path=z(1, 3))
    for bad in (dict(logits=z(1, 4, 9)), dict(hist_tok=z(2, 3)), dict(allow=z(1, 4, 2)), dict(bias_tok=z(1, 3)),
                dict(repetition=z(1)), dict(path=z(2, 3))):
        args = {**dict(tok=z(1, 4), parent=z(1, 4), n_nodes=z(1), logits=z(1, 4, 9, dt=h)), **outs, **bad}
        with pytest.raises((ValueError, spec.SpecError)):
            spec.spec_verify_tree(**args)
    kv, cache = z(1, 1, 4, 2, 64, dt=h), z(1, 3, 16, 2, 64, dt=h)
    for bad in (dict(path=z(1, 3).long()), dict(slots=z(1, 3)), dict(k_cache=cache[..., :32]),
                dict(v_cache=cache[:, :1].expand(1, 3, 16, 2, 64)), dict(v=kv.float())):
        args = {**dict(k=kv, v=kv, k_cache=cache, v_cache=cache, path=z(1, 3), accept_len=z(1), slots=z(1, 3, dt=torch.int64)), **bad}
        with pytest.raises(ValueError):
            spec.spec_kv_commit(**args)


def test_host_threads_call_with_different_sizes(spec):
    """Small and large tables in shared memory in turn, from several host threads at once."""
    import threading
    rng = np.random.default_rng(8)
    large = gpu(ref.random_candidates(rng, 1, 4096, 2, 50)), gpu([3], torch.int32), gpu([4], torch.int32)
    middle = gpu(ref.random_candidates(rng, 1, 700, 8, 9)), gpu([3], torch.int32), gpu([4], torch.int32)
    V = 300000
    logits = torch.zeros(1, 1, V, dtype=torch.bfloat16, device="cuda")
    node = gpu([[5]], torch.int32), gpu([[-1]], torch.int32), gpu([1], torch.int32)
    long, short = (gpu(rng.integers(0, V, (1, m)), torch.int32) for m in (9000, 40))
    size = lambda h: gpu([h.shape[1]], torch.int32)
    sizes = {long: size(long), short: size(short)}
    walk = lambda h: spec.spec_verify_tree(*node, logits, 1, hist_tok=h, hist_len=sizes[h])
    jobs = [lambda: spec.spec_tree_plan(*large, 64), lambda: spec.spec_tree_plan(*middle, 64), lambda: walk(long),
            lambda: walk(short)]
    want = [[t.clone() for t in job()] for job in jobs]
    torch.cuda.synchronize()
    wrong, start = [], threading.Barrier(len(jobs))

    def work(job, expected):
        try:
            start.wait()
            for _ in range(300):
                got = job()
            torch.cuda.current_stream().synchronize()
            if not all(torch.equal(g, w) for g, w in zip(got, expected)):
                wrong.append("values")
        except Exception as e:                                        # noqa: BLE001
            wrong.append(repr(e))

    threads = [threading.Thread(target=work, args=a) for a in zip(jobs, want)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not wrong
