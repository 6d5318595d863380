"""Attention of a tree of drafted tokens over a paged cache, against softmax attention in 64 bits."""
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


class Case:
    def __init__(self, B, T, Hq, Hkv, D, lens, page, dtype=torch.bfloat16, layout="nhd", levels=3, nodes=None, seed=0, std=1.0,
                 empty_rows=0.0, scale=None):
        rng = np.random.default_rng(seed + T * 1000 + D)
        gen = torch.Generator(device="cuda").manual_seed(seed)
        lens = np.resize(np.asarray(lens), B)
        nodes = np.full(B, T) if nodes is None else np.resize(np.asarray(nodes), B)
        held = (lens + page - 1) // page
        width, pages = max(1, int(held.max())), int(held.sum()) + 3
        order, table, at = rng.permutation(pages), np.full((B, width), -1, np.int32), 0
        for b in range(B):
            table[b, :held[b]] = order[at:at + held[b]]
            at += held[b]
        rand = lambda *s: (torch.randn(s, generator=gen, device="cuda") * std).to(dtype)
        cache = lambda: rand(pages, Hkv, page, D).transpose(1, 2) if layout == "hnd" else rand(pages, page, Hkv, D)
        self.q, self.k, self.v, self.k_cache, self.v_cache = rand(B, T, Hq, D), rand(B, T, Hkv, D), rand(B, T, Hkv, D), cache(), cache()
        self.lens, self.nodes, self.table, self.scale = lens, nodes, table, D ** -0.5 if scale is None else scale
        self.seen = np.tril(np.ones((B, T, T), bool)) if levels == 0 else ref.random_tree(rng, B, T, levels, empty_rows)
        self.mask = None if levels == 0 else gpu(ref.pack_mask(self.seen))
        self.g_lens, self.g_nodes, self.g_table = gpu(lens, torch.int32), gpu(nodes, torch.int32), gpu(table)
        self.shape = (B, T, Hq, Hkv, D)

    def run(self, spec, **given):
        B, T, Hq, Hkv, D = self.shape
        args = dict(mask=self.mask, n_nodes=self.g_nodes, scale=self.scale,
                    out=torch.full((B, T, Hq, D), 7.0, dtype=self.q.dtype, device="cuda"),
                    lse=torch.full((B, T, Hq), 7.0, device="cuda"), err_workspace=torch.zeros(1, dtype=torch.int32, device="cuda"))
        args.update(given)
        self.err = args["err_workspace"]
        out = spec.spec_tree_attention(self.q, self.k, self.v, self.k_cache, self.v_cache, self.g_table, self.g_lens, **args)
        return out, args["lse"]

    def check(self, spec, out, lse):
        want, w_lse, tol, lse_tol = ref.attention(self.q, self.k, self.v, self.k_cache, self.v_cache, self.g_table, self.lens,
                                                  self.nodes, self.seen, self.scale)
        for b, N in enumerate(self.nodes):
            bad = (out[b, :N].double() - want[b, :N]).abs() > tol[b, :N]
            assert not bad.any(), (b, bad.nonzero()[:5].tolist(), out[b, :N][bad][:5], want[b, :N][bad][:5], tol[b, :N][bad][:5])
            empty = torch.isinf(w_lse[b, :N])
            assert torch.equal(lse[b, :N][empty], w_lse[b, :N][empty].float())
            assert ((lse[b, :N].double() - w_lse[b, :N]).abs()[~empty] <= lse_tol[b, :N][~empty]).all()
            assert (out[b, N:] == 7).all() and (lse[b, N:] == 7).all()          # rows behind the tree stay as they were
        assert spec.spec_poll_error(self.err) == 0

    def run_and_check(self, spec, **given):
        self.check(spec, *self.run(spec, **given))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("D", [8, 64, 80, 96, 128])
@pytest.mark.parametrize("lens", [[0], [1], [63, 64, 65], [127, 128, 129], [0, 300, 17]])
def test_single_tokens(spec, D, lens, dtype):
    Case(len(lens), 1, 4, 2, D, lens, 16, dtype, levels=0).run_and_check(spec)


@pytest.mark.parametrize("page,layout", [(1, "nhd"), (7, "hnd"), (8, "nhd"), (16, "hnd"), (24, "nhd"), (64, "hnd"), (200, "nhd"),
                                         (32, "nhd"), (128, "hnd"), (256, "nhd"), (384, "hnd")])
@pytest.mark.parametrize("T,lens,nodes", [(5, [250, 3], None), (33, [0, 100], [33, 20]), (61, [511, 90], [1, 61])])
def test_pages_that_end_inside_a_tile(spec, page, layout, T, lens, nodes):
    Case(2, T, 4, 4, 64, lens, page, layout=layout, nodes=nodes).run_and_check(spec)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("Hq,Hkv", [(1, 1), (3, 3), (8, 1), (6, 2), (48, 1), (5, 5)])
@pytest.mark.parametrize("T,levels", [(2, 0), (13, 3), (50, 4)])
def test_grouped_heads(spec, Hq, Hkv, T, levels, dtype):
    Case(2, T, Hq, Hkv, 128, [130, 77], 16, dtype, levels=levels, nodes=[T, (T + 1) // 2]).run_and_check(spec)


@pytest.mark.parametrize("T,Hq,Hkv,D", [(1024, 1, 1, 64), (257, 2, 1, 128), (129, 8, 2, 96), (128, 1, 1, 128), (64, 4, 1, 128)])
def test_large_trees(spec, T, Hq, Hkv, D):
    Case(1, T, Hq, Hkv, D, [200], 16, levels=5).run_and_check(spec)


@pytest.mark.parametrize("B,T,Hq,Hkv,lens", [(1, 1, 2, 1, [20000]), (1, 9, 8, 1, [5001]), (3, 3, 2, 2, [3000, 0, 7001]),
                                            (40, 2, 1, 1, list(range(0, 2000, 50))), (1, 40, 16, 1, [4100])])
def test_long_and_uneven_contexts(spec, B, T, Hq, Hkv, lens):
    Case(B, T, Hq, Hkv, 128, lens, 16, levels=0).run_and_check(spec)


def test_rows_that_see_nothing(spec):
    c = Case(4, 20, 4, 2, 64, [0, 0, 5, 0], 16, empty_rows=0.5, nodes=[20, 0, 20, 7])
    out, lse = c.run(spec)
    c.check(spec, out, lse)
    empty = gpu(~c.seen[0].any(1))
    assert empty.any() and (out[0][empty] == 0).all() and torch.isinf(lse[0][empty]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("lens", [[0], [100], [250]])
def test_keys_that_a_row_does_not_see_do_not_touch_it(spec, lens, value, dtype):
    """Values that are not finite in the tree's other branches, behind its nodes, behind the cache's length and in pages that
    belong to nobody."""
    c = Case(1, 30, 4, 2, 128, lens, 16, dtype, nodes=[25])
    clean, lse = c.run(spec)
    c.check(spec, clean, lse)
    L = lens[0]
    for cache in (c.k_cache, c.v_cache):
        used = torch.zeros(cache.shape[:2], dtype=torch.bool, device="cuda")
        at = torch.arange(L, device="cuda")
        used[c.g_table[0].long()[at // 16], at % 16] = True
        cache[~used] = value
    c.k[0, 25:] = value
    c.v[0, 25:] = value
    poisoned = [3, 11]
    for t in poisoned:
        c.k[0, t, :, ::3] = value
        c.v[0, t, :, ::5] = value
    out, got = c.run(spec)
    hit = torch.as_tensor(c.seen[0, :25][:, poisoned].any(1)).cuda()
    assert hit.any() and not hit.all()
    assert torch.equal(out[0, :25][~hit], clean[0, :25][~hit]) and torch.equal(got[0, :25][~hit], lse[0, :25][~hit])
    assert (out[0, 25:] == 7).all()
    assert not torch.isfinite(out[0, :25][hit][:, :, ::5]).any()


@pytest.mark.parametrize("lens", [[0], [100], [250], [9000]])
def test_values_that_are_not_finite_reach_the_rows_that_see_them(spec, lens):
    c = Case(1, 20, 2, 1, 64, lens, 16)
    c.v[0, 4, 0, 7], c.v[0, 9, 0, 8], c.v[0, 12, 0, 9] = float("inf"), float("-inf"), float("nan")
    if lens[0]:
        c.v_cache[c.g_table[0, lens[0] // 32], 3, 0, 20] = float("inf")
    out, _ = c.run(spec)
    for t, d, what in ((4, 7, float("inf")), (9, 8, float("-inf")), (12, 9, float("nan"))):
        for i in range(20):
            got = out[0, i, :, d].float()
            if not c.seen[0, i, t]: assert torch.isfinite(got).all()
            elif what != what: assert torch.isnan(got).all()
            else: assert (got == what).all()
    if lens[0]:
        assert not torch.isfinite(out[0, :, :, 20].float()).any()
    assert torch.isfinite(out[0, :, :, 21:].float()).all()


@pytest.mark.parametrize("std,scale", [(8.0, None), (30.0, 1.0), (1.0, 0.0), (1.0, -0.5), (0.0, None)])
def test_large_and_degenerate_scores(spec, std, scale):
    Case(2, 9, 2, 1, 64, [700, 90], 16, std=std, scale=scale).run_and_check(spec)


def test_rising_scores_move_the_running_maximum_in_every_tile(spec):
    c = Case(1, 4, 2, 1, 64, [3000], 16, levels=0)
    at = torch.arange(3000, device="cuda")
    c.q.copy_(torch.ones_like(c.q))
    c.k_cache[c.g_table[0].long()[at // 16], at % 16, 0] = (at[:, None] / 1000.0).expand(3000, 64).to(torch.bfloat16)
    c.run_and_check(spec)
    c.k_cache.neg_()                          # falling: the first tile holds the maximum
    c.run_and_check(spec)


def test_strides(spec):
    """Queries, keys and values as slices of one projection, results into a slice, tables with longer rows."""
    c = Case(3, 7, 6, 2, 64, [40, 0, 99], 16, nodes=[7, 3, 6])
    qkv = torch.randn(3, 9, 10, 64, device="cuda").to(torch.bfloat16)
    c.q, c.k, c.v = qkv[:, 1:8, :6], qkv[:, 1:8, 6:8], qkv[:, 1:8, 8:]
    wide = torch.full((3, 9), 10 ** 6, dtype=torch.int32, device="cuda")
    wide[:, :c.g_table.shape[1]] = c.g_table
    c.g_table = wide[:, :c.g_table.shape[1]]
    out = torch.full((6, 3, 7, 72), 7.0, dtype=torch.bfloat16, device="cuda")
    c.run_and_check(spec, out=out[..., 8:].permute(1, 2, 0, 3))
    assert (out[..., :8] == 7).all()


@pytest.mark.parametrize("page", [16, 24, 256])
def test_keys_and_values_interleaved_in_one_pool(spec, page):
    c = Case(2, 11, 4, 2, 128, [700, 390], page)
    pool = torch.full((c.k_cache.shape[0], 2, page, 2, 128), 9.0, dtype=torch.bfloat16, device="cuda")
    pool[:, 0], pool[:, 1] = c.k_cache, c.v_cache
    c.k_cache, c.v_cache = pool[:, 0], pool[:, 1]
    c.run_and_check(spec)


@pytest.mark.parametrize("T", [7, 130])
def test_one_head_of_keys_seen_as_several(spec, T):
    """Expanded inputs: what TMA does not take as a tensor comes row by row."""
    c = Case(2, T, 4, 1, 64, [300, 129], 16)
    c.k, c.v = c.k.expand(-1, -1, 4, -1), c.v.expand(-1, -1, 4, -1)
    c.k_cache, c.v_cache = c.k_cache.expand(-1, -1, 4, -1), c.v_cache.expand(-1, -1, 4, -1)
    c.shape = (2, T, 4, 4, 64)
    c.run_and_check(spec)


@pytest.mark.parametrize("seed", range(12))
def test_random_batches(spec, seed):
    """Lengths, trees, heads and pages at random: units of every kind side by side, in one CTA and across several."""
    rng = np.random.default_rng(100 + seed)
    Hkv = int(rng.choice([1, 2, 3, 5]))
    T = int(rng.choice([1, 2, 17, 40, 90, 200]))
    B = int(rng.integers(1, 9))
    G = int(rng.choice([1, 2, 4, 9] if T < 90 else [1, 2]))
    lens = np.where(rng.random(B) < 0.3, rng.integers(0, 130, B), rng.integers(0, int(rng.choice([300, 3000, 9000])), B))
    Case(B, T, G * Hkv, Hkv, int(rng.choice([64, 88, 128])), lens, int(rng.choice([5, 8, 16, 64, 128])),
         torch.bfloat16 if seed % 2 else torch.float16, layout=["nhd", "hnd"][seed // 2 % 2], levels=int(rng.choice([0, 1, 4])),
         nodes=rng.integers(0, T + 1, B), empty_rows=0.1 * (seed % 3 == 0), seed=seed).run_and_check(spec)


def test_defaults(spec):
    c = Case(2, 3, 2, 1, 64, [40, 70], 16, levels=0)
    out = spec.spec_tree_attention(c.q, c.k, c.v, c.k_cache, c.v_cache, c.g_table, c.g_lens)
    c.err = torch.zeros(1, dtype=torch.int32, device="cuda")
    c.check(spec, out, c.run(spec)[1])


def test_offsets_beyond_32_bits(spec):
    """A cache of more than 2^32 elements, its last pages in use."""
    pages, page, Hkv, D = 33000, 16, 64, 128
    store = torch.empty((2, pages, page, Hkv, D), dtype=torch.bfloat16, device="cuda")
    assert store[0].numel() > 2 ** 32
    c = Case(1, 3, 64, 64, D, [100], page, levels=0)
    held = c.g_table.shape[1]
    for new, old in zip(store, (c.k_cache, c.v_cache)):
        new[-held:] = old[c.g_table[0].long()]
    c.k_cache, c.v_cache = store[0], store[1]
    c.g_table = torch.arange(pages - held, pages, dtype=torch.int32, device="cuda")[None]
    c.run_and_check(spec)


def test_indices_out_of_range(spec):
    c = Case(4, 5, 2, 1, 64, [40, 40, 40, 40], 16, levels=0)
    c.run_and_check(spec)
    table = c.g_table.clone()
    for bad in (-1, c.k_cache.shape[0], 2 ** 31 - 1, -2 ** 31):
        c.g_table = table.clone()
        c.g_table[2, 1] = bad
        out, lse = c.run(spec)
        assert spec.spec_poll_error(c.err) == spec.SPEC_ERR_INDEX_RANGE
        # the page reads as zeros; the other sequences do not notice
        k, v, t = (torch.cat([x, torch.zeros_like(x[:1])]) for x in (c.k_cache, c.v_cache, c.v_cache))
        zeroed = c.g_table.clone()
        zeroed[2, 1] = len(k) - 1
        want, _, tol, _ = ref.attention(c.q, c.k, c.v, k, v, zeroed, c.lens, c.nodes, c.seen, c.scale)
        assert ((out.double() - want).abs() <= tol).all()
    c.g_table = table
    for lens, nodes, w_lens, w_nodes in (([-4, 40, 40, 40], [5, 5, 5, 5], [0, 40, 40, 40], [5, 5, 5, 5]),
                                         ([40, 900, 40, 40], [5, 5, 5, 5], [40, 48, 40, 40], [5, 5, 5, 5]),
                                         ([40, 40, 40, 40], [5, -1, 99, 5], [40, 40, 40, 40], [5, 0, 5, 5])):
        c.g_lens, c.g_nodes = gpu(lens, torch.int32), gpu(nodes, torch.int32)
        out, lse = c.run(spec)
        assert spec.spec_poll_error(c.err) == spec.SPEC_ERR_INDEX_RANGE
        c.lens, c.nodes, c.err = np.array(w_lens), np.array(w_nodes), torch.zeros(1, dtype=torch.int32, device="cuda")
        c.check(spec, out, lse)


def test_another_stream_and_a_captured_graph(spec):
    c = Case(3, 21, 4, 2, 128, [300, 1000, 41], 16)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    out, lse = c.run(spec, stream=side)
    side.synchronize()
    c.check(spec, out, lse)
    B, T, Hq, Hkv, D = c.shape
    ws = torch.empty(spec.spec_tree_attention_workspace_bytes(B, T, Hq, Hkv, D), dtype=torch.uint8, device="cuda")
    args = dict(out=torch.full_like(out, 7.0), lse=torch.full_like(lse, 7.0), workspace=ws,
                err_workspace=torch.zeros(1, dtype=torch.int32, device="cuda"))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(spec, **args)
    # other lengths, trees and values than at capture
    other = Case(3, 21, 4, 2, 128, [999, 2, 640], 16, nodes=[21, 4, 13], seed=5)
    other.g_table = c.g_table.clone().fill_(-1)
    assert other.table.shape[1] <= c.g_table.shape[1]
    pages = c.k_cache.shape[0]
    for b in range(3):                        # into c's pool: the other case's page i is page i mod pages here
        other.g_table[b, :other.table.shape[1]] = gpu(np.where(other.table[b] >= 0, other.table[b] % pages, -1))
    n = min(pages, other.k_cache.shape[0])
    c.k_cache[:n], c.v_cache[:n] = other.k_cache[:n], other.v_cache[:n]
    for name in ("q", "k", "v", "mask", "g_lens", "g_nodes", "g_table"):
        getattr(c, name).copy_(getattr(other, name))
    c.lens, c.nodes, c.seen = other.lens, other.nodes, other.seen
    for _ in range(3):
        args["out"].fill_(7.0)
        args["lse"].fill_(7.0)
        graph.replay()
        c.err = args["err_workspace"]
        c.check(spec, args["out"], args["lse"])


def test_a_batch_without_a_node(spec):
    c = Case(3, 5, 2, 1, 64, [0, 70, 300], 16, nodes=[0, 0, 0])
    out, lse = c.run(spec)
    assert (out == 7).all() and (lse == 7).all() and spec.spec_poll_error(c.err) == 0


def test_calls_on_two_streams_at_once(spec):
    cases = [Case(4, 30, 8, 4, 128, [2000, 900, 30, 4000], 16, seed=1), Case(3, 90, 8, 2, 64, [700, 3000, 1], 64, seed=2)]
    args, streams = [], [torch.cuda.Stream(), torch.cuda.Stream()]
    for c in cases:
        B, T, Hq, Hkv, D = c.shape
        args.append(dict(out=torch.full_like(c.q, 7.0), lse=torch.full((B, T, Hq), 7.0, device="cuda"),
                         workspace=torch.empty(spec.spec_tree_attention_workspace_bytes(B, T, Hq, Hkv, D), dtype=torch.uint8,
                                               device="cuda"), err_workspace=torch.zeros(1, dtype=torch.int32, device="cuda")))
    torch.cuda.synchronize()
    for _ in range(20):
        for c, a, s in zip(cases, args, streams):
            c.run(spec, stream=s, **a)
    torch.cuda.synchronize()
    for c, a in zip(cases, args):
        c.check(spec, a["out"], a["lse"])


def test_graphs_that_share_a_workspace_one_after_the_other(spec):
    cases = [Case(4, 30, 8, 4, 128, [2000, 900, 30, 4000], 16, seed=1), Case(2, 30, 8, 4, 128, [700, 3000], 64, seed=2)]
    ws = torch.empty(max(spec.spec_tree_attention_workspace_bytes(*c.shape) for c in cases), dtype=torch.uint8, device="cuda")
    graphs, args = [], []
    for c in cases:
        B, T, Hq, Hkv, D = c.shape
        args.append(dict(out=torch.full_like(c.q, 7.0), lse=torch.full((B, T, Hq), 7.0, device="cuda"), workspace=ws,
                         err_workspace=torch.zeros(1, dtype=torch.int32, device="cuda")))
        c.run(spec, **args[-1])
        torch.cuda.synchronize()
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            c.run(spec, **args[-1])
    for _ in range(3):
        for c, a, graph in zip(cases, args, graphs):
            a["out"].fill_(7.0)
            a["lse"].fill_(7.0)
            graph.replay()
        for c, a in zip(cases, args):
            c.err = a["err_workspace"]
            c.check(spec, a["out"], a["lse"])


def test_results_repeat_bit_for_bit(spec):
    c = Case(5, 30, 8, 2, 128, [900, 20, 3000, 0, 411], 16)
    first = c.run(spec)
    for _ in range(5):
        again = c.run(spec)
        assert torch.equal(first[0], again[0]) and torch.equal(first[1], again[1])


def test_binding_refusals(spec):
    c = Case(2, 3, 4, 2, 64, [40, 70], 16)
    good = dict(q=c.q, k=c.k, v=c.v, k_cache=c.k_cache, v_cache=c.v_cache, block_table=c.g_table, seq_len=c.g_lens, mask=c.mask,
                n_nodes=c.g_nodes)
    spec.spec_tree_attention(**good)
    half = lambda t: t.to(torch.float16)
    wrong = [dict(q=c.q.float()), dict(k=half(c.k)), dict(v=c.v[:, :2]), dict(k_cache=half(c.k_cache)), dict(v_cache=c.v_cache[:-1]),
             dict(block_table=c.g_table.long()), dict(seq_len=c.g_lens.long()), dict(seq_len=c.g_lens[:1]), dict(mask=c.mask[:, :2]),
             dict(n_nodes=c.g_nodes.cpu()), dict(q=c.q.transpose(2, 3).contiguous().transpose(2, 3)), dict(out=torch.empty_like(c.q[:1])),
             dict(out=torch.empty_like(c.q[:1]).expand(2, -1, -1, -1)), dict(lse=torch.empty(2, 3, 4)),
             dict(lse=torch.empty((2, 3, 4), dtype=torch.float64, device="cuda"))]
    for bad in wrong:
        with pytest.raises((ValueError, spec.SpecError)):
            spec.spec_tree_attention(**{**good, **bad})
    with pytest.raises(spec.SpecError) as e:
        spec.spec_tree_attention(**good, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == spec.SPEC_ERR_WORKSPACE
