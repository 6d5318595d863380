"""The calls around a tree of drafted tokens as a serving program chains them, over several steps and in a captured graph, against a
plain loop over the accepted text."""
import numpy as np
import pytest
import torch

import tree_reference as ref

pytestmark = pytest.mark.gpu

B, K, N, T, V, L, HQ, HKV, D, PAGE = 3, 6, 3, 16, 300, 2, 4, 2, 64, 16
WIDTH, POOL = 12, 3 * 12 + 4


@pytest.fixture(scope="module")
def spec():
    from paper_2404_19124_b200 import build
    build.build()
    from paper_2404_19124_b200 import binding
    return binding


class ToyModel:
    """Queries, keys and values are rows of tables by token and position; the logits are the layers' results, summed, through one
    matrix.  Enough for what a token predicts to depend on all the text before it."""

    def __init__(self):
        g = torch.Generator(device="cuda").manual_seed(1)
        rand = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.tok, self.pos = rand(L, V, (HQ + 2 * HKV) * D), rand(L, 1000, (HQ + 2 * HKV) * D) * 0.5
        self.head = rand(HQ * D, V)

    def qkv(self, tok, pos):
        """[L, .., heads, D] each, bf16"""
        x = (self.tok[:, tok.long()] + self.pos[:, pos.long()]).to(torch.bfloat16)
        x = x.unflatten(-1, (HQ + 2 * HKV, D))
        return x[..., :HQ, :], x[..., HQ:HQ + HKV, :], x[..., HQ + HKV:, :]

    def logits_of_text(self, text):
        """fp64 logits of the last position, from the definition."""
        q, k, v = (t.double() for t in self.qkv(torch.tensor(text, device="cuda"), torch.arange(len(text), device="cuda")))
        total = 0
        for l in range(L):
            out = []
            for h in range(HQ):
                s = k[l, :, h // (HQ // HKV)] @ q[l, -1, h] * D ** -0.5
                out.append(torch.softmax(s, 0) @ v[l, :, h // (HQ // HKV)])
            total = total + torch.cat(out)
        return (total @ self.head.double()).cpu().numpy()


def words(*shape, dtype=torch.int32, value=0):
    return torch.full(shape, value, dtype=dtype, device="cuda")


class Server:
    def __init__(self, spec):
        self.spec, self.model = spec, ToyModel()
        self.caches = [torch.full((L, POOL, PAGE, HKV, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        self.table, self.held = words(B, WIDTH, value=-1), words(B)
        self.free, self.count = torch.randperm(POOL, device="cuda").to(torch.int32), words(1, value=POOL)
        self.len, self.last, self.cand, self.err = words(B), words(B), words(B, K, N), words(1)
        self.tree = spec.SpecTree(words(B, T), words(B, T), words(B, T), words(B, T, 1), words(B, K, N + 1), words(B))
        self.slots = words(B, N + 1, dtype=torch.int64)
        self.out = torch.zeros(L, B, T, HQ, D, dtype=torch.bfloat16, device="cuda")
        self.ws = torch.empty(spec.spec_tree_attention_workspace_bytes(B, T, HQ, HKV, D), dtype=torch.uint8, device="cuda")
        self.accept, self.node, self.next, self.path = words(B), words(B), words(B), words(B, N + 1)
        self.state = torch.zeros(B, T, 8, dtype=torch.bfloat16, device="cuda")
        self.ctx, self.zero = torch.zeros(B, 8, dtype=torch.bfloat16, device="cuda"), words(B)

    def step(self):
        """Candidates after `last` are in `cand`; on return the accepted tokens are in the cache and `last` is the token behind them."""
        s, tree = self.spec, self.tree
        s.spec_tree_plan(self.cand, self.last, self.len, T, tree=tree)
        s.spec_page_tables(self.len, None, self.table, self.held, self.free, self.count, PAGE, slots=self.slots)
        q, k, v = self.model.qkv(tree.tok, tree.pos)
        for l in range(L):
            s.spec_tree_attention(q[l], k[l], v[l], self.caches[0][l], self.caches[1][l], self.table, self.len, mask=tree.mask,
                                  n_nodes=tree.n_nodes, out=self.out[l], workspace=self.ws)
        logits = self.out.float().sum(0).flatten(2) @ self.model.head
        s.spec_verify_tree(tree.tok, tree.parent, tree.n_nodes, logits, accept_len=self.accept, last_node=self.node,
                           next_tok=self.next, path=self.path)
        s.spec_kv_commit(k, v, *self.caches, self.path, self.accept, self.slots, self.len, new_len=self.len)
        self.state.copy_(tree.tok[..., None].expand(-1, -1, 8))        # a state that tells which node it is from
        s.spec_next_ctx(self.state.view(B, 1, T, 8), self.zero, self.node, ctx_state=self.ctx)
        self.last.copy_(self.next)


def drafts(rng, model, texts):
    """Candidates of which some follow what the model would say for a while."""
    cand = ref.random_candidates(rng, B, K, N, V)
    for b, text in enumerate(texts):
        good = list(text)
        for j in range(int(rng.integers(0, N + 1))):
            best = int(np.argmax(model.logits_of_text(good)))
            cand[b, K // 2, j] = best
            good.append(best)
    return torch.from_numpy(cand).cuda()


@pytest.mark.parametrize("captured", [False, True])
def test_steps_of_a_serving_program(spec, captured):
    rng, server = np.random.default_rng(5), Server(spec)
    texts = [[int(t)] for t in rng.integers(0, V, B)]
    first = torch.tensor([t[-1] for t in texts], dtype=torch.int32, device="cuda")
    graph = None
    if captured:
        server.step()                                                  # (candidates of zeros: warms up, then everything is put back)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            server.step()
        for t in (server.len, server.held):
            t.zero_()
        server.count.fill_(POOL)
        server.table.fill_(-1)
        for c in server.caches:
            c.fill_(float("nan"))                                      # pages that belong to nobody
    server.last.copy_(first)
    taken = 0
    for step in range(12):
        server.cand.copy_(drafts(rng, server.model, texts))
        before = [len(t) for t in texts]
        graph.replay() if captured else server.step()
        accept, nxt, path, tok = (t.cpu().numpy() for t in (server.accept, server.next, server.path, server.tree.tok))
        for b in range(B):
            new = [int(tok[b, i]) for i in path[b, 1:accept[b] + 1]] + [int(nxt[b])]
            for t in new:                                              # every token is the model's choice after the text before it
                x = server.model.logits_of_text(texts[b])
                # bf16 results of D-long sums: 2^-8 of probabilities and results over HQ * D products each
                assert x[t] >= x.max() - 2 ** -6 * np.abs(x).max(), (step, b, t)
                texts[b].append(t)
            assert server.ctx[b, 0].item() == float(torch.tensor(float(tok[b, path[b, accept[b]]])).to(torch.bfloat16))
        assert server.len.tolist() == [len(t) - 1 for t in texts] and server.last.tolist() == [t[-1] for t in texts]
        taken += int(accept.sum())
        assert all(len(t) == n + a + 1 for t, n, a in zip(texts, before, accept))
    assert taken > 10                                                  # tokens were accepted, and the cache holds what they need:
    for b in range(B):
        for l in range(L):
            _, k, v = server.model.qkv(torch.tensor(texts[b][:-1], device="cuda"), torch.arange(len(texts[b]) - 1, device="cuda"))
            at = torch.arange(len(texts[b]) - 1, device="cuda")
            for cache, want in zip(server.caches, (k, v)):
                assert torch.equal(cache[l, server.table[b].long()[at // PAGE], at % PAGE], want[l])
    assert sorted(server.table[server.table >= 0].tolist() + server.free[:server.count.item()].tolist()) == list(range(POOL))
