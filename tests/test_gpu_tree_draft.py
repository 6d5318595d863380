"""Steps of a serving program from its draft to its next context, call by call and from one captured graph: spec_draft, the calls
around the tree of its candidates, spec_next_ctx and the next spec_draft, with a sequence that is idle at times."""
import numpy as np
import pytest
import torch

import oracle
import tree_reference as ref
from helpers import small_cfg, to_oracle_weights, weights_to_cuda
from paper_2404_19124_b200 import synth

pytestmark = pytest.mark.gpu

CFG = small_cfg(d_base=64, d_inner=64, V=520, topk=(3, 2, 2), K=5, B=4, seed=77)
B, K, N, V, T = CFG.B, CFG.K, 3, CFG.V, 1 + 5 * 3
L, HQ, HKV, D, PAGE, WIDTH = 2, 4, 2, 64, 8, 10
POOL = B * WIDTH
IDLE, STEPS = 2, 8                                    # the sequence that is idle in every third step


@pytest.fixture(scope="module")
def spec():
    from paper_2404_19124_b200 import build
    build.build()
    from paper_2404_19124_b200 import binding
    return binding


def words(*shape, dtype=torch.int32, value=0):
    return torch.full(shape, value, dtype=dtype, device="cuda")


class Server:
    """Everything on the device; `busy` [B] and `agree` [B, T] (nodes that the base model will say after their parents) are inputs."""

    def __init__(self, spec, weights):
        self.spec, self.h = spec, spec.spec_create(weights)
        g = torch.Generator(device="cuda").manual_seed(3)
        rand = lambda *s: torch.randn(s, generator=g, device="cuda")
        self.tok_rows, self.pos_rows, self.head = rand(L, V, (HQ + 2 * HKV) * D), rand(L, 200, (HQ + 2 * HKV) * D), rand(HQ * D, V)
        half = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
        self.ctx, self.last = rand(B, CFG.d_base).to(torch.bfloat16), torch.arange(7, 7 + B, dtype=torch.int32, device="cuda")
        self.cand, self.logp = words(B, K, N), words(B, K, dtype=torch.float32)
        self.draft_ws = words(spec.spec_draft_workspace_bytes(self.h, B, CFG.topk, K), dtype=torch.uint8)
        self.tree = spec.SpecTree(words(B, T), words(B, T), words(B, T), words(B, T, 1), words(B, K, N + 1), words(B))
        self.len, self.held, self.table = words(B), words(B), words(B, WIDTH, value=-1)
        self.free, self.count = torch.randperm(POOL, generator=g, device="cuda").to(torch.int32), words(1, value=POOL)
        self.slots = words(B, N + 1, dtype=torch.int64)
        self.caches = [torch.full((L, POOL, PAGE, HKV, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
        self.out, self.ws = half(L, B, T, HQ, D), words(spec.spec_tree_attention_workspace_bytes(B, T, HQ, HKV, D), dtype=torch.uint8)
        self.accept, self.node, self.next, self.path = words(B), words(B), words(B), words(B, N + 1)
        self.logits, self.state, self.new_ctx = words(B, T, V, dtype=torch.float32), half(B, T, CFG.d_base), half(B, CFG.d_base)
        self.busy, self.agree, self.zero, self.err = words(B, value=1), words(B, T, dtype=torch.bool), words(B), words(1)

    def qkv(self, tok, pos):
        x = (self.tok_rows[:, tok.long()] + self.pos_rows[:, pos.long()]).to(torch.bfloat16).unflatten(-1, (HQ + 2 * HKV, D))
        return x[..., :HQ, :], x[..., HQ:HQ + HKV, :], x[..., HQ + HKV:, :]

    def step(self):
        s, tree = self.spec, self.tree
        s.spec_draft(self.h, self.ctx, self.last, CFG.topk, K, cand_tok=self.cand, cand_logp=self.logp, workspace=self.draft_ws)
        s.spec_tree_plan(self.cand, self.last, self.len, T, tree=tree)
        tree.n_nodes.mul_(self.busy)
        s.spec_page_tables(self.len, self.busy * (N + 1), self.table, self.held, self.free, self.count, PAGE, slots=self.slots,
                           err_workspace=self.err)
        q, k, v = self.qkv(tree.tok, tree.pos)
        for l in range(L):
            s.spec_tree_attention(q[l], k[l], v[l], self.caches[0][l], self.caches[1][l], self.table, self.len, mask=tree.mask,
                                  n_nodes=tree.n_nodes, out=self.out[l], workspace=self.ws, err_workspace=self.err)
        torch.matmul(self.out.float().sum(0).flatten(2), self.head, out=self.logits)
        row = tree.parent.clamp_min(0).long()                          # what a node that agrees says of its parent's row
        self.logits.view(-1).index_add_(0, (torch.arange(B, device="cuda")[:, None] * T + row).flatten() * V + tree.tok.flatten(),
                                        (self.agree & (tree.parent >= 0)).flatten().float() * 1e4)
        s.spec_verify_tree(tree.tok, tree.parent, tree.n_nodes, self.logits, accept_len=self.accept, last_node=self.node,
                           next_tok=self.next, path=self.path)
        s.spec_kv_commit(k, v, *self.caches, self.path, self.accept, self.slots, self.len, new_len=self.len, err_workspace=self.err)
        self.state.copy_(self.tok_rows[0, tree.tok.long(), :CFG.d_base] + self.pos_rows[0, tree.pos.long(), :CFG.d_base])
        s.spec_next_ctx(self.state.view(B, 1, T, CFG.d_base), self.zero, self.node, ctx_state=self.new_ctx, err_workspace=self.err)
        keep = self.busy == 0                                          # an idle sequence goes on where it was
        self.ctx.copy_(torch.where(keep[:, None], self.ctx, self.new_ctx))
        self.last.copy_(torch.where(keep, self.last, self.next))


@pytest.mark.parametrize("captured", [False, True])
def test_from_draft_to_draft(spec, captured):
    rng, sw = np.random.default_rng(11), synth.make_weights(CFG)
    ow, server = to_oracle_weights(sw), Server(spec, weights_to_cuda(sw))
    graph = None
    if captured:
        kept = [t.clone() for t in (server.ctx, server.last)]
        server.step()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            server.step()
        for t, value in zip((server.ctx, server.last, server.len, server.held, server.count, server.table), (*kept, 0, 0, POOL, -1)):
            t.copy_(value) if torch.is_tensor(value) else t.fill_(value)
        for c in server.caches:
            c.fill_(float("nan"))
    texts, taken = [[int(t)] for t in server.last], 0
    for step in range(STEPS):
        busy = np.ones(B, np.int32)
        busy[IDLE] = step % 3 != 1
        server.busy.copy_(torch.from_numpy(busy))
        server.agree.copy_(torch.from_numpy(rng.random((B, T)) < 0.6))
        ctx, last, lens = server.ctx.clone(), server.last.cpu().numpy(), server.len.cpu().numpy()
        graph.replay() if captured else server.step()
        # the draft, its tree, the walk, the next context
        cand = server.cand.cpu().numpy()
        assert np.array_equal(cand, oracle.draft(ow, synth.bf16_bits(ctx.cpu()), last, CFG.topk, K)[0])
        want = list(ref.plan(cand, last, lens, T))
        want[5] = want[5] * busy
        for got, w in zip(server.tree, want):
            assert np.array_equal(got.cpu().numpy(), w)
        walk = ref.walk(want[0], want[2], want[5], server.logits.double().cpu().numpy(), N)
        for got, w in zip((server.accept, server.node, server.next, server.path), walk):
            assert np.array_equal(got.cpu().numpy(), w)
        accept, node, nxt, path = walk
        for b in range(B):
            if busy[b]:
                assert torch.equal(server.new_ctx[b], server.state[b, node[b]]) and torch.equal(server.ctx[b], server.new_ctx[b])
                texts[b] += [int(want[0][b, i]) for i in path[b, 1:accept[b] + 1]] + [int(nxt[b])]
                taken += int(accept[b])
            else:
                assert node[b] == -1 and (server.new_ctx[b] == 0).all() and torch.equal(server.ctx[b], ctx[b])
        assert server.len.tolist() == [len(t) - 1 for t in texts] and server.last.tolist() == [t[-1] for t in texts]
        assert spec.spec_poll_error(server.err) == spec.SPEC_OK and spec.spec_poll_error(server.draft_ws) == spec.SPEC_OK
    assert taken > STEPS                               # tokens were accepted, and the cache holds what they need:
    for b, text in enumerate(texts):
        at = torch.arange(len(text) - 1, device="cuda")
        _, k, v = server.qkv(torch.tensor(text[:-1], device="cuda"), at)
        for cache, want in zip(server.caches, (k, v)):
            assert torch.equal(cache[:, server.table[b].long()[at // PAGE], at % PAGE], want)
    spec.spec_destroy(server.h)
