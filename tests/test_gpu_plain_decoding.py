"""Decoding steps without drafted tokens through the calls around a tree of them: trees of one node, n = 0."""
import pytest
import torch

pytestmark = pytest.mark.gpu

B, V, HQ, HKV, D, PAGE, WIDTH, STEPS = 3, 97, 4, 2, 64, 4, 8, 21


@pytest.fixture(scope="module")
def spec():
    from paper_2404_19124_b200 import build
    build.build()
    from paper_2404_19124_b200 import binding
    return binding


def words(*shape, dtype=torch.int32, value=0):
    return torch.full(shape, value, dtype=dtype, device="cuda")


@pytest.mark.parametrize("native", [True, False])
def test_steps_of_single_tokens(spec, monkeypatch, native):
    if not native:
        monkeypatch.setattr(spec, "_pycall", None)
    g = torch.Generator(device="cuda").manual_seed(2)
    rows = torch.randn(V, (HQ + 2 * HKV) * D, generator=g, device="cuda").to(torch.bfloat16)
    head = torch.randn(HQ * D, V, generator=g, device="cuda")
    pool = B * WIDTH
    table, held, count = words(B, WIDTH, value=-1), words(B), words(1, value=pool)
    free = torch.randperm(pool, generator=g, device="cuda").to(torch.int32)
    caches = [torch.full((1, pool, PAGE, HKV, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    lens, last, err = words(B), torch.tensor([5, 17, 80], dtype=torch.int32, device="cuda"), words(1)
    parent, nodes, slots = words(B, 1, value=-1), words(B, value=1), words(B, 1, dtype=torch.int64)
    out = torch.zeros(B, 1, HQ, D, dtype=torch.bfloat16, device="cuda")
    ws = words(spec.spec_tree_attention_workspace_bytes(B, 1, HQ, HKV, D), dtype=torch.uint8)
    accept, node, nxt, path = words(B), words(B), words(B), words(B, 1)
    ctx, texts = torch.zeros(B, D, dtype=torch.bfloat16, device="cuda"), [[int(t)] for t in last]
    for _ in range(STEPS):
        spec.spec_page_tables(lens, None, table, held, free, count, PAGE, slots=slots, err_workspace=err)
        qkv = rows[last.long()].view(B, 1, HQ + 2 * HKV, D)
        q, k, v = qkv[:, :, :HQ], qkv[:, :, HQ:HQ + HKV], qkv[:, :, HQ + HKV:]
        spec.spec_tree_attention(q, k, v, caches[0][0], caches[1][0], table, lens, out=out, workspace=ws, err_workspace=err)
        logits = out.float().flatten(2) @ head
        spec.spec_verify_tree(last[:, None], parent, nodes, logits, accept_len=accept, last_node=node, next_tok=nxt, path=path)
        spec.spec_kv_commit(k[None], v[None], *caches, path, accept, slots, lens, new_len=lens, err_workspace=err)
        state = k[:, :, 0].contiguous().view(B, 1, 1, D)
        assert spec.spec_next_ctx(state, words(B), node, ctx_state=ctx, err_workspace=err) is ctx
        assert torch.equal(ctx, state[:, 0, 0])
        assert torch.equal(nxt, logits[:, 0].argmax(-1).to(torch.int32)) and accept.tolist() == [0] * B
        for b in range(B):                             # attention over the text so far, from the definition
            x = rows[torch.tensor(texts[b], device="cuda")].view(-1, HQ + 2 * HKV, D).double()
            for h in range(HQ):
                p = torch.softmax(x[:, HQ + h // 2] @ x[-1, h] * D ** -0.5, 0)
                values = x[:, HQ + HKV + h // 2]
                tol = (p @ values.abs()) * 2.0 ** -8 + (p @ values).abs() * 2.0 ** -8 + 2.0 ** -12
                assert ((out[b, 0, h].double() - p @ values).abs() <= tol).all()
            texts[b].append(int(nxt[b]))
        last.copy_(nxt)
    assert lens.tolist() == [STEPS] * B and spec.spec_poll_error(err) == spec.SPEC_OK
    for b in range(B):
        at, x = torch.arange(STEPS, device="cuda"), rows[torch.tensor(texts[b][:-1], device="cuda")].view(-1, HQ + 2 * HKV, D)
        for c, want in zip(caches, (x[:, HQ:HQ + HKV], x[:, HQ + HKV:])):
            assert torch.equal(c[0, table[b].long()[at // PAGE], at % PAGE], want)
