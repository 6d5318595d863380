"""What the calls around a tree of drafted tokens tell about their errors, and what they leave behind them."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def spec():
    from paper_2404_19124_b200 import build
    build.build()
    from paper_2404_19124_b200 import binding
    return binding


def i32(*values):
    return torch.tensor(values[0] if len(values) == 1 else values, dtype=torch.int32, device="cuda")


def zeros(*shape, dtype=torch.int32):
    return torch.zeros(shape, dtype=dtype, device="cuda")


# ---- error words through the native marshalling ---------------------------------------------------------------------
class Calls:
    """The three calls that take an error word, with all outputs given, one index of each out of range where `bad`."""

    def __init__(self, spec, bad):
        self.spec = spec
        h = torch.bfloat16
        self.table, self.held = i32([[0, 1, -1]]), i32([2])
        self.free, self.count = i32([3]), i32([0 if bad else 1])                        # the third page: there is none
        self.slots = zeros(1, 3, dtype=torch.int64)
        self.q, self.cache = torch.ones(1, 3, 2, 64, dtype=h, device="cuda"), torch.ones(2, 1, 4, 16, 2, 64, dtype=h, device="cuda")
        self.pages = i32([[0, 99 if bad else 1]])                                       # the cache has four pages
        self.out = torch.zeros_like(self.q)
        self.ws = zeros(spec.spec_tree_attention_workspace_bytes(1, 3, 2, 2, 64), dtype=torch.uint8)
        self.path, self.accept = i32([[0, 9 if bad else 1, 2]]), i32([2])               # the tree has three nodes

    def tables(self, err):
        self.spec.spec_page_tables(i32([30]), i32([3]), self.table, self.held, self.free, self.count, 16, slots=self.slots,
                                   err_workspace=err)

    def attention(self, err):
        self.spec.spec_tree_attention(self.q, self.q, self.q, self.cache[0, 0], self.cache[1, 0], self.pages, i32([20]), out=self.out,
                                      workspace=self.ws, err_workspace=err)

    def commit(self, err):
        slots = torch.tensor([[20, 21, 22]], device="cuda")
        self.spec.spec_kv_commit(self.q[None], self.q[None], self.cache[0], self.cache[1], self.path, self.accept, slots,
                                 err_workspace=err)

    def state(self):
        return [t.clone() for t in (self.table, self.held, self.count, self.slots, self.out, self.cache)]


@pytest.mark.parametrize("bad", [False, True])
@pytest.mark.parametrize("dtype,words", [(torch.int32, 1), (torch.int32, 64), (torch.uint8, 256), (torch.uint8, 4)])
def test_an_error_word_does_not_leave_the_native_marshalling(spec, monkeypatch, bad, dtype, words):
    if spec._pycall is None:
        pytest.skip("built without the interpreter's headers")
    want = {"tables": spec.SPEC_ERR_PAGES, "attention": spec.SPEC_ERR_INDEX_RANGE, "commit": spec.SPEC_ERR_INDEX_RANGE}
    native = []
    for name in ("page_tables", "tree_attention", "kv_commit"):
        real = getattr(spec._pycall, name)
        monkeypatch.setattr(spec._pycall, name, lambda *a, _r=real: native.append(_r(*a)) or native[-1])
    results = []
    for marshalled in (True, False):
        if not marshalled:
            monkeypatch.setattr(spec, "_pycall", None)
        calls, quiet = Calls(spec, bad), Calls(spec, bad)
        for name in ("tables", "attention", "commit"):
            err = zeros(words, dtype=dtype)
            getattr(calls, name)(err)
            assert spec.spec_poll_error(err) == (want[name] if bad else spec.SPEC_OK), name
            getattr(quiet, name)(None)
        results += [calls.state(), quiet.state()]
    assert native == [spec.SPEC_OK] * 6
    for r in results[1:]:
        assert all(torch.equal(a, b) for a, b in zip(results[0], r))


def test_error_words_that_are_none_are_refused(spec):
    calls = Calls(spec, False)
    for err in (zeros(1).cpu(), zeros(3, dtype=torch.uint8), zeros(8, dtype=torch.uint8)[1:5]):
        for call in (calls.tables, calls.attention, calls.commit):
            with pytest.raises(ValueError, match="err_workspace"):
                call(err)


# ---- lengths after a shortage of pages ------------------------------------------------------------------------------
def test_a_commit_counts_the_rows_that_have_a_slot(spec):
    """Sequences that get all, some or none of their pages: the new length ends where their slots end."""
    B, n, page, pages, D = 5, 4, 4, 16, 8
    lens, held = i32([6, 6, 8, 3, 7]), i32([2, 2, 2, 1, 2])
    table = torch.full((B, 6), -1, dtype=torch.int32, device="cuda")
    table[0, :2], table[1, :2], table[2, :2], table[3, :1], table[4, :2] = i32([0, 1]), i32([2, 3]), i32([4, 5]), i32([6]), i32([7, 8])
    err, count = zeros(1), i32([1])
    slots = spec.spec_page_tables(lens, None, table, held, i32([9]), count, page, max_new=n + 1, err_workspace=err)
    assert spec.spec_poll_error(err) == spec.SPEC_ERR_PAGES and (slots >= 0).sum(1).tolist() == [5, 2, 0, 1, 1]
    accept = i32([4, 4, 2, 0, 3])                                     # 5, 5, 3, 1 and 4 rows, for 5, 2, none, 1 and 1 slots
    path = torch.arange(n + 1, dtype=torch.int32, device="cuda").repeat(B, 1)
    k = torch.arange(B * (n + 1) * D, dtype=torch.int16, device="cuda").view(1, B, n + 1, 1, D)
    caches = [torch.full((1, pages, page, 1, D), -1, dtype=torch.int16, device="cuda") for _ in range(2)]
    new_len, err = zeros(B), zeros(1)
    spec.spec_kv_commit(k, k, *caches, path, accept, slots, lens, new_len=new_len, err_workspace=err)
    assert new_len.tolist() == [11, 8, 8, 4, 8] and spec.spec_poll_error(err) == spec.SPEC_ERR_INDEX_RANGE
    for b in range(B):                                                # every token that a length counts is where the table says
        for j in range(int(lens[b]), int(new_len[b])):
            for c in caches:
                assert torch.equal(c[0, table[b, j // page], j % page, 0], k[0, b, j - int(lens[b]), 0])
    assert sum(int((c.view(-1, D) >= 0).all(1).sum()) for c in caches) == 2 * (5 + 2 + 0 + 1 + 1)


def test_a_commit_in_place_after_a_shortage(spec):
    """new_len may be seq_len; more sequences than a block has threads, rows of every number."""
    B, n, page = 700, 3, 4
    accept = torch.arange(B, device="cuda").remainder(n + 1).to(torch.int32)
    room = torch.arange(B, device="cuda").remainder(n + 3)            # slots that the sequence has; n + 1 or more: all
    slots = torch.arange(B * (n + 1), device="cuda").view(B, n + 1)
    slots[torch.arange(n + 1, device="cuda")[None] >= room[:, None]] = -1
    path = torch.arange(n + 1, dtype=torch.int32, device="cuda").repeat(B, 1)
    k = torch.zeros(2, B, n + 1, 1, 8, dtype=torch.bfloat16, device="cuda")
    cache = torch.ones(2, B * (n + 1) // page, page, 1, 8, dtype=torch.bfloat16, device="cuda")
    lens = torch.arange(B, dtype=torch.int32, device="cuda")
    spec.spec_kv_commit(k, k, cache, cache.clone(), path, accept, slots, lens, new_len=lens)
    want = torch.arange(B, device="cuda") + torch.minimum(accept + 1, room)
    assert torch.equal(lens.long(), want)


# ---- a row of the batch that is idle --------------------------------------------------------------------------------
def test_an_idle_row_does_not_trip_the_next_context(spec):
    """Its last node is -1: its state becomes zeros, without an error that would hide a real one."""
    B, T, V, d = 4, 3, 40, 24
    tok, parent, nodes = i32([[1, 2, 3]] * B), i32([[-1, 0, 1]] * B), i32([3, 0, 1, 0])
    logits = zeros(B, T, V, dtype=torch.float32)
    logits[:, 0, 2] = logits[:, 1, 3] = 1
    accept, last, _, _ = spec.spec_verify_tree(tok, parent, nodes, logits, n=2)
    assert accept.tolist() == [2, 0, 0, 0] and last.tolist() == [2, -1, 0, -1]
    state = torch.randn(B, 1, T, d, device="cuda").to(torch.bfloat16)
    want = state[:, 0].gather(1, last.long().clamp_min(0)[:, None, None].expand(-1, 1, d))[:, 0]
    want[1], want[3] = 0, 0
    err = zeros(1)
    got = spec.spec_next_ctx(state, zeros(B), last, err_workspace=err)
    assert torch.equal(got, want) and spec.spec_poll_error(err) == spec.SPEC_OK
    odd = torch.empty(B * T * d + 1, dtype=torch.bfloat16, device="cuda")[1:].view(B, 1, T, d)
    odd.copy_(state)
    given = torch.ones(B, d, dtype=torch.bfloat16, device="cuda")
    assert spec.spec_next_ctx(odd, zeros(B), last, ctx_state=given, err_workspace=err) is given
    assert torch.equal(given, want) and spec.spec_poll_error(err) == spec.SPEC_OK


@pytest.mark.parametrize("best,accept", [(0, -2), (0, 3), (1, 0), (-1, 0), (-1, -1), (0, -2 ** 31)])
def test_other_indices_out_of_range_are_still_errors(spec, best, accept):
    err = zeros(1)
    got = spec.spec_next_ctx(torch.ones(1, 1, 3, 8, dtype=torch.bfloat16, device="cuda"), i32([best]), i32([accept]), err_workspace=err)
    assert (got == 0).all() and spec.spec_poll_error(err) == spec.SPEC_ERR_INDEX_RANGE
