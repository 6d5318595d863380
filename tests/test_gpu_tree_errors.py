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
