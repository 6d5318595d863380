"""Error words that are not aligned are refused on the host, before any device is touched."""
import pytest

P = 4096          # an address that is never read: every call below is refused first


@pytest.fixture(scope="module")
def b():
    from paper_2404_19124_b200 import build
    build.build()
    from paper_2404_19124_b200 import binding
    return binding


@pytest.mark.parametrize("off", [1, 2, 3])
def test_an_error_word_is_four_bytes_at_a_multiple_of_four(b, off):
    assert b._lib.spec_page_tables(P, P, 2, 16, 5, P, 8, 8, P, P, P, 9, P, P, P, P + off, None) == b.SPEC_ERR_INVALID_ARG
    args = b._ATTENTION.pack(0, 2, 5, 8, 2, 64, 16, 9, 4, 0.1, *[P] * 6, P, 0, 0, P, 0, P + off, 4, *[64] * 18)
    assert b._lib.spec_tree_attention(args, P, 1 << 40, None) == b.SPEC_ERR_INVALID_ARG
    args = b._COMMIT.pack(3, 2, 5, 3, 2, 64, 16, 9, *[P] * 4, P, P, P, P, P, P + off, *[64] * 16)
    assert b._lib.spec_kv_commit(args, None) == b.SPEC_ERR_INVALID_ARG


def test_what_the_marshalling_takes_none_of_is_left_to_the_checks(b):
    import torch
    if b._pycall is None:
        pytest.skip("built without the interpreter's headers")
    z = torch.zeros(2, 3, dtype=torch.int32)
    for err in (None, z):
        assert b._pycall.page_tables(z, None, z, z, z, z, 16, z, z, z, err, None) is None
        assert b._pycall.tree_attention(z, z, z, z, z, z, z, None, None, 0.1, z, None, z, err, None) is None
        assert b._pycall.kv_commit(z, z, z, z, z, z, z, z, z, err, None) is None
