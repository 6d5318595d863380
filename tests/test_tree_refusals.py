"""What the calls around a tree of drafted tokens refuse on the host, before any device is touched."""
import ctypes as C

import pytest

P = 4096          # an address that is never read: every call below is refused first


@pytest.fixture(scope="module")
def b():
    from paper_2404_19124_b200 import build
    build.build()
    from paper_2404_19124_b200 import binding
    return binding


def _plan(b, B=2, K=4, n=3, T=13, null=None):
    ptr = [P] * 9
    if null is not None:
        ptr[null] = None
    return b._lib.spec_tree_plan(*ptr[:3], B, K, n, T, *ptr[3:], None)


def test_plan(b):
    for i in range(9):
        assert _plan(b, null=i) == b.SPEC_ERR_INVALID_ARG
    for bad in (dict(B=0), dict(K=0), dict(n=0), dict(T=0), dict(T=-3)):
        assert _plan(b, **bad) == b.SPEC_ERR_INVALID_ARG
    for bad in (dict(T=b.MAX_TREE_NODES + 1), dict(n=b.MAX_TREE_DEPTH + 1), dict(K=b.MAX_TREE_ENTRIES // 3 + 1),
                dict(K=b.MAX_LEAVES + 1, n=1)):
        assert _plan(b, **bad) == b.SPEC_ERR_SHAPE


def _tables(b, null=None, B=2, page=16, new=5, stride=8, width=8, n_free=9):
    ptr = [P] * 10
    if null is not None:
        ptr[null] = None
    return b._lib.spec_page_tables(ptr[0], ptr[1], B, page, new, ptr[2], stride, width, ptr[3], ptr[4], ptr[5], n_free, ptr[6],
                                   ptr[7], ptr[8], None, None)


def test_page_tables(b):
    for i in (0, 2, 3, 4, 5, 6, 7, 8):           # n_new and err_word may be null
        assert _tables(b, null=i) == b.SPEC_ERR_INVALID_ARG
    for bad in (dict(B=0), dict(page=0), dict(new=0), dict(width=0, stride=0), dict(n_free=0)):
        assert _tables(b, **bad) == b.SPEC_ERR_INVALID_ARG
    for bad in (dict(stride=7), dict(B=1 << 16, new=1 << 15), dict(B=1 << 16, width=1 << 15, stride=1 << 15)):
        assert _tables(b, **bad) == b.SPEC_ERR_SHAPE


def _attention(b, **bad):
    f = dict(dtype=0, B=2, T=5, Hq=8, Hkv=2, D=64, page=16, pages=9, width=4, scale=0.1, ptrs=[P] * 6, lens=P, nodes=0, mask=0,
             out=P, lse=0, err=0, stride=4, strides=[64] * 18, ws=P, ws_bytes=1 << 40)
    f.update(bad)
    args = b._ATTENTION.pack(f["dtype"], f["B"], f["T"], f["Hq"], f["Hkv"], f["D"], f["page"], f["pages"], f["width"], f["scale"],
                             *f["ptrs"], f["lens"], f["nodes"], f["mask"], f["out"], f["lse"], f["err"], f["stride"],
                             *f["strides"])
    return b._lib.spec_tree_attention(args, f["ws"], f["ws_bytes"], None)


def test_attention(b):
    null = lambda i: [0 if j == i else P for j in range(6)]
    odd = lambda i: [P + 8 if j == i else P for j in range(6)]
    invalid = [dict(ptrs=null(i)) for i in range(6)] + [dict(ptrs=odd(i)) for i in range(5)] + [
        dict(lens=0), dict(out=0), dict(out=P + 2), dict(dtype=1), dict(dtype=3), dict(B=0), dict(T=0), dict(Hq=0), dict(Hkv=0),
        dict(D=0), dict(page=0), dict(pages=0), dict(width=0), dict(scale=float("nan"))]
    for bad in invalid:
        assert _attention(b, **bad) == b.SPEC_ERR_INVALID_ARG, bad
    shapes = [dict(D=60), dict(D=136), dict(Hq=7), dict(T=b.MAX_TREE_NODES + 1), dict(stride=3)] + [
        dict(strides=[64] * i + [x] + [64] * (17 - i)) for i in (0, 4, 8, 11, 14, 17) for x in (63, -64)]
    for bad in shapes:
        assert _attention(b, **bad) == b.SPEC_ERR_SHAPE, bad
    for bad in (dict(ws=0), dict(ws=P + 16), dict(ws_bytes=b.spec_tree_attention_workspace_bytes(2, 5, 8, 2, 64) - 1)):
        assert _attention(b, **bad) == b.SPEC_ERR_WORKSPACE, bad
    assert b._lib.spec_tree_attention(None, P, 1 << 40, None) == b.SPEC_ERR_INVALID_ARG
    for bad in ((0, 1, 8, 8, 64), (1, 1, 8, 3, 64), (1, 1, 8, 8, 12), (1, 1, 8, 8, 256), (1, 4096, 8, 8, 64)):
        assert b.spec_tree_attention_workspace_bytes(*bad) == 0
    assert b.spec_tree_attention_workspace_bytes(64, 129, 32, 8, 128) % 256 == 0


def _verify(b, **bad):
    f = dict(dtype=0, B=2, T=5, V=100, n=3, max_hist=7, max_bias=4, tree=[P] * 3, logits=P, strides=[500, 100], hist=[P] * 6,
             bias=[P] * 3, allow=P, out=[P] * 4)
    f.update(bad)
    args = b._TREE_VERIFY.pack(f["dtype"], f["B"], f["T"], f["V"], f["n"], f["max_hist"], f["max_bias"], *f["tree"], f["logits"],
                               *f["strides"], *f["hist"], *f["bias"], f["allow"], *f["out"])
    return b._lib.spec_verify_tree(args, None)


def test_verify_tree(b):
    null = lambda i, n: [0 if j == i else P for j in range(n)]
    invalid = [dict(tree=null(i, 3)) for i in range(3)] + [dict(out=null(i, 4)) for i in range(4)] + [
        dict(logits=0), dict(logits=P + 1), dict(dtype=1, logits=P + 2), dict(dtype=5), dict(B=0), dict(T=0), dict(V=0), dict(n=-1),
        dict(strides=[-1, 100]), dict(strides=[500, -100]), dict(hist=null(0, 6)), dict(hist=null(1, 6)), dict(max_hist=0),
        dict(bias=null(1, 3)), dict(max_bias=0)]
    for bad in invalid:
        assert _verify(b, **bad) == b.SPEC_ERR_INVALID_ARG, bad
    for bad in (dict(n=b.MAX_TREE_DEPTH + 1), dict(T=b.MAX_TREE_NODES + 1), dict(V=(1 << 30) + 1), dict(B=(1 << 20) + 1)):
        assert _verify(b, **bad) == b.SPEC_ERR_SHAPE, bad
    assert b._lib.spec_verify_tree(None, None) == b.SPEC_ERR_INVALID_ARG


def test_constraints_that_fit_no_table(b):
    assert _verify(b, V=1 << 22, max_hist=1 << 20) == b.SPEC_ERR_SHAPE


def _commit(b, **bad):
    f = dict(L=3, B=2, T=5, n=3, H=2, D=64, page=16, pages=9, ptrs=[P] * 4, path=P, accept=P, slots=P, lens=P, new=P, err=0,
             strides=[64] * 16)
    f.update(bad)
    args = b._COMMIT.pack(f["L"], f["B"], f["T"], f["n"], f["H"], f["D"], f["page"], f["pages"], *f["ptrs"], f["path"],
                          f["accept"], f["slots"], f["lens"], f["new"], f["err"], *f["strides"])
    return b._lib.spec_kv_commit(args, None)


def test_kv_commit(b):
    null = lambda i: [0 if j == i else P for j in range(4)]
    odd = lambda i: [P + 8 if j == i else P for j in range(4)]
    invalid = [dict(ptrs=null(i)) for i in range(4)] + [dict(ptrs=odd(i)) for i in range(4)] + [
        dict(path=0), dict(accept=0), dict(slots=0), dict(lens=0), dict(L=0), dict(B=0), dict(T=0), dict(n=-1), dict(H=0), dict(D=0),
        dict(page=0), dict(pages=0), dict(strides=[-64] + [64] * 15)]
    for bad in invalid:
        assert _commit(b, **bad) == b.SPEC_ERR_INVALID_ARG, bad
    for bad in (dict(D=60), dict(B=65536), dict(strides=[64] * 15 + [60]), dict(pages=1 << 28)):
        assert _commit(b, **bad) == b.SPEC_ERR_SHAPE, bad
    assert b._lib.spec_kv_commit(None, None) == b.SPEC_ERR_INVALID_ARG


def test_structures_have_the_size_of_the_headers(b, tmp_path):
    """The binding packs the three argument structures by format strings."""
    import os
    import shutil
    import subprocess
    gcc = shutil.which("gcc")
    if gcc is None:
        pytest.skip("no C compiler")
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "size.c"
    src.write_text('#include <stdio.h>\n#include "spec_b200.h"\nint main(void) { printf("%zu %zu %zu %zu %zu %zu", '
                   'sizeof(spec_tree_attention_t), sizeof(spec_tree_verify_t), sizeof(spec_kv_commit_t), '
                   'offsetof(spec_tree_attention_t, table_stride), offsetof(spec_tree_verify_t, hist_tok), '
                   'offsetof(spec_kv_commit_t, k_stride)); return 0; }')
    subprocess.check_call([gcc, "-I", os.path.join(root, "include"), str(src), "-o", str(tmp_path / "size")])
    sizes = [int(x) for x in subprocess.check_output([str(tmp_path / "size")]).split()]
    assert sizes[:3] == [b._ATTENTION.size, b._TREE_VERIFY.size, b._COMMIT.size]
    assert sizes[3:] == [C.sizeof(C.c_int32) * 10 + 8 * 12, 8 * 4 + 8 * 4 + 8 * 2, 8 * 4 + 8 * 10]


def test_the_binding_refuses_host_tensors(b):
    import torch
    z = lambda *s, dt=torch.int32: torch.zeros(s, dtype=dt)
    h = torch.bfloat16
    with pytest.raises(ValueError):
        b.spec_tree_plan(z(1, 2, 3), z(1), z(1), 7)
    with pytest.raises(ValueError):
        b.spec_page_tables(z(1), None, z(1, 4), z(1), z(8), z(1), 16, max_new=4)
    with pytest.raises(ValueError):
        b.spec_tree_attention(z(1, 2, 2, 64, dt=h), z(1, 2, 2, 64, dt=h), z(1, 2, 2, 64, dt=h), z(3, 16, 2, 64, dt=h),
                              z(3, 16, 2, 64, dt=h), z(1, 3), z(1))
    with pytest.raises(ValueError):
        b.spec_verify_tree(z(1, 2), z(1, 2), z(1), z(1, 2, 50, dt=h), n=1)
    with pytest.raises(ValueError):
        b.spec_kv_commit(z(1, 1, 2, 2, 64, dt=h), z(1, 1, 2, 2, 64, dt=h), z(1, 3, 16, 2, 64, dt=h), z(1, 3, 16, 2, 64, dt=h),
                         z(1, 2), z(1), z(1, 2, dt=torch.int64), z(1))
