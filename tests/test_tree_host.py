"""Host side of the operators for several new tokens: the header against the binding, refusals, the page book's cut, and the
oracle's own values. Nothing here launches a kernel."""

import os
import re
import shutil
import subprocess

import numpy as np
import pytest
import torch

import paper_2609_38095_amd as zo
from oracle import decode as single
from oracle import tree as oracle
from paper_2609_38095_amd import decode, tree

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_38095_amd", "csrc")


def test_header_declares_what_the_binding_names():
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "zo_tree.h")).read(), flags=re.S)
    names = sorted(set(re.findall(r"^\w[\w* ]*?\b(zo_\w+)\s*\(", text, flags=re.M)))
    assert names == sorted(tree.EXPORTS)
    assert all(hasattr(zo.library(), name) for name in names)
    assert int(re.search(r"ZO_TREE_WORDS (\d+)u", text).group(1)) == zo.ZO_TREE_WORDS


def test_header_is_plain_c(tmp_path):
    cc = shutil.which("gcc")
    if cc is None:
        pytest.skip("no gcc")
    (tmp_path / "a.c").write_text('#include "zo_tree.h"\nint f(const zo_tree* t) { return zo_tree_lay(t, 0); }\n')
    r = subprocess.run([cc, "-std=c99", "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), "-c", str(tmp_path / "a.c"),
                        "-o", str(tmp_path / "a.o")], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_host_code_under_asan_ubsan(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "tree_check")
    cmd = [cxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           os.path.join(ROOT, "tests", "helpers", "tree_check.cpp"), os.path.join(CSRC, "zo_checks.cpp"),
           os.path.join(CSRC, "zo_pages.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "tree_check ok" in r.stdout, r.stdout + r.stderr


def test_null_structs_are_refused():
    lib = decode._lib()
    for name in ("zo_tree_lay", "zo_tree_attend", "zo_tree_accept", "zo_tree_keep"):
        assert getattr(lib, name)(None, None) == zo.ZO_ERR_NULL
    assert lib.zo_norm_rotate_put_at(None, None, None) == zo.ZO_ERR_NULL


def test_binding_refuses_what_is_not_on_the_device():
    x, i = torch.zeros(2, 4, 64), torch.zeros(2, dtype=torch.int32)
    for call, args in ((zo.zo_tree_lay, (i, i, 2)), (zo.zo_tree_attend, (x, x, x, i, i, i)), (zo.zo_tree_attend, (None, x, x, i, i, i)),
                       (zo.zo_tree_accept, (i, i, i, 3)), (zo.zo_tree_accept, (None, i, i, 3)), (zo.zo_tree_keep, ([x], [x], i, i, i)),
                       (zo.zo_tree_lay, (None, None, 2))):
        with pytest.raises(TypeError):
            call(*args)


def test_book_cut():
    book = zo.ZoPages(8, 4)
    a = book.add(6)
    b = book.fork(a)
    book.extend(b, 9)
    assert book.left() == 8 - 5 and book.length(b) == 15
    book.cut(b, 7)
    assert book.left() == 5 and book.length(b) == 7
    book.cut(b, 7)
    with pytest.raises(zo.ZoError):
        book.cut(b, 8)
    book.cut(b, 0)
    assert book.left() == 6 and book.length(b) == 0 and book.length(a) == 6
    with pytest.raises(zo.ZoError):
        book.cut(9, 0)
    with pytest.raises(zo.ZoError):
        book.cut(a, -1)


def test_oracle_of_chains_and_trees():
    """A chain is the attention of single tokens whose lengths grow; a tree that of each token's branch put one after another."""
    rng = np.random.default_rng(0)
    k, v = rng.standard_normal((2, 8, 2, 4, 8))
    table = np.array([[3, 1, 5, 0], [2, 7, 6, 4]])
    q = rng.standard_normal((9, 4, 8))
    cached, starts = [5, 3], [0, 4, 9]
    out, lse, _, _ = oracle.attend(q, k, v, table, cached, starts, None, 0.5)
    for s in range(2):
        for i, t in enumerate(range(starts[s], starts[s + 1])):
            want = single.attend(q[t:t + 1], k, v, table[s:s + 1], [cached[s] + i + 1], 0.5)
            np.testing.assert_allclose(out[t], want[0][0], rtol=1e-13)
            np.testing.assert_allclose(lse[t], want[1][0], rtol=1e-13)
    parents = np.array([-1, 0, 0, 2, -1, 0, 1, -1, 2], np.int32)
    seq_of, positions, places, seen = oracle.lay(starts, cached, 9, parents, 1)
    assert seq_of.tolist() == [0] * 4 + [1] * 5 and places.tolist() == [5, 6, 7, 8, 3, 4, 5, 6, 7]
    assert positions.tolist() == [5, 6, 6, 7, 3, 4, 5, 3, 6]
    assert seen[:, 0].tolist() == [1, 3, 5, 13, 1, 3, 7, 8, 23]
    out, _, _, _ = oracle.attend(q, k, v, table, cached, starts, seen, 0.5)
    for s in range(2):
        for i, t in enumerate(range(starts[s], starts[s + 1])):
            on = sorted(oracle.branch(parents[starts[s]:starts[s + 1]], i))
            at = list(range(cached[s])) + [cached[s] + j for j in on]
            line = lambda c: np.stack([c[table[s, j // 4], :, j % 4] for j in at])  # noqa: E731
            kk, vv = line(k), line(v)
            for h in range(4):
                w = np.exp(0.5 * kk[:, h // 2] @ q[t, h])
                np.testing.assert_allclose(out[t, h], w @ vv[:, h // 2] / w.sum(), rtol=1e-12)


def test_oracle_of_the_walk_and_its_moves():
    parents = [-1, 0, 0, 2, 2, -1, 0]
    path, won, counts = oracle.accept([9, 4, 7, 1, 2, 8, 8], [7, 0, 2, 0, 5, 8, 3], [0, 5, 5, 7], 4, parents)
    assert path.tolist() == [[0, 2, 4, -1], [-1] * 4, [0, 1, -1, -1]]
    assert won.tolist() == [[7, 2, 5, -1], [-1] * 4, [8, 3, -1, -1]] and counts.tolist() == [3, 0, 2]
    assert oracle.accept([9, -1, 7], [-1, -1, 1], [0, 3], 4)[2].tolist() == [1]  # not a token
    path, won, counts = oracle.accept([9, 4, 7], [4, 6, 1], [0, 3], 4)
    assert path.tolist() == [[0, 1, -1, -1]] and won.tolist() == [[4, 6, -1, -1]] and counts.tolist() == [2]
    c = np.arange(6 * 1 * 2 * 1.0).reshape(6, 1, 2, 1)
    got = oracle.keep(c, np.array([[1, 4, 0]]), [1], np.array([[0, 2, 3, 2]]))
    want = c.copy()
    want[4, 0, 0], want[4, 0, 1] = c[4, 0, 1], c[0, 0, 0]  # places 3 and 4 to 2 and 3
    assert np.array_equal(got, want)


def test_masked_attention_sees_only_its_tokens():
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((2, 2, 1, 4, 4))
    q, seen = rng.standard_normal((3, 1, 4)), np.array([[0], [1], [-1]], np.int64)
    out, lse, _, _ = oracle.attend(q, k, v, np.array([[0, 1]]), [0], [0, 3], seen, 1.0)
    assert not out[0].any() and lse[0, 0] == -np.inf
    np.testing.assert_allclose(out[1, 0], v[0, 0, 0], rtol=1e-15)
    w = np.exp(k[0, 0, :3] @ q[2, 0])
    np.testing.assert_allclose(out[2, 0], w @ v[0, 0, :3] / w.sum(), rtol=1e-13)
