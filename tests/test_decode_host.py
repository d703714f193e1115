"""Host side of the decode-step operators: the header against the binding, refusals, rotation
frequencies, the page book, and the oracle's own values. Nothing here launches a kernel."""

import ctypes
import math
import os
import re
import shutil
import struct
import subprocess

import numpy as np
import pytest
import torch

import paper_2609_38095_amd as zo
from oracle import decode as oracle
from paper_2609_38095_amd import decode

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_38095_amd", "csrc")


def _header():
    text = open(os.path.join(ROOT, "include", "zo_decode.h")).read()
    return re.sub(r"/\*.*?\*/", "", text, flags=re.S)


def test_header_declares_what_the_binding_names():
    names = sorted(set(re.findall(r"^\w[\w* ]*?\b(zo_\w+)\s*\(", _header(), flags=re.M)))
    assert names == sorted(decode.EXPORTS)
    lib = zo.library()
    for name in names:
        assert hasattr(lib, name), name
    for name in ("ZO_ERR_MEMORY", "ZO_ERR_FULL"):
        assert int(re.search(name + r"\s*=\s*(-?\d+)", _header()).group(1)) == getattr(zo, name)
    assert int(re.search(r"ZO_DIM_MAX (\d+)u", _header()).group(1)) == zo.ZO_DIM_MAX
    for status in (zo.ZO_ERR_MEMORY, zo.ZO_ERR_FULL):
        assert b"unknown" not in lib.zo_strerror(status)


def test_binding_module_is_built_and_bound():
    """The module that marshals tensors is in the tree, takes the entry points' addresses and refuses anything else."""
    module = decode._tensors()
    assert os.path.exists(os.path.join(ROOT, "paper_2609_38095_amd", "_tensors.so"))
    for args in ((), (0,) * 8, (1, 2)):
        with pytest.raises((TypeError, ValueError)):
            module.bind(*args)
    with pytest.raises(TypeError):
        module.norm_rotate(0, 0)
    with pytest.raises(TypeError):
        module.cache_attend("x", 0, *[None] * 9)


def test_host_code_under_asan_ubsan(tmp_path):
    cxx = shutil.which("g++")
    if cxx is None:
        pytest.skip("no g++")
    exe = str(tmp_path / "decode_check")
    cmd = [cxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
           "-Wall", "-Wextra", "-Werror", "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           os.path.join(ROOT, "tests", "helpers", "decode_check.cpp"), os.path.join(CSRC, "zo_checks.cpp"),
           os.path.join(CSRC, "zo_pages.cpp"), "-o", exe]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "decode_check ok" in r.stdout, r.stdout + r.stderr


def test_rotary_turns():
    for rotary, base in ((2, 1e4), (64, 1e4), (128, 1e6), (256, 500.0)):
        i = np.arange(rotary // 2)
        plain = base ** (-2.0 * i / rotary) / (2 * math.pi)
        np.testing.assert_allclose(zo.zo_rotary_turns(rotary, base), plain, rtol=1e-14)
        np.testing.assert_allclose(zo.zo_rotary_turns(rotary, base, zo.ZO_ROTARY_LINEAR, 4.0), plain / 4, rtol=1e-14)
        if rotary > 2:
            got = zo.zo_rotary_turns(rotary, base, zo.ZO_ROTARY_BASE, 8.0)
            np.testing.assert_allclose([got[0], got[-1]], [plain[0], plain[-1] / 8], rtol=1e-12)
        got = zo.zo_rotary_turns(rotary, base, zo.ZO_ROTARY_BANDS, 8.0, 4096.0, 1.0, 32.0)
        s = np.clip((4096 * plain - 1) / 31, 0, 1)
        np.testing.assert_allclose(got, plain * ((1 - s) / 8 + s), rtol=1e-14)
    lib = zo.library()
    decode._lib()
    out = (ctypes.c_double * 128)(*([-7.0] * 128))
    at = ctypes.addressof(out)
    for args, code in (((0, 64, 1e4, 1.0, 0, 0, 0, None), zo.ZO_ERR_NULL), ((3, 64, 1e4, 1.0, 0, 0, 0, at), zo.ZO_ERR_ARG),
                       ((0, 63, 1e4, 1.0, 0, 0, 0, at), zo.ZO_ERR_ARG), ((0, 0, 1e4, 1.0, 0, 0, 0, at), zo.ZO_ERR_ARG),
                       ((0, 258, 1e4, 1.0, 0, 0, 0, at), zo.ZO_ERR_ARG), ((0, 64, 1.0, 1.0, 0, 0, 0, at), zo.ZO_ERR_ARG),
                       ((0, 64, 1e4, 0.5, 0, 0, 0, at), zo.ZO_ERR_ARG), ((1, 2, 1e4, 2.0, 0, 0, 0, at), zo.ZO_ERR_ARG),
                       ((2, 64, 1e4, 2.0, 0.0, 1, 2, at), zo.ZO_ERR_ARG), ((2, 64, 1e4, 2.0, 100.0, 2, 2, at), zo.ZO_ERR_ARG),
                       ((2, 64, 1e4, 2.0, 100.0, -1, 2, at), zo.ZO_ERR_ARG),
                       ((0, 64, math.inf, 1.0, 0, 0, 0, at), zo.ZO_ERR_NONFINITE),
                       ((2, 64, 1e4, 1.0, math.nan, 0, 1, at), zo.ZO_ERR_NONFINITE)):
        assert lib.zo_rotary_turns(*args) == code, args
    assert all(v == -7.0 for v in out)


def test_null_and_invalid_structs_are_refused():
    """Refusals come before any HIP call."""
    lib = decode._lib()
    for name in ("zo_norm_rotate", "zo_norm_rotate_put", "zo_norm_rotate_back", "zo_cache_attend", "zo_draw"):
        assert getattr(lib, name)(None, None) == zo.ZO_ERR_NULL
    packed = struct.Struct("QqQQQQQQQIIi4x")  # zo_draw_args
    draw = lambda **kw: lib.zo_draw(packed.pack(*{**dict(  # noqa: E731
        logits=0x1000, stride=100, u=0x2000, t=0, k=0, p=0, m=0, tokens=0x3000, lp=0, rows=4, vocab=100, dtype=0), **kw}.values()), None)
    assert draw(vocab=0) == draw(vocab=(1 << 18) + 1) == draw(dtype=5) == draw(stride=-1) == draw(logits=0x1002) == zo.ZO_ERR_ARG
    assert draw(u=0x2001) == draw(t=0x2002) == draw(tokens=0x3001) == draw(lp=0x3002) == zo.ZO_ERR_ARG
    assert draw(logits=0) == draw(u=0) == draw(tokens=0) == zo.ZO_ERR_NULL
    assert draw(rows=0, logits=0, u=0, tokens=0) == zo.ZO_OK
    cache = struct.pack("QQqqqIIII", 0x1000, 0x9000, 64, 64, 8, 4, 1, 8, 8)
    moves = np.array([[0, 1, 8]], np.int32)
    two = np.array([0x1000, 0x9000], np.uint64).tobytes()
    at = moves.ctypes.data
    assert lib.zo_cache_copy(cache, two, 2, None, 1, 0, None) == lib.zo_cache_copy(None, two, 2, at, 1, 0, None) == zo.ZO_ERR_NULL
    assert lib.zo_cache_copy(cache, None, 2, at, 1, 0, None) == zo.ZO_ERR_NULL
    assert lib.zo_cache_copy(cache, two, 0, at, 1, 0, None) == lib.zo_cache_copy(cache, two, 2, None, 0, 0, None) == zo.ZO_OK
    assert lib.zo_cache_copy(cache, two, 2, at, 1, 9, None) == zo.ZO_ERR_ARG


def test_binding_refuses_what_is_not_on_the_device():
    x = torch.zeros(2, 4, 64)
    i = torch.zeros(2, dtype=torch.int32)
    with pytest.raises(TypeError):
        zo.zo_norm_rotate(x, None, i)
    with pytest.raises(TypeError):
        zo.zo_norm_rotate(x.double(), None, i)
    with pytest.raises(ValueError):
        zo.zo_norm_rotate(None, None, i)
    with pytest.raises(TypeError):
        zo.zo_cache_attend(x, x, x, i, i)
    with pytest.raises(TypeError):
        zo.zo_cache_attend(None, x, x, i, i)
    with pytest.raises(TypeError):
        zo.zo_draw(x[0], i)
    with pytest.raises(ValueError):
        zo.zo_cache_copy([x], [], [0], [1])


def test_page_book():
    book = zo.ZoPages(8, 4)
    a = book.add(6)
    b = book.fork(a)
    assert book.left() == 6 and book.length(b) == 6
    src, dst, rows = book.extend(b, 1)
    ids, lengths = book.table([a, b])
    assert (src, dst, rows) == (ids[0, 1], ids[1, 1], 2) and ids[0, 0] == ids[1, 0] and lengths.tolist() == [6, 7]
    assert book.extend(a, 2) is None and book.extend(a, 1) is None
    with pytest.raises(zo.ZoError) as e:
        book.extend(a, 100)
    assert e.value.status == zo.ZO_ERR_FULL and book.length(a) == 9
    with pytest.raises(zo.ZoError):
        book.table([a], width=1)
    book.drop(a)
    with pytest.raises(zo.ZoError):
        book.drop(a)
    before, _ = book.table([b])
    moved = dict(zip(*[m.tolist() for m in book.compact()[:2]]))
    after, _ = book.table([b])
    assert after.tolist() == [[moved.get(i, i) for i in before[0].tolist()]] and after.max() < 8 - book.left()
    with pytest.raises(ValueError):
        zo.ZoPages(0, 4)


def test_oracle_rows():
    """Rotation keeps lengths and composes; the norm is 1; the gradient is the formula's, by differences."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((5, 2, 8))
    turns = np.array([0.1, 0.01, 0.3])
    at = np.array([0, 1, 7, -1, 100])
    one = np.ones(8)
    for interleaved in (False, True):
        y, _ = oracle.norm_rotate(x, None, at, turns, interleaved)
        live = at >= 0
        np.testing.assert_allclose((y[live] ** 2).sum(-1), (x[live] ** 2).sum(-1), rtol=1e-13)
        assert np.array_equal(y[0], x[0]) and not y[3].any() and np.array_equal(y[..., 6:][live], x[..., 6:][live])
        twice, _ = oracle.norm_rotate(y, None, at, turns, interleaved)
        np.testing.assert_allclose(twice[live], oracle.norm_rotate(x, None, 2 * at, turns, interleaved)[0][live], rtol=1e-10, atol=1e-12)
        n, _ = oracle.norm_rotate(x, one, at, turns, interleaved, eps=0.0)
        np.testing.assert_allclose((n[live] ** 2).mean(-1), 1.0, rtol=1e-13)
        w, g = rng.standard_normal(x.shape), 1 + 0.1 * rng.standard_normal(8)
        dx, _, dg, _ = oracle.norm_rotate_back(w, x, g, at, turns, interleaved, 0.7)
        loss = lambda a, b: (w * oracle.norm_rotate(a, b, at, turns, interleaved, 0.7)[0]).sum()  # noqa: E731
        for i in ((0, 0, 0), (1, 1, 5), (2, 0, 7), (4, 1, 2), (3, 0, 0)):
            e = np.zeros_like(x)
            e[i] = 1e-6
            np.testing.assert_allclose((loss(x + e, g) - loss(x - e, g)) / 2e-6, dx[i], rtol=1e-6, atol=1e-8)
        e = np.zeros(8)
        e[3] = 1e-6
        np.testing.assert_allclose((loss(x, g + e) - loss(x, g - e)) / 2e-6, dg[3], rtol=1e-6, atol=1e-8)
    # a quarter of a turn swaps a pair
    y, _ = oracle.norm_rotate(np.array([[[3.0, 4.0]]]), None, np.array([1]), np.array([0.25]))
    np.testing.assert_allclose(y, [[[-4.0, 3.0]]], atol=1e-15)


def test_oracle_attention_and_draw():
    rng = np.random.default_rng(1)
    k, v = rng.standard_normal((2, 6, 1, 4, 8))
    table = np.array([[3, 1, 5], [0, -1, 2]])
    q = rng.standard_normal((2, 2, 8))
    out, lse, _, _ = oracle.attend(q, k, v, table, [10, 12], 0.5)
    kk, vv = np.concatenate([k[3, 0], k[1, 0], k[5, 0]])[:10], np.concatenate([v[3, 0], v[1, 0], v[5, 0]])[:10]
    s = torch.softmax(torch.from_numpy(0.5 * q[0] @ kk.T), -1).numpy()
    np.testing.assert_allclose(out[0], s @ vv, rtol=1e-12)
    kk, vv = np.concatenate([k[0, 0], k[2, 0]]), np.concatenate([v[0, 0], v[2, 0]])
    np.testing.assert_allclose(lse[1], np.log(np.exp(0.5 * q[1] @ kk.T).sum(-1)), rtol=1e-12)
    l = np.log(np.array([0.1, 0.4, 0.2, 0.3], np.float32))
    assert [oracle.draw(l, u)[0] for u in (0.05, 0.2, 0.6, 0.9)] == [0, 1, 2, 3]
    assert [oracle.draw(l, u, top_k=2)[0] for u in (0.0, 0.5, 0.6, 0.99)] == [1, 1, 3, 3]
    assert [oracle.draw(l, u, top_p=0.5)[0] for u in (0.5, 0.6)] == [1, 3] and oracle.draw(l, 0.99, top_p=0.3)[0] == 1
    assert [oracle.draw(l, u, min_p=0.6)[0] for u in (0.5, 0.6)] == [1, 3] and oracle.draw(l, 0.9, temperature=0.0) == (1, 0.0)
    assert oracle.draw(np.full(3, -np.inf, np.float32), 0.3) == (-1, -math.inf)
    np.testing.assert_allclose(oracle.draw(l, 0.9)[1], math.log(0.3), rtol=1e-6)


def test_launches_of_2_to_the_32_threads_are_refused():
    """A launch takes fewer; what would need more is turned away before any HIP call."""
    lib = decode._lib()
    draw = struct.Struct("QqQQQQQQQIIi4x")  # zo_draw_args
    for rows in (1 << 22, 1 << 31, (1 << 32) - 1):
        assert lib.zo_draw(draw.pack(0x1000, 100, 0x2000, 0, 0, 0, 0, 0x3000, 0, rows, 100, 0), None) == zo.ZO_ERR_ARG
    moves = np.array([[0, 1, 8]], np.int32)
    one = np.array([1 << 20], np.uint64).tobytes()
    for tokens, heads in ((1 << 15, 5), (1 << 20, 1), (1 << 12, 64)):  # pages of 64-dim heads above 2^23 elements
        cache = struct.pack("QQqqqIIII", 1 << 20, 1 << 40, tokens * heads * 64, tokens * 64, 64, 4, heads, tokens, 64)
        assert lib.zo_cache_copy(cache, one, 1, moves.ctypes.data, 1, 0, None) == zo.ZO_ERR_ARG


def test_draw_split_workspace_is_checked():
    lib = decode._lib()
    draw = struct.Struct("QqQQQQQQQIIi4x")  # zo_draw_args
    call = lambda work, size, rows=4, vocab=50_272, top_p=0, stride=50_272: lib.zo_draw_split(  # noqa: E731
        draw.pack(0x1000, stride, 0x2000, 0, 0, top_p, 0, 0x3000, 0, rows, vocab, 0), work, size, None)
    need = lib.zo_draw_work(4, 50_272, 0)
    assert need > 0 and need % 8 == 0
    assert call(None, need) == zo.ZO_ERR_NULL
    assert call(0x10000, need - 1) == call(0x10008, need) == call(0x10000, 0) == call(0x10000, need, stride=-1) == zo.ZO_ERR_ARG
    assert call(0x10000, need, top_p=0x2002) == call(0x10000, need, vocab=0) == zo.ZO_ERR_ARG
    assert lib.zo_draw_split(None, 0x10000, need, None) == zo.ZO_ERR_NULL
    assert call(None, 0, rows=0) == zo.ZO_OK
    for rows, vocab, top_k in ((0, 50_272, 0), (33, 151_936, 0), (4, 16_383, 0), (4, (1 << 18) + 1, 0), (17, 151_936, 1), (4, 50_272, 1)):
        assert lib.zo_draw_work(rows, vocab, top_k) == 0
