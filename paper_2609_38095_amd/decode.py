"""Python binding of libzo's decode-step operators (include/zo_decode.h): from trained weights to
answers.

Argument marshalling only, as in the package itself (in _tensors.so for the calls that take tensors), under
the C names:

  zo_rotary_turns(rotary, base, kind, factor, ...)      rotation frequencies (host, float64)
  zo_norm_rotate(q, k, positions, turns, ...)           head norms and rotation, one pass
  zo_norm_rotate_back(dq_out, dk_out, q, k, ...)        its gradient
  zo_norm_rotate_put(q, k, v, k_cache, v_cache, ...)    the same, keys and values into the paged cache
  zo_cache_attend(q, k_cache, v_cache, table, lengths)  one new token of each sequence over the cache
  zo_cache_copy(k_caches, v_caches, src, dst, rows)     copies of pages, every layer
  zo_draw(logits, u, temperature, top_k, top_p, min_p)  tokens from given random numbers
  ZoPages(pages, page_tokens)                           the page book: add, fork, extend, cut, drop, compact

Rows of heads are tensors [tokens, heads, dim], caches [pages, heads, page_tokens, dim] (any strides,
the last dimension contiguous: permute a cache that is laid out otherwise). Results are allocated by
torch where no output is given. All tensors of a call live on the current device; a call with a
stream of its own allocates on that stream, and waiting for tensors that other streams still write
is the caller's. torch's autograd sees none of these calls: results carry no gradient, whatever their
inputs require, and zo_norm_rotate_back is called by the program.
"""

import contextlib
import ctypes
import operator
import os

import numpy as np
import torch

from . import PKG_DIR, ZO_ERR_ARG, ZoError, ZoLibraryMissing, _check, _lib as _base_lib, _stream

ZO_ERR_MEMORY, ZO_ERR_FULL = -5, -6
ZO_DIM_MAX = 256
ZO_ROTARY_LINEAR, ZO_ROTARY_BASE, ZO_ROTARY_BANDS = 0, 1, 2

EXPORTS = ("zo_rotary_turns", "zo_norm_rotate", "zo_norm_rotate_put", "zo_norm_rotate_back",
           "zo_norm_rotate_back_work", "zo_cache_attend", "zo_cache_attend_work", "zo_cache_copy", "zo_draw",
           "zo_draw_split", "zo_draw_work", "zo_pages_open", "zo_pages_close", "zo_pages_add", "zo_pages_fork",
           "zo_pages_extend", "zo_pages_drop", "zo_pages_left", "zo_pages_length", "zo_pages_table", "zo_pages_compact")
# entry points that _tensors.so calls, in the order that it takes their addresses in
_CALLED = ("zo_norm_rotate", "zo_norm_rotate_put_at", "zo_norm_rotate_back", "zo_norm_rotate_back_work", "zo_cache_attend",
           "zo_cache_attend_work", "zo_cache_copy", "zo_draw_split", "zo_draw_work", "zo_tree_lay", "zo_tree_attend",
           "zo_tree_attend_work", "zo_tree_accept", "zo_tree_keep")

_READY = None
_TENSORS = None


class ZoPageMove(ctypes.Structure):
    _fields_ = [("src", ctypes.c_int32), ("dst", ctypes.c_int32), ("rows", ctypes.c_int32)]


def _lib():
    global _READY
    if _READY is None:
        lib = _base_lib()
        u64, u32, f64, vp, i32 = ctypes.c_uint64, ctypes.c_uint32, ctypes.c_double, ctypes.c_void_p, ctypes.c_int
        args = ctypes.c_char_p  # a packed struct
        pu, move = ctypes.POINTER(u32), ctypes.POINTER(ZoPageMove)
        for name, argtypes, restype in (
                ("zo_rotary_turns", [i32, u32, f64, f64, f64, f64, f64, vp], i32),
                ("zo_norm_rotate", [args, vp], i32), ("zo_norm_rotate_put", [args, vp], i32),
                ("zo_norm_rotate_back", [args, vp], i32), ("zo_norm_rotate_back_work", [u32, u32, u32, u32], u64),
                ("zo_cache_attend", [args, vp], i32), ("zo_cache_attend_work", [u32, u32, u32, u32], u64),
                ("zo_cache_copy", [args, args, u32, vp, u32, i32, vp], i32), ("zo_draw", [args, vp], i32),
                ("zo_draw_split", [args, vp, u64, vp], i32), ("zo_draw_work", [u32, u32, i32], u64),
                ("zo_pages_open", [u32, u32], vp), ("zo_pages_close", [vp], None),
                ("zo_pages_add", [vp, u32, pu], i32), ("zo_pages_fork", [vp, u32, pu], i32),
                ("zo_pages_extend", [vp, u32, u32, move], i32), ("zo_pages_drop", [vp, u32], i32),
                ("zo_pages_left", [vp], u32), ("zo_pages_length", [vp, u32], ctypes.c_int64),
                ("zo_pages_table", [vp, vp, u32, vp, u64, u32, vp], i32),
                ("zo_pages_compact", [vp, vp, u32, pu], i32), ("zo_pages_cut", [vp, u32, u32], i32),
                ("zo_norm_rotate_put_at", [args, vp, vp], i32), ("zo_tree_lay", [args, vp], i32),
                ("zo_tree_attend", [args, vp], i32), ("zo_tree_attend_work", [u32, u32, u32, u32, u32, i32], u64),
                ("zo_tree_accept", [args, vp], i32), ("zo_tree_keep", [args, vp], i32)):
            f = getattr(lib, name)
            f.argtypes, f.restype = argtypes, restype
        _READY = lib
    return _READY


def _tensors():
    global _TENSORS
    if _TENSORS is None:
        lib = _lib()
        if not os.path.exists(os.path.join(PKG_DIR, "_tensors.so")):
            raise ZoLibraryMissing(f"{os.path.join(PKG_DIR, '_tensors.so')} is not built; run __graft_entry__.build()")
        from . import _tensors as module
        module.bind(*[ctypes.cast(getattr(lib, name), ctypes.c_void_p).value for name in _CALLED])
        _TENSORS = module
    return _TENSORS


def _on(stream):
    """Allocations of a call with a stream of its own belong to that stream."""
    if stream is None:
        return contextlib.nullcontext()
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(getattr(stream, "cuda_stream", stream)))
    return torch.cuda.stream(stream)


_INITIALIZED = False


def _initialized():
    global _INITIALIZED
    _INITIALIZED = torch.cuda.is_initialized()
    return _INITIALIZED


_device, _raw_stream = torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream


def _call(f, stream, like, *args):
    """f on the current device and stream, or on the stream given, which must belong to like's device."""
    if stream is None:
        if _INITIALIZED or _initialized():
            device = _device()
            got = f(device, _raw_stream(device), *args)
        else:  # then no argument is on a device, and f says so
            got = f(-1, 0, *args)
    else:
        # f itself refuses what is on no device, as it does without a stream
        handle = _stream(like if getattr(like, "is_cuda", False) else None, stream).value or 0
        with _on(stream):
            got = f(_device(), handle, *args)
    if type(got) is int:
        _check(got, "zo_" + f.__name__)
    return got


def _whole(x, dtype, call):
    """x as an array of a whole type that holds every number of it."""
    x = np.asarray(x)
    try:
        with np.errstate(invalid="ignore"):
            whole = x.astype(dtype)
    except OverflowError:
        raise ZoError(ZO_ERR_ARG, call) from None
    if not np.array_equal(whole, x):
        raise ZoError(ZO_ERR_ARG, call)
    return whole


def _count(n, call):
    """n where it fits the 32 bits that the library takes (ctypes would hand on the lowest ones)."""
    if not 0 <= operator.index(n) < 1 << 32:
        raise ZoError(ZO_ERR_ARG, call)
    return n


def _doubles(turns):
    """Frequencies as an array of float64; None for none."""
    if turns is None or type(turns) is np.ndarray and turns.dtype == np.float64 and turns.flags.c_contiguous:
        return turns
    return np.array(turns, np.float64, order="C")


def zo_rotary_turns(rotary, base=10000.0, kind=ZO_ROTARY_LINEAR, factor=1.0, original=0.0, low=1.0, high=4.0):
    """Rotation frequencies in turns per position, float64 [rotary / 2]; factor > 1 scales them for long contexts."""
    out = np.zeros(max(_count(rotary, "zo_rotary_turns") // 2, 1))
    _check(_lib().zo_rotary_turns(kind, rotary, base, factor, original, low, high, out.ctypes.data), "zo_rotary_turns")
    return out


def zo_norm_rotate(q, k, positions, turns=None, interleaved=False, magnitude=1.0, q_gamma=None, k_gamma=None,
                   norm_eps=1e-6, q_out=None, k_out=None, stream=None):
    """(q_out, k_out): each head of q and k [tokens, heads, dim] normed (where it has a gamma) and its first
    2 len(turns) dims rotated by its token's position. q or k may be None. In place: q_out = q."""
    return _call((_TENSORS or _tensors()).norm_rotate, stream, q if q is not None else k, q, k, positions, _doubles(turns),
                 interleaved, magnitude, q_gamma, k_gamma, norm_eps, q_out, k_out)


def zo_norm_rotate_put(q, k, v, k_cache, v_cache, table, positions, turns=None, interleaved=False, magnitude=1.0,
                       q_gamma=None, k_gamma=None, norm_eps=1e-6, seqs=None, q_out=None, stream=None, places=None):
    """zo_norm_rotate whose keys, with the values v, are put at token positions[t] of sequence seqs[t] (t itself
    where seqs is None) of the paged cache, or at token places[t] where places are given (zo_norm_rotate_put_at: tokens of
    different branches share positions). Returns q_out. q may be None."""
    return _call((_TENSORS or _tensors()).norm_rotate_put, stream, k, q, k, v, k_cache, v_cache, table, positions, _doubles(turns),
                 interleaved, magnitude, q_gamma, k_gamma, norm_eps, seqs, q_out, places)


def zo_norm_rotate_back(dq_out, dk_out, q, k, positions, turns=None, interleaved=False, magnitude=1.0, q_gamma=None,
                        k_gamma=None, norm_eps=1e-6, dq=None, dk=None, work=None, stream=None):
    """(dq, dk, dq_gamma, dk_gamma) of zo_norm_rotate(q, k, ...) for the gradients of its outputs; the gammas'
    are float32 (None without the gamma). q and k are read only where there is a gamma."""
    return _call((_TENSORS or _tensors()).norm_rotate_back, stream, dq_out if dq_out is not None else dk_out, dq_out, dk_out, q, k,
                 positions, _doubles(turns), interleaved, magnitude, q_gamma, k_gamma, norm_eps, dq, dk, work)


def zo_cache_attend(q, k_cache, v_cache, table, lengths, scale=None, out=None, lse=False, work=None, stream=None):
    """out [sequences, heads, dim] of one new token of each sequence: attention of its queries q over the first
    lengths[s] tokens of its pages table[s]. scale: dim ** -0.5 by default. lse: also returns log sum exp
    of the scores, float32 [sequences, heads]. work: a tensor of zo_cache_attend_work() bytes (allocated if None)."""
    return _call((_TENSORS or _tensors()).cache_attend, stream, q, q, k_cache, v_cache, table, lengths, scale, out, lse, work)


def _int32s(x):
    if x is None or type(x) is np.ndarray and x.dtype == np.int32 and x.flags.c_contiguous:
        return x
    return np.ascontiguousarray(_whole(x, np.int32, "zo_cache_copy"))


def zo_cache_copy(k_caches, v_caches, src, dst, rows=None, stream=None):
    """In each layer's cache: tokens 0 .. rows[i] - 1 (all if None) of page src[i] to page dst[i]. src, dst and rows
    are host arrays; no dst is repeated or a src of the same call."""
    k_caches = list(k_caches)
    _call((_TENSORS or _tensors()).cache_copy, stream, k_caches[0] if k_caches else None, k_caches, list(v_caches), _int32s(src),
          _int32s(dst), _int32s(rows))


def zo_draw(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, logprobs=False, tokens=None, work=None, stream=None):
    """int32 tokens [rows] drawn from logits [rows, vocab] with the random numbers u [rows] in [0, 1), each row with
    its temperature, top_k (int32), top_p and min_p (device tensors [rows] or None). logprobs: also returns
    the drawn tokens' log probabilities among what was kept, float32. work: a tensor of zo_draw_work() bytes
    (allocated if None)."""
    return _call((_TENSORS or _tensors()).draw, stream, logits, logits, u, temperature, top_k, top_p, min_p, logprobs, tokens,
                 work)


class ZoPages:
    """The book of a cache's pages (host only): which sequence holds which pages, which are shared, which are free."""

    def __init__(self, pages, page_tokens):
        self._book = None
        if 0 <= pages < 1 << 32 and 0 <= page_tokens < 1 << 32:
            self._book = _lib().zo_pages_open(pages, page_tokens)
        if not self._book:
            raise ValueError(f"no page book of {pages} pages of {page_tokens} tokens")
        self._close = _lib().zo_pages_close
        self.pages, self.page_tokens = pages, page_tokens

    def __del__(self):
        if self._book:
            self._close(self._book)
            self._book = None

    def add(self, tokens=0):
        """A new sequence with room for `tokens` tokens; returns its number."""
        seq = ctypes.c_uint32()
        _check(_lib().zo_pages_add(self._book, _count(tokens, "zo_pages_add"), ctypes.byref(seq)), "zo_pages_add")
        return seq.value

    def fork(self, seq):
        """A new sequence with the tokens of seq, sharing its pages; returns its number."""
        forked = ctypes.c_uint32()
        _check(_lib().zo_pages_fork(self._book, _count(seq, "zo_pages_fork"), ctypes.byref(forked)), "zo_pages_fork")
        return forked.value

    def extend(self, seq, tokens=1):
        """Room for more tokens; returns the copy that this needs first, (src, dst, rows), or None."""
        move = ZoPageMove()
        _check(_lib().zo_pages_extend(self._book, _count(seq, "zo_pages_extend"), _count(tokens, "zo_pages_extend"),
                                      ctypes.byref(move)), "zo_pages_extend")
        return (move.src, move.dst, move.rows) if move.rows else None

    def cut(self, seq, tokens):
        """The sequence keeps its first tokens; pages behind them are free again where no other holds them."""
        _check(_lib().zo_pages_cut(self._book, _count(seq, "zo_pages_cut"), _count(tokens, "zo_pages_cut")), "zo_pages_cut")

    def drop(self, seq):
        _check(_lib().zo_pages_drop(self._book, _count(seq, "zo_pages_drop")), "zo_pages_drop")

    def left(self):
        """How many pages are free."""
        return _lib().zo_pages_left(self._book)

    def length(self, seq):
        """The tokens of a sequence, -1 if there is none of that number."""
        return _lib().zo_pages_length(self._book, seq) if 0 <= seq < 1 << 32 else -1

    def table(self, seqs, width=None):
        """(page ids int32 [sequences, width], lengths int32 [sequences]) as numpy arrays."""
        seqs = np.ascontiguousarray(_whole(seqs, np.uint32, "zo_pages_table").reshape(-1))
        lengths = np.zeros(len(seqs), np.int32)
        if width is None:
            width = max([1] + [-(-self.length(s) // self.page_tokens) for s in seqs.tolist()])
        ids = np.full((len(seqs), width), -1, np.int32)
        _check(_lib().zo_pages_table(self._book, seqs.ctypes.data, len(seqs), ids.ctypes.data, width, width,
                                     lengths.ctypes.data), "zo_pages_table")
        return ids, lengths

    def compact(self, room=None):
        """Moves pages in use to the lowest ids; returns (src, dst, rows) to hand to zo_cache_copy."""
        room = self.pages if room is None else min(room, self.pages)
        if room < 0:
            raise ZoError(ZO_ERR_ARG, "zo_pages_compact")
        moves = np.zeros((max(room, 1), 3), np.int32)
        n = ctypes.c_uint32()
        _check(_lib().zo_pages_compact(self._book, moves.ctypes.data, room, ctypes.byref(n)), "zo_pages_compact")
        return tuple(np.ascontiguousarray(moves[:n.value, i]) for i in range(3))
