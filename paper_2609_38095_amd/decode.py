"""Python binding of libzo's decode-step operators (include/zo_decode.h): from trained weights to
answers.

Argument marshalling only, as in the package itself, under the C names:

  zo_rotary_turns(rotary, base, kind, factor, ...)      rotation frequencies (host, float64)
  zo_norm_rotate(q, k, positions, turns, ...)           head norms and rotation, one pass
  zo_norm_rotate_back(dq_out, dk_out, q, k, ...)        its gradient
  zo_norm_rotate_put(q, k, v, k_cache, v_cache, ...)    the same, keys and values into the paged cache
  zo_cache_attend(q, k_cache, v_cache, table, lengths)  one new token of each sequence over the cache
  zo_cache_copy(k_caches, v_caches, src, dst, rows)     copies of pages, every layer
  zo_draw(logits, u, temperature, top_k, top_p, min_p)  tokens from given random numbers
  ZoPages(pages, page_tokens)                           the page book: add, fork, extend, drop, compact

Rows of heads are tensors [tokens, heads, dim], caches [pages, heads, page_tokens, dim] (any strides,
the last dimension contiguous: permute a cache that is laid out otherwise). Results are allocated by
torch where no output is given. All tensors of a call live on the current device; a call with a
stream of its own allocates on that stream, and waiting for tensors that other streams still write
is the caller's.
"""

import array
import ctypes
import struct

import numpy as np
import torch

from . import ZO_BF16, ZO_F32, _check, _lib as _base_lib, _stream

ZO_ERR_MEMORY, ZO_ERR_FULL = -5, -6
ZO_DIM_MAX = 256
ZO_ROTARY_LINEAR, ZO_ROTARY_BASE, ZO_ROTARY_BANDS = 0, 1, 2

EXPORTS = ("zo_rotary_turns", "zo_norm_rotate", "zo_norm_rotate_put", "zo_norm_rotate_back",
           "zo_norm_rotate_back_work", "zo_cache_attend", "zo_cache_attend_work", "zo_cache_copy", "zo_draw",
           "zo_pages_open", "zo_pages_close", "zo_pages_add", "zo_pages_fork", "zo_pages_extend", "zo_pages_drop",
           "zo_pages_left", "zo_pages_length", "zo_pages_table", "zo_pages_compact")

# the argument structs of zo_decode.h, packed by one call each (a ctypes structure takes longer to
# fill than a small kernel to run)
_ROTATE = struct.Struct("Qqq Qqq Qqq Qqq QQQQ IIIIII ff i4x".replace(" ", ""))
_PUT = struct.Struct(_ROTATE.format + "Qqq QQqqqIIII QqII Q".replace(" ", ""))
_BACK = struct.Struct(_ROTATE.format + "Qqq Qqq QQQQ".replace(" ", ""))
_ATTEND = struct.Struct("Qqq Qqq QQqqqIIII QqII QQQQ If i4x".replace(" ", ""))
_DRAW = struct.Struct("QqQQQQQQQIIi4x")
_CACHE = struct.Struct("QQqqqIIII")
_NO_ROWS = (0, 0, 0)
_TYPES = {torch.float32: ZO_F32, torch.bfloat16: ZO_BF16}

_TENSORS = {torch.Tensor, torch.nn.Parameter}
_READY = None


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
                ("zo_pages_open", [u32, u32], vp), ("zo_pages_close", [vp], None),
                ("zo_pages_add", [vp, u32, pu], i32), ("zo_pages_fork", [vp, u32, pu], i32),
                ("zo_pages_extend", [vp, u32, u32, move], i32), ("zo_pages_drop", [vp, u32], i32),
                ("zo_pages_left", [vp], u32), ("zo_pages_length", [vp, u32], ctypes.c_int64),
                ("zo_pages_table", [vp, vp, u32, vp, u64, u32, vp], i32),
                ("zo_pages_compact", [vp, vp, u32, pu], i32)):
            f = getattr(lib, name)
            f.argtypes, f.restype = argtypes, restype
        _READY = lib
    return _READY


def _on(stream):
    """Allocations of a call with a stream of its own belong to that stream."""
    if not isinstance(stream, torch.cuda.Stream):
        stream = torch.cuda.ExternalStream(int(getattr(stream, "cuda_stream", stream)))
    return torch.cuda.stream(stream)


def _new(like, shape, stream, dtype=None):
    """A tensor on `like`'s device for a result or a workspace."""
    if stream is None:
        return torch.empty(shape, dtype=dtype or like.dtype, device=like.device)
    with _on(stream):
        return torch.empty(shape, dtype=dtype or like.dtype, device=like.device)


def _launch_stream(like, stream):
    """The hipStream_t to launch on, torch's current one by default; the tensors are on the current device."""
    if stream is None:
        index = like.get_device()
        if index == torch._C._cuda_getDevice():
            return torch._C._cuda_getCurrentRawStream(index)
    return _stream(like, stream)


# Each check is one expression over what a sound argument has; what it does not take is named by _refuse. (A
# call on a few tokens takes less time on the GPU than ten tensors' checks one by one take here.)

def _refuse(t, name, dtype, like, shape, what):
    """Raises what is wrong with an argument."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) torch tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.get_device() != like.get_device():
        raise ValueError(f"{name} lives on {t.device}, the other tensors on {like.device}")
    if t.shape != shape:
        raise ValueError(f"{name} must be {tuple(shape)}, not {tuple(t.shape)}")
    raise ValueError(f"{name}: {what}")


def _dtype(t, name, dims):
    """The library's name of a tensor's type; the tensor that a call's others are compared with."""
    dtype = _TYPES.get(getattr(t, "dtype", None))
    if dtype is None:
        raise TypeError(f"{name} must be a float32 or bfloat16 tensor")
    if not t.is_cuda:
        raise TypeError(f"{name} must be a CUDA (HIP) torch tensor")
    if t.dim() != dims:
        raise ValueError(f"{name} must have {dims} dimensions")
    return dtype


def _rows(t, name, like, shape):
    """(address, token stride, head stride) of a tensor [tokens, heads, dim]."""
    if type(t) in _TENSORS and t.dtype is like.dtype and t.shape == shape and t.get_device() == like.get_device():
        a, b, c = t.stride()
        if c == 1 or shape[2] == 1:
            return t.data_ptr(), a, b
    _refuse(t, name, like.dtype, like, shape, "the last dimension must be contiguous")


def _vector(t, name, dtype, like, n):
    """The address of a contiguous tensor of n elements; 0 for None."""
    if t is None:
        return 0
    if type(t) in _TENSORS and t.dtype is dtype and t.shape == (n,) and t.get_device() == like.get_device() \
            and (n < 2 or t.stride(0) == 1):
        return t.data_ptr()
    _refuse(t, name, dtype, like, (n,), "must be contiguous")


def _cache(k, v, like):
    """The fields of a cache [pages, heads, page_tokens, dim]."""
    shape = getattr(k, "shape", None)
    if shape is not None and len(shape) == 4:
        strides = k.stride()
        if type(v) in _TENSORS and k.dtype is like.dtype and v.dtype is like.dtype and v.shape == shape \
                and v.stride() == strides and k.get_device() == like.get_device() == v.get_device() \
                and (strides[3] == 1 or shape[3] == 1):
            return (k.data_ptr(), v.data_ptr(), *strides[:3], *shape)
    else:
        raise ValueError("k_cache must be a tensor [pages, heads, page_tokens, dim]")
    _refuse(k, "k_cache", like.dtype, like, shape, "") if k.dtype != like.dtype or k.get_device() != like.get_device() else \
        _refuse(v, "v_cache", like.dtype, like, shape, "the strides of k_cache, the last dimension contiguous, are needed")


def _table(table, like):
    if type(table) in _TENSORS and table.dtype is torch.int32 and table.get_device() == like.get_device() and table.dim() == 2:
        n, width = table.shape
        a, b = table.stride()
        if b == 1 or width < 2:
            return table.data_ptr(), a, n, width
    _refuse(table, "table", torch.int32, like, getattr(table, "shape", ()), "must be [sequences, pages], its rows contiguous")


def zo_rotary_turns(rotary, base=10000.0, kind=ZO_ROTARY_LINEAR, factor=1.0, original=0.0, low=1.0, high=4.0):
    """Rotation frequencies in turns per position, float64 [rotary / 2]; factor > 1 scales them for long contexts."""
    out = np.zeros(max(int(rotary) // 2, 1))
    _check(_lib().zo_rotary_turns(kind, rotary, base, factor, original, low, high, out.ctypes.data), "zo_rotary_turns")
    return out


def _sides(q, k):
    like = q if q is not None else k
    if like is None:
        raise ValueError("queries or keys are needed")
    dtype = _dtype(like, "q and k", 3)
    tokens, heads, dim = like.shape
    if k is None:
        return like, dtype, tokens, dim, heads, 0
    if not isinstance(k, torch.Tensor) or k.dim() != 3:
        raise TypeError("k must be a CUDA (HIP) torch tensor [tokens, heads, dim]")
    return like, dtype, tokens, dim, 0 if q is None else heads, k.shape[1]


def _turns(turns):
    """(the frequencies as float64, their address, the rotated dims)."""
    if turns is None:
        return None, 0, 0
    if not (isinstance(turns, np.ndarray) and turns.dtype == np.float64 and turns.ndim == 1 and turns.flags.c_contiguous):
        turns = np.ascontiguousarray(np.asarray(turns, dtype=np.float64)).reshape(-1)
    return turns, turns.__array_interface__["data"][0], 2 * len(turns)


def zo_norm_rotate(q, k, positions, turns=None, interleaved=False, magnitude=1.0, q_gamma=None, k_gamma=None,
                   norm_eps=1e-6, q_out=None, k_out=None, stream=None):
    """(q_out, k_out): each head of q and k [tokens, heads, dim] normed (where it has a gamma) and its first
    2 len(turns) dims rotated by its token's position. q or k may be None. In place: q_out = q."""
    like, dtype, tokens, dim, hq, hk = _sides(q, k)
    if q is not None and q_out is None:
        q_out = _new(like, (tokens, hq, dim), stream)
    if k is not None and k_out is None:
        k_out = _new(like, (tokens, hk, dim), stream)
    qs = ks = qo = ko = _NO_ROWS
    if q is not None:
        qs, qo = _rows(q, "q", like, q.shape), _rows(q_out, "q_out", like, q.shape)
    if k is not None:
        shape = (tokens, hk, dim)
        ks, ko = _rows(k, "k", like, shape), _rows(k_out, "k_out", like, shape)
    turns, at, rotary = _turns(turns)
    args = _ROTATE.pack(*qs, *ks, *qo, *ko, _vector(q_gamma, "q_gamma", like.dtype, like, dim),
                        _vector(k_gamma, "k_gamma", like.dtype, like, dim),
                        _vector(positions, "positions", torch.int32, like, tokens), at, tokens, hq, hk, dim, rotary,
                        interleaved, norm_eps, magnitude, dtype)
    _check(_lib().zo_norm_rotate(args, _launch_stream(like, stream)), "zo_norm_rotate")
    return q_out, k_out


def zo_norm_rotate_put(q, k, v, k_cache, v_cache, table, positions, turns=None, interleaved=False, magnitude=1.0,
                       q_gamma=None, k_gamma=None, norm_eps=1e-6, seqs=None, q_out=None, stream=None):
    """zo_norm_rotate whose keys, with the values v, are put at token positions[t] of sequence seqs[t] (t itself
    where seqs is None) of the paged cache. Returns q_out. q may be None."""
    like, dtype, tokens, dim, hq, hk = _sides(q, k)
    qs = qo = _NO_ROWS
    if q is not None:
        qs = _rows(q, "q", like, q.shape)
        if q_out is None:
            q_out = _new(like, (tokens, hq, dim), stream)
        qo = _rows(q_out, "q_out", like, q.shape)
    shape = (tokens, hk, dim)
    turns, at, rotary = _turns(turns)
    args = _PUT.pack(*qs, *_rows(k, "k", like, shape), *qo, *_NO_ROWS, _vector(q_gamma, "q_gamma", like.dtype, like, dim),
                     _vector(k_gamma, "k_gamma", like.dtype, like, dim),
                     _vector(positions, "positions", torch.int32, like, tokens), at, tokens, hq, hk, dim, rotary,
                     interleaved, norm_eps, magnitude, dtype, *_rows(v, "v", like, shape), *_cache(k_cache, v_cache, like),
                     *_table(table, like), _vector(seqs, "seqs", torch.int32, like, tokens))
    _check(_lib().zo_norm_rotate_put(args, _launch_stream(like, stream)), "zo_norm_rotate_put")
    return q_out


def zo_norm_rotate_back(dq_out, dk_out, q, k, positions, turns=None, interleaved=False, magnitude=1.0, q_gamma=None,
                        k_gamma=None, norm_eps=1e-6, dq=None, dk=None, work=None, stream=None):
    """(dq, dk, dq_gamma, dk_gamma) of zo_norm_rotate(q, k, ...) for the gradients of its outputs; the gammas'
    are float32 (None without the gamma). q and k are read only where there is a gamma."""
    like, dtype, tokens, dim, hq, hk = _sides(dq_out, dk_out)
    lib = _lib()
    if dq_out is not None and dq is None:
        dq = _new(like, (tokens, hq, dim), stream)
    if dk_out is not None and dk is None:
        dk = _new(like, (tokens, hk, dim), stream)
    dq_gamma = _new(like, (dim,), stream, torch.float32) if q_gamma is not None and hq else None
    dk_gamma = _new(like, (dim,), stream, torch.float32) if k_gamma is not None and hk else None
    if work is None and (dq_gamma is not None or dk_gamma is not None):
        work = _new(like, (max(lib.zo_norm_rotate_back_work(tokens, hq, hk, dim), 16),), stream, torch.uint8)
    sq, sk = (tokens, hq, dim), (tokens, hk, dim)
    rows = lambda t, name, shape, on: _rows(t, name, like, shape) if on else _NO_ROWS  # noqa: E731
    turns, at, rotary = _turns(turns)
    args = _BACK.pack(*rows(q, "q", sq, dq_gamma is not None), *rows(k, "k", sk, dk_gamma is not None),
                      *rows(dq_out, "dq_out", sq, hq), *rows(dk_out, "dk_out", sk, hk),
                      _vector(q_gamma, "q_gamma", like.dtype, like, dim), _vector(k_gamma, "k_gamma", like.dtype, like, dim),
                      _vector(positions, "positions", torch.int32, like, tokens), at, tokens, hq, hk, dim, rotary,
                      interleaved, norm_eps, magnitude, dtype, *rows(dq, "dq", sq, hq), *rows(dk, "dk", sk, hk),
                      0 if dq_gamma is None else dq_gamma.data_ptr(), 0 if dk_gamma is None else dk_gamma.data_ptr(),
                      *_work(work, like))
    _check(lib.zo_norm_rotate_back(args, _launch_stream(like, stream)), "zo_norm_rotate_back")
    return dq, dk, dq_gamma, dk_gamma


def _work(work, like):
    """(address, bytes) of a workspace; (0, 0) for None."""
    if work is None:
        return 0, 0
    if not isinstance(work, torch.Tensor) or not work.is_cuda or not work.is_contiguous() or work.get_device() != like.get_device():
        raise TypeError("work must be a contiguous CUDA (HIP) tensor on the other tensors' device")
    return work.data_ptr(), work.numel() * work.element_size()


def zo_cache_attend(q, k_cache, v_cache, table, lengths, scale=None, out=None, lse=False, work=None, stream=None):
    """out [sequences, heads, dim] of one new token of each sequence: attention of its queries q over the first
    lengths[s] tokens of its pages table[s]. scale: dim ** -0.5 by default. lse: also returns log sum exp
    of the scores, float32 [sequences, heads]. work: a tensor of zo_cache_attend_work() bytes (allocated if None)."""
    dtype = _dtype(q, "q", 3)
    seqs, heads, dim = shape = q.shape
    qs = _rows(q, "q", q, shape)
    cache = _cache(k_cache, v_cache, q)
    if cache[8] != dim:
        raise ValueError(f"the cache's heads hold {cache[8]} dims, the queries' {dim}")
    ids = _table(table, q)
    if ids[2] != seqs:
        raise ValueError("the table has one row for each sequence")
    lib = _lib()
    if out is None:
        out = _new(q, shape, stream)
    sums = _new(q, (seqs, heads), stream, torch.float32) if lse else None
    if work is None:
        work = _new(q, (lib.zo_cache_attend_work(seqs, heads, cache[6], dim),), stream, torch.uint8)
    args = _ATTEND.pack(*qs, *_rows(out, "out", q, shape), *cache, *ids,
                        _vector(lengths, "lengths", torch.int32, q, seqs), 0 if sums is None else sums.data_ptr(),
                        *_work(work, q), heads, dim ** -0.5 if scale is None else scale, dtype)
    _check(lib.zo_cache_attend(args, _launch_stream(q, stream)), "zo_cache_attend")
    return (out, sums) if lse else out


def zo_cache_copy(k_caches, v_caches, src, dst, rows=None, stream=None):
    """In each layer's cache: tokens 0 .. rows[i] - 1 (all if None) of page src[i] to page dst[i]. src, dst and rows
    are host arrays; no dst is repeated or a src of the same call."""
    k_caches, v_caches = list(k_caches), list(v_caches)
    if len(k_caches) != len(v_caches):
        raise ValueError("one v_cache for each k_cache")
    if not k_caches:
        return
    like = k_caches[0]
    dtype = _dtype(like, "k_cache", 4)
    fields = _cache(like, v_caches[0], like)
    kind, device, shape, strides = like.dtype, like.get_device(), like.shape, like.stride()
    at = []
    for t in k_caches + v_caches:
        if not (type(t) in _TENSORS and t.dtype is kind and t.get_device() == device and t.shape == shape
                and t.stride() == strides):
            _refuse(t, "each cache", kind, like, shape, "must have the strides of the first")
        at.append(t.data_ptr())
    src = np.asarray(src, dtype=np.int32)
    moves = np.empty((src.size, 3), np.int32)
    moves[:, 0], moves[:, 1] = src, dst
    moves[:, 2] = shape[2] if rows is None else rows
    _check(_lib().zo_cache_copy(_CACHE.pack(*fields), array.array("Q", at).tobytes(), len(at), moves.ctypes.data, len(moves),
                                dtype, _launch_stream(like, stream)), "zo_cache_copy")


def zo_draw(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, logprobs=False, tokens=None, stream=None):
    """int32 tokens [rows] drawn from logits [rows, vocab] with the random numbers u [rows] in [0, 1), each row with
    its temperature, top_k (int32), top_p and min_p (device tensors [rows] or None). logprobs: also returns
    the drawn tokens' log probabilities among what was kept, float32."""
    dtype = _dtype(logits, "logits", 2)
    rows, vocab = logits.shape
    if vocab > 1 and logits.stride(1) != 1:
        raise ValueError("rows of logits must be contiguous")
    if tokens is None:
        tokens = _new(logits, (rows,), stream, torch.int32)
    probs = _new(logits, (rows,), stream, torch.float32) if logprobs else None
    f32 = torch.float32
    args = _DRAW.pack(logits.data_ptr(), logits.stride(0), _vector(u, "u", f32, logits, rows),
                      _vector(temperature, "temperature", f32, logits, rows), _vector(top_k, "top_k", torch.int32, logits, rows),
                      _vector(top_p, "top_p", f32, logits, rows), _vector(min_p, "min_p", f32, logits, rows),
                      _vector(tokens, "tokens", torch.int32, logits, rows), 0 if probs is None else probs.data_ptr(),
                      rows, vocab, dtype)
    _check(_lib().zo_draw(args, _launch_stream(logits, stream)), "zo_draw")
    return (tokens, probs) if logprobs else tokens


class ZoPages:
    """The book of a cache's pages (host only): which sequence holds which pages, which are shared, which are free."""

    def __init__(self, pages, page_tokens):
        self._book = None
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
        _check(_lib().zo_pages_add(self._book, tokens, ctypes.byref(seq)), "zo_pages_add")
        return seq.value

    def fork(self, seq):
        """A new sequence with the tokens of seq, sharing its pages; returns its number."""
        forked = ctypes.c_uint32()
        _check(_lib().zo_pages_fork(self._book, seq, ctypes.byref(forked)), "zo_pages_fork")
        return forked.value

    def extend(self, seq, tokens=1):
        """Room for more tokens; returns the copy that this needs first, (src, dst, rows), or None."""
        move = ZoPageMove()
        _check(_lib().zo_pages_extend(self._book, seq, tokens, ctypes.byref(move)), "zo_pages_extend")
        return (move.src, move.dst, move.rows) if move.rows else None

    def drop(self, seq):
        _check(_lib().zo_pages_drop(self._book, seq), "zo_pages_drop")

    def left(self):
        """How many pages are free."""
        return _lib().zo_pages_left(self._book)

    def length(self, seq):
        """The tokens of a sequence, -1 if there is none of that number."""
        return _lib().zo_pages_length(self._book, seq)

    def table(self, seqs, width=None):
        """(page ids int32 [sequences, width], lengths int32 [sequences]) as numpy arrays."""
        seqs = np.ascontiguousarray(np.asarray(seqs, dtype=np.uint32).reshape(-1))
        lengths = np.zeros(len(seqs), np.int32)
        if width is None:
            width = max([1] + [-(-self.length(s) // self.page_tokens) for s in seqs.tolist()])
        ids = np.full((len(seqs), width), -1, np.int32)
        _check(_lib().zo_pages_table(self._book, seqs.ctypes.data, len(seqs), ids.ctypes.data, width, width,
                                     lengths.ctypes.data), "zo_pages_table")
        return ids, lengths

    def compact(self, room=None):
        """Moves pages in use to the lowest ids; returns (src, dst, rows) to hand to zo_cache_copy."""
        room = self.pages if room is None else room
        moves = np.zeros((max(room, 1), 3), np.int32)
        n = ctypes.c_uint32()
        _check(_lib().zo_pages_compact(self._book, moves.ctypes.data, room, ctypes.byref(n)), "zo_pages_compact")
        return tuple(np.ascontiguousarray(moves[:n.value, i]) for i in range(3))
