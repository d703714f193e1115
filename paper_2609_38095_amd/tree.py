"""Python binding of libzo's operators for several new tokens of each sequence at a time (include/zo_tree.h): prompts, and
drafted answers that one pass of the model verifies.

Argument marshalling only, as in decode.py, under the C names:

  zo_tree_lay(starts, lengths, tokens, parents, words)  sequences, positions, places and masks of the new tokens
  zo_norm_rotate_put(..., seqs=, places=)               (decode.py) queries rotated, keys and values put at the places
  zo_tree_attend(q, k_cache, v_cache, table, lengths, starts, seen)
                                                        the new tokens over the cache and over each other
  zo_tree_accept(drafted, drawn, starts, most, parents, words=) the walk along the drafted tokens that the draws agree with
  zo_tree_keep(k_caches, v_caches, table, lengths, path) its keys and values brought together, every layer
  ZoPages.cut(seq, tokens)                              (decode.py) the rest of the draft's pages goes back

New tokens lie packed, sequence s has rows starts[s] .. starts[s + 1] - 1 (starts: int32 [sequences + 1]) behind its lengths[s]
cached tokens. parents (int32 [tokens], indices within the sequence, -1: behind the cached tokens) makes them a tree, None a
chain. Tensors, streams and errors as in decode.py.
"""

from . import decode

ZO_TREE_WORDS = 8

EXPORTS = ("zo_tree_lay", "zo_norm_rotate_put_at", "zo_tree_attend", "zo_tree_attend_work", "zo_tree_accept", "zo_tree_keep",
           "zo_pages_cut")


def zo_tree_lay(starts, lengths, tokens, parents=None, words=None, stream=None):
    """(seq_of, positions, places, seen) of the new tokens: int32 [tokens] each, and masks int64 [tokens, words] whose bit 64 w + b
    says that a token sees new token 64 w + b of its sequence. words: as many as the largest tree needs, 64 tokens each (by
    default what a tree of all the tokens needs, at most ZO_TREE_WORDS); 0 for chains (their default), whose seen is None."""
    if words is None:
        words = 0 if parents is None else min(ZO_TREE_WORDS, max(1, -(-tokens // 64)))
    return decode._call((decode._TENSORS or decode._tensors()).tree_lay, stream, starts, starts, lengths, tokens, parents, words)


def zo_tree_attend(q, k_cache, v_cache, table, lengths, starts, seen=None, scale=None, out=None, lse=False, work=None, stream=None):
    """out [tokens, heads, dim]: attention of the new tokens' queries q over the first lengths[s] tokens of their sequence's pages
    table[s] and over the new tokens behind them that they see (seen None: a chain, each sees itself and those before it).
    scale: dim ** -0.5 by default. lse: also returns log sum exp of the scores, float32 [tokens, heads]. Rows of no sequence are
    left as they were. work: a tensor of zo_tree_attend_work() bytes (allocated if None)."""
    return decode._call((decode._TENSORS or decode._tensors()).tree_attend, stream, q, q, k_cache, v_cache, table, lengths, starts, seen,
                        scale, out, lse, work)


def zo_tree_accept(drafted, drawn, starts, most, parents=None, stream=None, words=0):
    """(path, tokens, counts): int32 [sequences, most] indices of the walked tokens and the tokens drawn behind them, -1 behind
    the walk's end, and int32 [sequences] how many they are. drafted, drawn: int32 [tokens], the drafted tokens and those drawn
    behind each of them. words: the masks' of zo_tree_lay, whose trees end with them (0: no limit); new tokens behind have no place
    in the cache and are not walked."""
    return decode._call((decode._TENSORS or decode._tensors()).tree_accept, stream, drafted, drafted, drawn, starts, most, parents, words)


def zo_tree_keep(k_caches, v_caches, table, lengths, path, stream=None):
    """In each layer's cache: the keys and values of sequence s at token lengths[s] + path[s][i] go to token lengths[s] + i. Layers
    that share a cache may list it each; it moves once."""
    k_caches = list(k_caches)
    decode._call((decode._TENSORS or decode._tensors()).tree_keep, stream, k_caches[0] if k_caches else None, k_caches, list(v_caches),
                 table, lengths, path)
