"""Calls of the operators for several new tokens that are easy to forget, on the GPU."""

import numpy as np
import pytest
import torch

import paper_2609_38095_amd as zo
from oracle import tree as oracle
from test_gpu_tree import cache_of, dev, ints, wide

pytestmark = pytest.mark.gpu


# ---- moves

@pytest.mark.parametrize("layers", [1, 3, 150])
def test_keep_of_shared_caches(layers):
    """Layers that share a cache, and keys that are the values: each tensor's rows move once, in one launch or several."""
    kc, vc = cache_of("heads", 1, 12, 2, 4, 64, "bf16")
    table, lengths = np.arange(12, dtype=np.int32).reshape(3, 4), [0, 5, 2]
    path = np.array([[0, 2, 3, 5, 6], [1, 2, 4, 5, 7], [0, 1, 5, -1, -1]], np.int32)
    wants = [oracle.keep(wide(t), table, lengths, path) for t in (kc, vc)]
    for tensors in ((kc.clone(), vc.clone()), (kc.clone(), None)):
        k, v = tensors
        zo.zo_tree_keep([k] * layers, [k if v is None else v] * layers, dev(table), ints(lengths), dev(path))
        assert np.array_equal(wide(k), wants[0]) and (v is None or np.array_equal(wide(v), wants[1]))
