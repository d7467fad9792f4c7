"""Refusals of the drafted-token and cache-budget calls that need no device: they are made before any CUDA call."""
from paper_2503_05840_b200 import binding as B


def test_missing_arguments_are_refused():
    L = B.lib()
    assert L.slim_tree_workspace_bytes(None, 1, 16, 4) == 0
    assert L.slim_weights_workspace_bytes(None, 1, 16) == 0
    assert L.slim_evict_workspace_bytes(None, 1, 16) == 0
    assert L.slim_tree_decode(None, None, None, None, None, None, 1, None, None, None) == B.SLIM_ERR_INVALID_ARG
    assert L.slim_tree_verify(None, None, None, None, None, None, 1, 1, 1, None, None, None, None) == B.SLIM_ERR_INVALID_ARG
    assert L.slim_tree_commit(None, None, None, None, None, None, 1, None) == B.SLIM_ERR_INVALID_ARG
    assert L.slim_accumulate_weights(None, None, None, None, None, None, None) == B.SLIM_ERR_INVALID_ARG
    assert L.slim_evict(None, None, None, None, 1, 0, None, None, None) == B.SLIM_ERR_INVALID_ARG
    assert "tree" in B.strerror(B.SLIM_ERR_TREE)
