"""Limits of the calls around the sparse path at their edges, and arguments that are missing, on the host: nothing is launched (no GPU is needed)."""
import pytest
import torch

P = pytest.importorskip("paper_2605_23445_amd")
from paper_2605_23445_amd import binding as B  # noqa: E402
from tests.test_layer_host import QK, _rope  # noqa: E402


@pytest.mark.parametrize("batch,tokens", [(1, (1 << 27) - 7), (1, (1 << 27) - 1), (11, 12201611), (8193, 16382)])
def test_tokens_that_fill_a_grid_with_its_last_group_are_refused(batch, tokens):
    """32 lanes a token, in work-groups of 256: 2^27 - 7 tokens are 2^32 threads already, one more than a grid has."""
    assert (1 << 27) - 8 < batch * tokens < 1 << 27
    geom = dict(batch=batch, tokens=tokens)
    for back in (False, True):
        assert _rope(geom=geom, back=back) == -2 and b"tokens" in B._lib.dfs_last_error()
    assert P.dfs_qk_workspace_bytes(P.QkGeom(**dict(QK, **geom))) == 0


def test_the_most_tokens_are_taken():
    assert P.dfs_qk_workspace_bytes(P.QkGeom(**dict(QK, batch=1, tokens=(1 << 27) - 8))) > 0


def test_missing_tensors_raise_what_other_missing_ones_do():
    """On the host ValueError comes from the first tensor that is not the device's; what is None raises no AttributeError of the binding's own."""
    g = P.QkGeom(2, 5, 4, 2, 64, 1, 1, 64, 0, 0, 1e4, 1e-6)
    q, k = torch.zeros(2, 4, 5, 64), torch.zeros(2, 2, 5, 64)
    pos, start = torch.zeros(5, 1, dtype=torch.int32), torch.zeros(2, dtype=torch.int32)
    for args in ((q, k, k, None, None, None, q, k, k), (q, k, k, pos, None, None, q, None, k, start), (q, k, k, pos, None, None, q, k[0, 0, 0], k, start),
                 (q, k, k, None, None, None, q, None, None, start)):
        with pytest.raises((ValueError, P.DfsError)):
            P.dfs_qk_norm_rope(g, P.DFS_F32, *args)
    with pytest.raises((ValueError, P.DfsError)):
        P.dfs_qk_norm_rope_bwd(g, P.DFS_F32, q, k, None, None, None, q, k, k, q, k, k)
