"""Limits of the calls around the sparse path at their edges, on the host: nothing is launched (no GPU is needed)."""
import pytest

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
