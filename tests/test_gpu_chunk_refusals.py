"""Chunk calls that are refused on the host, whatever their buffers."""
import pytest

from paper_2608_23599_b200 import binding as B
from tests import test_gpu_chunk as tc

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n_new", [2 ** 30 + 1, 2 ** 31 - 130, 2 ** 31 - 1])
def test_more_new_tokens_than_any_memory_holds(n_new):
    """Counts from which the tiles' number does not fit 32 bits; only the question for the workspace, which reads no buffer."""
    c, _, _ = tc.caches(3, 1, 100, seed=1, plan=8, **tc.EXT)
    n = B.C.c_size_t(7)
    assert B.load().gkv_chunk_workspace_bytes(c.handle, 0, n_new, B.C.byref(n)) == B.ERR_INVALID_ARG and n.value == 7
