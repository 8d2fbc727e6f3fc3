"""Calls of more workgroups than a launch takes: refused by name, before anything is launched (so without a GPU, and not as a dry run)."""
import pytest

import paper_2105_04663_amd as g
from tests.test_tokens_host import UNSUPPORTED, bufs

ONE = g.Mesh((1,), (0,))
T = 1 << 24
ROUTE = g.RouteBuf(*((1 << 21) + 64 * j for j in range(5)))


def refused(call, *args, **kw):
    with pytest.raises(g.GspmdError) as e:
        call(*args, **kw)
    assert e.value.status == UNSUPPORTED


@pytest.mark.parametrize("dtype, M", [(g.BF16, 8200), (g.F32, 4100), (g.BF16, 1 << 21)])
def test_rows_of_the_vocabulary(dtype, M):
    """2^24 tokens of five pieces of a wave each, and of many."""
    refused(g.embed, ONE, [1 << 21], bufs(1, dtype), g.Sharding((50, M), (-1, -1)), bufs(1, dtype), g.Sharding((T, M), (-1, -1)))


@pytest.mark.parametrize("dtype, M", [(g.BF16, 4100), (g.F32, 2050)])
def test_combined_rows(dtype, M):
    refused(g.combine, ONE, bufs(1, dtype), g.Sharding((2, T, M), (-1, -1, -1)), 1, ROUTE, bufs(1, dtype), g.Sharding((T, M), (-1, -1)))


@pytest.mark.parametrize("dtype, M", [(g.BF16, 8200), (g.F32, 4100)])
def test_dispatched_rows(dtype, M):
    refused(g.dispatch, ONE, bufs(1, dtype), g.Sharding((T, M), (-1, -1)), 1, ROUTE, bufs(1, dtype), g.Sharding((2, T, M), (-1, -1, -1)))
