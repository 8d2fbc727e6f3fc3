"""Shards of one tensor have one row stride; 0 stands for that of a dense shard."""
import pytest

import paper_2105_04663_amd as g
from tests.pin import pinned
from tests.test_softmax_host import BUFFER, args, status


@pytest.mark.parametrize("vocab_dim", [0, 1])
@pytest.mark.parametrize("name", ["x_shards", "w_shards", "dx_shards", "dw_shards"])
def test_dense_shards_by_either_name(name, vocab_dim):
    ok = args(vocab_dim=vocab_dim, w_map=(1, -1) if vocab_dim == 0 else (-1, 1))
    dense = 20 if vocab_dim == 1 and name in ("w_shards", "dw_shards") else 16
    for at in (0, 2):
        shards = list(ok[name])
        shards[at] = g.ShardBuf(1 << 20, g.BF16, dense)
        with pinned(dry_run=True):
            g.softmax_xent(**{**ok, name: shards})
            g.softmax_distill(targets=3, **{**ok, name: shards})
        shards[at] = g.ShardBuf(1 << 20, g.BF16, dense + 8)
        assert status(g.softmax_xent, ok, **{name: shards}) == BUFFER
