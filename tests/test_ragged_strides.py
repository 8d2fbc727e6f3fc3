"""The longest rows that gspmd_ragged_dot takes, and what it says to longer ones: host work, before anything is launched."""
import pytest

import paper_2105_04663_amd as g
from tests.test_ragged_host import UNSUPPORTED, args, status

K_CONTIGUOUS, K_MAJOR = 1 << 22, 1 << 24        # elements between rows of a bfloat16 operand


@pytest.mark.parametrize("way, operand, most", [("rows", "lhs_shards", K_CONTIGUOUS), ("rows", "rhs_shards", K_MAJOR), ("back", "lhs_shards", K_CONTIGUOUS), ("back", "rhs_shards", K_CONTIGUOUS),
                                                ("matrices", "lhs_shards", K_MAJOR), ("matrices", "rhs_shards", K_MAJOR)])
def test_longest_rows(way, operand, most):
    for dtype, stride, expect in ((g.BF16, most, 0), (g.BF16, most + 1, UNSUPPORTED), (g.BF16, most + 8, UNSUPPORTED), (g.BF16, (1 << 31) - 1, UNSUPPORTED), (g.BF16, 1 << 31, UNSUPPORTED),
                                  (g.F32, most + 1, 0), (g.F32, (1 << 31) - 1, 0), (g.F32, 1 << 31, UNSUPPORTED)):
        ok = args(way=way, dtype=dtype)
        buf = ok[operand][0]
        assert status(ok, **{operand: [g.ShardBuf(buf.data, buf.dtype, stride)] * 4}) == expect, (dtype, stride)
        one = [g.ShardBuf(buf.data, buf.dtype, stride)] + ok[operand][1:]         # of one partition's shard (not of a replica that shares its out buffer, whose operands are not read)
        assert status(ok, **{operand: one}) == expect, (dtype, stride)


@pytest.mark.parametrize("way", ["rows", "back", "matrices"])
@pytest.mark.parametrize("dtype, out", [(g.BF16, g.BF16), (g.BF16, g.F32), (g.F32, g.F32)])
def test_rows_of_the_output_may_be_longer(way, dtype, out):
    ok = args(way=way, dtype=dtype, out_dtype=out)
    for stride, expect in ((K_MAJOR + 1, 0), ((1 << 31) - 1, 0), (1 << 31, UNSUPPORTED)):
        assert status(ok, out_shards=[g.ShardBuf(b.data, b.dtype, stride) for b in ok["out_shards"]]) == expect
