"""What gspmd_ragged_dot refuses, before anything is launched."""
import pytest

import paper_2105_04663_amd as g
from tests.pin import pinned

NULL, BAD_MESH, BAD_SHARDING, BAD_DIMS, RESHARD, UNSUPPORTED, BUFFER = 1, 2, 3, 5, 6, 7, 10


def args(E=4, S=50, M=16, H=24, way="rows", mesh=(2, 2), lhs_map=(1, -1, -1), rhs_map=(1, -1, -1), out_map=(1, -1, -1), dtype=g.BF16, out_dtype=None):
    m = g.Mesh(mesh, tuple(range(mesh[0] * mesh[1])))
    contract = {"rows": ((2,), (1,)), "back": ((2,), (2,)), "matrices": ((1,), (1,))}[way]
    rhs = {"rows": (E, M, H), "back": (E, H, M), "matrices": (E, S, H)}[way]
    buf = [g.ShardBuf(1 << 20, dtype, 0)] * m.n_partitions
    return dict(mesh=m, dims=g.DotDims((0,), (0,), *contract), lhs_shards=list(buf), lhs_sh=g.Sharding((E, S, M), lhs_map), rhs_shards=list(buf), rhs_sh=g.Sharding(rhs, rhs_map),
                out_shards=[g.ShardBuf(1 << 22, dtype if out_dtype is None else out_dtype, 0)] * m.n_partitions, out_sh=g.Sharding((E, M, H) if way == "matrices" else (E, S, H), out_map), sizes=1 << 21)


def status(kw, **more):
    try:
        with pinned(dry_run=True):
            g.ragged_dot(**{**kw, **more})
    except g.GspmdError as e:
        return e.status
    return 0


@pytest.mark.parametrize("way", ["rows", "back", "matrices"])
def test_refusals(way):
    ok = args(way=way)
    assert status(ok) == 0
    assert status(ok, sizes=0) == NULL
    assert status(ok, sizes=(1 << 21) + 2) == BUFFER
    assert status(ok, mesh=g.Mesh((2, 2), (0, 1, 2, 2))) == BAD_MESH
    assert status(args(way=way, lhs_map=(1, 1, -1))) == BAD_SHARDING
    assert status(ok, epilogue=7) == UNSUPPORTED
    assert status(args(way=way, dtype=3)) == UNSUPPORTED
    assert status(args(way=way, dtype=g.F32, out_dtype=g.BF16)) == UNSUPPORTED
    assert status(args(way=way, dtype=g.BF16, out_dtype=g.F32)) == 0
    assert status(args(way=way, S=(1 << 24) + 1)) == UNSUPPORTED
    assert status(args(way=way, rhs_map=(0, -1, -1))) == RESHARD                # experts split otherwise
    assert status(args(way=way, out_map=(-1, -1, -1))) == RESHARD
    for dim in (1, 2):                                                          # anything but the experts split
        split = tuple(0 if i == dim else 1 if i == 0 else -1 for i in range(3))
        assert status(args(way=way, lhs_map=split)) == RESHARD
        assert status(args(way=way, rhs_map=split, out_map=split)) == RESHARD
    for name in ("lhs_shards", "rhs_shards", "out_shards"):
        for wrong, expect in ((g.ShardBuf(1 << 20, g.F32, 0), UNSUPPORTED if name != "out_shards" else UNSUPPORTED), (g.ShardBuf(0, g.BF16, 0), NULL), (g.ShardBuf(1 << 20, g.BF16, 15), BUFFER),
                              (g.ShardBuf(1 << 20, g.BF16, -1), BUFFER), (g.ShardBuf((1 << 20) + 1, g.BF16, 0), BUFFER), (g.ShardBuf(1 << 20, g.BF16, 1 << 32), UNSUPPORTED)):
            shards = list(ok[name])
            shards[3] = wrong
            assert status(ok, **{name: shards}) == expect, (name, wrong)
        with pytest.raises(ValueError):
            g.ragged_dot(**{**ok, name: ok[name][:3]})
    # a mesh dimension of one partition splits nothing
    assert status(args(way=way, mesh=(1, 4), lhs_map=(1, 0, -1))) == 0


def test_other_forms_are_refused():
    ok = args()
    E, S, M, H = 4, 50, 16, 24
    assert status(ok, dims=g.DotDims((), (), (2,), (1,))) in (BAD_DIMS, UNSUPPORTED)
    assert status(ok, dims=g.DotDims((0,), (0,), (2,), (2,))) == BAD_DIMS
    assert status(ok, lhs_sh=g.Sharding((E, S, M + 1), (1, -1, -1))) == BAD_DIMS
    assert status(ok, out_sh=g.Sharding((E, H, S), (1, -1, -1))) == BAD_DIMS
    # the slots of lhs contracted with another dimension than the slots of rhs
    assert status(ok, dims=g.DotDims((0,), (0,), (1,), (2,)), lhs_sh=g.Sharding((E, S, M), (1, -1, -1)), rhs_sh=g.Sharding((E, H, S), (1, -1, -1)), out_sh=g.Sharding((E, M, H), (1, -1, -1))) == UNSUPPORTED
    assert status(ok, lhs_sh=g.Sharding((E, S, 2, 8), (1, -1, -1, -1)), dims=g.DotDims((0,), (0,), (3,), (1,)), rhs_sh=g.Sharding((E, 8, H), (1, -1, -1)),
                  out_sh=g.Sharding((E, S, 2, H), (1, -1, -1, -1))) == UNSUPPORTED
    # rows beyond 32-bit offsets inside a tile
    assert status(ok, lhs_shards=[g.ShardBuf(1 << 20, g.BF16, 1 << 23)] * 4) == UNSUPPORTED


def test_no_elements_need_no_buffers():
    nothing = [g.ShardBuf(0, g.BF16, 0)] * 4
    for kw in (dict(E=0), dict(H=0), dict(S=0)):
        ok = args(**kw)
        assert status(ok, lhs_shards=ok["lhs_shards"] if "H" in kw else nothing, rhs_shards=ok["rhs_shards"] if "S" in kw else nothing, out_shards=nothing, sizes=0) == 0
    ok = args(way="matrices", S=0)
    assert status(ok, lhs_shards=nothing, rhs_shards=nothing) == 0
    assert status(ok, out_shards=nothing) == NULL
