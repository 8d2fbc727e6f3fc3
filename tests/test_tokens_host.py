"""What the operators that choose by a token's index refuse, and their workspaces: host work, before anything is launched."""
import pytest

import paper_2105_04663_amd as g
from tests.pin import pinned

NULL, BAD_MESH, BAD_SHARDING, BAD_DIMS, RESHARD, UNSUPPORTED, WORKSPACE, BUFFER = 1, 2, 3, 5, 6, 7, 8, 10


def status(call, kw, **more):
    try:
        with pinned(dry_run=True):
            call(**{**kw, **more})
    except g.GspmdError as e:
        return e.status
    return 0


def bufs(n, dtype=g.BF16, at=1 << 20):
    return [g.ShardBuf(at, dtype, 0)] * n


WRONG = [(g.ShardBuf(1 << 20, g.F32, 0), UNSUPPORTED), (g.ShardBuf(0, g.BF16, 0), NULL), (g.ShardBuf(1 << 20, g.BF16, 15), BUFFER), (g.ShardBuf(1 << 20, g.BF16, -1), BUFFER),
         (g.ShardBuf((1 << 20) + 1, g.BF16, 0), BUFFER), (g.ShardBuf(1 << 20, g.BF16, 1 << 32), BUFFER), (g.ShardBuf(1 << 20, g.BF16, 24), BUFFER)]


def embed_args(T=9, M=16, V=40, mesh=(2, 2), t_map=(0, -1), w_map=None, vocab_dim=0, grad=False, dtype=g.BF16):
    m = g.Mesh(mesh, tuple(range(mesh[0] * mesh[1])))
    n = m.n_partitions
    w_map = w_map or ((1, -1) if vocab_dim == 0 else (-1, 1))
    rows, w = g.Sharding((T, M), t_map), g.Sharding((V, M) if vocab_dim == 0 else (M, V), w_map)
    kw = dict(mesh=m, ids=[1 << 21] * n, vocab_dim=vocab_dim)
    if grad:
        return dict(kw, dy_shards=bufs(n, dtype), dy_sh=rows, dw_shards=bufs(n, dtype), dw_sh=w, workspace=1 << 24, workspace_bytes=1 << 30)
    return dict(kw, w_shards=bufs(n, dtype), w_sh=w, y_shards=bufs(n, dtype), y_sh=rows)


@pytest.mark.parametrize("vocab_dim", [0, 1])
@pytest.mark.parametrize("grad", [False, True])
def test_embed_refusals(grad, vocab_dim):
    call = g.embed_grad if grad else g.embed
    make = lambda **kw: embed_args(grad=grad, vocab_dim=vocab_dim, **kw)
    ok = make()
    assert status(call, ok) == 0
    assert status(call, ok, mesh=g.Mesh((2, 2), (0, 1, 2, 2))) == BAD_MESH
    assert status(call, make(t_map=(0, 0))) == BAD_SHARDING
    assert status(call, make(t_map=(-1, 0))) == RESHARD
    assert status(call, make(w_map=(-1, 1) if vocab_dim == 0 else (1, -1))) == RESHARD
    assert status(call, make(w_map=(0, -1) if vocab_dim == 0 else (-1, 0))) == RESHARD          # over the tokens' mesh dimension
    assert status(call, ok, vocab_dim=2) == BAD_DIMS
    assert status(call, ok, **{"dy_sh" if grad else "y_sh": g.Sharding((9, 17), (0, -1))}) == BAD_DIMS
    assert status(call, ok, **{"dy_sh" if grad else "y_sh": g.Sharding((9, 16, 1), (0, -1, -1))}) == BAD_DIMS
    assert status(call, make(V=0)) == BAD_DIMS
    assert status(call, make(dtype=3)) == UNSUPPORTED
    assert status(call, make(T=1 << 25)) == UNSUPPORTED
    assert status(call, make(V=1 << 30)) == UNSUPPORTED
    assert status(call, make(mesh=(65, 1))) == UNSUPPORTED and status(call, make(mesh=(1, 65))) == UNSUPPORTED
    assert status(call, ok, ids=[1 << 21] * 3 + [0]) == NULL
    assert status(call, ok, ids=[1 << 21] * 3 + [(1 << 21) + 2]) == BUFFER
    for name in ("dy_shards", "dw_shards") if grad else ("w_shards", "y_shards"):
        for wrong, expect in WRONG:
            if wrong.row_stride == 15 and vocab_dim == 1 and name in ("dw_shards", "w_shards"):
                wrong = g.ShardBuf(1 << 20, g.BF16, 19)
            assert status(call, ok, **{name: ok[name][:3] + [wrong]}) == expect, (name, wrong)
        with pytest.raises(ValueError):
            call(**{**ok, name: ok[name][:3]})
    if grad:
        need = g.embed_grad_workspace_bytes(ok["mesh"], ok["dy_sh"], ok["dw_sh"], vocab_dim, g.BF16)
        assert need > 0
        assert status(call, ok, workspace_bytes=need) == 0
        for more in (dict(workspace_bytes=need - 1), dict(workspace=0), dict(workspace=(1 << 24) + 64)):
            assert status(call, ok, **more) == WORKSPACE
        assert status(call, make(T=0), workspace=0, workspace_bytes=0, ids=[0] * 4, dy_shards=bufs(4, at=0)) == 0
        with pytest.raises(g.GspmdError):
            g.embed_grad_workspace_bytes(ok["mesh"], ok["dy_sh"], ok["dw_sh"], vocab_dim, 9)
    else:
        assert status(call, make(T=0), ids=[0] * 4, y_shards=bufs(4, at=0)) == 0


def route_args(T=9, E=8, k=2, mesh=(2, 2), sh_map=(0, -1), dtype=g.F32, grad=False):
    m = g.Mesh(mesh, tuple(range(mesh[0] * mesh[1])))
    kw = dict(mesh=m, logits_shards=bufs(m.n_partitions, dtype), logits_sh=g.Sharding((T, E), sh_map), choices=k, route=g.RouteBuf(*[(1 << 21) + 64 * i for i in range(5)]))
    return dict(kw, dweights=1 << 22, dlogits_shards=bufs(m.n_partitions, dtype)) if grad else dict(kw, workspace=1 << 24, workspace_bytes=1 << 30)


@pytest.mark.parametrize("grad", [False, True])
def test_route_refusals(grad):
    call = g.route_grad if grad else g.route
    make = lambda **kw: route_args(grad=grad, **kw)
    ok = make()
    assert status(call, ok) == 0 and status(call, make(dtype=g.BF16)) == 0
    assert status(call, ok, mesh=g.Mesh((2, 2), (0, 1, 2, 2))) == BAD_MESH
    assert status(call, make(sh_map=(0, 0))) == BAD_SHARDING
    assert status(call, make(sh_map=(-1, 1))) == RESHARD
    assert status(call, make(k=0)) == BAD_DIMS and status(call, make(k=9)) == BAD_DIMS
    assert status(call, ok, logits_sh=g.Sharding((9, 8, 1), (0, -1, -1))) == BAD_DIMS
    assert status(call, make(E=g.MAX_EXPERTS)) == 0 and status(call, make(E=g.MAX_EXPERTS + 1)) == UNSUPPORTED
    assert status(call, make(E=40, k=g.MAX_CHOICES)) == 0 and status(call, make(E=40, k=g.MAX_CHOICES + 1)) == UNSUPPORTED
    assert status(call, make(T=1 << 24)) == UNSUPPORTED and status(call, make(mesh=(65, 1))) == UNSUPPORTED and status(call, make(dtype=2)) == UNSUPPORTED
    assert status(call, ok, logits_shards=ok["logits_shards"][:3] + [g.ShardBuf(1 << 20, g.F32, 12)]) == BUFFER
    assert status(call, ok, logits_shards=ok["logits_shards"][:3] + [g.ShardBuf(0, g.F32, 0)]) == NULL
    for i, name in enumerate(("experts", "weights", "slots", "order", "sizes")):
        needed = not grad or i < 2
        fields = [(1 << 21) + 64 * j for j in range(5)]
        assert status(call, ok, route=g.RouteBuf(*(fields[:i] + [0] + fields[i + 1:]))) == (NULL if needed else 0), name
        assert status(call, ok, route=g.RouteBuf(*(fields[:i] + [fields[i] + 2] + fields[i + 1:]))) == (BUFFER if needed else 0), name
    if grad:
        assert status(call, ok, dweights=0) == NULL and status(call, ok, dweights=(1 << 22) + 1) == BUFFER
        assert status(call, ok, dlogits_shards=bufs(4, g.BF16)) == UNSUPPORTED
    else:
        assert g.route_workspace_bytes(ok["mesh"], ok["logits_sh"], 2) == 0 and status(call, ok, workspace=0, workspace_bytes=0) == 0      # few tokens
        big = make(T=2000)
        need = g.route_workspace_bytes(big["mesh"], big["logits_sh"], 2)
        assert need > 0 and status(call, big, workspace_bytes=need) == 0
        for more in (dict(workspace_bytes=need - 1), dict(workspace=0), dict(workspace=(1 << 24) + 8)):
            assert status(call, big, **more) == WORKSPACE


def exchange_args(which, T=9, E=8, k=2, M=16, S=18, mesh=(2, 2), t_map=(0, -1), e_map=(1, -1, -1), dtype=g.BF16):
    m = g.Mesh(mesh, tuple(range(mesh[0] * mesh[1])))
    n = m.n_partitions
    kw = dict(mesh=m, choices=k, route=g.RouteBuf(*[(1 << 21) + 64 * i for i in range(5)]), rows_shards=bufs(n, dtype), rows_sh=g.Sharding((E, S, M), e_map))
    sh = g.Sharding((T, M), t_map)
    if which == "dispatch":
        return dict(kw, x_shards=bufs(n, dtype), x_sh=sh)
    if which == "combine":
        return dict(kw, y_shards=bufs(n, dtype), y_sh=sh)
    return dict(kw, dy_shards=bufs(n, dtype), dy_sh=sh, drows_shards=bufs(n, dtype), dweights=1 << 22)


@pytest.mark.parametrize("which", ["dispatch", "combine", "combine_grad"])
def test_exchange_refusals(which):
    call = getattr(g, which)
    make = lambda **kw: exchange_args(which, **kw)
    ok = make()
    assert status(call, ok) == 0 and status(call, make(S=1000)) == 0
    assert status(call, make(S=17)) == BAD_DIMS
    assert status(call, make(k=0)) == BAD_DIMS and status(call, make(k=9, S=1000)) == BAD_DIMS
    assert status(call, ok, rows_sh=g.Sharding((8, 18, 17), (1, -1, -1))) == BAD_DIMS
    assert status(call, ok, rows_sh=g.Sharding((18, 16), (1, -1))) == BAD_DIMS
    assert status(call, make(t_map=(-1, 0))) == RESHARD and status(call, make(e_map=(-1, 1, -1))) == RESHARD and status(call, make(e_map=(-1, -1, 1))) == RESHARD
    assert status(call, make(E=g.MAX_EXPERTS + 1)) == UNSUPPORTED and status(call, make(mesh=(1, 65))) == UNSUPPORTED and status(call, make(T=1 << 23, S=1 << 24, k=3)) in (BAD_DIMS, UNSUPPORTED)
    assert status(call, make(dtype=2)) == UNSUPPORTED
    for name in [n for n in ok if n.endswith("_shards")]:
        for wrong, expect in WRONG:
            assert status(call, ok, **{name: ok[name][:3] + [wrong]}) == expect, (name, wrong)
        with pytest.raises(ValueError):
            call(**{**ok, name: ok[name][:3]})
    needed = {"dispatch": (0, 2), "combine": (0, 1, 2), "combine_grad": (0, 1, 2)}[which]
    fields = [(1 << 21) + 64 * j for j in range(5)]
    for i in range(5):
        assert status(call, ok, route=g.RouteBuf(*(fields[:i] + [0] + fields[i + 1:]))) == (NULL if i in needed else 0), i
        assert status(call, ok, route=g.RouteBuf(*(fields[:i] + [fields[i] + 1] + fields[i + 1:]))) == (BUFFER if i in needed else 0), i
    if which == "combine":
        assert status(call, ok, weighted=False, route=g.RouteBuf(fields[0], 0, fields[2], 0, 0)) == 0
    if which == "combine_grad":
        assert status(call, ok, dweights=0) == NULL and status(call, ok, dweights=2) == BUFFER


@pytest.mark.parametrize("grad", [False, True])
@pytest.mark.parametrize("vocab_dim", [0, 1])
def test_rows_of_the_embedding_are_bounded(grad, vocab_dim):
    call = g.embed_grad if grad else g.embed
    ok = embed_args(grad=grad, vocab_dim=vocab_dim, M=1 << 21)
    more = dict(workspace_bytes=1 << 40) if grad else {}
    rows = "dy_shards" if grad else "y_shards"
    w = "dw_shards" if grad else "w_shards"
    dense = {name: [g.ShardBuf(b.data, b.dtype, 0) for b in ok[name]] for name in (rows, w)}
    assert status(call, ok, **dense, **more) == 0
    assert status(call, embed_args(grad=grad, vocab_dim=vocab_dim, M=(1 << 21) + 1), **dense, **more) == UNSUPPORTED


def test_the_same_through_ctypes(monkeypatch):
    """Refusals do not depend on which way a call takes into the library."""
    from paper_2105_04663_amd import binding
    g.load_library()
    monkeypatch.setattr(binding, "_CALL", None)
    for grad in (False, True):
        test_route_refusals(grad)
        for vocab_dim in (0, 1):
            test_embed_refusals(grad, vocab_dim)
            test_rows_of_the_embedding_are_bounded(grad, vocab_dim)
    for which in ("dispatch", "combine", "combine_grad"):
        test_exchange_refusals(which)
