"""Softmax cross entropy and distillation over a split vocabulary against float64, element by element, at the sizes, meshes and targets where they can go wrong."""
import numpy as np
import pytest
import torch

import paper_2105_04663_amd as g
from tests.losses import Problem
from tests.pin import MFMA, pinned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab_dim", [0, 1])
@pytest.mark.parametrize("T,M,V", [(1, 1, 1), (1, 8, 2), (2, 65, 7), (33, 64, 90), (65, 130, 257), (300, 72, 1025), (5, 257, 8200)])
def test_xent(dtype, vocab_dim, T, M, V):
    Problem(T, M, V, dtype, vocab_dim=vocab_dim, pad=(T + V) % 2 == 0).stage().call().check()


# rows of every variant of the row kernel, at and beside the sizes where one takes over from another
@pytest.mark.parametrize("V", [1023, 1024, 1025, 8191, 8192, 8193, 32768, 32769, 65536, 65537, 70001])
@pytest.mark.parametrize("dtype,K", [("bf16", None), ("bf16", 5), ("f32", 5)])
def test_rows(V, dtype, K):
    Problem(3, 16, V, dtype, K=K, tau=1.5 if K else 1.0, missing=0.0).stage().call().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("K,tau,logits_dtype", [(1, 1.0, "f32"), (3, 2.0, "bf16"), (64, 0.5, "f32"), (100, 3.0, "bf16"), (1024, 1.0, "f32")])
def test_distill(dtype, K, tau, logits_dtype):
    Problem(37, 48, 1500, dtype, K=K, tau=tau, logits_dtype=logits_dtype).stage().call().check()


MESHES = [dict(mesh=(1, 4)), dict(mesh=(3, 1)), dict(mesh=(2, 4), ids_order=(5, 2, 7, 0, 3, 1, 6, 4)), dict(mesh=(2, 2, 3), x_map=(2, -1), v_axis=0),
          dict(mesh=(2, 2, 3), x_map=(2, -1), v_axis=0, share=False), dict(mesh=(8, 2)), dict(mesh=(2, 3), x_map=(-1, -1), v_axis=-1, share=False),
          dict(mesh=(4, 1, 2), x_map=(0, 1), v_axis=2)]


@pytest.mark.parametrize("where", MESHES, ids=lambda m: "x".join(map(str, m["mesh"])) + ("" if m.get("share", True) else "_own"))
@pytest.mark.parametrize("dtype,K,vocab_dim,pad", [("bf16", None, 0, True), ("bf16", 7, 1, False), ("f32", None, 1, True)])
def test_meshes(where, dtype, K, vocab_dim, pad):
    Problem(41, 24, 203, dtype, K=K, vocab_dim=vocab_dim, pad=pad, **where).stage().call().check()


@pytest.mark.parametrize("T,V,mesh", [(5, 9, (4, 4)), (1, 3, (3, 8)), (9, 65, (4, 5)), (2, 1, (2, 2)), (40, 300, (40, 1)), (70, 40, (66, 1)), (20, 130, (3, 17))])
def test_partitions_without_tokens_or_entries(T, V, mesh):
    for dtype, vocab_dim in (("bf16", 0), ("f32", 1)):
        Problem(T, 24, V, dtype, vocab_dim=vocab_dim, mesh=mesh).stage().call().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_tokens_and_no_hidden_dimension(dtype):
    p = Problem(0, 24, 50, dtype, mesh=(1, 2)).stage().call()
    assert not p.results()["dw"].any()
    p = Problem(6, 0, 50, dtype).stage((False, False)).call()
    got = p.results()
    assert np.allclose(got["lse"], np.log(50.0), atol=1e-6)
    assert np.allclose(got["loss"], np.where(p.ids[:, 0] >= 0, np.log(50.0), 0.0), atol=1e-6)


@pytest.mark.parametrize("grad", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("K", [None, 4])
def test_fewer_gradients(grad, K):
    full = Problem(70, 40, 333, K=K).stage().call().results()
    some = Problem(70, 40, 333, K=K).stage(grad).call().check()
    for name in some:
        if name in ("dx", "dw"):
            assert np.array_equal(some[name], full[name])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_no_targets(dtype):
    """Labels outside the vocabulary are none: loss 0, nothing in the gradients, bits of zero in all of them if no token has one."""
    p = Problem(20, 16, 77, dtype, missing=0.0)
    p.ids[:] = np.array([-1, 77, 78, 2 ** 31 - 1, -2 ** 31] * 4, dtype=np.int64).astype(np.int32)[:, None]
    got = p.stage().call().check()
    assert not got["loss"].any() and not got["dx"].any() and not got["dw"].any()
    q = Problem(20, 16, 77, dtype, K=6, missing=1.0)
    q.logits_t[:] = float("nan")                       # of entries that are absent
    got = q.stage().call().results()
    assert not got["loss"].any() and not got["dx"].any() and not got["dw"].any()


def test_teachers_logits_at_the_ends():
    p = Problem(6, 16, 77, K=4, missing=0.0)
    p.ids[3] = [5, 5, 5, 9]                             # one entry given three times
    for a in (p.logits, p.logits_t):
        a[0, 1:] = -np.inf                              # one entry
        a[1, :] = -np.inf                               # none
        a[2, 0] = -3e38                                 # the type's lowest
        a[4, 2] = 200.0                                 # all of it on one entry
    got = p.stage().call().check()
    assert got["loss"][1] == 0.0 and not got["dx"][1].any()


def test_one_bad_token_leaves_the_others():
    """A NaN among a token's teacher's logits, or in its activations, is a NaN in its own results; a weight of 0 keeps it out of D."""
    ref = Problem(9, 16, 300, K=3, missing=0.0).stage((True, False)).call().results()
    p = Problem(9, 16, 300, K=3, missing=0.0)
    p.logits_t[2, 1] = float("nan")
    p.logits_t[3, 0] = float("inf")
    p.xt[5, 3] = float("nan")
    p.weights[6] = 0.0
    p.xt[6, 2] = float("inf")
    got = p.stage((True, False)).call().results()
    assert np.isnan(got["loss"][[2, 3, 5, 6]]).all() and np.isnan(got["dx"][[2, 3, 5]]).all()
    assert not got["dx"][6].any()
    for t in (0, 1, 4, 7, 8):
        assert got["loss"][t] == ref["loss"][t] and np.array_equal(got["dx"][t], ref["dx"][t])


def test_large_logits():
    """Far beyond what exp takes: the maximum is subtracted."""
    for dtype in ("bf16", "f32"):
        p = Problem(17, 64, 500, dtype, wscale=40.0)
        got = p.stage().call().check()
        assert np.isfinite(got["loss"]).all() and np.abs(got["lse"]).max() > 500


@pytest.mark.parametrize("dtype,K", [("bf16", None), ("bf16", 9), ("f32", None)])
@pytest.mark.parametrize("mesh", [(1, 1), (2, 3)])
def test_pieces(dtype, K, mesh):
    """Less workspace: more pieces, down to one row of every token shard, the same results within their bounds; one byte less than the least is refused."""
    p = Problem(75, 40, 600, dtype, K=K, mesh=mesh).stage()
    p.call()
    for n in (p.least, p.least + (p.bytes - p.least) // 3, max(p.least, p.bytes - 1), p.bytes, p.bytes + 100000):
        for s in (p.dxs, p.dws):
            for b in s:
                b[1].fill_(float("nan"))
        p.call(n).check()
    with pytest.raises(g.GspmdError) as e:
        p.call(p.least - 1)
    assert e.value.status == 8


def test_equal_calls_give_equal_bits():
    for kw in (dict(), dict(mesh=(2, 4)), dict(dtype="f32", K=5)):
        a, b = (Problem(200, 96, 1111, **kw).stage().call().results() for _ in range(2))
        for name in a:
            assert np.array_equal(a[name], b[name]), name


@pytest.mark.parametrize("vocab_dim", [0, 1])
def test_gradients_against_differences(vocab_dim):
    """float32: the loss along a direction.  Its third derivative is below 8 |s|^3 (s: the largest change of a logit), a loss is 2^-20 off at most, so with h s = 0.05 a
    central difference is within 8 * 0.05^2 s / 6 + 2^-20 T / h of the derivative."""
    rng = np.random.default_rng(5)
    for K in (None, 4):
        p = Problem(6, 12, 40, "f32", K=K, vocab_dim=vocab_dim, weights=False)
        got = p.stage().call().results()
        for which in ("x", "w"):
            base, grad = getattr(p, which), got["d" + which]
            direction = rng.standard_normal(base.shape)
            s = np.abs(direction @ p.w.T if which == "x" else p.x @ direction.T).max()
            h = 0.05 / s
            at = []
            for sign in (1, -1):
                q = Problem(6, 12, 40, "f32", K=K, vocab_dim=vocab_dim, weights=False)
                t = torch.from_numpy((base + sign * h * direction).astype(np.float32))
                setattr(q, which + "t", t)
                at.append((q.stage((False, False)).call().results()["loss"].sum(), t.double().numpy()))
            step = at[0][1] - at[1][1]                  # as the type holds it
            assert abs((at[0][0] - at[1][0]) / (2 * h) - (grad * step).sum() / (2 * h)) <= 6 * (8 * 0.05 ** 2 * s / 6) + 6 * 2.0 ** -20 / h


def test_another_stream_and_a_graph():
    p = Problem(130, 64, 700, mesh=(2, 2)).stage()
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    p.call(stream=stream.cuda_stream)
    stream.synchronize()
    ref = p.check()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.call(stream=torch.cuda.current_stream().cuda_stream)
    for turn in range(4):
        for s in (p.dxs, p.dws):
            for b in s:
                b[1].fill_(float(turn))
        p.xs[0][1][:3].mul_(-1.0)                       # other inputs for every replay
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        replayed = [b[1].clone() for b in p.dxs + p.dws] + [t[1]["loss"].clone() for t in p.ts]
        p.call()
        torch.cuda.synchronize()
        for a, b in zip(replayed, [b[1] for b in p.dxs + p.dws] + [t[1]["loss"] for t in p.ts]):
            assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))
    assert np.isfinite(ref["loss"]).all()


# a handful of tokens, which have kernels of their own: every number of them that these provide for, rows of fewer elements than a lane takes and of more than a workgroup's
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab_dim", [0, 1])
@pytest.mark.parametrize("T,M,V", [(1, 1, 1), (1, 5, 700), (2, 64, 129), (3, 515, 1000), (4, 1030, 333), (5, 72, 5003), (8, 2100, 90), (8, 17, 40), (11, 300, 777), (16, 520, 1300)])
def test_a_handful_of_tokens(dtype, vocab_dim, T, M, V):
    for K, pad in ((None, True), (6, False)):
        p = Problem(T, M, V, dtype, K=K, vocab_dim=vocab_dim, pad=pad, missing=0.1).stage()
        p.call().check()
        if p.least < p.bytes:                           # the other path
            p.call(p.least).check()


@pytest.mark.parametrize("vocab_dim", [0, 1])
@pytest.mark.parametrize("mesh,T,V", [((2, 3), 7, 1000), ((5, 8), 3, 61), ((16, 2), 16, 300), ((1, 64), 2, 100), ((1, 65), 2, 100), ((3, 4), 8, 9)])
def test_a_handful_of_tokens_on_meshes(mesh, T, V, vocab_dim):
    for dtype, K, share in (("bf16", None, True), ("f32", 3, False)):
        Problem(T, 96, V, dtype, K=K, vocab_dim=vocab_dim, mesh=mesh, pad=T % 2 == 0, share=share).stage().call().check()
        for grad in ((True, False), (False, True), (False, False)):
            Problem(T, 96, V, dtype, K=K, vocab_dim=vocab_dim, mesh=mesh, pad=T % 2 == 0, share=share).stage(grad).call().check()


@pytest.fixture
def big_tiles():
    """The calls of a test through dot_mfma_kernel, whose tiles reduce the logits of a call without gradients where they are."""
    with pinned(MFMA):
        yield


@pytest.mark.parametrize("vocab_dim", [0, 1])
@pytest.mark.parametrize("T,M,V,K", [(1, 64, 64, None), (17, 72, 65, None), (256, 64, 256, 1), (300, 130, 1025, 3), (513, 96, 700, 33), (40, 1000, 3000, 128), (33, 64, 500, 129)])
def test_logits_that_are_not_kept(big_tiles, vocab_dim, T, M, V, K):
    Problem(T, M, V, K=K, vocab_dim=vocab_dim).stage((False, False)).call().check()


@pytest.mark.parametrize("mesh,T,V", [((1, 4), 50, 901), ((2, 3), 600, 1300), ((5, 7), 33, 100), ((66, 2), 70, 300), ((3, 8), 1, 9)])
def test_logits_that_are_not_kept_on_meshes(big_tiles, mesh, T, V):
    for K, vocab_dim in ((None, 0), (5, 1)):
        Problem(T, 80, V, K=K, vocab_dim=vocab_dim, mesh=mesh, tau=1.7 if K else 1.0).stage((False, False)).call().check()


def test_targets_of_one_tile(big_tiles):
    """All of 256 tokens' 128 targets in one tile: more than it looks at between two barriers."""
    p = Problem(300, 64, 2000, K=128, missing=0.3)
    p.ids[:] = np.where(p.ids >= 0, 512 + p.ids % 256, -1)
    p.stage((False, False)).call().check()


def test_logits_that_are_not_kept_in_pieces(big_tiles):
    p = Problem(700, 64, 900, K=3, mesh=(2, 2)).stage((False, False))
    for n in (p.least + (p.bytes - p.least) // 3, p.bytes):
        p.call(n).check()


def test_logits_that_are_not_kept_at_their_ends(big_tiles):
    p = Problem(40, 64, 300, wscale=30.0).stage((False, False)).call()
    assert np.abs(p.check()["lse"]).max() > 300
    p = Problem(20, 64, 300, missing=1.0).stage((False, False)).call()
    assert not p.check()["loss"].any()
    p = Problem(20, 64, 300, K=2, missing=0.0)
    p.logits_t[3, 0] = float("nan")
    p.xt[5, 1] = float("nan")
    got = p.stage((False, False)).call().results()
    assert np.isnan(got["loss"][[3, 5]]).all() and np.isfinite(np.delete(got["loss"], [3, 5])).all()


def test_random_problems():
    """Sizes, meshes and layouts drawn together."""
    rng = np.random.default_rng(77)
    for n in range(40):
        T, M, V = (int(np.exp(rng.uniform(0, np.log(hi)))) for hi in (400, 300, 3000))
        K = None if rng.random() < 0.5 else int(rng.integers(1, 40))
        p = Problem(T, M, V, "bf16" if rng.random() < 0.7 else "f32", K=K, tau=float(rng.choice([0.7, 1.0, 2.5])) if K else 1.0, seed=n, vocab_dim=int(rng.integers(0, 2)),
                    mesh=(int(rng.integers(1, 5)), int(rng.integers(1, 7))), pad=bool(rng.integers(0, 2)), share=bool(rng.integers(0, 2)), weights=bool(rng.integers(0, 2)))
        print(n, T, M, V, p.dtype, K, p.mesh.shape, p.vocab_dim, p.pad, flush=True)
        p.stage().call().check()


@pytest.mark.parametrize("T,V,dtype,grad,K", [(2, 300, "f32", True, None), (9, 300, "bf16", True, None), (200, 300, "bf16", False, 3), (9, 70000, "bf16", True, None), (3, 3000, "bf16", False, None)])
def test_logits_of_minus_infinity_throughout(T, V, dtype, grad, K):
    """A token without any probability: lse is -infinity, its loss and gradient NaN, by every path; other tokens are as ever."""
    p = Problem(T, 16, V, dtype, K=K, missing=0.0)
    p.xt[:, 0] = 0.0
    ref = p.stage((grad, False)).call().results()
    p.xt[1, 0] = 3e38
    p.wt[:, 0] = -100.0
    got = p.stage((grad, False)).call().results()
    assert got["lse"][1] == -np.inf and np.isnan(got["loss"][1])
    if grad:
        assert np.isnan(got["dx"][1]).all()
    others = np.arange(T) != 1
    assert np.array_equal(got["lse"][others], ref["lse"][others]) and np.array_equal(got["loss"][others], ref["loss"][others])


@pytest.mark.parametrize("T,M,V,dtype,mesh", [(1100, 40, 300, "f32", (1, 1)), (1301, 33, 301, "f32", (2, 3)), (1100, 17, 9, "f32", (1, 8)), (2100, 40, 300, "bf16", (3, 1)), (4133, 77, 1003, "bf16", (2, 2)), (3001, 50, 130, "bf16", (3, 2)),
                                                                                            (2600, 8200, 101, "bf16", (2, 8)), (2600, 8200, 101, "f32", (1, 8))])
@pytest.mark.parametrize("vocab_dim", [0, 1])
@pytest.mark.parametrize("pad", [True, False])
def test_dw_over_ranges_of_the_tokens(T, M, V, dtype, mesh, vocab_dim, pad):
    """Long sums into few outputs, and narrow shards of the vocabulary: dw made for all shards together; with less workspace as everywhere else."""
    p = Problem(T, M, V, dtype, mesh=mesh, vocab_dim=vocab_dim, pad=pad, K=3 if T % 2 else None).stage()
    p.call().check()
    if M < 100:
        p.call(p.least + (p.bytes - p.least) // 2).check()


@pytest.mark.parametrize("T,M,V,dtype", [(2600, 8200, 101, "bf16"), (2600, 8200, 101, "f32"), (16500, 700, 202, "bf16")])
def test_losses_alone_over_narrow_shards(T, M, V, dtype):
    Problem(T, M, V, dtype, mesh=(2, 8)).stage((False, False)).call().check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("vocab_dim", [0, 1])
@pytest.mark.parametrize("T,M,V,mesh", [(1, 8, 8, (1, 1)), (7, 9, 1280, (1, 1)), (16, 24, 1281, (1, 1)), (16, 65, 301, (1, 3)), (17, 66, 77, (2, 8)), (15, 67, 90, (3, 4)), (129, 130, 200, (2, 2)), (4096, 11, 40, (2, 2)),
                                        (4097, 11, 40, (2, 2)), (3, 500, 60, (1, 6)), (33, 700, 33, (16, 2)), (12, 40, 81, (1, 9)), (260, 31, 512, (3, 16))])
def test_a_small_vocabulary_matrix(T, M, V, mesh, vocab_dim, dtype):
    """All in one launch, at the edges of its tiles, its rows and its shards."""
    for K, pad in ((None, True), (5, False), (128, True)):
        if K is None or K < V:
            Problem(T, M, V, dtype, K=K, mesh=mesh, vocab_dim=vocab_dim, pad=pad).stage().call().check()
    for grad in ((False, False), (True, False), (False, True)):
        Problem(T, M, V, dtype, mesh=mesh, vocab_dim=vocab_dim).stage(grad).call().check()


@pytest.mark.parametrize("vocab_dim", [0, 1])
@pytest.mark.parametrize("T,M,V", [(1, 8, 8), (2, 65, 7), (33, 64, 90), (65, 130, 257), (300, 72, 301)])
@pytest.mark.parametrize("dtype,K,pad", [("bf16", None, True), ("bf16", 5, False), ("f32", None, False), ("f32", 100, True)])
def test_small_sizes_by_products(T, M, V, vocab_dim, dtype, K, pad):
    """The same without the one launch: a pinned product kernel stands for any."""
    for mesh in ((1, 1), (2, 3)):
        p = Problem(T, M, V, dtype, K=K, vocab_dim=vocab_dim, mesh=mesh, pad=pad).stage()
        with pinned(MFMA):
            p.call().check()


@pytest.mark.parametrize("where", MESHES, ids=lambda m: "x".join(map(str, m["mesh"])) + ("" if m.get("share", True) else "_own"))
def test_meshes_by_products(where):
    for dtype, K, vocab_dim, pad in (("bf16", None, 0, True), ("bf16", 7, 1, False), ("f32", None, 1, True)):
        p = Problem(41, 24, 203, dtype, K=K, vocab_dim=vocab_dim, pad=pad, **where).stage()
        with pinned(MFMA):
            p.call().check()


@pytest.mark.parametrize("T,M,V,kw,grad", [(130, 64, 2000, dict(mesh=(2, 2)), True), (300, 72, 2003, dict(pad=False, vocab_dim=1), True), (3, 64, 2000, {}, True), (5, 300, 1000, dict(dtype="f32", vocab_dim=1, mesh=(1, 3)), True),
                                           (2100, 300, 400, dict(mesh=(2, 3), K=4), True), (9, 40, 300, dict(K=9), True), (40, 40, 300, dict(dtype="f32"), True), (700, 512, 30001, dict(mesh=(2, 1)), False),
                                           (1000, 1030, 5000, dict(pad=False, K=3), False)])
def test_graphs_of_every_path(T, M, V, kw, grad):
    """Recorded and replayed on other inputs, with eager calls between: the same bits as eager ones."""
    p = Problem(T, M, V, **kw).stage((grad, grad))
    outputs = [b[1] for b in (p.dxs or []) + (p.dws or [])] + [t[1][name] for t in p.ts for name in ("loss", "lse")]
    p.call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.call(stream=torch.cuda.current_stream().cuda_stream)
    for turn in range(3):
        p.xs[0][1][:3].mul_(-1.0)
        for o in outputs:
            o.fill_(float(turn))
        graph.replay()
        torch.cuda.synchronize()
        replayed = [o.clone() for o in outputs]
        p.space.fill_(255)                              # what the workspace holds is of no consequence
        for o in outputs:
            o.fill_(float(turn))
        p.call()
        torch.cuda.synchronize()
        for a, b in zip(replayed, outputs):
            assert torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))
