"""gspmd_ragged_dot on the GPU: every form, type, kernel and alignment against the product in float64, with gaps and other partitions' places poisoned."""
import pytest
import torch

import paper_2105_04663_amd as g
from tests.pin import MFMA, MID, PAIR, SPLIT, last, pinned
from tests.ragged import BACK, FORWARD, WEIGHT, Ragged

pytestmark = pytest.mark.gpu
WAYS = [FORWARD, BACK, WEIGHT]
SIZES = {"one token": [0, 0, 1, 0], "one expert": [37], "all to one": [0, 300, 0], "ends": [5, 0, 0, 9], "uneven": [1, 130, 0, 17, 256, 64, 3, 129], "single rows": [1] * 9}


@pytest.mark.parametrize("sizes", sorted(SIZES))
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_small(way, sizes, dtype):
    r = Ragged(way, SIZES[sizes], M=72, H=136, dtype=dtype).stage()
    r.call()
    r.check()


@pytest.mark.parametrize("kernel", [dict(kernel=MFMA), dict(kernel=MID), dict(kernel=PAIR), dict(kernel=SPLIT, row_blocks=1, col_blocks=4), dict(kernel=SPLIT, row_blocks=2, col_blocks=4),
                                    dict(kernel=SPLIT, row_blocks=4, col_blocks=4), dict(kernel=SPLIT, row_blocks=1, col_blocks=2), dict(kernel=SPLIT, row_blocks=2, col_blocks=2)],
                         ids=lambda k: "-".join(map(str, k.values())))
@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("out", ["same", "f32"])
def test_every_kernel(way, kernel, out):
    """K of whole steps and not, tiles that an expert's rows end inside, experts without rows."""
    for M, H, sizes in ((320, 264, [0, 257, 1, 0, 511, 33, 64]), (136, 712, [128, 0, 31, 300]), (96, 128, [700, 3])):
        r = Ragged(way, sizes, M=M, H=H, out=out, seed=1).stage()
        with pinned(**kernel):
            r.call()
            assert last()[0] == kernel["kernel"]
        r.check()


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("M, H, shift", [(65, 67, 0), (127, 130, 0), (130, 258, 2), (257, 131, 1), (3, 5, 0), (8, 1, 0), (1, 9, 3), (201, 301, 0), (140, 6, 0), (6, 140, 0)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_dense_rows_at_any_alignment(way, M, H, shift, dtype):
    r = Ragged(way, [70, 1, 0, 133, 18], M=M, H=H, dtype=dtype, pad=False, shift=shift, seed=2).stage()
    r.call()
    r.check()


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("E", [63, 64, 65, 130, 200])
def test_many_experts(way, E):
    """More experts than a wave has lanes; those that hold anything lie in any sixty-four."""
    for kind in range(3):
        sizes = [(e * 7 + 3) % 11 if kind == 0 else 40 * (e == E - 1) if kind == 1 else 5 * (e % 64 == 0) for e in range(E)]
        r = Ragged(way, sizes, M=40, H=72, seed=kind, y=3 if kind == 0 else 1).stage()
        r.call()
        r.check()


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("y, x, share", [(2, 1, True), (3, 1, False), (4, 2, False), (8, 1, True), (2, 3, False)])
def test_experts_over_a_mesh(way, y, x, share):
    """An uneven split (a partition may have none), buffers of a partition's own in which other experts' places hold NaN, replicas that are each written."""
    r = Ragged(way, [12, 0, 150, 7, 40], M=80, H=200, y=y, x=x, share=share, seed=3).stage()
    r.call()
    r.check()


@pytest.mark.parametrize("way", WAYS)
def test_more_parts_than_a_launch_takes(way):
    r = Ragged(way, [(5 * e) % 13 for e in range(80)], M=32, H=48, y=40, x=2, share=False, seed=4).stage()
    r.call()
    r.check()


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("sizes, slots", [([3, -5, 4], 12), ([10, 10, 10], 15), ([2 ** 31 - 1, 5], 20), ([-2 ** 31, 6, 2 ** 31 - 1, 3], 9), ([2 ** 31 - 1] * 130, 33)])
def test_sizes_that_do_not_fit(way, sizes, slots):
    """Negative ones count as 0, and slots end where the array does."""
    r = Ragged(way, sizes, M=48, H=64, slots=slots, seed=5).stage()
    r.call()
    r.check()


@pytest.mark.parametrize("way", WAYS)
def test_nothing_to_do(way):
    for kw in (dict(sizes=[0, 0], slots=7), dict(sizes=[0], slots=0), dict(sizes=[0, 0, 0], slots=0)):
        r = Ragged(way, kw["sizes"], M=16, H=24, slots=kw["slots"]).stage()
        r.call()
        r.check()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_of_no_columns_are_zeros(dtype):
    r = Ragged(FORWARD, [4, 0, 6], M=0, H=40, dtype=dtype).stage()
    r.call()
    r.check()


@pytest.mark.parametrize("way", WAYS)
def test_relu(way):
    r = Ragged(way, [50, 0, 9], M=64, H=96, relu=way != WEIGHT, seed=6).stage()
    r.call()
    r.check()


@pytest.mark.parametrize("way", WAYS)
@pytest.mark.parametrize("M, H, sizes", [(512, 1024, [700, 300, 1500, 20]), (2048, 1408, [900, 2, 60, 1100]), (1000, 2056, [40] * 16)])
def test_ordinary_sizes(way, M, H, sizes):
    for pad in (True, False):
        r = Ragged(way, sizes, M=M, H=H, pad=pad, seed=7).stage()
        r.call()
        r.check()


def test_infinities_and_nan_stay_in_their_rows():
    r = Ragged(FORWARD, [3, 4], M=64, H=64)
    r.lhs[1, 5] = float("inf")
    r.lhs[5, 7] = float("nan")
    r.stage().call()
    out = r.outs[0][1][:, :64].cpu().float()
    assert torch.isfinite(out[[0, 2, 3, 4, 6]]).all() and not torch.isfinite(out[1]).any() and torch.isnan(out[5]).all()
    want, mag, _ = r.expected(0)
    rows = [0, 2, 3, 4, 6]
    assert ((out[rows].double() - want[rows]).abs() <= 66 * 2.0 ** -23 * mag[rows] + 2.0 ** -8 * want[rows].abs()).all()


@pytest.mark.parametrize("way", WAYS)
def test_a_graph_reads_the_sizes_anew(way):
    """Replays with other sizes and rows, eager work between them: bits of the eager call."""
    r = Ragged(way, [100, 3, 0, 61], M=136, H=200, slots=200, seed=8).stage()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        r.call()
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        r.call()
    for sizes in ([100, 3, 0, 61], [0, 0, 200, 0], [1, 150, 20, 29], [64, 64, 64, 8], [0, 0, 0, 0]):
        r.sizes_t.copy_(torch.tensor(sizes, dtype=torch.int32))
        r.keep[0].copy_(torch.randint(-4, 5, r.keep[0].shape, device="cuda").to(r.dtype))
        r.keep[1].copy_(torch.randint(-4, 5, r.keep[1].shape, device="cuda").to(r.dtype))
        out = r.outs[0][1]
        out.fill_(5.0)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        out.fill_(5.0)
        r.call()
        torch.cuda.synchronize()
        assert torch.equal(got, out)


def test_two_streams_at_once():
    """Calls of two streams share nothing."""
    a, b = Ragged(FORWARD, [300, 20, 500], M=256, H=512, seed=9).stage(), Ragged(WEIGHT, [40, 900], M=384, H=256, seed=10).stage()
    torch.cuda.synchronize()
    streams = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        for r, s in zip((a, b), streams):
            r.call(s.cuda_stream)
    torch.cuda.synchronize()
    a.check()
    b.check()


def test_the_gradients_against_differences():
    """loss = sum of c * out: its differences along random directions of rows and matrices, small whole numbers in float32 so that every sum is exact."""
    sizes, M, H = [5, 0, 12, 3], 24, 40
    f = Ragged(FORWARD, sizes, M, H, dtype="f32", whole_numbers=True, seed=11)
    c = torch.randint(-3, 4, (f.S, H)).float()
    def forward(lhs, rhs):
        f.lhs, f.rhs = lhs, rhs
        f.stage().call()
        return f.outs[0][1][:, :H].cpu().double()
    lhs, rhs = f.lhs.clone(), f.rhs.clone()
    d_lhs, d_rhs = torch.randint(-2, 3, lhs.shape).float(), torch.randint(-2, 3, rhs.shape).float()
    back = Ragged(BACK, sizes, H, M, dtype="f32")
    back.lhs, back.rhs = c, rhs
    back.stage().call()
    weight = Ragged(WEIGHT, sizes, M, H, dtype="f32")
    weight.lhs, weight.rhs = lhs, c
    weight.stage().call()
    d_rows, d_w = back.outs[0][1][:, :M].cpu().double(), weight.outs[0][1][..., :H].cpu().double()
    for along, got in ((lambda s: forward(lhs + s * d_lhs, rhs), (d_rows * d_lhs).sum()), (lambda s: forward(lhs, rhs + s * d_rhs), (d_w * d_rhs).sum())):
        assert (((along(1) - along(-1)) / 2) * c).sum() == got


FEW = [[1], [0, 3, 0, 1, 0, 0, 16, 0], [17, 2, 0, 5, 1, 33, 0, 4], [1] * 70, [0] * 63 + [5, 20, 1]]


@pytest.mark.parametrize("way", [FORWARD, BACK])
@pytest.mark.parametrize("sizes", range(len(FEW)))
@pytest.mark.parametrize("M", [1, 3, 15, 16, 17, 64, 79, 128, 300, 1031])
def test_few_float32_rows(way, sizes, M):
    """K below a step, of whole steps for some waves and not for others, and what is left of it; columns that end inside a lane's four, at a tile's end, and fewer than four."""
    for H, kw in ((1, dict()), (3, dict(pad=False, shift=1)), (63, dict(pad=False)), (64, dict(relu=True)), (66, dict(pad=False, shift=3)), (130, dict(y=2, share=False)), (257, dict(slots=sum(FEW[sizes]) + 7))):
        r = Ragged(way, FEW[sizes], M=M, H=H, dtype="f32", seed=31, **kw).stage()
        r.call()
        r.check()


@pytest.mark.parametrize("way", [FORWARD, BACK])
def test_few_float32_rows_are_exact_in_whole_numbers(way):
    r = Ragged(way, [3, 0, 20, 1, 9], M=515, H=131, dtype="f32", seed=32, whole_numbers=True, pad=False, shift=1).stage()
    for _ in range(3):
        r.call()
    r.check()
    want, _, _ = r.expected(0)
    got = r.outs[0][1][:, :131].cpu().double()
    assert torch.equal(got[:r.used], want[:r.used])
