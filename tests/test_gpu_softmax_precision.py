"""The precision that gradients are promised: up to 128 tokens what D's rounding to bfloat16 loses takes part in the products, by every path; a handful of tokens and float32 keep D in float32."""
import numpy as np
import pytest

from tests.loss_bounds import D_FLOAT, check_gradients, exact_logits
from tests.losses import Problem
from tests.pin import MFMA, pinned

pytestmark = pytest.mark.gpu


def run(*a, grad=(True, True), workspace=None, precision=None, by_products=False, **kw):
    p = exact_logits(Problem(*a, **kw)).stage(grad)
    with pinned(MFMA) if by_products else pinned():
        p.call(None if workspace is None else workspace(p))
    check_gradients(p, p.check(), precision)


@pytest.mark.parametrize("vocab_dim", [0, 1])
@pytest.mark.parametrize("T,M,V,K", [(65, 130, 257, None), (33, 64, 90, None), (2, 65, 7, None), (16, 520, 1300, None), (41, 24, 203, 7), (128, 64, 2000, None), (129, 64, 2000, None), (100, 72, 33000, 5),
                                     (16, 24, 300, 9), (128, 300, 40, None), (1000, 40, 300, None), (300, 136, 3000, 3)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_each_size(T, M, V, K, vocab_dim, dtype):
    kw = dict(K=K, vocab_dim=vocab_dim, tau=1.0 if K is None else 2.0, pad=T % 2 == 0)
    run(T, M, V, dtype, **kw)
    run(T, M, V, dtype, by_products=True, **kw)                   # also where one launch would do
    for grad in ((True, False), (False, True)):
        run(T, M, V, dtype, grad=grad, **kw)


@pytest.mark.parametrize("mesh", [(1, 4), (3, 1), (2, 3), (66, 1), (100, 2)])
@pytest.mark.parametrize("T,M,V,vocab_dim", [(100, 24, 203, 0), (100, 130, 2003, 1), (70, 40, 5000, 0)])
def test_meshes_and_pieces(T, M, V, vocab_dim, mesh):
    for dtype in ("bf16", "f32"):
        run(T, M, V, dtype, mesh=mesh, vocab_dim=vocab_dim, pad=M == 24)
        run(T, M, V, dtype, mesh=mesh, vocab_dim=vocab_dim, workspace=lambda p: p.least + (p.bytes - p.least) // 2)


# kernels_few.h: w beyond 128 KiB
@pytest.mark.parametrize("dtype,vocab_dim,T", [("bf16", 0, 1), ("bf16", 0, 2), ("bf16", 0, 4), ("f32", 0, 1), ("f32", 0, 8), ("f32", 1, 3), ("f32", 1, 8)])
@pytest.mark.parametrize("M,V", [(16, 8193), (16, 65537), (515, 1003), (136, 2000)])
def test_a_handful_of_tokens(dtype, vocab_dim, T, M, V):
    run(T, M, V, dtype, vocab_dim=vocab_dim, precision=D_FLOAT, missing=0.0)
    run(T, M, V, dtype, vocab_dim=vocab_dim, precision=D_FLOAT, pad=False, mesh=(2, 3), K=4)


@pytest.mark.parametrize("T,dtype,vocab_dim", [(3, "bf16", 0), (3, "bf16", 1), (3, "f32", 0), (3, "f32", 1), (60, "bf16", 0), (60, "bf16", 1), (200, "f32", 0)])
@pytest.mark.parametrize("V", [8193, 65537])
def test_labels_in_the_last_columns(T, dtype, vocab_dim, V):
    p = exact_logits(Problem(T, 16, V, dtype, vocab_dim=vocab_dim, missing=0.0))
    p.ids[:, 0] = V - 1 - np.arange(T) % 3
    p.stage().call()
    check_gradients(p, p.check())
