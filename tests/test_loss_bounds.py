"""The bounds of the losses' gradients see what they are there for: results made from D in two bfloat16 parts pass, without the second part, with its sign turned, with it times another
token's activations, or without the last columns of a sum they do not.  Float64 on the CPU; the mistakes are in what is held against the bounds."""
import numpy as np
import pytest
import torch

from tests.loss_bounds import check_gradients, exact_logits
from tests.losses import Problem

SIZES = [(65, 130, 257, None), (33, 64, 90, None), (2, 65, 7, None), (16, 520, 1300, None), (41, 24, 203, 7), (128, 64, 2000, None), (16, 520, 1300, 30)]


def bf16(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16).double().numpy()


def made(p, second=1.0, x_second=None, dx_columns=None):
    d = p.expected()[2]
    high = bf16(d)
    low = second * bf16(d - high)
    n = p.V if dx_columns is None else dx_columns
    return {"dx": bf16((high + low)[:, :n] @ p.w[:n]), "dw": bf16(high.T @ p.x + low.T @ (p.x if x_second is None else x_second))}


@pytest.mark.parametrize("T,M,V,K", SIZES)
@pytest.mark.parametrize("vocab_dim", [0, 1])
def test_two_parts(T, M, V, K, vocab_dim):
    p = exact_logits(Problem(T, M, V, K=K, vocab_dim=vocab_dim, tau=1.0 if K is None else 2.0))
    good = made(p)
    check_gradients(p, good)
    for mistake in (made(p, second=0.0), made(p, second=-1.0)):
        for name in ("dx", "dw"):
            with pytest.raises(AssertionError):
                check_gradients(p, {name: mistake[name]})
    with pytest.raises(AssertionError):
        check_gradients(p, {"dw": made(p, x_second=np.roll(p.x, 1, axis=0))["dw"]})


@pytest.mark.parametrize("V", [8193, 65537])
def test_last_columns_of_a_long_sum(V):
    p = exact_logits(Problem(3, 16, V, missing=0.0))
    p.ids[:, 0] = V - 1 - np.arange(3)                    # labels among them
    check_gradients(p, made(p))
    with pytest.raises(AssertionError):
        check_gradients(p, {"dx": made(p, dx_columns=V - 3)["dx"]})
