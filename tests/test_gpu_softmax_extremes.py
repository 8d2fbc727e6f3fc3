"""Teacher's logits at the ends of their type, at a temperature below 1: what counts is how far they lie apart, not what one of them divided by the temperature would be."""
import numpy as np
import pytest
import torch

from tests.losses import Problem
from tests.pin import MFMA, pinned

pytestmark = pytest.mark.gpu


# in one launch, a handful of tokens, by products, and with logits that are not kept
@pytest.mark.parametrize("T,M,V,dtype,grad,kernel", [(6, 16, 77, "bf16", True, None), (200, 16, 77, "f32", True, None), (3, 64, 2000, "bf16", True, None), (7, 64, 2000, "f32", True, None),
                                                     (60, 64, 2000, "bf16", True, None), (200, 64, 2000, "bf16", True, None), (40, 64, 3000, "bf16", False, MFMA)])
@pytest.mark.parametrize("K", [1, 4, 70])
@pytest.mark.parametrize("logits_dtype", ["f32", "bf16"])
def test_equal_entries_at_the_ends_of_the_type(T, M, V, dtype, grad, kernel, K, logits_dtype):
    most = torch.finfo(torch.float32 if logits_dtype == "f32" else torch.bfloat16).max
    ref = None
    for value in (0.0, -most, most, -1.0):
        p = Problem(T, M, V, dtype, K=K, tau=0.5, logits_dtype=logits_dtype)
        p.logits_t[:] = value
        p.logits[:] = 0.0                                        # (equal ones are as good as any)
        if kernel is None:
            p.stage((grad, grad)).call()
        else:
            with pinned(kernel):
                p.stage((grad, grad)).call()
        got = p.check()
        ref = ref or got
        for name in ref:
            assert np.array_equal(got[name], ref[name]), (value, name)


def test_one_entry_far_above_the_others():
    p = Problem(9, 32, 500, K=3, tau=0.5, missing=0.0)
    for a in (p.logits, p.logits_t):
        a[:, 0] = 0.0
        a[:, 1:] = -torch.finfo(torch.float32).max
    got = p.stage().call().results()
    q = Problem(9, 32, 500, K=3, tau=0.5, missing=0.0)
    for a in (q.logits, q.logits_t):
        a[:, 0] = 0.0
        a[:, 1:] = -np.inf
    want = q.stage().call().check()
    for name in want:
        assert np.array_equal(got[name], want[name]), name
