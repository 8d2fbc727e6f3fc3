"""The losses refuse arrays of tokens that are not at their elements' alignment, before anything is launched."""
import dataclasses

import pytest

import paper_2105_04663_amd as g
from tests.pin import pinned
from tests.test_softmax_host import BUFFER, args, status

TOKEN = g.TokenBuf(ids=1 << 21, loss=1 << 22, lse=1 << 25, weights=1 << 26, logits=1 << 23)


@pytest.mark.parametrize("field,by,distill_only", [("ids", 2, False), ("ids", 1, False), ("loss", 2, False), ("lse", 1, False), ("weights", 2, False), ("weights", 3, False), ("logits", 2, True)])
def test_arrays_at_odd_addresses(field, by, distill_only):
    ok = args()
    for at in (0, 3):
        tokens = [TOKEN] * 4
        tokens[at] = dataclasses.replace(TOKEN, **{field: getattr(TOKEN, field) + by})
        assert status(lambda **kw: g.softmax_distill(targets=3, **kw), ok, tokens=tokens) == BUFFER
        if distill_only:
            with pinned(dry_run=True):
                g.softmax_xent(**{**ok, "tokens": tokens})         # ignored there
        else:
            assert status(g.softmax_xent, ok, tokens=tokens) == BUFFER


def test_bfloat16_logits_at_two_bytes():
    ok = args()
    for by, good in ((2, True), (1, False)):
        tokens = [dataclasses.replace(TOKEN, logits=TOKEN.logits + by, logits_dtype=g.BF16)] * 4
        if good:
            with pinned(dry_run=True):
                g.softmax_distill(targets=3, **{**ok, "tokens": tokens})
        else:
            assert status(lambda **kw: g.softmax_distill(targets=3, **kw), ok, tokens=tokens) == BUFFER


def test_without_tokens_any_address():
    with pinned(dry_run=True):
        g.softmax_xent(**{**args(T=0), "tokens": [g.TokenBuf(ids=1, loss=3)] * 4})
