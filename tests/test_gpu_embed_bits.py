"""What a gradient of the embedding leaves alone when it is added to one that is there: bit for bit."""
import pytest
import torch

from tests.tokens import KEPT, Embed

pytestmark = pytest.mark.gpu


def patterns(dtype, V, M):
    """Elements of every kind, signalling NaN with their payloads among them."""
    if dtype == "bf16":
        return (torch.arange(V * M, dtype=torch.int32) * 7919 % 2 ** 16 - 2 ** 15).to(torch.int16).view(V, M).view(torch.bfloat16)
    return ((torch.arange(V * M, dtype=torch.int64) * 65537 + 2 ** 23 * 255 - 7) % 2 ** 32).to(torch.uint32).view(torch.int32).view(V, M).view(torch.float32)


@pytest.mark.parametrize("order", ["vm", "mv"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [0, 3, 100, 128, 129, 500, 8193])
def test_entries_without_tokens_keep_their_bits(order, dtype, T):
    """Few tokens and many, entries with tokens among ones without, tiles with none at all, shards behind the last entry, rows that are whole 16 bytes or not."""
    for M, V, kw in ((64, 1024, dict()), (37, 331, dict(pad=False, y=3)), (5, 200, dict(pad=False, shift=1, y=64))):
        ids = torch.arange(T) * 5 % 60 * (V // 64)                        # entries below 60 / 64 V, multiples of V / 64
        e = Embed(T, M, V, order=order, dtype=dtype, ids=ids, accumulate=True, scale=0.5, **kw)
        view = torch.int16 if dtype == "bf16" else torch.int32
        e.w = patterns(dtype, V, M)
        used = torch.zeros(V, dtype=torch.bool)
        used[ids] = True
        e.w[used] = torch.arange(M).to(e.dtype)                          # ordinary numbers where something is added
        e.dy = torch.ones_like(e.dy)
        e.stage_gradient().gradient()
        got = e.dwc.whole() if order == "vm" else e.dwc.whole().t().contiguous()
        assert torch.equal(got[:V][~used].view(view), e.w[~used].view(view))
        count = torch.bincount(ids, minlength=V)[used].double()
        want = torch.arange(M).double() + 0.5 * count[:, None]           # exact in float32, then one rounding
        assert torch.equal(got[:V][used], want.to(e.dtype))
        assert (got[V:] == 0).all() and (e.dwc.gaps() == KEPT).all()
