"""Test-side driver of gspmd_ragged_dot: packed rows and matrices cut into shard buffers, gaps and other experts' places poisoned, the plain product in float64 and the bound."""
from __future__ import annotations

import numpy as np
import torch

import paper_2105_04663_amd as g

FORWARD, BACK, WEIGHT = "rows", "rows by transposed matrices", "matrices"
DIMS = {FORWARD: g.DotDims((0,), (0,), (2,), (1,)), BACK: g.DotDims((0,), (0,), (2,), (2,)), WEIGHT: g.DotDims((0,), (0,), (1,), (1,))}
KEPT = 77.0            # what out holds before: places that the call leaves alone keep it


def spread(sizes, slots):
    """(first slot, number) of every expert by the documented rule: negative sizes are 0, slots end at `slots`."""
    out, at = [], 0
    for n in sizes:
        n = min(max(int(n), 0), slots - at)
        out.append((at, n))
        at += n
    return out


class Ragged:
    """way: of DIMS.  The rows have M columns (BACK: the matrices are [H-side, M]), the other extent is H.  `pad`: row strides are multiples of 8; `y`: the experts' mesh dimension,
    `x` replicas; `share`: one buffer for all partitions of the packed arrays."""

    def __init__(self, way, sizes, M, H, slots=None, dtype="bf16", out="same", y=1, x=1, share=True, pad=True, relu=False, seed=0, whole_numbers=False, shift=0):
        self.way, self.sizes, self.E, self.M, self.H = way, list(sizes), len(sizes), M, H
        self.S = sum(max(n, 0) for n in sizes) if slots is None else slots
        self.dtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.out_dtype = self.dtype if out == "same" else torch.float32
        self.relu, self.pad, self.share, self.shift = relu, pad, share, shift
        self.x, self.y, self.es = x, y, -(-self.E // y)
        self.mesh = g.Mesh((x, y), tuple(range(x * y)))
        rng = torch.Generator().manual_seed(100 * seed + M + 3 * H + self.S)
        def draw(*shape):
            t = torch.randint(-3, 4, shape, generator=rng).float() if whole_numbers else torch.randn(shape, generator=rng)
            return t.to(self.dtype)
        self.lhs = draw(self.S, M)
        self.rhs = draw(self.S, H) if way == WEIGHT else draw(self.E, H, M) if way == BACK else draw(self.E, M, H)
        self.lhs_sh = g.Sharding((self.E, self.S, M), (1, -1, -1))
        self.rhs_sh = g.Sharding(((self.E, self.S, H) if way == WEIGHT else tuple(self.rhs.shape)), (1, -1, -1))
        self.out_sh = g.Sharding((self.E, M, H) if way == WEIGHT else (self.E, self.S, H), (1, -1, -1))
        self.ranges = spread(self.sizes, self.S)
        self.used = sum(n for _, n in self.ranges)

    def ld(self, cols):
        return -(-cols // 8) * 8 if self.pad else cols

    def place(self, t, fill):
        """`t` [.., rows, cols] on the GPU with the row stride, gaps poisoned, `shift` elements into its allocation."""
        cols = t.shape[-1]
        ld = self.ld(cols)
        flat = torch.full((t.numel() // max(cols, 1) * ld + self.shift + 8,), fill, dtype=t.dtype)
        body = flat[self.shift:self.shift + t.numel() // max(cols, 1) * ld].view(t.shape[:-1] + (ld,))
        body[..., :cols] = t
        flat = flat.cuda()
        return flat, flat[self.shift:self.shift + body.numel()].view(body.shape)

    def packed(self, t, j):
        """The rows as partition coordinate j may see them: its experts' slots; all else NaN."""
        seen = torch.full_like(t, float("nan"))
        for e in range(j * self.es, min((j + 1) * self.es, self.E)):
            a, n = self.ranges[e]
            seen[a:a + n] = t[a:a + n]
        return seen

    def matrices(self, t, j):
        shard = torch.full((self.es,) + tuple(t.shape[1:]), float("nan"), dtype=t.dtype)
        part = t[j * self.es:(j + 1) * self.es]
        shard[:part.shape[0]] = part
        return shard

    def stage(self):
        self.keep, self.bufs = [], {"lhs": [], "rhs": [], "out": []}
        self.outs = []                               # (coordinate j, tensor), distinct ones
        seen = {}
        def held(key, make, fill=float("nan")):
            if key not in seen:
                flat, body = self.place(make(), fill)
                seen[key] = (g.ShardBuf.of(body, body.shape[-1]), body)
                self.keep.append(flat)
            return seen[key]
        everywhere = torch.full((self.S, self.M), float("nan"), dtype=self.dtype)
        everywhere[:self.used] = self.lhs[:self.used]
        for p in range(self.x * self.y):
            i, j = divmod(p, self.y)
            self.bufs["lhs"].append(held(("lhs", 0) if self.share else ("lhs", j), (lambda: everywhere) if self.share else (lambda: self.packed(self.lhs, j)))[0])
            if self.way == WEIGHT:
                self.bufs["rhs"].append(held(("rhs", j), lambda: self.packed(self.rhs, j))[0])
                o = held(("out", i, j), lambda: torch.full((self.es, self.M, self.H), KEPT, dtype=self.out_dtype), KEPT)
            else:
                self.bufs["rhs"].append(held(("rhs", j), lambda: self.matrices(self.rhs, j))[0])
                o = held(("out", 0) if self.share else ("out", i, j), lambda: torch.full((self.S, self.H), KEPT, dtype=self.out_dtype), KEPT)
            self.bufs["out"].append(o[0])
            self.outs.append((j, o[1]))
        self.sizes_t = torch.tensor(self.sizes, dtype=torch.int32).cuda()
        return self

    def call(self, stream=None):
        g.ragged_dot(self.mesh, DIMS[self.way], self.bufs["lhs"], self.lhs_sh, self.bufs["rhs"], self.rhs_sh, self.bufs["out"], self.out_sh, self.sizes_t.data_ptr(),
                     stream=torch.cuda.current_stream().cuda_stream if stream is None else stream, epilogue=g.EPILOGUE_RELU if self.relu else g.EPILOGUE_NONE)

    def expected(self, j):
        """(values, sum of absolute products, terms) of partition coordinate j's out; NaN where the call leaves what was there."""
        lhs, rhs = self.lhs.double(), self.rhs.double()
        if self.way == WEIGHT:
            v, a = torch.zeros(self.es, self.M, self.H, dtype=torch.float64), torch.zeros(self.es, self.M, self.H, dtype=torch.float64)
            for i, e in enumerate(range(j * self.es, min((j + 1) * self.es, self.E))):
                s, n = self.ranges[e]
                v[i], a[i] = lhs[s:s + n].T @ rhs[s:s + n], lhs[s:s + n].abs().T @ rhs[s:s + n].abs()
            return v, a, max([n for _, n in self.ranges], default=0)
        v = torch.full((self.S, self.H), float("nan"), dtype=torch.float64)
        a = torch.zeros(self.S, self.H, dtype=torch.float64)
        for e in range(self.E) if self.share else range(j * self.es, min((j + 1) * self.es, self.E)):
            s, n = self.ranges[e]
            w = rhs[e].T if self.way == BACK else rhs[e]
            v[s:s + n], a[s:s + n] = lhs[s:s + n] @ w, lhs[s:s + n].abs() @ w.abs()
        return v.clamp(min=0) if self.relu else v, a, self.M

    def check(self):
        """Each output within its own rounding (half a step: 2^-8 of a bfloat16, 2^-24 of a float32) and that of a sum of `terms` products in fp32: each of at most terms additions
        is off by 2^-24 of a partial sum, which the sum of absolute products bounds (products of bfloat16 are exact in fp32, those of float32 rounded once more); 2^-126 for results below normal."""
        for j, out in self.outs:
            got = out[..., :self.H].cpu().double()
            want, mag, terms = self.expected(j)
            left = torch.isnan(want)
            assert torch.equal(got[left], torch.full_like(got[left], KEPT)), "a place that is not this call's was written"
            half = 2.0 ** -8 if self.out_dtype == torch.bfloat16 else 2.0 ** -24
            most = (1 + 2.0 ** -8) * (terms + 2) * 2.0 ** -24 * mag + half * want.abs() + 2.0 ** -126
            bad = ~((got - want).abs() <= most) & ~left
            assert not bad.any(), (self.way, int(bad.sum()), got[bad][:4], want[bad][:4])
            if self.way != WEIGHT:                                        # row gaps of a packed out are not this call's either
                gap = out[..., self.H:].cpu().double()
                assert torch.equal(gap, torch.full_like(gap, KEPT))
