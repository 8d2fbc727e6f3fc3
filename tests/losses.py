"""Test-side driver of the losses over a split vocabulary: global operands cut into shard buffers (padding and gaps NaN), the
library's call, results put together again, and the bounds that they are held to.  Expected values come from oracle/softmax.py."""
from __future__ import annotations

import numpy as np
import torch

import paper_2105_04663_amd as g
from oracle import bounds as ob
from oracle import softmax as osm

ROUND = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}       # of one rounding to the operands' type
FLOAT = 2.0 ** -24


def as_type(a, dtype):
    """The nearest values that the operands' type has, as float64, and the tensor of them."""
    t = torch.from_numpy(np.asarray(a, dtype=np.float32))
    t = t.to(torch.bfloat16) if dtype == "bf16" else t
    return t.double().numpy(), t


class Problem:
    def __init__(self, T, M, V, dtype="bf16", K=None, tau=1.0, seed=0, wscale=0.1, missing=0.15, vocab_dim=0, mesh=(1, 1), x_map=(0, -1), v_axis=1, ids_order=None,
                 pad=True, share=True, logits_dtype="f32", weights=True):
        rng = np.random.default_rng(1000 * seed + 7 * T + 11 * M + 13 * V)
        self.T, self.M, self.V, self.dtype, self.K, self.tau, self.vocab_dim = T, M, V, dtype, K, tau, vocab_dim
        self.x, self.xt = as_type(rng.standard_normal((T, M)), dtype)
        self.w, self.wt = as_type(rng.standard_normal((V, M)) * wscale, dtype)
        k = K or 1
        self.ids = rng.integers(0, V, size=(T, k)).astype(np.int32)
        self.ids[rng.random((T, k)) < missing] = -1
        self.logits = None
        if K is not None:
            self.logits, self.logits_t = as_type(rng.standard_normal((T, k)) * 2.0, logits_dtype)
        self.logits_dtype = logits_dtype
        self.weights = (rng.random(T).astype(np.float32) + np.float32(0.25)) / np.float32(max(T, 1)) if weights else None
        self.mesh = g.Mesh(tuple(mesh), tuple(ids_order) if ids_order is not None else tuple(range(int(np.prod(mesh)))))
        self.x_sh = g.Sharding((T, M), tuple(x_map))
        self.w_sh = g.Sharding((V, M), (v_axis, -1)) if vocab_dim == 0 else g.Sharding((M, V), (-1, v_axis))
        self.pad, self.share = pad, share

    # ---- shards
    def _cut(self, sharding, full, kept, fill=float("nan")):
        """Shard buffers of a tensor (one per distinct offset, or one per partition), as (ShardBuf, tensor, offset, valid, shard)."""
        out = []
        for p in range(self.mesh.n_partitions):
            off, valid, shard = ob.shard_bounds(self.mesh.shape, self.mesh.device_ids, sharding.global_shape, sharding.dims_mapping, p)
            if self.share and off in kept:
                out.append(kept[off])
                continue
            ld = -(-max(shard[1], 1) // 8) * 8 if self.pad else max(shard[1], 1)
            t = torch.full((max(shard[0], 1), ld), fill, dtype=torch.bfloat16 if self.dtype == "bf16" else torch.float32)
            if full is not None and min(valid) > 0:
                t[:valid[0], :valid[1]] = full[off[0]:off[0] + valid[0], off[1]:off[1] + valid[1]]
            t = t.cuda()
            kept[off] = (g.ShardBuf.of(t, ld), t, off, valid, shard)
            out.append(kept[off])
        return out

    def _tokens(self):
        kept, out = {}, []
        k = self.K or 1
        for p in range(self.mesh.n_partitions):
            off, valid, shard = ob.shard_bounds(self.mesh.shape, self.mesh.device_ids, self.x_sh.global_shape, self.x_sh.dims_mapping, p)
            if not (self.share and off[0] in kept):
                n = max(shard[0], 1)
                held = {"ids": torch.full((n, k), 12345678, dtype=torch.int32), "loss": torch.full((n,), float("nan")), "lse": torch.full((n,), float("nan")),
                        "weights": torch.full((n,), float("nan"))}
                held["ids"][:valid[0]] = torch.from_numpy(self.ids[off[0]:off[0] + valid[0]])
                if self.weights is not None:
                    held["weights"][:valid[0]] = torch.from_numpy(self.weights[off[0]:off[0] + valid[0]])
                if self.logits is not None:
                    held["logits"] = torch.full((n, k), float("nan"), dtype=self.logits_t.dtype)
                    held["logits"][:valid[0]] = self.logits_t[off[0]:off[0] + valid[0]]
                kept[off[0]] = {n: t.cuda() for n, t in held.items()}, off[0], valid[0], shard[0]
            held = kept[off[0]][0]
            out.append((g.TokenBuf(held["ids"].data_ptr(), held["loss"].data_ptr(), held["lse"].data_ptr(), held["weights"].data_ptr() if self.weights is not None else 0,
                                   held["logits"].data_ptr() if self.logits is not None else 0, g.BF16 if self.logits_dtype == "bf16" else g.F32),) + kept[off[0]])
        return out

    def stage(self, grad=(True, True)):
        w_full = self.wt if self.vocab_dim == 0 else self.wt.t()
        self.xs, self.ws, self.ts = self._cut(self.x_sh, self.xt, {}), self._cut(self.w_sh, w_full, {}), self._tokens()
        self.dxs = self._cut(self.x_sh, None, {}) if grad[0] else None
        self.dws = self._cut(self.w_sh, None, {}) if grad[1] else None
        self.bytes = g.softmax_workspace_bytes(self.mesh, self.x_sh, self.w_sh, self.vocab_dim, g.BF16 if self.dtype == "bf16" else g.F32, any(grad))
        self.least = g.softmax_workspace_bytes(self.mesh, self.x_sh, self.w_sh, self.vocab_dim, g.BF16 if self.dtype == "bf16" else g.F32, any(grad), least=True)
        return self

    def call(self, workspace=None, stream=None):
        n = self.bytes if workspace is None else workspace
        # NaN beyond what the call is told of and in it, so that what is not written shows
        if getattr(self, "space", None) is None or self.space.numel() < n + 512:
            self.space = torch.full((n + 512,), 255, dtype=torch.uint8, device="cuda")
        base = (self.space.data_ptr() + 255) // 256 * 256
        bufs = lambda s: None if s is None else [b[0] for b in s]
        args = (self.mesh, bufs(self.xs), self.x_sh, bufs(self.ws), self.w_sh, [t[0] for t in self.ts])
        kw = dict(vocab_dim=self.vocab_dim, dx_shards=bufs(self.dxs), dw_shards=bufs(self.dws), workspace=base, workspace_bytes=n,
                  stream=torch.cuda.current_stream().cuda_stream if stream is None else stream)
        if self.K is None:
            g.softmax_xent(*args, **kw)
        else:
            g.softmax_distill(*args, self.K, self.tau, **kw)
        return self

    def _join(self, shards, shape):
        full = np.full(shape, np.nan)
        for buf, t, off, valid, shard in shards:
            v = t[:shard[0], :shard[1]].double().cpu().numpy()
            assert not v[valid[0]:].any() and not v[:, valid[1]:].any(), "padding is written as zeros"
            gap = t[:shard[0], shard[1]:]
            assert gap.numel() == 0 or bool(torch.isnan(gap).all()), "the gap between rows is not written"
            here = full[off[0]:off[0] + valid[0], off[1]:off[1] + valid[1]]
            assert np.isnan(here).all() or np.array_equal(here, v[:valid[0], :valid[1]], equal_nan=True), "partitions of the same data agree"
            full[off[0]:off[0] + valid[0], off[1]:off[1] + valid[1]] = v[:valid[0], :valid[1]]
        return full

    def results(self):
        torch.cuda.synchronize()
        out = {"loss": np.full(self.T, np.nan), "lse": np.full(self.T, np.nan)}
        for _, held, off, valid, shard in self.ts:
            for name in ("loss", "lse"):
                v = held[name][:shard].double().cpu().numpy()
                assert not v[valid:].any(), "padding is written as zeros"
                out[name][off:off + valid] = v[:valid]
        if self.dxs is not None:
            out["dx"] = self._join(self.dxs, (self.T, self.M))
        if self.dws is not None:
            dw = self._join(self.dws, (self.V, self.M) if self.vocab_dim == 0 else (self.M, self.V))
            out["dw"] = dw if self.vocab_dim == 0 else dw.T
        return out

    def expected(self):
        weights = np.ones(self.T) if self.weights is None else self.weights.astype(np.float64)
        return osm.loss_and_gradients(self.x, self.w, self.ids, weights, self.logits, self.tau)

    def check(self):
        """Every result element by element against the oracle, within what the roundings that the path makes can amount to.
        z: an fp32 sum of M exact (bf16) or rounded (f32) products, at most (M + 2) 2^-24 of sum |x||w| off; u, exp, log: a few roundings of values up to |u|; the sum of V
        terms adds (V + 8) 2^-24 to log at most in theory, its tree here no more than 2^-18 of it.  D: those errors times its terms, and one rounding to the operands' type."""
        got = self.results()
        loss, lse, d, dx, dw = self.expected()
        if self.T == 0:
            assert got.get("dw") is None or not got["dw"].any()
            return got
        u = (self.x @ self.w.T) / self.tau
        size = (np.abs(self.x) @ np.abs(self.w).T).max(axis=1) / self.tau
        du = (self.M + 2) * FLOAT * size + 8 * FLOAT * (np.abs(u).max(axis=1) + 1)            # of any u of a token
        dl = 2 * du + 2.0 ** -18 + 4 * FLOAT * np.abs(lse)                                       # of its lse
        assert (np.abs(got["lse"] - lse) <= dl).all(), np.abs(got["lse"] - lse).max()
        q = 0.0 if self.logits is None else 16 * FLOAT * (np.abs(self.logits[np.isfinite(self.logits)]).max(initial=0.0) / self.tau + 2)
        assert (np.abs(got["loss"] - loss) <= 2 * dl + q * (1 + np.abs(loss))).all(), np.abs(got["loss"] - loss).max()
        r = ROUND[self.dtype]
        weights = np.ones(self.T) if self.weights is None else self.weights.astype(np.float64)
        terms = np.exp(u - lse[:, None]) * (weights / self.tau)[:, None]                       # D's: the share of the model ..
        terms = terms + np.abs(d - terms) * (loss != 0)[:, None]                               # .. and the target's (d = the first - the second)
        off = 1.01 * r * np.abs(d) + (2 * dl[:, None] + q + 16 * FLOAT) * terms
        for name, ref, a, b, n in (("dx", dx, off, np.abs(self.w), self.V), ("dw", dw, off.T, np.abs(self.x), self.T)):
            if name in got:
                most = 1.02 * (a @ b) + 1.01 * r * np.abs(ref) + (min(n, 4096) + 8) * FLOAT * ((np.abs(d) if name == "dx" else np.abs(d).T) @ b) + 1e-38
                bad = ~(np.abs(got[name] - ref) <= most)
                assert not bad.any(), (name, int(bad.sum()), float((np.abs(got[name] - ref) / most)[bad].max()))
        return got
