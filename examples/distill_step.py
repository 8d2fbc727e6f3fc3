"""A small language model's last layers trained on a mesh, by labels and by a teacher's top logits.

    python examples/distill_step.py [steps]

Tokens are split two ways and the vocabulary four ways, unevenly (virtual partitions on one GPU).  A step is
  h  = x W1                       gspmd_grouped_dot, tokens split
  L1 = cross entropy(h w^T)       gspmd_softmax_xent, with dh, dw
  L2 = distillation from the teacher's 16 top logits at temperature 2     gspmd_softmax_distill, with dh, dw
  dW1 = x^T dh                    gspmd_grouped_dot, the sum over tokens an AllReduce
and a plain update.  The teacher is a wider model of the same kind; its logits come from a Dot too, its top entries from torch.topk.
After the steps the labels are scored by the forward loss alone, whose logits are not kept."""
import os
import sys

import torch

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import paper_2105_04663_amd as g  # noqa: E402

T, IN, M, V, K, TAU = 500, 200, 96, 1003, 16, 2.0
MESH = g.Mesh((2, 4), tuple(range(8)))          # tokens over dimension 0, vocabulary over dimension 1
PLACES = [(i, j) for i in range(2) for j in range(4)]
TS, VS = -(-T // 2), -(-V // 4)                 # static shard extents


def up(n, to=8):
    return -(-n // to) * to


class Shards:
    """A tensor's shards in one stacked buffer [shards, rows, row stride]: `which` of a partition's two mesh positions a shard belongs to (None: one for all)."""

    def __init__(self, rows, cols, which, dtype=torch.bfloat16):
        self.ld = up(cols)
        self.cols = cols
        self.t = torch.zeros((1 if which is None else (2, 4)[which], rows, self.ld), dtype=dtype, device="cuda")
        self.bufs = [g.ShardBuf.of(self.t[0 if which is None else p[which]], self.ld) for p in PLACES]

    def fill(self, full):
        flat = self.t.view(-1, self.ld)
        flat[:full.shape[0], :self.cols] = full.to(self.t.dtype)
        return self

    def full(self, rows):
        return self.t.view(-1, self.ld)[:rows, :self.cols]


def workspace(n):
    space = torch.empty(n + 256, dtype=torch.uint8, device="cuda")
    return space, up(space.data_ptr(), 256)


def dot(dims, lhs, lhs_sh, rhs, rhs_sh, out, out_sh):
    n = g.dot_workspace_bytes(MESH, dims, lhs_sh, rhs_sh, out_sh, -1)
    space, base = workspace(n)
    g.grouped_dot(MESH, dims, lhs.bufs, lhs_sh, rhs.bufs, rhs_sh, out.bufs, out_sh, None, base, n, torch.cuda.current_stream().cuda_stream)
    return space                                # kept until the stream has run the call


def main(steps=30):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(3)
    rand = lambda *s: torch.randn(s, generator=gen, device="cuda")
    stream = torch.cuda.current_stream().cuda_stream
    x_sh, w1_sh = g.Sharding((T, IN), (0, -1)), g.Sharding((IN, M), (-1, -1))
    h_sh, w_sh = g.Sharding((T, M), (0, -1)), g.Sharding((V, M), (1, -1))
    x = Shards(TS, IN, 0).fill(rand(T, IN))
    w1, w = Shards(IN, M, None).fill(rand(IN, M) * 0.07), Shards(VS, M, 1).fill(rand(V, M) * 0.05)
    h, dh = Shards(TS, M, 0), (Shards(TS, M, 0), Shards(TS, M, 0))
    dw, dw1 = (Shards(VS, M, 1), Shards(VS, M, 1)), Shards(IN, M, None, torch.float32)

    # the teacher: its logits on this mesh, its top entries, and labels drawn from it
    z_sh = g.Sharding((T, V), (0, 1))
    rows_by_columns = g.DotDims((), (), (1,), (1,))
    teacher_w = Shards(VS, IN, 1).fill(rand(V, IN) * 0.15)
    z = torch.zeros((2, 4, TS, up(VS)), device="cuda")
    z_bufs = [g.ShardBuf.of(z[p], up(VS)) for p in PLACES]
    n = g.dot_workspace_bytes(MESH, rows_by_columns, x_sh, g.Sharding((V, IN), (1, -1)), z_sh, -1)
    space, base = workspace(n)
    g.grouped_dot(MESH, rows_by_columns, x.bufs, x_sh, teacher_w.bufs, g.Sharding((V, IN), (1, -1)), z_bufs, z_sh, None, base, n, stream)
    logits = z[..., :VS].permute(0, 2, 1, 3).reshape(2 * TS, 4 * VS)[:T, :V]
    top, entries = torch.topk(logits, K, dim=1)
    labels = torch.multinomial(torch.softmax(logits, dim=1), 1, generator=gen)
    labels[::17] = -1                           # tokens without a label

    def per_token(values, dtype):
        t = torch.zeros((2 * TS, values.shape[1]), dtype=dtype, device="cuda")
        t[:T] = values
        return t

    arrays = {"labels": per_token(labels, torch.int32), "entries": per_token(entries, torch.int32), "top": per_token(top, torch.float32)}
    weights = torch.full((2 * TS,), 1.0 / T, device="cuda")
    losses = torch.zeros((2, 2 * TS), device="cuda")
    at = lambda t, i: t.data_ptr() + i * TS * t[0].numel() * t.element_size()
    by_label = [g.TokenBuf(ids=at(arrays["labels"], i), loss=at(losses[0], i), weights=at(weights, i)) for i, _ in PLACES]
    by_teacher = [g.TokenBuf(ids=at(arrays["entries"], i), loss=at(losses[1], i), weights=at(weights, i), logits=at(arrays["top"], i)) for i, _ in PLACES]

    n = g.softmax_workspace_bytes(MESH, h_sh, w_sh, 0, g.BF16, True)
    space, base = workspace(n)
    common = dict(vocab_dim=0, workspace=base, workspace_bytes=n, stream=stream)
    params = [w1.t.float(), w.t.float()]        # kept in float32, used in bfloat16
    history = []
    for step in range(steps):
        held = [dot(g.DotDims((), (), (1,), (0,)), x, x_sh, w1, w1_sh, h, h_sh)]
        g.softmax_xent(MESH, h.bufs, h_sh, w.bufs, w_sh, by_label, dx_shards=dh[0].bufs, dw_shards=dw[0].bufs, **common)
        g.softmax_distill(MESH, h.bufs, h_sh, w.bufs, w_sh, by_teacher, K, TAU, dx_shards=dh[1].bufs, dw_shards=dw[1].bufs, **common)
        dh[0].t.add_(dh[1].t)
        held.append(dot(g.DotDims((), (), (0,), (0,)), x, x_sh, dh[0], h_sh, dw1, w1_sh))
        params[0].sub_(dw1.t, alpha=2.0)
        params[1].sub_(dw[0].t.float() + dw[1].t.float(), alpha=20.0)
        w1.t.copy_(params[0])
        w.t.copy_(params[1])
        history.append(losses[:, :T].mean(dim=1).tolist())
        if step % 10 == 0 or step == steps - 1:
            print("step %3d   cross entropy %.4f   distance from the teacher %.4f" % (step, *history[-1]), flush=True)
    dot(g.DotDims((), (), (1,), (0,)), x, x_sh, w1, w1_sh, h, h_sh)
    n = g.softmax_workspace_bytes(MESH, h_sh, w_sh, 0, g.BF16, False)
    space, base = workspace(n)
    g.softmax_xent(MESH, h.bufs, h_sh, w.bufs, w_sh, by_label, vocab_dim=0, workspace=base, workspace_bytes=n, stream=stream)
    history.append([losses[0, :T].mean().item(), history[-1][1]])
    print("scored     cross entropy %.4f" % history[-1][0], flush=True)
    return history


if __name__ == "__main__":
    main(int(sys.argv[1]) if len(sys.argv) > 1 else 30)
