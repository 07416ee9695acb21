"""Softmax weights enter the sums of attention over an uncompressed cache held to 2^-15: results are rounded once, at the end.

The bound is that of cache_reference.attend without the half step that it allows for weights rounded to the storage type.  Instead: a
weight as two bf16 numbers, the second one for what the first one leaves (at most 2^-7 of it), itself rounded (half a step, 2^-8):
2^-15 of it; and twice as many additions, T 2^-24 more.  Queries are small and few tokens carry values, so that the other terms of the
bound (errors of logits, additions) stay far below the half step of bf16 that such a weight would be off by.
"""
import pytest
import torch

import cache_reference as ref
from paper_2503_18893_amd import binding as xb
from test_gpu_cache import ints, need_gpu, random_trees, run_tree, scale_of, shape_of, within, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


def attend(q, K, V, sees, scale):
    out, p, _, rel = ref.attend(q, K, V, sees, scale)
    rel = rel + 2.0 ** -15 + len(K) * 2.0 ** -24
    return out, rel * (p @ V.double().abs()) + ref.EPS[q.dtype] * out.abs() + 1e-30


def inputs(s, N, seed):
    g = torch.Generator().manual_seed(seed)
    q = 0.1 * torch.randn((s.batch, N, s.H_q, s.d_h), generator=g)
    K, V = (torch.randn((s.batch, s.H_kv, s.L, s.d_h), generator=g) for _ in "KV")
    return g, q.bfloat16(), K.bfloat16(), V.bfloat16()


# up to 16, 32, 64, 128 and 256 rows of a workgroup, two tiles of 256
@pytest.mark.parametrize("n_rep,N", [(4, 1), (1, 16), (4, 8), (4, 16), (4, 32), (4, 64), (4, 100)])
def test_trees(n_rep, N):
    lengths = [7, 20]
    s = shape_of(2, n_rep, 128, 20, 2, "bf16")
    g, q, K, V = inputs(s, N, 500 + N)
    Kd, Vd = (torch.randn((2, 2, N, 128), generator=g).bfloat16() for _ in "KV")
    sees = random_trees(g, 2, N)
    out = run_tree(s, ints(lengths), N, K, V, q, Kd, Vd, ref.pack_mask(sees).cuda())
    for b, n in enumerate(lengths):
        mask = torch.cat((torch.ones((N, n), dtype=torch.bool), sees[b]), 1).repeat_interleave(n_rep, 0)
        for h in range(2):
            rows = slice(h * n_rep, (h + 1) * n_rep)
            want, bound = attend(q[b, :, rows].reshape(-1, 128), torch.cat((K[b, h, :n], Kd[b, h])), torch.cat((V[b, h, :n], Vd[b, h])), mask,
                                 scale_of(s))
            within(out[b, :, rows].reshape(-1, 128), want, bound, f"{N} {b} {h}")


@pytest.mark.parametrize("n_rep,N", [(4, 1), (4, 8), (4, 16), (4, 32), (4, 64)])
def test_trees_over_many_tiles(n_rep, N):
    """Six rows of the cache have values, far apart; the draft has none."""
    L, hot = 2000, [3, 400, 777, 1200, 1333, 1999]
    s = shape_of(1, n_rep, 128, L, 1, "bf16")
    g, q, K, V = inputs(s, N, 600 + N)
    V[:, :, [t for t in range(L) if t not in hot]] = 0.0
    Kd, Vd = torch.randn((1, 1, N, 128), generator=g).bfloat16(), torch.zeros((1, 1, N, 128), dtype=torch.bfloat16)
    out = run_tree(s, None, N, K, V, q, Kd, Vd, None)
    mask = torch.cat((torch.ones((N, L), dtype=torch.bool), torch.ones((N, N), dtype=torch.bool).tril()), 1).repeat_interleave(n_rep, 0)
    want, bound = attend(q[0].reshape(-1, 128), torch.cat((K[0, 0], Kd[0, 0])), torch.cat((V[0, 0], Vd[0, 0])), mask, scale_of(s))
    within(out[0].reshape(-1, 128), want, bound, f"{N}")


@pytest.mark.parametrize("n_rep", [1, 4, 7, 16])
def test_weights(n_rep):
    """Kept weights and the result belong together: both are those of unrounded weights."""
    lengths = [20, 7, 1500]
    s = shape_of(2, n_rep, 128, 1500, 3, "bf16")
    _, q, K, V = inputs(s, 1, 700 + n_rep)
    V[2, :, 6:] = 0.0
    out, total = torch.empty((3, s.H_q, 128), dtype=torch.bfloat16, device="cuda"), torch.zeros((3, 2, 1500), device="cuda")
    xb.xkv_dense_decode_weights(s, K.cuda(), V.cuda(), ints(lengths), q[:, 0].contiguous().cuda(), out, total, workspace(s))
    torch.cuda.synchronize()
    for b, n in enumerate(lengths):
        for h in range(2):
            heads = slice(h * n_rep, (h + 1) * n_rep)
            want, bound = attend(q[b, 0, heads], K[b, h, :n], V[b, h, :n], torch.ones((n_rep, n), dtype=torch.bool), scale_of(s))
            within(out.cpu()[b, heads], want, bound, f"{b} {h}")


@pytest.mark.parametrize("batch,N", [(1, 1), (2, 2), (4, 32)])
def test_blocks(batch, N):
    """One part a query or several; values in six rows of the query's own block."""
    L, c, k = 600, 50, 400
    s = shape_of(2, 4, 128, L, batch, "bf16", k=k)
    _, q, K, V = inputs(s, N, 800 + N)
    V[:, :, :594] = 0.0
    marks = K.view(batch, 2, 12, 50, 128).double().mean(3).bfloat16()
    out = torch.empty((batch, N, 8, 128), dtype=torch.bfloat16, device="cuda")
    blocks = torch.empty((batch, N, 2, 8), dtype=torch.int32, device="cuda")
    xb.xkv_block_decode(s, K.cuda(), V.cuda(), None, q.cuda(), N, marks.cuda(), c, out, blocks, workspace(s, N, c))
    torch.cuda.synchronize()
    for b in range(batch):
        for i in range(N):
            for h in range(2):
                heads = slice(4 * h, 4 * h + 4)
                t = torch.tensor([j * c + x for j in blocks.cpu()[b, i, h].tolist() for x in range(c)])
                want, bound = attend(q[b, i, heads], K[b, h, t], V[b, h, t], torch.ones((4, len(t)), dtype=torch.bool), scale_of(s))
                within(out.cpu()[b, i, heads], want, bound, f"{b} {i} {h}")
