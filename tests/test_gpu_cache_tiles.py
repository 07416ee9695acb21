"""Attention over an uncompressed cache with parts of many tiles, several of a workgroup's buffers in turn and more than one tile of rows,
against a plain implementation in double precision on the device.  tests/test_cache_plan.py holds how many tiles a part of each has."""
import pytest
import torch

import cache_reference as ref
from paper_2503_18893_amd import binding as xb
from test_gpu_cache import DT, ints, need_gpu, random_trees, run_tree, scale_of, shape_of, within, workspace  # noqa: F401

pytestmark = pytest.mark.gpu

TREES = {
    # name: dtype, H_kv, n_rep, d, lengths, N, rows of a workgroup, the fewest rounds of a part
    "rows_16": ("bf16", 32, 4, 128, [5000, 3017], 4, 16, 8),
    "rows_16_odd": ("bf16", 32, 2, 128, [7700], 7, 16, 7),
    "rows_32": ("bf16", 32, 1, 128, [5000, 3017], 32, 32, 8),
    "rows_32_odd": ("bf16", 32, 4, 128, [7103], 8, 32, 7),
    "rows_64": ("bf16", 32, 2, 128, [5000, 3017], 32, 64, 8),
    "rows_64_odd": ("bf16", 32, 4, 128, [7101], 13, 64, 7),
    "rows_128": ("bf16", 32, 4, 128, [5000, 3017], 32, 128, 8),
    "rows_128_odd": ("bf16", 32, 7, 128, [7001], 18, 128, 7),
    "rows_256": ("bf16", 32, 4, 128, [5000, 3017], 64, 256, 16),
    "rows_256_odd": ("bf16", 32, 7, 128, [7000, 1, 999], 33, 256, 16),
    "rows_256_two_tiles": ("bf16", 32, 4, 128, [1500, 1501], 100, 256, 12),
    "rows_256_two_full_tiles": ("bf16", 32, 4, 128, [3000], 128, 256, 12),
    "rows_128_three_tiles": ("bf16", 16, 4, 128, [3000], 96, 128, 4),
    "general_f32": ("f32", 32, 1, 64, [5000, 1200], 16, 16, 3),
    "general_bf16": ("bf16", 32, 2, 96, [3001, 3000], 24, 16, 5),
}


def tree_shape(name):
    dtype, H_kv, n_rep, d, lengths, N, _, _ = TREES[name]
    return shape_of(H_kv, n_rep, d, max(lengths), len(lengths), dtype), lengths, N


@pytest.mark.parametrize("grow", (False, True))
@pytest.mark.parametrize("name", list(TREES))
def test_trees(name, grow):
    """grow: keys whose logits rise with their place up to about 60, so that the maximum is raised again and again."""
    s, lengths, N = tree_shape(name)
    n_rep, d = s.H_q // s.H_kv, s.d_h
    g = torch.Generator(device="cuda").manual_seed(1000 + len(name))
    q = torch.randn((s.batch, N, s.H_kv, n_rep, d), generator=g, device="cuda")
    K, V = (torch.randn((s.batch, s.H_kv, s.L, d), generator=g, device="cuda") for _ in "KV")
    Kd, Vd = (torch.randn((s.batch, s.H_kv, N, d), generator=g, device="cuda") for _ in "KV")
    if grow:
        u = torch.randn((s.batch, s.H_kv, d), generator=g, device="cuda")
        u *= d ** 0.25 / u.norm(dim=-1, keepdim=True)  # scale |u|^2 = 1
        q = 0.3 * q + 8.0 * u[:, None, :, None]
        K = 0.3 * K + 8.0 * u[:, :, None] * torch.linspace(0, 1, s.L, device="cuda")[:, None]
    for b, n in enumerate(lengths):
        K[b, :, n:], V[b, :, n:] = float("nan"), float("nan")
    q = q.reshape(s.batch, N, s.H_q, d)
    q, K, V, Kd, Vd = (x.to(DT[s.dtype]) for x in (q, K, V, Kd, Vd))
    sees = random_trees(torch.Generator().manual_seed(1), s.batch, N)
    out = run_tree(s, ints(lengths), N, K, V, q, Kd, Vd, ref.pack_mask(sees).cuda()).cuda()
    for b, n in enumerate(lengths):
        mask = torch.cat((torch.ones((N, n), dtype=torch.bool), sees[b]), 1).repeat_interleave(n_rep, 0).cuda()
        for h in range(s.H_kv):
            heads = slice(h * n_rep, (h + 1) * n_rep)
            want, _, bound, _ = ref.attend(q[b, :, heads].reshape(-1, d), torch.cat((K[b, h, :n], Kd[b, h])), torch.cat((V[b, h, :n], Vd[b, h])), mask, scale_of(s))
            within(out[b, :, heads].reshape(-1, d), want, bound, f"{name} {b} {h}")


@pytest.mark.parametrize("grow", (False, True))
def test_weights(grow):
    """Logits of several tiles leave together: full groups of tiles and a rest of them, and a part that ends inside a tile."""
    lengths, n_rep, d = [5000, 3017, 1027], 4, 128
    s = shape_of(32, n_rep, d, 5000, 3, "bf16")
    g = torch.Generator(device="cuda").manual_seed(1100)
    q, K, V = (torch.randn(x, generator=g, device="cuda") for x in ((3, 32, n_rep, d), (3, 32, 5000, d), (3, 32, 5000, d)))
    if grow:
        u = torch.randn((3, 32, d), generator=g, device="cuda")
        u *= d ** 0.25 / u.norm(dim=-1, keepdim=True)
        q, K = 0.3 * q + 8.0 * u[:, :, None], 0.3 * K + 8.0 * u[:, :, None] * torch.linspace(0, 1, 5000, device="cuda")[:, None]
    q, K, V = q.reshape(3, s.H_q, d).bfloat16(), K.bfloat16(), V.bfloat16()
    out, total = torch.full_like(q, float("nan")), torch.zeros((3, 32, 5000), device="cuda")
    xb.xkv_dense_decode_weights(s, K, V, ints(lengths), q, out, total, workspace(s))
    for b, n in enumerate(lengths):
        for h in range(32):
            heads = slice(h * n_rep, (h + 1) * n_rep)
            want, p, bound, rel = ref.attend(q[b, heads], K[b, h, :n], V[b, h, :n], torch.ones((n_rep, n), dtype=torch.bool, device="cuda"), scale_of(s))
            within(out[b, heads], want, bound, f"{b} {h}")
            p = p.sum(0)
            assert ((total[b, h, :n].double() - p).abs() <= (2 * rel + (n_rep + 2) * 2.0 ** -24) * p + 1e-30).all(), (b, h)
            assert (total[b, h, n:] == 0).all()


BLOCKS = {
    # name: dtype, H_kv, n_rep, d, batch, N, L, k, parts
    "one_part": ("bf16", 8, 4, 128, 4, 8, 3500, 1500, 1),
    "two_parts": ("bf16", 8, 4, 128, 4, 4, 3500, 1500, 2),
    "sixteen_heads": ("bf16", 8, 16, 128, 4, 8, 2001, 1000, 1),
    "general_f32": ("f32", 32, 2, 64, 4, 8, 2000, 700, 1),
    "general_bf16": ("bf16", 32, 2, 96, 4, 4, 2000, 700, 2),
}


@pytest.mark.parametrize("c", (1, 5, 24, 64, 129, 500))
@pytest.mark.parametrize("name", list(BLOCKS))
def test_blocks(name, c):
    dtype, H_kv, n_rep, d, batch, N, L, k, _ = BLOCKS[name]
    s = shape_of(H_kv, n_rep, d, L, batch, dtype, k=k)
    g = torch.Generator(device="cuda").manual_seed(1200 + c)
    n_c, k_ch = -(-L // c), min(-(-k // c), -(-L // c))
    q, K, V, marks = (torch.randn(x, generator=g, device="cuda").to(DT[dtype]) for x in ((batch, N, s.H_q, d), (batch, H_kv, L, d), (batch, H_kv, L, d),
                                                                                        (batch, H_kv, n_c, d)))
    visible = L - torch.randint(0, L // 4, (batch, N), generator=g, device="cuda", dtype=torch.int32)
    visible[0, 0], visible[1, 0], visible[2, 0] = L, (L // c) * c, min(L, (k_ch - 1) * c + 1)
    out = torch.full((batch, N, s.H_q, d), float("nan"), dtype=DT[dtype], device="cuda")
    blocks = torch.full((batch, N, H_kv, k_ch), -7, dtype=torch.int32, device="cuda")
    xb.xkv_block_decode(s, K, V, visible, q, N, marks, c, out, blocks, workspace(s, N, c))
    got = blocks.cpu()
    for b in range(batch):
        for i in range(N):
            v = visible[b, i].item()
            for h in range(0, H_kv, 5):
                heads = slice(h * n_rep, (h + 1) * n_rep)
                want = ref.choose_blocks(q[b, i, heads].cpu(), marks[b, h].cpu(), v, c, k_ch)
                assert got[b, i, h, :len(want)].tolist() == want, (b, i, h)
                t = (torch.tensor(want, device="cuda")[:, None] * c + torch.arange(c, device="cuda")).flatten()
                t = t[t < v]
                o, _, bound, _ = ref.attend(q[b, i, heads], K[b, h, t], V[b, h, t], torch.ones((n_rep, len(t)), dtype=torch.bool, device="cuda"), scale_of(s))
                within(out[b, i, heads], o, bound, f"{name} {c}: {b} {i} {h}")


@pytest.mark.parametrize("in_place", (False, True))
@pytest.mark.parametrize("L", (8192, 8193, 12001, 16384, 16385, 32768, 32769))
def test_evictions_at_the_borders_of_the_selection(L, in_place):
    """As many keys per lane as the room for rows needs, and from 32769 rows on another selection."""
    lengths, H_kv, d = [L, L - 77, L // 2], 2, 64
    k, sink, recent = L // 3, 4, 1000
    s = shape_of(H_kv, 1, d, L, 3, "bf16", k=k)
    g = torch.Generator().manual_seed(1300 + L)
    K, V = (torch.randn((3, H_kv, L, d), generator=g).bfloat16() for _ in "KV")
    w = torch.randn((3, H_kv, L), generator=g).exp()
    w[0, :, ::3] = 0.25  # ties
    w[:, :, 1::7] = 0.0
    w[1, 1] = 1.0
    src = [x.cuda() for x in (K, V, w)]
    dst = src if in_place else [torch.full((3, H_kv, k, *x), 3.0, dtype=t, device="cuda") for x, t in (((d,), torch.bfloat16), ((d,), torch.bfloat16), ((), torch.float32))]
    rows, n_out = torch.full((3, H_kv, k), -9, dtype=torch.int32, device="cuda"), torch.full((3,), -9, dtype=torch.int32, device="cuda")
    xb.xkv_evict(s, *src, ints(lengths), sink, recent, L if in_place else k, *dst, rows, n_out, workspace(s))
    torch.cuda.synchronize()
    assert n_out.tolist() == [min(n, k) for n in lengths]
    for b, n in enumerate(lengths):
        for h in range(H_kv):
            keep = ref.keep_rows(w[b, h], n, k, sink, recent)
            assert rows[b, h].tolist() == keep, (b, h)
            for x, y in zip(dst, (K, V, w)):
                assert torch.equal(x[b, h, :k].cpu(), y[b, h, keep]), (b, h)
                if in_place:
                    assert torch.equal(x[b, h, k:].cpu(), y[b, h, k:]), (b, h)


@pytest.mark.parametrize("dtype,d,n_rep,N", [("f32", 40, 1, 3), ("bf16", 128, 4, 2), ("bf16", 128, 4, 8), ("bf16", 128, 2, 40)])
@pytest.mark.parametrize("batch", (33, 65, 150))
def test_many_sequences_of_any_lengths(dtype, d, n_rep, N, batch):
    """More sequences than a wavefront has lanes, with fewer and more parts than sequences."""
    g = torch.Generator(device="cuda").manual_seed(1400 + batch)
    L = 700
    lengths = torch.randint(0, L + 1, (batch,), generator=g, device="cuda", dtype=torch.int32)
    lengths[3], lengths[-1], lengths[7] = 0, L, 1
    s = shape_of(1, n_rep, d, L, batch, dtype)
    q, K, V, Kd, Vd = (torch.randn(x, generator=g, device="cuda").to(DT[dtype]) for x in ((batch, N, n_rep, d), (batch, 1, L, d), (batch, 1, L, d), (batch, 1, N, d),
                                                                                      (batch, 1, N, d)))
    sees = random_trees(torch.Generator().manual_seed(2), batch, N)
    out = run_tree(s, lengths, N, K, V, q, Kd, Vd, ref.pack_mask(sees).cuda()).cuda()
    q1, one, total = q[:, 0].contiguous(), torch.full((batch, n_rep, d), float("nan"), dtype=DT[dtype], device="cuda"), torch.zeros((batch, 1, L), device="cuda")
    xb.xkv_dense_decode_weights(s, K, V, lengths, q1, one, total, workspace(s))
    for b, n in enumerate(lengths.tolist()):
        mask = torch.cat((torch.ones((N, n), dtype=torch.bool), sees[b]), 1).repeat_interleave(n_rep, 0).cuda()
        want, _, bound, _ = ref.attend(q[b].reshape(-1, d), torch.cat((K[b, 0, :n], Kd[b, 0])), torch.cat((V[b, 0, :n], Vd[b, 0])), mask, scale_of(s))
        within(out[b].reshape(-1, d), want, bound, f"{b}")
        if n == 0:
            assert (one[b] == 0).all()
            continue
        want, p, bound, rel = ref.attend(q1[b], K[b, 0, :n], V[b, 0, :n], mask[:n_rep, :1].new_ones((n_rep, n)), scale_of(s))
        within(one[b], want, bound, f"{b}")
        assert ((total[b, 0, :n].double() - p.sum(0)).abs() <= (2 * rel + (n_rep + 2) * 2.0 ** -24) * p.sum(0) + 1e-30).all(), b
        assert (total[b, 0, n:] == 0).all()
