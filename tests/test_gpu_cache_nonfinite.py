"""Infinities and NaN in what attention over an uncompressed cache reads: results are those of the formulas, and the same on every path.
Only a query that sees nothing has a result of zeros; a NaN query or key, or an infinite logit, gives NaN."""
import pytest
import torch

import cache_reference as ref
from paper_2503_18893_amd import binding as xb
from test_gpu_cache import DT, ints, need_gpu, random_trees, run_tree, scale_of, shape_of, workspace  # noqa: F401

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")


def attend(q, K, V, sees, scale):
    """The formulas in double precision, hidden tokens left out row by row -> out, weights, bound of the errors of finite results (that of
    cache_reference.attend, with sums over what is finite)."""
    half = ref.EPS[q.dtype]
    q, K, V = q.double(), K.double(), V.double()
    z = torch.where(sees, scale * (q @ K.T), -INF)
    p = torch.where(sees.any(1, keepdim=True), torch.softmax(z, 1), torch.zeros_like(z))
    finite = torch.isfinite(V)
    out = p @ torch.where(finite, V, 0.0)
    for t in (~finite).any(1).nonzero().flatten().tolist():
        odd = torch.where(finite[t], 0.0, V[t])
        out = torch.where(sees[:, t, None] & ~finite[t], out + p[:, t, None] * odd, out)
    plain = lambda x: torch.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0).abs()  # noqa: E731
    dz = (q.shape[1] + 4) * 2.0 ** -24 * scale * (plain(q) @ plain(K).T).max().item()
    rel = 2 * dz + 2.0 ** -20 + (2 * len(K) + 64) * 2.0 ** -24 + 2.0 ** -15
    return out, p, rel * (p @ plain(V)) + half * out.abs() + 1e-30, rel


def same(got, want, bound, what):
    got = got.double()
    assert torch.equal(torch.isnan(got), torch.isnan(want)), f"{what}: NaN in {torch.isnan(got).sum()} of {got.numel()}, due {torch.isnan(want).sum()}"
    wide = torch.isinf(want)
    assert torch.equal(torch.isinf(got), wide) and torch.equal(got[wide], want[wide]), f"{what}: infinities"
    ok = torch.isfinite(want)
    assert ((got - want).abs() <= bound)[ok].all(), f"{what}: {((got - want).abs() / bound)[ok].max().item():.3g} of the bound"


TREES = {
    # name: dtype, n_rep, d, L, N
    "f32": ("f32", 4, 64, 700, 6),
    "bf16_96": ("bf16", 4, 96, 700, 6),
    "rows_4": ("bf16", 4, 128, 700, 1),
    "rows_16": ("bf16", 2, 128, 700, 8),
    "rows_32": ("bf16", 4, 128, 700, 8),
    "rows_64": ("bf16", 4, 128, 700, 16),
    "rows_128": ("bf16", 4, 128, 700, 32),
    "rows_256": ("bf16", 4, 128, 700, 64),
    "rows_400": ("bf16", 4, 128, 90, 100),
    "rows_1024": ("bf16", 1, 128, 70, 1024),  # every word of a mask
}


def tree_inputs(name, seed):
    dtype, n_rep, d, L, N = TREES[name]
    s = shape_of(2, n_rep, d, L, 2, dtype)
    g = torch.Generator().manual_seed(seed)
    q = torch.randn((2, N, s.H_q, d), generator=g)
    q[..., 0] = q[..., 0].abs() + 0.5  # a key of -inf in channel 0 has logits of -inf, all of them
    K, V = (torch.randn((2, 2, L, d), generator=g) for _ in "KV")
    Kd, Vd = (torch.randn((2, 2, N, d), generator=g) for _ in "KV")
    return s, N, [L, L // 2], [x.to(DT[dtype]) for x in (q, K, V, Kd, Vd)], random_trees(g, 2, N)


def check_tree(s, N, lengths, tensors, sees, what):
    q, K, V, Kd, Vd = tensors
    n_rep = s.H_q // s.H_kv
    out = run_tree(s, ints(lengths), N, K, V, q, Kd, Vd, ref.pack_mask(sees).cuda())
    for b, n in enumerate(lengths):
        mask = torch.cat((torch.ones((N, n), dtype=torch.bool), sees[b]), 1).repeat_interleave(n_rep, 0)
        for h in range(s.H_kv):
            rows = slice(h * n_rep, (h + 1) * n_rep)
            want, _, bound, _ = attend(q[b, :, rows].reshape(-1, s.d_h), torch.cat((K[b, h, :n], Kd[b, h])), torch.cat((V[b, h, :n], Vd[b, h])), mask,
                                       scale_of(s))
            same(out[b, :, rows].reshape(-1, s.d_h), want, bound, f"{what} {b} {h}")


def spoil_keys(K, lengths, how):
    """K [2][2][L][d]: the first sequence's, some of them or half of them or all."""
    n = lengths[0]
    if how == "nan_key":
        K[0, 1, n // 3] = NAN
    elif how == "nan_keys":
        K[0, 1, :n // 2] = NAN
    elif how == "plus_inf_key":
        K[0, 1, n - 1, 0] = INF
    elif how == "minus_inf_key":
        K[0, 1, n // 3, 0] = -INF
    elif how == "minus_inf_keys":
        K[0, 1, :n // 2, 0] = -INF
    else:
        K[0, 1, :n, 0] = -INF


KEYS = ("nan_key", "nan_keys", "plus_inf_key", "minus_inf_key", "minus_inf_keys", "all_minus_inf")


@pytest.mark.parametrize("name,how", [(n, h) for n in TREES for h in ("nan_query",) + KEYS if h != "nan_query" or n.startswith("rows")])
def test_trees(name, how):
    s, N, lengths, x, sees = tree_inputs(name, 900)
    if how == "nan_query":
        x[0][0, N - 1, 1, 3] = NAN
        x[0][1, 0, s.H_q - 1] = NAN
    else:
        spoil_keys(x[1], lengths, how)
        if how == "all_minus_inf":
            x[3][0, 1, :, 0] = -INF
    check_tree(s, N, lengths, x, sees, how)


@pytest.mark.parametrize("name", list(TREES))
def test_queries_that_see_nothing_beside_others(name):
    """An empty cache: tokens that see no drafted one get zeros, the others' NaN stay theirs."""
    s, N, _, x, sees = tree_inputs(name, 901)
    sees[:, ::2] = False
    x[0][0, N - 1] = NAN
    x[0][1, 0] = NAN  # sees nothing: its query does not matter
    check_tree(s, N, [0, 3], x, sees, "empty")


ONE = {
    # name: dtype, n_rep, d, L
    "f32": ("f32", 4, 64, 900),
    "bf16_64": ("bf16", 8, 64, 900),
    "bf16": ("bf16", 4, 128, 900),
    "bf16_16_heads": ("bf16", 16, 128, 900),
}


@pytest.mark.parametrize("how", ("nan_query",) + KEYS)
@pytest.mark.parametrize("name", list(ONE))
def test_weights(name, how):
    dtype, n_rep, d, L = ONE[name]
    lengths = [L, 0, 33]
    s = shape_of(2, n_rep, d, L, 3, dtype)
    g = torch.Generator().manual_seed(902)
    q, K, V = torch.randn((3, s.H_q, d), generator=g), torch.randn((3, 2, L, d), generator=g), torch.randn((3, 2, L, d), generator=g)
    q[..., 0] = q[..., 0].abs() + 0.5
    if how == "nan_query":
        q[0, 0, d - 1] = NAN
        q[1] = NAN  # sees nothing
    else:
        spoil_keys(K, lengths, how)
    q, K, V = (x.to(DT[dtype]) for x in (q, K, V))
    out, total = torch.full_like(q, 7.0, device="cuda"), torch.zeros((3, 2, L), device="cuda")
    xb.xkv_dense_decode_weights(s, K.cuda(), V.cuda(), ints(lengths), q.cuda(), out, total, workspace(s))
    torch.cuda.synchronize()
    for b, n in enumerate(lengths):
        for h in range(2):
            heads = slice(h * n_rep, (h + 1) * n_rep)
            want, p, bound, rel = attend(q[b, heads], K[b, h, :n], V[b, h, :n], torch.ones((n_rep, n), dtype=torch.bool), scale_of(s)) if n else (
                torch.zeros((n_rep, d), dtype=torch.float64), torch.zeros((n_rep, 0), dtype=torch.float64), torch.ones((n_rep, d)), 0.0)
            same(out.cpu()[b, heads], want, bound, f"{how} {b} {h}")
            p = p.sum(0)
            same(total.cpu()[b, h, :n], p, (2 * rel + (n_rep + 2) * 2.0 ** -24) * p + 1e-30, f"{how} weights {b} {h}")
            assert (total[b, h, n:] == 0).all()


@pytest.mark.parametrize("how", ("nan_query",) + KEYS)
@pytest.mark.parametrize("batch", (2, 40))  # queries in several parts, and in one
@pytest.mark.parametrize("name", list(ONE))
def test_blocks(name, batch, how):
    dtype, n_rep, d, L = ONE[name]
    N, c, k = 4, 60, 600
    s = shape_of(2, n_rep, d, L, batch, dtype, k=k)
    g = torch.Generator().manual_seed(903)
    q, K, V = torch.randn((batch, N, s.H_q, d), generator=g), torch.randn((batch, 2, L, d), generator=g), torch.randn((batch, 2, L, d), generator=g)
    q[..., 0] = q[..., 0].abs() + 0.5
    visible = torch.full((batch, N), L, dtype=torch.int32)
    visible[:, 1:] = torch.tensor([0, 31, 555])
    if how == "nan_query":
        q[0, 0, 0, d - 1] = NAN
        q[:, 1] = NAN  # sees nothing
    else:
        spoil_keys(K, [L], how)
    q, K, V = (x.to(DT[dtype]) for x in (q, K, V))
    marks = torch.randn((batch, 2, L // c, d), generator=g).to(DT[dtype])
    out, blocks = torch.full_like(q, 7.0, device="cuda"), torch.full((batch, N, 2, k // c), -7, dtype=torch.int32, device="cuda")
    xb.xkv_block_decode(s, K.cuda(), V.cuda(), visible.cuda(), q.cuda(), N, marks.cuda(), c, out, blocks, workspace(s, N, c))
    torch.cuda.synchronize()
    out, blocks = out.cpu(), blocks.cpu()
    for b in (0, 1, batch - 1):
        for i in range(N):
            for h in range(2):
                heads = slice(h * n_rep, (h + 1) * n_rep)
                t = torch.tensor([j * c + x for j in blocks[b, i, h].tolist() for x in range(c) if j * c + x < visible[b, i]], dtype=torch.long)
                if len(t) == 0:
                    assert (out[b, i, heads] == 0).all()
                    continue
                want, _, bound, _ = attend(q[b, i, heads], K[b, h, t], V[b, h, t], torch.ones((n_rep, len(t)), dtype=torch.bool), scale_of(s))
                same(out[b, i, heads], want, bound, f"{how} {b} {i} {h}")


GENERAL = ("f32", "bf16_96")


@pytest.mark.parametrize("name", GENERAL)
def test_a_nan_query_leaves_other_rows_alone(name):
    s, N, lengths, x, sees = tree_inputs(name, 904)
    x[0][0, N - 1, 1, 3] = NAN
    x[0][1, 0, s.H_q - 1] = NAN
    check_tree(s, N, lengths, x, sees, "NaN query")


def spoil_draft(x, sees, how):
    """Drafted tokens that some tokens see and others do not."""
    N = sees.shape[-1]
    Kd, Vd = x[3], x[4]
    j = N // 2
    for t in (j, N - 1):
        sees[:, :, t] = False
        sees[:, t, t] = True  # only itself
    if how == "nan":
        Kd[:, :, j], Vd[:, :, j] = NAN, NAN
        Vd[1, 0, N - 1] = NAN
    elif how == "inf_values":
        Vd[:, :, j] = INF
        Vd[0, 1, N - 1] = -INF
    elif how == "inf_in_places":
        Vd[0, :, j, 5], Vd[0, :, j, -1] = -INF, INF
        Vd[1, :, N - 1, 0] = NAN
    else:  # +inf and -inf in one place, seen together by some rows and alone by others
        Vd[:, :, 0, 7], Vd[:, :, j, 7], Vd[:, :, N - 1, 7] = INF, -INF, INF
        sees[:, N // 3:, j] = True
        sees[:, N // 2:, N - 1] = True


DRAFTS = ("nan", "inf_values", "inf_in_places", "inf_and_minus_inf")


@pytest.mark.parametrize("empty", (False, True))
@pytest.mark.parametrize("how", DRAFTS)
@pytest.mark.parametrize("name", [n for n in TREES if TREES[n][4] > 1])
def test_what_a_drafted_token_holds_reaches_only_those_who_see_it(name, how, empty):
    s, N, lengths, x, sees = tree_inputs(name, 905)
    spoil_draft(x, sees, how)
    check_tree(s, N, [0, 33] if empty else lengths, x, sees, how)


@pytest.mark.parametrize("name", [n for n in TREES if TREES[n][4] > 1])
def test_many_drafted_tokens_with_infinite_values(name):
    """Most of the draft: every word and every row of a tile has some."""
    s, N, lengths, x, sees = tree_inputs(name, 906)
    for t in range(0, N, 3):
        x[4][:, :, t, t % s.d_h] = INF if t % 2 else NAN
    x[2][1, 1, lengths[1] - 1, 2] = INF  # and the last row of the cache, which all see
    check_tree(s, N, lengths, x, sees, "many")


@pytest.mark.parametrize("name", list(ONE))
def test_infinite_values_of_the_last_row(name):
    """Tokens behind the last one are not that one again, with weight zero."""
    dtype, n_rep, d, L = ONE[name]
    lengths, c, k = [L, 1, 33], 60, 600
    s = shape_of(2, n_rep, d, L, 3, dtype, k=k)
    g = torch.Generator().manual_seed(907)
    q, K, V = (torch.randn(x, generator=g).to(DT[dtype]) for x in ((3, s.H_q, d), (3, 2, L, d), (3, 2, L, d)))
    for b, n in enumerate(lengths):
        V[b, :, n - 1], V[b, 1, n - 1, 3] = INF, -INF
    marks = torch.randn((3, 2, L // c, d), generator=g).to(DT[dtype])
    dev = [x.cuda() for x in (K, V, q, marks)]
    out, sparse = torch.full_like(q, 7.0, device="cuda"), torch.full_like(q, 7.0, device="cuda")
    blocks, ws = torch.full((3, 1, 2, k // c), -7, dtype=torch.int32, device="cuda"), workspace(s, 1, c)
    xb.xkv_dense_decode_weights(s, dev[0], dev[1], ints(lengths), dev[2], out, torch.zeros((3, 2, L), device="cuda"), ws)
    xb.xkv_block_decode(s, dev[0], dev[1], ints(lengths), dev[2], 1, dev[3], c, sparse, blocks, ws)
    torch.cuda.synchronize()
    for b, n in enumerate(lengths):
        for h in range(2):
            heads = slice(h * n_rep, (h + 1) * n_rep)
            t = torch.tensor([j * c + x for j in blocks.cpu()[b, 0, h].tolist() for x in range(c) if j * c + x < n], dtype=torch.long)
            for got, rows in ((out, torch.arange(n)), (sparse, t)):
                want, _, bound, _ = attend(q[b, heads], K[b, h, rows], V[b, h, rows], torch.ones((n_rep, len(rows)), dtype=torch.bool), scale_of(s))
                same(got.cpu()[b, heads], want, bound, f"{b} {h}")
