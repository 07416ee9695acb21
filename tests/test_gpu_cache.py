"""The calls on an uncompressed cache that grows and shrinks, through the C ABI, against a plain implementation in double precision
(cache_reference.py, which also derives the tolerances).  Rows that are not in use and drafted tokens that nothing sees hold NaN."""
import pytest
import torch

import cache_reference as ref
from paper_2503_18893_amd import binding as xb

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def shape_of(H_kv, n_rep, d, L, batch, dtype, k=1, scale=0.0):
    return xb.Shape(1, H_kv, H_kv * n_rep, d, 1, 1, L, k, batch, dtype, scale)


def workspace(s, N=1, c=0):
    # whatever is in it: nothing may depend on it
    return torch.full((xb.xkv_cache_workspace_bytes(s, N, c),), 0xFF, dtype=torch.uint8, device="cuda")


def cache(s, lengths, seed, key_scale=1.0):
    """K, V on the CPU, NaN in rows that are not in use."""
    g = torch.Generator().manual_seed(seed)
    K, V = (torch.randn((s.batch, s.H_kv, s.L, s.d_h), generator=g) for _ in "KV")
    K *= key_scale
    for b, n in enumerate(lengths):
        K[b, :, n:] = float("nan")
        V[b, :, n:] = float("nan")
    return g, K.to(DT[s.dtype]), V.to(DT[s.dtype])


def scale_of(s):
    return s.scale if s.scale > 0 else s.d_h ** -0.5


def within(got, want, bound, what):
    err = (got.double() - want).abs()
    assert torch.isfinite(got.double()).all(), what
    worst = (err / bound).max().item()
    assert worst <= 1.0, f"{what}: {worst:.3g} of the bound, largest error {err.max().item():.3g}"


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------------------------------------------------- trees
TREES = {
    # name: dtype, H_kv, n_rep, d, L, lengths, N, key scale
    "f32_tiny": ("f32", 1, 4, 64, 512, [512], 8, 1.0),
    "f32_one_of_everything": ("f32", 1, 1, 1, 1, [1], 1, 1.0),
    "f32_odd_width": ("f32", 2, 3, 33, 130, [130, 0, 7], 5, 1.0),
    "f32_wide": ("f32", 1, 2, 256, 200, [65, 200], 40, 1.0),
    "bf16_odd_width": ("bf16", 2, 5, 96, 300, [300, 64], 17, 1.0),
    "bf16_64": ("bf16", 2, 8, 64, 500, [1, 500, 499], 9, 1.0),
    "bf16_one_token": ("bf16", 2, 4, 128, 1000, [1000, 33], 1, 1.0),
    "bf16_few_rows": ("bf16", 2, 4, 128, 3000, [3000, 2999, 31], 7, 1.0),
    "bf16_two_tiles": ("bf16", 1, 4, 128, 2500, [2047, 2500], 16, 1.0),
    "bf16_four_tiles": ("bf16", 2, 4, 128, 2000, [2000, 1], 32, 1.0),
    "bf16_seven_heads": ("bf16", 2, 7, 128, 1500, [1500, 777, 0], 33, 1.0),
    "bf16_many_rows": ("bf16", 2, 4, 128, 1100, [1100, 64], 64, 1.0),
    "bf16_sixteen_heads": ("bf16", 1, 16, 128, 700, [700, 129], 100, 1.0),
    "bf16_long_draft": ("bf16", 1, 1, 128, 90, [90, 0], 300, 1.0),
    "bf16_peaked": ("bf16", 2, 4, 128, 2000, [2000, 1500], 24, 12.0),
    "bf16_long": ("bf16", 1, 4, 128, 20011, [20011], 20, 1.0),
}


def random_trees(g, batch, N):
    sees = torch.eye(N, dtype=torch.bool).repeat(batch, 1, 1)
    for j in range(1, N):
        sees[:, j] |= sees[torch.arange(batch), (torch.rand(batch, generator=g) * j).long()]
    return sees


def run_tree(s, lengths, N, K, V, q, Kd, Vd, words, ws=None):
    out = torch.full((s.batch, N, s.H_q, s.d_h), float("nan"), dtype=DT[s.dtype], device="cuda")
    dev = [x.cuda() for x in (K, V, q, Kd, Vd)]
    ws = workspace(s, N) if ws is None else ws
    xb.xkv_tree_decode(s, dev[0], dev[1], lengths, dev[2], dev[3], dev[4], words, N, out, ws)
    torch.cuda.synchronize()
    return out.cpu()


def check_tree(s, lengths, N, K, V, q, Kd, Vd, sees, out, what):
    n_rep = s.H_q // s.H_kv
    for b, n in enumerate(lengths):
        mask = torch.cat((torch.ones((N, n), dtype=torch.bool), sees[b]), 1).repeat_interleave(n_rep, 0)
        for g in range(s.H_kv):
            rows = q[b, :, g * n_rep:(g + 1) * n_rep].reshape(-1, s.d_h)
            want, _, bound, _ = ref.attend(rows, torch.cat((K[b, g, :n], Kd[b, g])), torch.cat((V[b, g, :n], Vd[b, g])), mask, scale_of(s))
            within(out[b, :, g * n_rep:(g + 1) * n_rep].reshape(-1, s.d_h), want, bound, f"{what} sequence {b} head {g}")


@pytest.mark.parametrize("name", list(TREES))
def test_tree(name):
    dtype, H_kv, n_rep, d, L, lengths, N, key_scale = TREES[name]
    s = shape_of(H_kv, n_rep, d, L, len(lengths), dtype)
    g, K, V = cache(s, lengths, 100 + len(name), key_scale)
    q = torch.randn((s.batch, N, s.H_q, d), generator=g).to(DT[dtype])
    Kd, Vd = (torch.randn((s.batch, H_kv, N, d), generator=g).to(DT[dtype]) for _ in "KV")
    sees = random_trees(g, s.batch, N)
    if N > 4:  # padding at the end of the draft: no token sees it, and it sees nothing of the draft; one more sees no draft at all
        sees[:, :, N - 2:] = False
        sees[:, N - 2:] = False
        sees[:, 1] = False
        Kd[:, :, N - 2:] = float("nan")
        Vd[:, :, N - 2:] = float("nan")
    out = run_tree(s, ints(lengths), N, K, V, q, Kd, Vd, ref.pack_mask(sees).cuda())
    check_tree(s, lengths, N, K, V, q, Kd, Vd, sees, out, name)
    for b, n in enumerate(lengths):
        if n == 0 and N > 4:
            assert (out[b, 1] == 0).all() and (out[b, N - 1] == 0).all()  # they see nothing


@pytest.mark.parametrize("dtype,N", [("f32", 6), ("bf16", 6), ("bf16", 70)])
def test_tree_without_a_mask_is_a_chain(dtype, N):
    s = shape_of(2, 4, 128, 200, 2, dtype)
    g, K, V = cache(s, [200, 200], 5)
    q = torch.randn((2, N, s.H_q, 128), generator=g).to(DT[dtype])
    Kd, Vd = (torch.randn((2, 2, N, 128), generator=g).to(DT[dtype]) for _ in "KV")
    out = run_tree(s, None, N, K, V, q, Kd, Vd, None)
    sees = torch.ones((N, N), dtype=torch.bool).tril().repeat(2, 1, 1)
    check_tree(s, [200, 200], N, K, V, q, Kd, Vd, sees, out, "chain")


def test_tree_lengths_outside_the_cache_count_as_the_nearer_end():
    s = shape_of(1, 4, 128, 100, 2, "bf16")
    g, K, V = cache(s, [100, 0], 6)
    q = torch.randn((2, 3, 4, 128), generator=g).bfloat16()
    Kd, Vd = (torch.randn((2, 1, 3, 128), generator=g).bfloat16() for _ in "KV")
    assert torch.equal(run_tree(s, ints([1000, -5]), 3, K, V, q, Kd, Vd, None), run_tree(s, ints([100, 0]), 3, K, V, q, Kd, Vd, None))


# ------------------------------------------------------------------------------------------------------------ blocks
BLOCKS = {
    # name: dtype, H_kv, n_rep, d, L, N, c, k, visible
    "f32_tiny": ("f32", 1, 4, 64, 512, 1, 16, 128, [[512]]),
    "f32_blocks_of_one": ("f32", 2, 3, 33, 70, 2, 1, 9, [[70, 5], [0, 1]]),
    "f32_wide": ("f32", 1, 2, 256, 300, 1, 7, 50, [[300], [299], [7], [8]]),
    "bf16_64": ("bf16", 2, 8, 64, 400, 2, 8, 65, [[400, 399], [9, 8]]),
    "bf16_one": ("bf16", 2, 4, 128, 4000, 1, 16, 512, [[4000], [3999], [16], [17], [1], [0]]),
    "bf16_blocks_of_24": ("bf16", 2, 7, 128, 2500, 1, 24, 480, [[2500], [2401]]),
    "bf16_blocks_of_5": ("bf16", 1, 16, 128, 999, 1, 5, 333, [[999], [500]]),
    "bf16_everything": ("bf16", 2, 4, 128, 700, 1, 32, 700, [[700], [333]]),
    "bf16_only_its_own": ("bf16", 2, 4, 128, 700, 1, 64, 64, [[700], [641], [640]]),
    "bf16_prompt": ("bf16", 2, 4, 128, 600, 40, 16, 128, [list(range(561, 601)), list(range(0, 40))]),
    "bf16_prompt_in_one_part": ("bf16", 2, 4, 128, 300, 150, 16, 64, [list(range(0, 150)), list(range(151, 301))]),
    "bf16_large_blocks": ("bf16", 1, 4, 128, 6000, 1, 500, 2000, [[6000], [5555]]),
    "bf16_one_head": ("bf16", 3, 1, 128, 2000, 3, 64, 640, [[2000, 1990, 64]]),
}


def means_of(K, lengths, c):
    """Block means over the rows in use, in the storage type; NaN for blocks without any."""
    b, H_kv, L, d = K.shape
    n_c = -(-L // c)
    m = torch.full((b, H_kv, n_c, d), float("nan"), dtype=torch.float64)
    for i, n in enumerate(lengths):
        for j in range(-(-n // c)):
            m[i, :, j] = K[i, :, j * c:min(n, (j + 1) * c)].double().mean(1)
    return m.to(K.dtype)


@pytest.mark.parametrize("name", list(BLOCKS))
def test_blocks(name):
    dtype, H_kv, n_rep, d, L, N, c, k, visible = BLOCKS[name]
    s = shape_of(H_kv, n_rep, d, L, len(visible), dtype, k=k)
    rows = [max(v) for v in visible]
    g, K, V = cache(s, rows, 200 + len(name))
    q = torch.randn((s.batch, N, s.H_q, d), generator=g).to(DT[dtype])
    marks = means_of(K, rows, c)
    n_c, k_ch = -(-L // c), min(-(-k // c), -(-L // c))
    out = torch.full((s.batch, N, s.H_q, d), float("nan"), dtype=DT[dtype], device="cuda")
    blocks = torch.full((s.batch, N, H_kv, k_ch), -7, dtype=torch.int32, device="cuda")
    args = [K.cuda(), V.cuda(), ints(visible), q.cuda(), N, marks.cuda(), c]
    xb.xkv_block_decode(s, *args, out, blocks, workspace(s, N, c))
    again = torch.full_like(out, float("nan"))
    xb.xkv_block_decode(s, *args, again, None, workspace(s, N, c))
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    out, blocks = out.cpu(), blocks.cpu()
    for b in range(s.batch):
        for i in range(N):
            v = visible[b][i]
            for h in range(H_kv):
                heads = slice(h * n_rep, (h + 1) * n_rep)
                want = ref.choose_blocks(q[b, i, heads], marks[b, h], v, c, k_ch)
                got = blocks[b, i, h].tolist()
                assert got[:len(want)] == want, (b, i, h)
                assert got[len(want):] == list(range(-(-v // c), -(-v // c) + k_ch - len(want))), (b, i, h)
                t = torch.tensor([j * c + x for j in want for x in range(c) if j * c + x < v], dtype=torch.long)
                o, _, bound, _ = ref.attend(q[b, i, heads], K[b, h, t], V[b, h, t], torch.ones((n_rep, len(t)), dtype=torch.bool), scale_of(s))
                within(out[b, i, heads], o, bound, f"{name} {b} {i} {h}")


@pytest.mark.parametrize("L,c,k", [(1500, 1, 300), (4000, 1, 64), (9000, 1, 1000), (17000, 1, 500), (3000, 2, 700)])
@pytest.mark.parametrize("spread", [1.0, 2.0 ** -7, 2.0 ** -12, 0.0])
def test_blocks_whose_scores_lie_close_together(L, c, k, spread):
    """Means that differ by a few roundings, or not at all: the selection is that of the sums in double precision, rounded once."""
    s = shape_of(1, 4, 128, L, 2, "bf16", k=k)
    g, K, V = cache(s, [L, L], 14)
    n_c, k_ch = -(-L // c), -(-k // c)
    marks = (1.0 + spread * torch.randn((2, 1, n_c, 128), generator=g)).bfloat16()
    marks[:, :, n_c // 2:n_c // 2 + 50] = marks[:, :, :50]  # and some twice
    visible = [L, L - L // 3]
    q = torch.randn((2, 1, 4, 128), generator=g).bfloat16()
    out, blocks = torch.empty_like(q).cuda(), torch.empty((2, 1, 1, k_ch), dtype=torch.int32, device="cuda")
    xb.xkv_block_decode(s, K.cuda(), V.cuda(), ints(visible), q.cuda(), 1, marks.cuda(), c, out, blocks, workspace(s, 1, c))
    for b in range(2):
        assert blocks.cpu()[b, 0, 0].tolist() == ref.choose_blocks(q[b, 0], marks[b, 0], visible[b], c, k_ch)


@pytest.mark.parametrize("L,N", [(1100, 3), (2049, 2), (1100, 150), (2049, 140)])
def test_blocks_with_few_and_many_queries(L, N):
    """More than 1024 and 2048 blocks, for fewer and more queries than compute units."""
    s = shape_of(2, 2, 128, L, 1, "bf16", k=40)
    g, K, V = cache(s, [L], 81)
    marks, q = torch.randn((1, 2, L, 128), generator=g).bfloat16(), torch.randn((1, N, 4, 128), generator=g).bfloat16()
    visible = torch.randint(1, L + 1, (1, N), generator=g, dtype=torch.int32)
    visible[0, 0] = L
    out, blocks = torch.empty_like(q, device="cuda"), torch.empty((1, N, 2, 40), dtype=torch.int32, device="cuda")
    xb.xkv_block_decode(s, K.cuda(), V.cuda(), visible.cuda(), q.cuda(), N, marks.cuda(), 1, out, blocks, workspace(s, N, 1))
    torch.cuda.synchronize()
    for i in range(N):
        n = visible[0, i].item()
        for h in range(2):
            want = ref.choose_blocks(q[0, i, 2 * h:2 * h + 2], marks[0, h], n, 1, 40)
            assert blocks.cpu()[0, i, h].tolist() == want + list(range(n, n + 40 - len(want))), (i, h)
            o, _, bound, _ = ref.attend(q[0, i, 2 * h:2 * h + 2], K[0, h, want], V[0, h, want], torch.ones((2, len(want)), dtype=torch.bool), scale_of(s))
            within(out.cpu()[0, i, 2 * h:2 * h + 2], o, bound, f"{i} {h}")


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("f32", 64), ("f32", 20)])
@pytest.mark.parametrize("L", [3000, 17000])
def test_blocks_whose_scores_overflow(dtype, d, L):
    """Scores that are infinite in single precision rank like any other; the query's own block is read all the same."""
    k = 50
    s = shape_of(1, 2, d, L, 2, dtype, k=k)
    g, K, V = cache(s, [L, L], 71)
    marks = torch.randn((2, 1, L, d), generator=g)
    marks[:, :, ::5] *= 1e20
    marks[1, :, 7] = float("nan")  # a mean that is no number counts below all others
    q = torch.randn((2, 2, d), generator=g) * 1e20
    q, marks = q.to(DT[dtype]), marks.to(DT[dtype])
    out, blocks = torch.empty((2, 2, d), dtype=DT[dtype], device="cuda"), torch.empty((2, 1, 1, k), dtype=torch.int32, device="cuda")
    xb.xkv_block_decode(s, K.cuda(), V.cuda(), None, q.cuda(), 1, marks.cuda(), 1, out, blocks, workspace(s, 1, 1))
    torch.cuda.synchronize()
    marks[1, :, 7] = 0.0  # (among hundreds of positive scores neither this nor a NaN is chosen)
    for b in range(2):
        assert blocks.cpu()[b, 0, 0].tolist() == ref.choose_blocks(q[b], marks[b, 0], L, 1, k), b


def test_blocks_tie_towards_the_smaller_block():
    s = shape_of(1, 2, 128, 320, 1, "bf16", k=64)
    g, K, V = cache(s, [320], 9)
    marks = torch.ones((1, 1, 20, 128), dtype=torch.bfloat16)
    q = torch.randn((1, 1, 2, 128), generator=g).bfloat16()
    out, blocks = torch.empty_like(q).cuda(), torch.empty((1, 1, 1, 4), dtype=torch.int32, device="cuda")
    xb.xkv_block_decode(s, K.cuda(), V.cuda(), None, q.cuda(), 1, marks.cuda(), 16, out, blocks, workspace(s, 1, 16))
    assert blocks.cpu().flatten().tolist() == [0, 1, 2, 19]


@pytest.mark.parametrize("dtype,d,c,N", [("f32", 64, 7, 1), ("bf16", 128, 16, 1), ("bf16", 128, 16, 40), ("bf16", 96, 5, 1000), ("bf16", 128, 64, 3)])
def test_landmarks_update(dtype, d, c, N):
    L, lengths = 333, [333, 320, 0, 1, 17]
    s = shape_of(2, 1, d, L, len(lengths), dtype)
    _, K, _ = cache(s, lengths, 11)
    n_c = -(-L // c)
    marks = torch.full((5, 2, n_c, d), 7.0, dtype=DT[dtype], device="cuda")
    xb.xkv_landmarks_update(s, K.cuda(), ints(lengths), N, c, marks)
    got, want = marks.cpu().double(), means_of(K, lengths, c)
    for b, n in enumerate(lengths):
        first = max(0, n - N) // c
        for j in range(n_c):
            if n > 0 and first <= j <= (n - 1) // c:
                rows = K[b, :, j * c:min(n, (j + 1) * c)].double()
                # c additions and a product in fp32, rounded to the type; the reference is rounded as well
                bound = (c + 2) * 2.0 ** -24 * rows.abs().mean(1) + 2 * ref.EPS[DT[dtype]] * rows.mean(1).abs() + 1e-30
                assert ((got[b, :, j] - want[b, :, j].double()).abs() <= bound).all(), (b, j)
            else:
                assert (got[b, :, j] == 7.0).all(), (b, j)


def test_landmarks_update_agrees_with_landmarks():
    s = shape_of(2, 4, 128, 640, 1, "bf16")
    _, K, _ = cache(s, [640], 12)
    whole = torch.empty((1, 2, 40, 128), dtype=torch.bfloat16, device="cuda")
    xb.xkv_landmarks(s, K.cuda(), 16, 0, whole, None, None, None)
    marks = torch.empty_like(whole)
    xb.xkv_landmarks_update(s, K.cuda(), None, 640, 16, marks)
    near = (whole.double() - marks.double()).abs() <= 2 * 2.0 ** -8 * whole.double().abs() + 16 * 2.0 ** -24
    assert near.all()


# ----------------------------------------------------------------------------------------------------------- weights
WEIGHTS = {
    "f32_tiny": ("f32", 1, 4, 64, 512, [512], 1.0),
    "f32_odd": ("f32", 2, 3, 33, 1, [1, 0], 1.0),
    "f32_wide": ("f32", 1, 16, 256, 300, [300, 129], 1.0),
    "bf16_64": ("bf16", 2, 8, 64, 900, [900, 65], 1.0),
    "bf16": ("bf16", 2, 4, 128, 3001, [3001, 2048, 1, 0], 1.0),
    "bf16_seven_heads": ("bf16", 2, 7, 128, 1025, [1025, 1024], 1.0),
    "bf16_sixteen_heads": ("bf16", 1, 16, 128, 333, [333, 32], 1.0),
    "bf16_one_head": ("bf16", 4, 1, 128, 5000, [5000, 33], 1.0),
    "bf16_peaked": ("bf16", 2, 4, 128, 2000, [2000, 1999], 12.0),
    "bf16_long": ("bf16", 1, 4, 128, 40001, [40001], 1.0),
}


@pytest.mark.parametrize("name", list(WEIGHTS))
def test_weights(name):
    dtype, H_kv, n_rep, d, L, lengths, key_scale = WEIGHTS[name]
    s = shape_of(H_kv, n_rep, d, L, len(lengths), dtype)
    g, K, V = cache(s, lengths, 300 + len(name), key_scale)
    before = torch.rand((s.batch, H_kv, L), generator=g)
    for b, n in enumerate(lengths):
        before[b, :, n:] = float("nan")
    total, ws = before.cuda(), workspace(s)
    Kc, Vc = K.cuda(), V.cuda()
    want = before.double()
    slack = torch.zeros_like(want)
    for step in range(2):
        q = torch.randn((s.batch, s.H_q, d), generator=g).to(DT[dtype])
        out = torch.full((s.batch, s.H_q, d), float("nan"), dtype=DT[dtype], device="cuda")
        xb.xkv_dense_decode_weights(s, Kc, Vc, ints(lengths), q.cuda(), out, total, ws)
        torch.cuda.synchronize()
        for b, n in enumerate(lengths):
            for h in range(H_kv):
                heads = slice(h * n_rep, (h + 1) * n_rep)
                o, p, bound, rel = ref.attend(q[b, heads], K[b, h, :n], V[b, h, :n], torch.ones((n_rep, n), dtype=torch.bool), scale_of(s))
                within(out.cpu()[b, heads], o, bound, f"{name} {b} {h}")
                want[b, h, :n] += p.sum(0)
                # the weights' own errors (twice: the sum below the fraction has them, too), n_rep additions, one to the total
                slack[b, h, :n] += (2 * rel + (n_rep + 2) * 2.0 ** -24) * p.sum(0) + 2.0 ** -24 * want[b, h, :n]
    got = total.cpu().double()
    for b, n in enumerate(lengths):
        assert torch.isnan(got[b, :, n:]).all()  # left as they were
        assert ((got[b, :, :n] - want[b, :, :n]).abs() <= slack[b, :, :n]).all(), (name, b)


# ---------------------------------------------------------------------------------------------------------- eviction
EVICT = {
    # name: dtype, H_kv, d, L, lengths, k, sink, recent, L_out (None: in place)
    "f32_out": ("f32", 1, 64, 512, [512, 100], 128, 4, 16, 200),
    "f32_odd": ("f32", 2, 33, 70, [70, 0, 1, 20], 20, 1, 3, 20),
    "f32_odd_in_place": ("f32", 2, 33, 70, [70, 0, 1, 20], 20, 1, 3, None),
    "bf16_odd_in_place": ("bf16", 2, 33, 700, [700, 333], 321, 0, 0, None),
    "bf16_out": ("bf16", 2, 128, 3000, [3000, 2999, 1024, 1025], 1024, 4, 200, 1024),
    "bf16_in_place": ("bf16", 2, 128, 3000, [3000, 2999, 1024, 1025], 1024, 4, 200, None),
    "bf16_nothing_to_do": ("bf16", 2, 128, 300, [300, 200], 300, 0, 0, None),
    "bf16_only_protected": ("bf16", 1, 128, 300, [300, 290], 40, 10, 30, 50),
    "bf16_one_row": ("bf16", 3, 128, 300, [300], 1, 0, 0, 1),
    "bf16_most_in_place": ("bf16", 1, 128, 5000, [5000], 4900, 0, 100, None),
    "bf16_long": ("bf16", 1, 64, 70000, [70000], 9000, 4, 1000, 9001),
    "bf16_long_in_place": ("bf16", 1, 128, 20000, [20000, 16000], 17000, 4, 1000, None),
}


@pytest.mark.parametrize("name", list(EVICT))
def test_evict(name):
    dtype, H_kv, d, L, lengths, k, sink, recent, L_out = EVICT[name]
    s = shape_of(H_kv, 1, d, L, len(lengths), dtype, k=k)
    g, K, V = cache(s, lengths, 400 + len(name))
    w = torch.randn((s.batch, H_kv, L), generator=g).exp()
    w[:, :, ::3] = 0.25  # ties
    w[:, :, 1::7] = 0.0
    w[:, :, 2::14] = -0.0
    for b, n in enumerate(lengths):
        w[b, :, n:] = float("nan")
    n_dev = ints(lengths)
    src = [x.cuda() for x in (K, V, w)]
    room = L if L_out is None else L_out
    if L_out is None:
        dst = src
    else:
        dst = [torch.full((s.batch, H_kv, room, d), 3.0, dtype=DT[dtype], device="cuda") for _ in "KV"]
        dst.append(torch.full((s.batch, H_kv, room), 3.0, device="cuda"))
    rows = torch.full((s.batch, H_kv, k), -9, dtype=torch.int32, device="cuda")
    n_out = n_dev if L_out is None else torch.full_like(n_dev, -9)
    xb.xkv_evict(s, *src, n_dev, sink, recent, room, *dst, rows, n_out, workspace(s))
    torch.cuda.synchronize()
    assert n_out.tolist() == [min(n, k) for n in lengths]
    same = lambda x, y: torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))  # noqa: E731
    got = [x.cpu() for x in dst]
    for b, n in enumerate(lengths):
        for h in range(H_kv):
            keep = ref.keep_rows(w[b, h], n, k, sink, recent)
            m = len(keep)
            assert rows[b, h].tolist() == keep + [-1] * (k - m), (b, h)
            for x, y in zip(got, (K, V, w)):
                assert same(x[b, h, :m], y[b, h, keep]), (b, h)
                if L_out is not None:
                    assert (x[b, h, m:] == 3.0).all()
                else:
                    assert same(x[b, h, m:], y[b, h, m:])  # rows behind are as they were


def test_evict_without_optional_results_and_lengths():
    s = shape_of(2, 1, 128, 500, 1, "bf16", k=77)
    g, K, V = cache(s, [500], 13)
    w = torch.rand((1, 2, 500), generator=g)
    Kc, Vc, wc = K.cuda(), V.cuda(), w.cuda()
    xb.xkv_evict(s, Kc, Vc, wc, None, 0, 0, 500, Kc, Vc, wc, None, None, workspace(s))
    for h in range(2):
        keep = ref.keep_rows(w[0, h], 500, 77, 0, 0)
        assert torch.equal(Kc.cpu()[0, h, :77], K[0, h, keep]) and torch.equal(wc.cpu()[0, h, :77], w[0, h, keep])


@pytest.mark.parametrize("L,lengths", [(5000, [5000, 3000]), (20000, [20000, 700]), (40000, [40000, 1000, 900])])
def test_evict_weights_that_are_no_numbers(L, lengths):
    """Infinities and NaN of both signs are ordered by their bits like the rest, below the rows that stay anyway.  (The two NaN at either
    end of that order count as one: only one of each end is here.)"""
    k, sink, recent = 1000, 5, 300
    s = shape_of(2, 1, 16, L, len(lengths), "f32", k=k)
    g, K, V = cache(s, lengths, 61)
    w = torch.rand((s.batch, 2, L), generator=g)
    odd = torch.tensor([0x7F800000, 0x7FC00000, 0x7FFFFFFF, 0x7F800001, -0x800000, -0x400000, -1, -3], dtype=torch.int32).view(torch.float32)
    for b, n in enumerate(lengths):
        for h in range(2):
            at = torch.randperm(n, generator=g)[: n // 2 if h else 40]
            w[b, h, at] = odd[torch.randint(0, 8, (len(at),), generator=g)]
    w[0, 1, :lengths[0]] = odd[torch.randint(4, 8, (lengths[0],), generator=g)]  # nothing but negative ones
    rows = torch.full((s.batch, 2, k), -9, dtype=torch.int32, device="cuda")
    dst = [torch.zeros((s.batch, 2, k, 16), device="cuda") for _ in "KV"] + [torch.zeros((s.batch, 2, k), device="cuda")]
    xb.xkv_evict(s, K.cuda(), V.cuda(), w.cuda(), ints(lengths), sink, recent, k, *dst, rows, None, workspace(s))
    torch.cuda.synchronize()
    for b, n in enumerate(lengths):
        for h in range(2):
            keep = ref.keep_rows(w[b, h], n, k, sink, recent)
            assert rows[b, h].tolist() == keep + [-1] * (k - len(keep)), (b, h)
            assert torch.equal(dst[0].cpu()[b, h, :len(keep)], K[b, h, keep])


# ------------------------------------------------------------------------------------------------- shapes of a program
@pytest.mark.parametrize("dtype,d,batch,H_kv", [("f32", 64, 100, 1), ("bf16", 128, 100, 1), ("bf16", 128, 300, 2)])
def test_one_long_sequence_among_empty_ones(dtype, d, batch, H_kv):
    """All parts that a launch has go to one sequence."""
    L = 30000
    s = shape_of(H_kv, 2, d, L, batch, dtype)
    g = torch.Generator(device="cuda").manual_seed(15)
    K, V = (torch.zeros((batch, H_kv, L, d), dtype=DT[dtype], device="cuda") for _ in "KV")
    at = batch - 3
    K[at], V[at] = (torch.randn((H_kv, L, d), generator=g, device="cuda") for _ in "KV")
    lengths = [0] * batch
    lengths[at] = L
    q = torch.randn((batch, s.H_q, d), generator=g, device="cuda").to(DT[dtype])
    out, w = torch.full_like(q, float("nan")), torch.zeros((batch, H_kv, L), device="cuda")
    xb.xkv_dense_decode_weights(s, K, V, ints(lengths), q, out, w, workspace(s))
    rest = torch.arange(batch) != at
    assert (out.cpu()[rest] == 0).all() and (w.cpu()[rest] == 0).all()
    for h in range(H_kv):
        o, p, bound, rel = ref.attend(q.cpu()[at, 2 * h:2 * h + 2], K.cpu()[at, h], V.cpu()[at, h], torch.ones((2, L), dtype=torch.bool), scale_of(s))
        within(out.cpu()[at, 2 * h:2 * h + 2], o, bound, "long")
        assert ((w.cpu()[at, h].double() - p.sum(0)).abs() <= (2 * rel + 4 * 2.0 ** -24) * p.sum(0)).all()


def test_pointers_that_are_not_aligned_take_the_general_kernels():
    s = shape_of(1, 4, 128, 333, 1, "bf16", k=64)
    g, K, V = cache(s, [333], 16)
    q, Kd, Vd = (torch.randn(x, generator=g).bfloat16() for x in ((1, 9, 4, 128), (1, 1, 9, 128), (1, 1, 9, 128)))

    def shifted(x):  # 8 bytes behind an aligned address
        flat = torch.empty(x.numel() + 4, dtype=x.dtype, device="cuda")
        flat[4:] = x.flatten().cuda()
        return flat[4:].view(x.shape)

    out, ws = torch.full_like(q, float("nan"), device="cuda"), workspace(s, 9, 16)
    xb.xkv_tree_decode(s, shifted(K), shifted(V), None, shifted(q), shifted(Kd), shifted(Vd), None, 9, out, ws)
    check_tree(s, [333], 9, K, V, q, Kd, Vd, torch.ones((1, 9, 9), dtype=torch.bool).tril(), out.cpu(), "shifted")
    marks = means_of(K, [333], 16)
    blocks = torch.empty((1, 9, 1, 4), dtype=torch.int32, device="cuda")
    xb.xkv_block_decode(s, shifted(K), shifted(V), None, shifted(q), 9, shifted(marks), 16, out, blocks, ws)
    for i in range(9):
        want = ref.choose_blocks(q[0, i], marks[0, 0], 333, 16, 4)
        assert blocks.cpu()[0, i, 0].tolist() == want
        t = torch.tensor([j * 16 + x for j in want for x in range(16) if j * 16 + x < 333])
        o, _, bound, _ = ref.attend(q[0, i], K[0, 0, t], V[0, 0, t], torch.ones((4, len(t)), dtype=torch.bool), scale_of(s))
        within(out.cpu()[0, i], o, bound, "shifted blocks")
    w = torch.rand((1, 1, 333), generator=g)
    Ko, Vo, wo = shifted(torch.zeros((1, 1, 64, 128), dtype=torch.bfloat16)), shifted(torch.zeros((1, 1, 64, 128), dtype=torch.bfloat16)), torch.zeros((1, 1, 64), device="cuda")
    xb.xkv_evict(s, shifted(K), shifted(V), w.cuda(), None, 1, 2, 64, Ko, Vo, wo, None, None, ws)
    keep = ref.keep_rows(w[0, 0], 333, 64, 1, 2)
    assert torch.equal(Ko.cpu()[0, 0], K[0, 0, keep]) and torch.equal(Vo.cpu()[0, 0], V[0, 0, keep])


def test_a_cache_of_more_than_two_to_the_31_elements():
    """Everything is at the end of it: the last sequence's last KV head is compared."""
    batch, H_kv, L, d, N, c = 5, 4, 860000, 128, 5, 64
    s = shape_of(H_kv, 2, d, L, batch, "bf16", k=640)
    assert batch * H_kv * L * d > 2 ** 31
    g = torch.Generator(device="cuda").manual_seed(17)
    K, V = (torch.zeros((batch, H_kv, L, d), dtype=torch.bfloat16, device="cuda") for _ in "KV")
    k, v = torch.randn((L, d), generator=g, device="cuda").bfloat16(), torch.randn((L, d), generator=g, device="cuda").bfloat16()
    K[-1, -1], V[-1, -1] = k, v
    lengths = ints([1, 0, 5, 64, L])
    q = torch.randn((batch, N, s.H_q, d), generator=g, device="cuda").bfloat16()
    Kd, Vd = (torch.randn((batch, H_kv, N, d), generator=g, device="cuda").bfloat16() for _ in "KV")
    ws, out = workspace(s, N, c), torch.full_like(q, float("nan"))
    xb.xkv_tree_decode(s, K, V, lengths, q, Kd, Vd, None, N, out, ws)
    mask = torch.cat((torch.ones((N, L), dtype=torch.bool), torch.ones((N, N), dtype=torch.bool).tril()), 1).repeat_interleave(2, 0)
    o, _, bound, _ = ref.attend(q[-1, :, 6:].reshape(-1, d).cpu(), torch.cat((k, Kd[-1, -1])).cpu(), torch.cat((v, Vd[-1, -1])).cpu(), mask, scale_of(s))
    within(out[-1, :, 6:].reshape(-1, d).cpu(), o, bound, "tree")
    w = torch.zeros((batch, H_kv, L), device="cuda")
    q1, out1 = q[:, 0].contiguous(), torch.full((batch, s.H_q, d), float("nan"), dtype=torch.bfloat16, device="cuda")
    xb.xkv_dense_decode_weights(s, K, V, lengths, q1, out1, w, ws)
    o, p, bound, rel = ref.attend(q1[-1, 6:].cpu(), k.cpu(), v.cpu(), torch.ones((2, L), dtype=torch.bool), scale_of(s))
    within(out1[-1, 6:].cpu(), o, bound, "weights")
    assert ((w[-1, -1].cpu().double() - p.sum(0)).abs() <= (2 * rel + 4 * 2.0 ** -24) * p.sum(0)).all()
    marks = torch.zeros((batch, H_kv, -(-L // c), d), dtype=torch.bfloat16, device="cuda")
    xb.xkv_landmarks_update(s, K, lengths, L, c, marks)
    blocks = torch.empty((batch, 1, H_kv, 10), dtype=torch.int32, device="cuda")
    xb.xkv_block_decode(s, K, V, lengths, q1, 1, marks, c, out1, blocks, ws)
    want = ref.choose_blocks(q1[-1, 6:].cpu(), marks[-1, -1].cpu(), L, c, 10)
    assert blocks[-1, 0, -1].tolist() == want
    t = torch.tensor([j * c + x for j in want for x in range(c) if j * c + x < L])
    o, _, bound, _ = ref.attend(q1[-1, 6:].cpu(), k.cpu()[t], v.cpu()[t], torch.ones((2, len(t)), dtype=torch.bool), scale_of(s))
    within(out1[-1, 6:].cpu(), o, bound, "blocks")
    keep = ref.keep_rows(w[-1, -1].cpu(), L, 640, 4, 100)
    rows = torch.empty((batch, H_kv, 640), dtype=torch.int32, device="cuda")
    xb.xkv_evict(s, K, V, w, lengths, 4, 100, L, K, V, w, rows, None, ws)
    assert rows[-1, -1].tolist() == keep
    assert torch.equal(K[-1, -1, :640], k[torch.tensor(keep, device="cuda")]) and torch.equal(V[-1, -1, :640], v[torch.tensor(keep, device="cuda")])
    assert torch.equal(K[-1, -1, 640:], k[640:])


# ---------------------------------------------------------------------------------------------------------- together
def serve(s, c, N, steps, state, stream=None):
    """Draft, verify, append, decode with weights, evict, refresh the block means, decode sparsely; all on device lengths."""
    K, V, w, n, marks, ws = (state[x] for x in ("K", "V", "w", "n", "marks", "ws"))
    at = torch.arange(s.batch, device="cuda")
    for q, Kd, Vd, words, q1 in steps:
        xb.xkv_tree_decode(s, K, V, n, q, Kd, Vd, words, N, state["tree_out"], ws, stream)
        for j in (0, 1):  # two drafted tokens are accepted
            K[at, :, n.long()] = Kd[:, :, j]
            V[at, :, n.long()] = Vd[:, :, j]
            w[at, :, n.long()] = state["zero"]
            n += 1
        xb.xkv_dense_decode_weights(s, K, V, n, q1, state["out"], w, ws, stream)
        xb.xkv_evict(s, K, V, w, n, 2, 16, s.L, K, V, w, None, n, ws, stream)
        xb.xkv_landmarks_update(s, K, n, s.L, c, marks, stream)
        xb.xkv_block_decode(s, K, V, n, q1, 1, marks, c, state["block_out"], None, ws, stream)


def loop_state(s, c, N, lengths, seed):
    g, K, V = cache(s, lengths, seed)
    dt = DT[s.dtype]
    w = torch.rand((s.batch, s.H_kv, s.L), generator=g)
    steps = []
    for _ in range(3):
        x = [torch.randn((s.batch, N, s.H_q, s.d_h), generator=g), torch.randn((s.batch, s.H_kv, N, s.d_h), generator=g),
             torch.randn((s.batch, s.H_kv, N, s.d_h), generator=g)]
        steps.append([t.to(dt).cuda() for t in x] + [ref.pack_mask(random_trees(g, s.batch, N)).cuda(),
                                                      torch.randn((s.batch, s.H_q, s.d_h), generator=g).to(dt).cuda()])
    n_c = -(-s.L // c)
    state = dict(zero=torch.zeros((s.batch, s.H_kv), device="cuda"), K=K.cuda(), V=V.cuda(), w=w.cuda(), n=ints(lengths), ws=workspace(s, N, c),
                 marks=torch.zeros((s.batch, s.H_kv, n_c, s.d_h), dtype=dt, device="cuda"),
                 tree_out=torch.empty((s.batch, N, s.H_q, s.d_h), dtype=dt, device="cuda"),
                 out=torch.empty((s.batch, s.H_q, s.d_h), dtype=dt, device="cuda"),
                 block_out=torch.empty((s.batch, s.H_q, s.d_h), dtype=dt, device="cuda"))
    return state, steps


@pytest.mark.parametrize("dtype,d,n_rep", [("bf16", 128, 4), ("f32", 64, 2)])
def test_a_serving_loop(dtype, d, n_rep):
    """The last step of the loop, from the state that the kernels left before it."""
    c, N, lengths = 16, 6, [200, 190]
    s = shape_of(2, n_rep, d, 256, 2, dtype, k=192)
    state, steps = loop_state(s, c, N, lengths, 21)
    serve(s, c, N, steps[:2], state)
    torch.cuda.synchronize()
    assert state["n"].tolist() == [192, 192]
    K, V, w, n = (state[x].cpu().clone() for x in ("K", "V", "w", "n"))
    q, Kd, Vd, words, q1 = (x.cpu() for x in steps[2])
    serve(s, c, N, steps[2:], state)
    torch.cuda.synchronize()
    sees = torch.stack([ref.tree_mask(words[b], N) for b in range(2)])
    check_tree(s, n.tolist(), N, K, V, q, Kd, Vd, sees, state["tree_out"].cpu(), "loop")
    for b in range(2):
        for h in range(2):
            heads = slice(h * n_rep, (h + 1) * n_rep)
            k2, v2 = torch.cat((K[b, h, :192], Kd[b, h, :2])), torch.cat((V[b, h, :192], Vd[b, h, :2]))
            all_rows = torch.ones((n_rep, 194), dtype=torch.bool)
            o, p, bound, rel = ref.attend(q1[b, heads], k2, v2, all_rows, scale_of(s))
            within(state["out"].cpu()[b, heads], o, bound, "loop: one token")
            # which rows stay, from the weights as the kernel left them is not visible any more: the kept ones are its own, in order
            kept_w = torch.cat((w[b, h, :192].double(), torch.zeros(2).double())) + p.sum(0)
            got_w = state["w"].cpu()[b, h, :192].double()
            keep = ref.keep_rows(kept_w.float(), 194, 192, 2, 16)
            assert ((got_w - kept_w[keep]).abs() <= (2 * rel + 1e-6) * kept_w[keep] + 1e-7).all()
            assert torch.equal(state["K"].cpu()[b, h, :192], k2[keep]) and torch.equal(state["V"].cpu()[b, h, :192], v2[keep])
            k3, v3, marks = state["K"].cpu()[b, h], state["V"].cpu()[b, h], state["marks"].cpu()[b, h]
            rows = torch.tensor([j * c + x for j in ref.choose_blocks(q1[b, heads], marks, 192, c, 12) for x in range(c)])
            o, _, bound, _ = ref.attend(q1[b, heads], k3[rows], v3[rows], torch.ones((n_rep, len(rows)), dtype=torch.bool), scale_of(s))
            within(state["block_out"].cpu()[b, heads], o, bound, "loop: blocks")


def test_the_loop_on_another_stream_and_in_a_graph():
    """Two captured loops with workspaces of their own, replayed in turn, against eager runs from the same states."""
    c, N = 16, 40
    s = shape_of(2, 4, 128, 320, 2, "bf16", k=192)
    names = ("K", "V", "w", "n", "marks", "tree_out", "out", "block_out")
    cases = [loop_state(s, c, N, lengths, 31 + i) for i, lengths in enumerate(([280, 200], [200, 64]))]
    start = [{x: st[x].clone() for x in names} for st, _ in cases]

    def reset(i):
        for x in names:
            cases[i][0][x].copy_(start[i][x])

    want = []
    for i, (st, steps) in enumerate(cases):
        serve(s, c, N, steps, st)
        torch.cuda.synchronize()
        want.append({x: st[x].clone() for x in names})
    same = lambda x, y: torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8))  # noqa: E731
    side = torch.cuda.Stream()
    graphs = []
    for i, (st, steps) in enumerate(cases):
        reset(i)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            serve(s, c, N, steps, st)  # eager on another stream
        side.synchronize()
        for x in names:
            assert same(st[x], want[i][x]), (i, x, "another stream")
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            serve(s, c, N, steps, st)
        graphs.append(graph)
    for replay in range(3):
        for i in (0, 1):
            reset(i)
        torch.cuda.synchronize()
        graphs[0].replay()
        graphs[1].replay()
        torch.cuda.synchronize()
        for i, (st, _) in enumerate(cases):
            for x in names:
                assert same(st[x], want[i][x]), (replay, i, x)


def test_results_do_not_change_from_call_to_call():
    s = shape_of(2, 4, 128, 5000, 2, "bf16")
    g, K, V = cache(s, [5000, 3333], 41)
    q = torch.randn((2, 20, 8, 128), generator=g).bfloat16()
    Kd, Vd = (torch.randn((2, 2, 20, 128), generator=g).bfloat16() for _ in "KV")
    words = ref.pack_mask(random_trees(g, 2, 20)).cuda()
    first = run_tree(s, ints([5000, 3333]), 20, K, V, q, Kd, Vd, words)
    dev = [x.cuda() for x in (K, V, q, Kd, Vd)]
    ws, n = workspace(s, 20), ints([5000, 3333])
    for _ in range(50):
        out = torch.full_like(first, float("nan"), device="cuda")
        xb.xkv_tree_decode(s, dev[0], dev[1], n, dev[2], dev[3], dev[4], words, 20, out, ws)
        assert torch.equal(out.cpu(), first)
