"""xkv_cache8_decode on caches that several workgroups share, each a part of the rows, and their merge: what a part of no weight says (NaN), queries
and scales that are NaN, parts without rows for some of the queries, and a captured step.  Every test asks for room for partials first, so
that it is the merge that answers."""
import pytest
import torch

import cache8_reference as ref8
from paper_2503_18893_amd import binding as xb
from test_gpu_cache8_attend import DT, cache, check, run, shape_of, workspace

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def several_parts(s, N):
    """Whether there are partials: a workspace has more than the table of the sequences' parts."""
    return xb.xkv_cache8_workspace_bytes(s, N) > (4 * (s.batch + 1) + 255) // 256 * 256


# dtype, d, queries, rows of a block, KV heads, sequences: streams of 16 and 32 rows, tiles of 256 rows, blocks of one row, single precision, the general kernel;
# the last has as many workgroups of a part as the card has places, so that parts are not cut by the lengths
KINDS = [("bf16", 128, 1, 16, 2, 2), ("bf16", 128, 5, 16, 2, 2), ("bf16", 128, 50, 32, 2, 2), ("bf16", 64, 5, 4, 2, 2), ("bf16", 256, 2, 64, 2, 2), ("bf16", 128, 3, 1, 2, 2),
         ("f32", 128, 3, 16, 2, 2), ("f32", 64, 2, 2, 2, 2), ("bf16", 48, 3, 8, 2, 2), ("f32", 96, 1, 32, 2, 2), ("bf16", 128, 1, 16, 1, 1), ("f32", 40, 2, 4, 1, 1),
         ("bf16", 64, 64, 16, 2, 33)]


def leading_key(state, code, c, b, g, t, q):
    """Row t of sequence b and KV head g leads all others by more than 110 in the logits of all queries, so that others weigh less than 2^-149
    of it: its block's keys are zeros but for channel 0, where every query is 1."""
    q[..., 0] = 1.0
    n0 = t // c * c
    codes = state[0][b, g, n0:n0 + c]
    codes.view(torch.uint8).zero_()
    state[0][b, g, t, 0] = ref8.encode(torch.tensor(ref8.HIGHEST[code]), code)
    state[2][b, g, t // c] = 250.0 / ref8.HIGHEST[code] * q.shape[-1] ** 0.5  # a logit of 250; those of the others are below 100 (asserted)


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,d,N,c,H_kv,batch", KINDS)
def test_nan_in_a_part_of_no_weight(dtype, d, N, c, H_kv, batch, code):
    """One key far larger than all others, and a NaN among the values of another part: its weight is zero in single precision, and zero times NaN is
    NaN, as it is where one workgroup takes all rows."""
    L = 3000
    s = shape_of(H_kv, 4, d, L, batch, dtype)
    assert several_parts(s, N)
    n = [L - 40] * batch
    seen = [[n[b] - N + 1 + i for i in range(N)] for b in range(batch)]
    g, *state = cache(s, code, c, n, 21, 0.2)
    q = torch.randn((batch, N, 4 * H_kv, d), generator=g).to(DT[dtype])
    last, h = batch - 1, H_kv - 1
    for hot, odd in ((7, n[last] - 1), (7, 2001), (n[last] - N, 9)):
        now = [x.clone() for x in state]
        qs = q.clone()
        leading_key(now, code, c, last, h, hot, qs)
        K = ref8.rows(now[0], now[2], c)[last, h, :n[last]]
        z = (qs[last, :, 4 * h:].double().reshape(-1, d) @ K.T) / d ** 0.5
        assert ((z.max(1).values == z[:, hot]) & (z.topk(2).values.diff().squeeze(1) < -110)).all()
        clean = run(s, code, c, seen, qs, now)
        check(s, code, c, seen, qs, now, clean, f"leading row {hot}")
        for what in ("scale",) + (("code",) if code == "e4m3" else ()):
            bad = [x.clone() for x in now]
            if what == "scale":
                bad[3][last, h, odd // c] = float("nan")
                t, ch = odd // c * c, slice(None)
            else:
                bad[1].view(torch.uint8)[last, h, odd, d - 1] = 0x7F
                t, ch = odd, d - 1
            out = run(s, code, c, seen, qs, bad)
            hit = torch.zeros_like(clean, dtype=torch.bool)
            for i in range(N):
                if t < seen[last][i]:
                    hit[last, i, 4 * h:, ch] = True
            assert torch.equal(out.isnan(), hit), (hot, odd, what)
            assert torch.equal(out[~hit], clean[~hit]), (hot, odd, what)


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype,d,N,c,H_kv,batch", KINDS)
def test_nan_reaches_those_that_see_it(dtype, d, N, c, H_kv, batch, code):
    """Scales, codes and queries that are NaN, among rows of ordinary weight."""
    L = 3000
    s = shape_of(H_kv, 4, d, L, batch, dtype)
    assert several_parts(s, N)
    seen = [[L - N + 1 + i - 700 * (b % 4) for i in range(N)] for b in range(batch)]
    g, *state = cache(s, code, c, [max(x) for x in seen], 22)
    q = torch.randn((batch, N, 4 * H_kv, d), generator=g).to(DT[dtype])
    clean = run(s, code, c, seen, q, state)
    check(s, code, c, seen, q, state, clean, "clean")
    last, h = batch - 1, H_kv - 1
    for what in ("k_scale", "v_scale") + (("k_code", "v_code") if code == "e4m3" else ()):
        for t in (5, 1300, seen[last][N // 2] - 1):
            bad = [x.clone() for x in state]
            if what.endswith("scale"):
                bad[2 if what[0] == "k" else 3][last, h, t // c] = float("nan")
                t = t // c * c
            else:
                bad[0 if what[0] == "k" else 1].view(torch.uint8)[last, h, t, 7] = 0xFF
            out = run(s, code, c, seen, q, bad)
            hit = torch.zeros_like(clean, dtype=torch.bool)
            for i in range(N):
                if t < seen[last][i]:
                    hit[last, i, 4 * h:, 7 if what == "v_code" else slice(None)] = True
            assert torch.equal(out.isnan(), hit), (what, t)
            assert torch.equal(out[~hit], clean[~hit]), (what, t)
    odd = q.clone()
    odd[last, N - 1, 1, 3] = float("nan")
    out = run(s, code, c, seen, odd, state)
    assert out[last, N - 1, 1].isnan().all() and out.isnan().sum() == d
    out[last, N - 1, 1] = clean[last, N - 1, 1]
    check(s, code, c, seen, q, state, out, "the other queries")  # (not equal: rows of a wavefront raise their maxima together)


@pytest.mark.parametrize("dtype,d,N", [("bf16", 128, 4), ("bf16", 128, 60), ("f32", 64, 3), ("bf16", 80, 3)])
@pytest.mark.parametrize("batch", [1, 3])
def test_queries_that_see_no_row_of_most_parts(dtype, d, N, batch):
    """The first queries see nothing or one row, the last ones all; rows of the workspace that no workgroup writes hold NaN (workspace())."""
    L, code, c = 4000, "e4m3", 16
    s = shape_of(1, 4, d, L, batch, dtype)
    assert several_parts(s, N)
    seen = [[0, 1] + [L - 500 * b] * (N - 2) for b in range(batch)]
    g, *state = cache(s, code, c, [max(x) for x in seen], 23)
    q = torch.randn((batch, N, 4, d), generator=g).to(DT[dtype])
    check(s, code, c, seen, q, state, run(s, code, c, seen, q, state), "few rows")
    seen = [[0] * N] + [[L] * N] * (batch - 1)
    _, *state = cache(s, code, c, [max(x) for x in seen], 24)
    check(s, code, c, seen, q, state, run(s, code, c, seen, q, state), "an empty sequence")


def test_a_captured_step_that_merges():
    """Rotate, append and attend as a serving loop does, on a cache of several parts, captured once and replayed for token after token; every replay
    against the same calls made one by one, with other work between."""
    s, c, code, n0 = shape_of(2, 4, 128, 2500, 2, "bf16"), 32, "int8", [2000, 777]
    assert several_parts(s, 1)
    g = torch.Generator().manual_seed(5)
    f = ref8.frequencies(128, 1e4).cuda()
    _, *start = cache(s, code, c, n0, 25)
    for x in start[2:]:
        x.nan_to_num_(0.0)

    def fresh():
        return dict(state=[x.cuda() for x in start], lengths=torch.tensor(n0, dtype=torch.int32, device="cuda"), ws=workspace(s),
                    qkv=torch.zeros((2, 1, 12, 128), dtype=torch.bfloat16, device="cuda"), q=torch.zeros((2, 1, 8, 128), dtype=torch.bfloat16, device="cuda"),
                    K=torch.zeros((2, 1, 2, 128), dtype=torch.bfloat16, device="cuda"), out=torch.zeros((2, 1, 8, 128), dtype=torch.bfloat16, device="cuda"))

    def step(t):
        x = t["qkv"]
        xb.xkv_rotate(s, 128, "half", "forward", 1.0, f, t["lengths"], 1, x[:, :, :8], t["q"], x[:, :, 8:10], t["K"])
        xb.xkv_cache8_append(s, t["K"], x[:, :, 10:], t["lengths"], None, 1, code, c, *t["state"])
        t["lengths"] += 1
        xb.xkv_cache8_decode(s, *t["state"], code, c, t["lengths"], t["q"], 1, t["out"], t["ws"])

    eager, held, graph = fresh(), fresh(), torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        step(held)
    for i in range(40):
        x = torch.randn((2, 1, 12, 128), generator=g).bfloat16()
        for t in (eager, held):
            t["qkv"].copy_(x)
        step(eager)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager["state"] + [eager["out"], eager["lengths"]], held["state"] + [held["out"], held["lengths"]]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), i
    check(s, code, c, [[2040], [817]], eager["q"].cpu(), [x.cpu() for x in eager["state"]], eager["out"].cpu(), "serving")
