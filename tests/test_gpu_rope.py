"""xkv_rotate and xkv_rope_frequencies through the C ABI against a plain implementation in double precision (cache8_reference.py, which
also derives the tolerances)."""
import pytest
import torch

import cache8_reference as ref
from paper_2503_18893_amd import binding as xb

pytestmark = pytest.mark.gpu

DT = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(autouse=True)
def need_gpu():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")


def shape_of(H_kv, n_rep, d, batch, dtype):
    return xb.Shape(1, H_kv, H_kv * n_rep, d, 1, 1, 1, 1, batch, dtype)


def within(got, want, bound, what):
    err = (got.double().cpu() - want).abs()
    assert torch.isfinite(got.double()).all(), what
    assert (err <= bound).all(), f"{what}: {(err / bound.clamp_min(1e-300)).max().item():.3g} of the bound, largest error {err.max().item():.3g}"


SCALINGS = {"plain": (), "linear": (4.0,), "base": (8.0,), "turns": (8.0, 1.0, 4.0, 8192.0)}


@pytest.mark.parametrize("scaling", list(SCALINGS))
@pytest.mark.parametrize("d_rot,theta", [(128, 500000.0), (64, 10000.0), (6, 1e6), (256, 2.0)])
def test_frequencies(scaling, d_rot, theta):
    f = torch.full((d_rot // 2 + 1,), -1.0, dtype=torch.float64, device="cuda")
    more = SCALINGS[scaling] + (0.0,) * (4 - len(SCALINGS[scaling]))
    xb.xkv_rope_frequencies(d_rot, theta, scaling, *more, f)
    want = ref.frequencies(d_rot, theta, scaling, *SCALINGS[scaling])
    # a power in double precision: a relative error of its logarithm, at most 13, by 2^-53, and a few roundings
    assert (f.cpu()[:-1] / want - 1).abs().max() < 40 * 2.0 ** -52
    assert f[-1] == -1.0


CASES = {
    # name: dtype, H_kv, n_rep, d, d_rot, layout, batch, N, first position
    "f32_tiny": ("f32", 1, 4, 64, 64, "half", 1, 1, 0),
    "f32_two_channels": ("f32", 1, 1, 2, 2, "interleaved", 2, 3, 5),
    "f32_odd_width": ("f32", 2, 3, 33, 6, "half", 2, 7, 100),
    "f32_pairs_of_neighbours": ("f32", 2, 2, 96, 96, "interleaved", 1, 19, 1 << 20),
    "f32_wide": ("f32", 1, 2, 256, 256, "half", 2, 65, 70000),
    "bf16_step": ("bf16", 8, 4, 128, 128, "half", 3, 1, 65535),
    "bf16_far": ("bf16", 2, 7, 128, 128, "half", 1, 33, (1 << 31) - 40),
    "bf16_part": ("bf16", 2, 7, 128, 64, "half", 2, 31, 1000),
    "bf16_part_of_neighbours": ("bf16", 4, 7, 128, 32, "interleaved", 2, 50, 40000),
    "bf16_neighbours": ("bf16", 2, 4, 128, 128, "interleaved", 1, 9, 7),
    "bf16_no_whole_pieces": ("bf16", 3, 2, 80, 20, "half", 2, 21, 9),
    "bf16_odd_width": ("bf16", 1, 3, 127, 126, "interleaved", 2, 13, 9),
    "bf16_prompt": ("bf16", 8, 4, 128, 128, "half", 2, 1500, 0),
}


def run(case, direction, amplitude=1.0, seed=0, views=False):
    dtype, H_kv, n_rep, d, d_rot, layout, batch, N, first = CASES[case]
    g = torch.Generator().manual_seed(seed)
    s, H_q = shape_of(H_kv, n_rep, d, batch, dtype), H_kv * n_rep
    x = torch.randn((batch, N, H_q + 2 * H_kv, d), generator=g).to(DT[dtype]).cuda()
    q, K = x[:, :, :H_q], x[:, :, H_q:H_q + H_kv]
    if not views:
        q, K = q.contiguous(), K.contiguous()
    p = first + torch.arange(N) + torch.randint(0, 5, (batch, 1), generator=g)
    p[0, N // 2] = -3  # any number
    p = p.to(torch.int32)
    f = ref.frequencies(d_rot, 500000.0, "turns", 8.0, 1.0, 4.0, 8192.0)
    q_out = torch.full((batch, N, H_q, d), float("nan"), dtype=DT[dtype], device="cuda")
    K_out = torch.full((batch, H_kv, N, d), float("nan"), dtype=DT[dtype], device="cuda").transpose(1, 2)
    xb.xkv_rotate(s, d_rot, layout, direction, amplitude, f.cuda(), p.cuda(), N, q, q_out, K, K_out)
    for name, a, b in (("q", q, q_out), ("K", K, K_out)):
        want, bound = ref.rotate(a.cpu(), p, f, layout, direction, amplitude)
        within(b, want, bound, f"{case} {direction} {name}")


@pytest.mark.parametrize("direction", ["forward", "inverse", "gradient"])
@pytest.mark.parametrize("case", list(CASES))
def test_rotate(case, direction):
    run(case, direction, 1.25, len(case))


@pytest.mark.parametrize("case", ["bf16_step", "bf16_part", "f32_odd_width", "bf16_neighbours", "bf16_prompt"])
def test_slices_of_a_projection(case):
    run(case, "forward", 1.0, 3, views=True)


def test_amplitude_of_zero_is_one_and_positions_are_counted():
    s = shape_of(2, 2, 64, 2, "f32")
    x = torch.randn((2, 5, 4, 64), device="cuda")
    f = ref.frequencies(64, 1e4).cuda()
    p = torch.arange(5, dtype=torch.int32, device="cuda").repeat(2, 1)
    a, b = torch.empty_like(x), torch.empty_like(x)
    xb.xkv_rotate(s, 64, "half", "forward", 0.0, f, None, 5, x, a, None, None)
    xb.xkv_rotate(s, 64, "half", "forward", 1.0, f, p, 5, x, b, None, None)
    assert torch.equal(a, b)


def test_inverse_undoes_and_gradient_is_the_transpose():
    s = shape_of(1, 3, 128, 2, "f32")
    g = torch.Generator().manual_seed(1)
    x, y = (torch.randn((2, 9, 3, 128), generator=g).cuda() for _ in "xy")
    f = ref.frequencies(96, 1e4).cuda()
    p = torch.randint(0, 1 << 20, (2, 9), generator=g).to(torch.int32).cuda()

    def rotated(z, direction):
        out = torch.empty_like(z)
        xb.xkv_rotate(s, 96, "interleaved", direction, 1.5, f, p, 9, z, out, None, None)
        return out

    # two rotations, each off by 2^-21 of a pair's sum of magnitudes and three roundings (ref.rotate)
    reach = (x[..., 0:96:2].abs() + x[..., 1:96:2].abs()).max().item()
    assert (rotated(rotated(x, "forward"), "inverse") - x).abs().max() <= 4 * (2.0 ** -21 + 4 * 2.0 ** -24) * reach
    lhs, rhs = (rotated(x, "forward").double() * y).sum(), (x.double() * rotated(y, "gradient")).sum()
    assert (lhs - rhs).abs() <= 2 * 1.5 * 2 * (2.0 ** -21 + 4 * 2.0 ** -24) * (x.abs().double() * y.abs().max()).sum()
    # differences, in the directions of single channels: the rotation is linear, so a step of one is exact but for rounding
    e = torch.zeros_like(x)
    e[1, 4, 2, 7] = 1.0
    assert ((rotated(x + e, "forward") - rotated(x, "forward")).double() * y).sum().sub(rotated(y, "gradient")[1, 4, 2, 7]).abs() <= 2e-4


@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_in_place_and_with_rows_of_a_cache(layout, dtype):
    s = shape_of(2, 2, 128, 2, dtype)
    x = torch.randn((2, 2, 40, 128), device="cuda").to(DT[dtype])
    f = ref.frequencies(64, 1e4).cuda()
    rows = x.transpose(1, 2)[:, 10:31]      # rows 10 .. 30 of a cache [batch][H_kv][L][d]
    want = torch.empty((2, 21, 2, 128), dtype=DT[dtype], device="cuda")
    xb.xkv_rotate(s, 64, layout, "forward", 1.0, f, None, 21, None, None, rows, want)
    before = x.clone()
    xb.xkv_rotate(s, 64, layout, "forward", 1.0, f, None, 21, None, None, rows, rows)
    assert torch.equal(rows, want)
    assert torch.equal(x[:, :, :10], before[:, :, :10]) and torch.equal(x[:, :, 31:], before[:, :, 31:])
    assert torch.equal(x[..., 64:], before[..., 64:])


def test_broadcast_queries_and_rows_that_are_not_aligned():
    s = shape_of(2, 2, 64, 3, "bf16")
    f = ref.frequencies(64, 1e4)
    one = torch.randn((1, 1, 4, 64), device="cuda").bfloat16()
    out = torch.empty((3, 6, 4, 64), dtype=torch.bfloat16, device="cuda")
    p = torch.randint(0, 1000, (3, 6)).to(torch.int32)
    xb.xkv_rotate(s, 64, "half", "forward", 1.0, f.cuda(), p.cuda(), 6, one.expand(3, 6, 4, 64), out, None, None)
    want, bound = ref.rotate(one.expand(3, 6, 4, 64).cpu(), p, f, "half", "forward", 1.0)
    within(out, want, bound, "broadcast")
    odd = torch.randn(3 * 6 * 4 * 65 + 8, device="cuda").bfloat16()[3:].as_strided((3, 6, 4, 64), (6 * 4 * 65, 4 * 65, 65, 1))
    xb.xkv_rotate(s, 64, "half", "forward", 1.0, f.cuda(), p.cuda(), 6, odd, out, None, None)
    want, bound = ref.rotate(odd.cpu(), p, f, "half", "forward", 1.0)
    within(out, want, bound, "not aligned")


def test_infinities_and_nan_stay_in_their_pairs():
    s = shape_of(1, 1, 64, 1, "bf16")
    x = torch.randn((1, 4, 1, 64), device="cuda").bfloat16()
    x[0, 1, 0, 3] = float("nan")
    x[0, 2, 0, 40] = float("inf")
    out = torch.empty_like(x)
    xb.xkv_rotate(s, 32, "half", "forward", 1.0, ref.frequencies(32, 1e4).cuda(), None, 4, x, out, None, None)
    bad = ~torch.isfinite(out)
    want = torch.zeros_like(bad)
    want[0, 1, 0, [3, 19]] = True
    want[0, 2, 0, 40] = True  # not turned
    assert torch.equal(bad, want) and out[0, 1, 0, 3].isnan() and out[0, 2, 0, 40] == float("inf")


def test_more_workgroups_than_a_launch_has_in_one_direction():
    """2^27 tokens and more of one pair, eight a workgroup of 256 threads: 2^32 threads."""
    N = (1 << 27) + 101
    s = shape_of(1, 1, 2, 1, "bf16")
    x = torch.randn((1, N, 1, 2), device="cuda").bfloat16()
    f = ref.frequencies(2, 1e4)
    out = torch.empty_like(x)
    xb.xkv_rotate(s, 2, "half", "forward", 1.0, f.cuda(), None, N, x, out, None, None)
    for start in (0, (1 << 25) - 50, (1 << 26) - 50, (1 << 27) - 50, N - 100):
        p = torch.arange(start, start + 100)
        want, bound = ref.rotate(x[:, start:start + 100].cpu(), p[None].to(torch.int32), f, "half", "forward", 1.0)
        within(out[:, start:start + 100], want, bound, f"tokens from {start}")
