"""xkv_cache8_append through the C ABI: codes and scales are those of a plain implementation (cache8_reference.py), bit for bit, and nothing
else is written."""
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


def shape_of(H_kv, d, L, batch, dtype):
    return xb.Shape(1, H_kv, H_kv, d, 1, 1, L, 1, batch, dtype)


def empty(s, c, code, seed):
    """K8, V8, k_scales, v_scales on the CPU: anything."""
    g = torch.Generator().manual_seed(seed)
    n_c = -(-s.L // c)
    return [torch.randint(0, 256, (s.batch, s.H_kv, s.L, s.d_h), generator=g).to(torch.uint8).view(ref.TYPE[code]) for _ in "KV"] + \
           [torch.randn((s.batch, s.H_kv, n_c), generator=g).abs() for _ in "KV"]


def both(s, K, V, lengths, counts, code, c, state, views=None):
    """One append by the library, on the state on the GPU, and by the reference, on the one on the CPU."""
    N = K.shape[1]
    dev = [x.cuda() for x in state]
    ints = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    Kd, Vd = (K.cuda(), V.cuda()) if views is None else views
    xb.xkv_cache8_append(s, Kd, Vd, ints(lengths), ints(counts), N, code, c, *dev)
    for new, codes, scales in ((K, state[0], state[2]), (V, state[1], state[3])):
        for b in range(s.batch):
            for g in range(s.H_kv):
                ref.append(new[b, :, g].float(), lengths[b] if lengths else 0, counts[b] if counts else N, codes[b, g], scales[b, g], c, code)
    return dev


def same(dev, state, what):
    for name, x, y in zip(("K8", "V8", "k_scales", "v_scales"), dev, state):
        kind = torch.uint8 if name.endswith("8") else torch.int32  # (bits: NaN too)
        x, y = x.cpu().view(kind), y.view(kind)
        assert torch.equal(x, y), f"{what} {name}: {(x != y).sum().item()} of {x.numel()} differ, first at {(x != y).nonzero()[0].tolist()}"


CASES = {
    # name: dtype, H_kv, d, L, c, N, lengths, counts
    "f32_tiny": ("f32", 1, 64, 512, 16, 1, [100], None),
    "f32_one_of_everything": ("f32", 1, 1, 1, 1, 1, None, None),
    "f32_odd_width": ("f32", 2, 33, 70, 4, 9, [61, 0, 70], [9, 5, 9]),
    "f32_wide": ("f32", 1, 256, 200, 64, 130, [63, 65], None),
    "bf16_step": ("bf16", 8, 128, 1000, 32, 1, [0, 31, 32, 999, 1000], None),
    "bf16_every_row_its_own": ("bf16", 2, 128, 300, 1, 40, [0, 17], None),
    "bf16_pairs": ("bf16", 2, 64, 301, 2, 41, [0, 18], [40, 41]),
    "bf16_padded": ("bf16", 2, 128, 2000, 32, 100, [5, 1990, 640, 0], [100, 50, 0, 1]),
    "bf16_prompt": ("bf16", 4, 128, 1500, 64, 1500, [0, 0], [1500, 777]),
    "bf16_from_odd_places": ("bf16", 2, 128, 1100, 16, 1001, [99, 3, 50], None),
    "bf16_large_blocks": ("bf16", 2, 128, 3000, 1024, 2000, [1000, 1024], None),
    "bf16_one_block": ("bf16", 1, 96, 100, 1 << 30, 30, [70, 50], None),
    "bf16_odd_width": ("bf16", 3, 80, 90, 8, 17, [2, 80], None),
}


@pytest.mark.parametrize("code", ["e4m3", "int8"])
@pytest.mark.parametrize("case", list(CASES))
def test_append(case, code):
    dtype, H_kv, d, L, c, N, lengths, counts = CASES[case]
    batch = len(lengths) if lengths else 1
    s = shape_of(H_kv, d, L, batch, dtype)
    g = torch.Generator().manual_seed(len(case))
    state = empty(s, c, code, 7)
    for x in state[2:]:
        x.mul_(0.01)
    for x in state[:2]:  # (rows in use hold numbers)
        if code == "e4m3":
            x.view(torch.uint8).masked_fill_((x.view(torch.uint8) & 0x7F) == 0x7F, 0x7E)
    K, V = (torch.randn((batch, N, H_kv, d), generator=g).mul(torch.randn((batch, N, 1, 1), generator=g).mul(2).exp()).to(DT[dtype]) for _ in "KV")
    dev = both(s, K, V, lengths, counts, code, c, state)
    same(dev, state, case)


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_a_cache_that_grows_by_steps(code):
    """Rows one or a few at a time, ever larger, from an empty cache: the same codes all the way, and no row off by more than one step."""
    s, c, g = shape_of(2, 128, 200, 2, "bf16"), 16, torch.Generator().manual_seed(3)
    state, n, kept = empty(s, c, code, 1), [0, 5], []
    both_n = [0, 5]
    for step in range(12):
        N = 1 + step % 4
        K, V = (torch.randn((2, N, 2, 128), generator=g).mul(1.3 ** step).bfloat16() for _ in "KV")
        dev = both(s, K, V, both_n, None, code, c, state)
        same(dev, state, f"step {step}")
        state = [x.cpu() for x in dev]
        kept.append((list(both_n), K))
        both_n = [x + N for x in both_n]
    values = ref.rows(state[0], state[2], c)
    for at, K in kept:
        for b in range(2):
            for i in range(K.shape[1]):
                t = at[b] + i
                step = state[2][b, :, t // c].double()[:, None]
                err, x = (values[b, :, t] - K[b, i].double()).abs(), K[b, i].double().abs()
                if b == 1 and t // c == 0:
                    continue  # (rows 0 .. 4 of that block are said to be in use)
                # int8: half a step of every scale it had, of which each is at most half the next; e4m3: half a step relative, 2^-4, and
                # half of the smallest step, 2^-10, of every scale
                assert (err <= (step if code == "int8" else 2.0 ** -4 * x + 2.0 ** -9 * step) * (1 + 2.0 ** -20)).all()


def test_lengths_and_counts_outside_their_bounds():
    s = shape_of(1, 64, 50, 3, "bf16")
    K, V = (torch.randn((3, 4, 1, 64)).bfloat16() for _ in "KV")
    state = empty(s, 16, "int8", 2)
    same(both(s, K, V, [-7, 60, 10], [9, 2, -1], "int8", 16, state), state, "bounds")


@pytest.mark.parametrize("code", ["e4m3", "int8"])
def test_zeros_tiny_large_and_odd_numbers(code):
    s, c = shape_of(1, 64, 200, 1, "f32"), 8
    state = empty(s, c, code, 4)
    x = torch.randn((1, 160, 1, 64), generator=torch.Generator().manual_seed(1))
    x[0, 0:8] = 0.0                 # a block of zeros
    x[0, 8:16] *= 1e-44             # subnormal
    x[0, 16:24] *= 1e-37            # scales next to the smallest
    x[0, 24:32] *= 3e37             # large
    x[0, 33, 0, 5] = float("nan")   # block 4
    x[0, 47, 0, 6] = float("inf")   # block 5
    x[0, 48, 0, 7] = float("-inf")  # block 6
    for n, m in ((0, 60), (60, 1), (61, 3), (64, 96)):  # (block 7 is continued)
        state = [y.cpu() for y in both(s, x[:, n:n + m], x.flip(3)[:, n:n + m], [n], None, code, c, state)]
        if n == 0:
            assert state[2][0, 0, 0] == 0 and (state[0][0, 0, :8].float() == 0).all()
            assert state[2][0, 0, 4:7].isnan().all() and (state[0][0, 0, 32:56].view(torch.uint8) == 0).all()
            assert torch.isfinite(state[2][0, 0, [0, 1, 2, 3, 7]]).all()
    dev = both(s, x[:, 30:70], x[:, 30:70], [30], None, code, c, state)  # anew from the middle of block 3 on
    same(dev, state, "odd numbers")
    # a block of zeros that gets numbers, one whose scale is NaN, and that one again from its first row
    dev = both(s, x[:, 100:104], x[:, 100:104], [4], None, code, c, state)
    same(dev, state, "after zeros")
    dev = both(s, x[:, 100:104], x[:, 100:104], [44], None, code, c, state)
    same(dev, state, "after NaN")
    dev = both(s, x[:, 100:104], x[:, 100:104], [40], None, code, c, state)
    same(dev, state, "anew")
    assert torch.isfinite(state[2][0, 0, 5])


def test_slices_of_a_projection_and_rows_that_are_not_aligned():
    for d, H, off in ((128, 4, 0), (128, 4, 1), (64, 2, 8), (100, 3, 4)):
        s = shape_of(H, d, 300, 2, "bf16")
        N = 37
        flat = torch.randn(2 * N * (6 * H * d) + 16, generator=torch.Generator().manual_seed(d + off)).bfloat16()
        x = flat[off:off + 2 * N * 6 * H * d].view(2, N, 6 * H, d)
        gpu = flat.cuda()[off:off + 2 * N * 6 * H * d].view(2, N, 6 * H, d)
        state = empty(s, 16, "e4m3", 5)
        dev = both(s, x[:, :, 4 * H:5 * H], x[:, :, 5 * H:], [0, 48], None, "e4m3", 16, state, (gpu[:, :, 4 * H:5 * H], gpu[:, :, 5 * H:]))
        same(dev, state, f"slices {d} {H} {off}")
    # drafted rows, heads before tokens, and one row for all
    s = shape_of(3, 128, 64, 2, "f32")
    x = torch.randn((2, 3, 9, 128))
    state = empty(s, 8, "int8", 6)
    K, V = x.transpose(1, 2), torch.randn((1, 1, 3, 128)).expand(2, 9, 3, 128)
    gpu = x.cuda().transpose(1, 2), V[:1, :1].cuda().expand(2, 9, 3, 128)
    same(both(s, K, V, [0, 16], None, "int8", 8, state, gpu), state, "drafts")


def test_codes_that_are_not_aligned():
    s, c = shape_of(2, 128, 60, 1, "bf16"), 16
    K, V = (torch.randn((1, 20, 2, 128)).bfloat16() for _ in "KV")
    state = empty(s, c, "e4m3", 8)
    room = torch.zeros(2 * 60 * 128 + 3, dtype=torch.uint8, device="cuda")
    dev = [x.cuda() for x in state]
    K8 = room[3:].view(torch.float8_e4m3fn).view(1, 2, 60, 128)
    K8.view(torch.uint8).copy_(dev[0].view(torch.uint8))
    xb.xkv_cache8_append(s, K.cuda(), V.cuda(), None, None, 20, "e4m3", c, K8, *dev[1:])
    for new, codes, scales in ((K, state[0], state[2]), (V, state[1], state[3])):
        for g in range(2):
            ref.append(new[0, :, g].float(), 0, 20, codes[0, g], scales[0, g], c, "e4m3")
    same([K8.contiguous()] + dev[1:], state, "not aligned")
    assert (room[:3] == 0).all()


def test_no_strides_are_contiguous_rows():
    """NULL in the place of strides, as a C program may pass it: rows one after the other, [batch][N][heads][d_h]; here and in xkv_rotate."""
    import ctypes
    s = shape_of(3, 64, 90, 2, "bf16")
    K, V = (torch.randn((2, 20, 3, 64)).bfloat16() for _ in "KV")
    state = empty(s, 16, "int8", 9)
    dev, Kd, Vd = [x.cuda() for x in state], K.cuda(), V.cuda()
    lib, st = xb.load(), torch.cuda.current_stream().cuda_stream
    assert lib.xkv_cache8_append(s.ref, Kd.data_ptr(), None, Vd.data_ptr(), None, None, None, 20, 1, 16, *(x.data_ptr() for x in dev), st) == 0
    for new, codes, scales in ((K, state[0], state[2]), (V, state[1], state[3])):
        for b in range(2):
            for g in range(3):
                ref.append(new[b, :, g].float(), 0, 20, codes[b, g], scales[b, g], 16, "int8")
    same(dev, state, "no strides")
    f = ref.frequencies(64, 1e4).cuda()
    a, b = torch.empty_like(Kd), torch.empty_like(Kd)
    xb.xkv_rotate(s, 64, "half", "forward", 1.0, f, None, 20, None, None, Kd, a)
    nothing = ctypes.c_void_p(0)
    assert lib.xkv_rotate(s.ref, 64, 0, 0, 1.0, f.data_ptr(), None, 20, nothing, None, nothing, None, Kd.data_ptr(), None, b.data_ptr(), None, st) == 0
    assert torch.equal(a, b)


def test_more_workgroups_than_a_launch_has_in_one_direction():
    """2^25 rows and more, each its own block, four a workgroup of 256 threads, of keys and values: 2^32 threads."""
    N = (1 << 25) + 4099
    s = shape_of(1, 1, N, 1, "bf16")
    K, V = (torch.randn((1, N, 1, 1), device="cuda").bfloat16() for _ in "KV")
    codes = [torch.full((1, 1, N, 1), 77, dtype=torch.uint8, device="cuda") for _ in "KV"]
    scales = [torch.full((1, 1, N), 5.0, device="cuda") for _ in "KV"]
    xb.xkv_cache8_append(s, K, V, None, None, N, "int8", 1, codes[0], codes[1], scales[0], scales[1])
    for x, y, z in ((K, codes[0], scales[0]), (V, codes[1], scales[1])):
        x, code = x.flatten().double(), y.flatten().view(torch.int8)
        assert torch.equal(code, (127 * x.sign()).to(torch.int8))  # a row of one number is its own largest
        assert bool(((z.flatten().double() * 127 - x.abs()).abs() <= x.abs() * 2.0**-24).all())  # one quotient in fp32
