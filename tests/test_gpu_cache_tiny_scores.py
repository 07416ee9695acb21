"""Selection of blocks by scores so small that products or means are subnormal numbers: still that of the sums in double precision."""
import pytest
import torch

import cache_reference as ref
from paper_2503_18893_amd import binding as xb
from test_gpu_cache import cache, need_gpu, shape_of, workspace  # noqa: F401

pytestmark = pytest.mark.gpu


def check(q, marks, k):
    L = marks.shape[2]
    s = shape_of(1, q.shape[1], 128, L, 1, "bf16", k=k)
    _, K, V = cache(s, [L], 91)
    out, blocks = torch.empty_like(q, device="cuda"), torch.empty((1, 1, 1, k), dtype=torch.int32, device="cuda")
    xb.xkv_block_decode(s, K.cuda(), V.cuda(), None, q.cuda(), 1, marks.cuda(), 1, out, blocks, workspace(s, 1, 1))
    assert blocks.cpu().flatten().tolist() == ref.choose_blocks(q[0], marks[0, 0], L, 1, k)


@pytest.mark.parametrize("n_c,k", [(100, 20), (900, 40), (5000, 300)])
def test_subnormal_means(n_c, k):
    """One channel of normal numbers; the others are below 2^-126 and decide most comparisons."""
    g = torch.Generator().manual_seed(92)
    marks = torch.randint(-127, 128, (1, 1, n_c, 128), generator=g).double() * 2.0 ** -133
    marks[..., 0] = 2.0 ** -124 * (1 + 7 * torch.rand((1, 1, n_c), generator=g).double())
    q = torch.full((1, 2, 128), 2.0 ** 100)
    q[0, 1] = -(2.0 ** 100)
    check(q.bfloat16(), marks.bfloat16(), k)


@pytest.mark.parametrize("n_c,k", [(100, 20), (900, 40), (5000, 300)])
def test_subnormal_products(n_c, k):
    """Normal numbers whose products are not, beside larger ones."""
    g = torch.Generator().manual_seed(93)
    marks = 2.0 ** -63 * torch.randn((1, 1, n_c, 128), generator=g).double()
    marks[..., 1] *= 2.0 ** 4
    marks[..., 0] = 2.0 ** -50
    marks[0, 0, ::30, 0] *= 1.25
    q = torch.full((1, 2, 128), 2.0 ** -64)
    q[0, 1] *= -1
    check(q.bfloat16(), marks.bfloat16(), k)


@pytest.mark.parametrize("power", (-60, -75))
def test_subnormal_scores(power):
    g = torch.Generator().manual_seed(94)
    marks, q = 2.0 ** power * torch.randn((1, 1, 900, 128), generator=g), 2.0 ** -66 * torch.randn((1, 2, 128), generator=g)
    check(q.bfloat16(), marks.bfloat16(), 40)
