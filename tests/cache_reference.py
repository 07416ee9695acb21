"""The operators on a cache that grows and shrinks, in double precision on the CPU, plainly; and how far rounding may take a
kernel from them.  Tensors are torch CPU tensors; results are float64."""
import torch

EPS = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8}  # half a step, relative to the value


def attend(q, keys, values, sees, scale):
    """q [rows][d], keys / values [T][d], sees [rows][T] -> (out, weights, bound of |out| errors, bound of relative errors of weights).

    The bounds: a logit is a sum of d products in fp32 (in any order: at most d roundings of the sum of magnitudes, and a few of the
    scaling), so it is off by dz = (d + 4) 2^-24 scale max sum |q k|, twice over with the maximum that is subtracted; a weight then by
    a factor exp(2 dz), by 2^-20 from the exponential, and by half a step where it is rounded to the storage type as an operand of the
    matrix cores; sums over T tokens, by (T + 64) 2^-24; the result by half a step of its type.
    """
    out_type = q.dtype
    q, keys, values = q.double(), keys.double(), values.double()
    z = (scale * (q @ keys.T)).masked_fill(~sees, -torch.inf)
    some = sees.any(1, keepdim=True)
    p = torch.where(some, torch.softmax(z.masked_fill(~some, 0.0), 1), torch.zeros_like(z)) * sees
    used = sees.any(0)
    v = torch.where(used[:, None], values, torch.zeros_like(values))
    out = p @ v
    reach = (q.abs() @ torch.where(used[:, None], keys, torch.zeros_like(keys)).abs().T).max().item() if len(keys) else 0.0
    dz = (q.shape[1] + 4) * 2.0 ** -24 * scale * reach
    rel = 2 * dz + 2.0 ** -20 + (len(keys) + 64) * 2.0 ** -24
    half = EPS[out_type]
    bound = (rel + (half if out_type != torch.float32 else 0.0)) * (p @ v.abs()) + half * out.abs()
    return out, p, bound + 1e-30, rel


def tree_mask(words, N):
    """int32 words [N][..] -> bool [N][N]."""
    bits = (words.long()[:, :, None] >> torch.arange(32)) & 1
    return bits.reshape(words.shape[0], -1)[:, :N] > 0


def pack_mask(sees):
    """bool [..][N][N] -> int32 [..][N][ceil(N / 32)]."""
    N = sees.shape[-1]
    bits = torch.nn.functional.pad(sees, (0, -N % 32)).reshape(*sees.shape[:-1], -1, 32).long() << torch.arange(32)
    words = bits.sum(-1)
    return torch.where(words >= 2 ** 31, words - 2 ** 32, words).to(torch.int32)


def choose_blocks(q, landmarks, visible, c, k_ch):
    """q [n_rep][d], landmarks [n_c][d] of one KV head -> the blocks, ascending (only those that exist)."""
    if visible < 1:
        return []
    own = (visible - 1) // c
    S = (landmarks[:own].double() @ q.double().T).float()
    S = S.max(1).values if own else S[:, 0]
    order = sorted(range(own), key=lambda j: (-S[j].item(), j))
    return sorted(order[: k_ch - 1] + [own])


def keep_rows(weights, n, k, sink, recent):
    """weights [L] fp32 of one KV head -> the rows that stay, ascending.  Larger weights first, -0 below +0, smaller rows first."""
    import numpy as np
    u = weights[:n].numpy().view(np.uint32).astype(np.int64)
    key = np.where(u >> 31, 0xFFFFFFFF - u, u + 0x80000000)
    protected = [t for t in range(n) if t < sink or t >= n - recent]
    rest = sorted((t for t in range(n) if sink <= t < n - recent), key=lambda t: (-key[t], t))
    return sorted((protected + rest)[:k])
