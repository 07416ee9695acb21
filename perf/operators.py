"""Attention over an uncompressed cache that grows and shrinks, as cases that can be timed and compared.

K, V [batch][H_kv][L][d_h] have room for L rows, of which the first `lengths` of each sequence are in use.  A case is a
dict of plain values.  `kind` is the operator:

  tree     N drafted tokens, which form a tree, attend to the cache and to their ancestors in the draft
  block    each of N queries attends to the blocks of c rows whose means agree with it best, and to its own block
  weights  one token attends to the cache, and what every row got is added up
  evict    the rows that got most, the first and the last ones are kept, in order, in a smaller cache

Keys are those of a text: rows of a stretch of 64 tokens resemble one another.  Logits of a query have a spread of about one.
"""
import math

import torch

own = False

# Model shapes: Llama-3.1-8B and Qwen2.5-7B attention (32 / 28 query heads), and a small single-precision one.
LLAMA = dict(H_kv=8, H_q=32, d_h=128, dtype="bf16")
QWEN = dict(H_kv=4, H_q=28, d_h=128, dtype="bf16")
TINY = dict(H_kv=1, H_q=4, d_h=64, dtype="f32")


def listed():
    return [
        # the smallest call: a toy model in single precision, a short draft
        dict(TINY, name="tree_f32_tiny", kind="tree", L=512, batch=1, N=8, ragged=False),
        # interactive decoding of one user with 32K tokens, 16 drafted tokens
        dict(LLAMA, name="tree_llama_b1_32k", kind="tree", L=32768, batch=1, N=16, ragged=False),
        # four users with wide trees and contexts of different lengths up to 64K
        dict(LLAMA, name="tree_llama_b4_64k", kind="tree", L=65536, batch=4, N=64, ragged=True),
        # odd sizes everywhere, seven query heads per KV head
        dict(QWEN, name="tree_qwen_b3_40k", kind="tree", L=40001, batch=3, N=33, ragged=True),
        # a toy model's blocks
        dict(TINY, name="block_f32_tiny", kind="block", L=512, batch=1, N=1, c=16, k=128, ragged=False),
        # one user with 32K tokens, blocks of 16, a sixteenth of the context
        dict(LLAMA, name="block_llama_b1_32k", kind="block", L=32768, batch=1, N=1, c=16, k=2048, ragged=False),
        # the benchmark's serving batch: 16 users with up to 64K tokens, blocks of 32
        dict(LLAMA, name="block_llama_b16_64k", kind="block", L=65536, batch=16, N=1, c=32, k=4096, ragged=True),
        # the last 256 tokens of a 128K prompt, each with its own blocks
        dict(QWEN, name="block_qwen_prompt_128k", kind="block", L=131072, batch=1, N=256, c=64, k=4096, ragged=False),
        # one user with 32K tokens
        dict(LLAMA, name="weights_llama_b1_32k", kind="weights", L=32768, batch=1, ragged=False),
        # 16 users with up to 64K tokens
        dict(LLAMA, name="weights_llama_b16_64k", kind="weights", L=65536, batch=16, ragged=True),
        # a cache that has outgrown its budget of 4096 rows by 256
        dict(LLAMA, name="evict_llama_b4_4k", kind="evict", L=4352, batch=4, k=4096, sink=4, recent=256, ragged=False),
        # prompts of up to 64K tokens cut down to 8192 rows
        dict(QWEN, name="evict_qwen_b8_64k", kind="evict", L=65536, batch=8, k=8192, sink=4, recent=1024, ragged=True),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        c = _draw_any(rng)
        if _cost(c) <= most:
            return c


def _draw_any(rng):
    kind = rng.choice(("tree", "block", "weights", "evict"))
    toy = rng.random() < 0.15
    c = dict(TINY if toy else rng.choice((LLAMA, QWEN)), kind=kind)
    c["L"] = _log_int(rng, 64, 4096 if toy else 131072)
    c["batch"] = _log_int(rng, 1, 4 if toy else 16)
    c["ragged"] = rng.random() < 0.5
    if kind == "tree":
        c["N"] = _log_int(rng, 1, 128)
    elif kind == "block":
        c["c"] = rng.choice((8, 16, 24, 32, 64))
        c["k"] = min(_log_int(rng, 64, 6000), c["L"])
        c["N"] = rng.choice((1, 1, 1, _log_int(rng, 2, 256)))
        c["N"] = min(c["N"], c["L"])
    elif kind == "evict":
        c["k"] = max(2, int(c["L"] * rng.uniform(0.05, 1.0)))
        c["sink"] = rng.choice((0, 1, 4))
        c["sink"] = min(c["sink"], c["k"] // 2)
        c["recent"] = rng.randint(0, c["k"] // 2)
    return c


def _cost(c):
    """Rough nanoseconds of a pass of the plain forms, for keeping drawn cases below the largest listed one."""
    w = work(c)
    b = w["bytes"] * 5
    if c["kind"] == "tree":
        b += 20 * c["batch"] * c["H_q"] * c["N"] * c["L"]
    elif c["kind"] == "block":
        b += 16 * c["batch"] * c["N"] * c["H_kv"] * _blocks(c) * c["c"] * c["d_h"]
    return b / 4000.0 + w["flops"] / 1e5


def _lengths(c):
    """Rows in use of every sequence: all, or evenly down to L / batch."""
    return [c["L"] - (i * c["L"] // c["batch"] if c["ragged"] else 0) for i in range(c["batch"])]


def _blocks(c):
    """Blocks that a query attends to."""
    return min(-(-c["k"] // c["c"]), -(-c["L"] // c["c"]))


# ---------------------------------------------------------------------------------------------------------- inputs
def _dtype(c):
    return torch.float32 if c["dtype"] == "f32" else torch.bfloat16


def prepare(case, seed):
    c, dt = dict(case), _dtype(case)
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    b, H_kv, H_q, d, L = c["batch"], c["H_kv"], c["H_q"], c["d_h"], c["L"]

    def randn(*shape):
        return torch.randn(shape, generator=g, device="cuda")

    K, V = (torch.empty((b, H_kv, L, d), dtype=dt, device="cuda") for _ in "KV")
    for i in range(b):
        stretch = 0.8 * randn(H_kv, -(-L // 64), d)
        K[i] = (stretch.repeat_interleave(64, 1)[:, :L] + 0.6 * randn(H_kv, L, d)).to(dt)
        V[i] = randn(H_kv, L, d).to(dt)
    n = torch.tensor(_lengths(c), dtype=torch.int32, device="cuda")
    st = {"c": c, "K": K, "V": V, "lengths": n}
    if c["kind"] in ("tree", "block"):
        st["q"] = randn(b, c["N"], H_q, d).to(dt)
    if c["kind"] == "tree":
        N = c["N"]
        st["K_draft"], st["V_draft"] = randn(b, H_kv, N, d).to(dt), randn(b, H_kv, N, d).to(dt)
        # every drafted token but the first continues one of those before it
        cpu = torch.Generator()
        cpu.manual_seed(int(seed))
        sees = torch.eye(N, dtype=torch.bool).repeat(b, 1, 1)
        for j in range(1, N):
            sees[:, j] |= sees[torch.arange(b), (torch.rand(b, generator=cpu) * j).long()]
        bits = torch.nn.functional.pad(sees, (0, -N % 32)).view(b, N, -1, 32).long() << torch.arange(32)
        words = bits.sum(-1)
        st["tree"] = torch.where(words >= 2**31, words - 2**32, words).to(torch.int32).cuda()
    elif c["kind"] == "block":
        # the queries are the last tokens of each sequence
        st["visible"] = (n[:, None] - c["N"] + 1 + torch.arange(c["N"], device="cuda", dtype=torch.int32)).clamp_min(0).contiguous()
        n_c = -(-L // c["c"])
        full = torch.nn.functional.pad(K, (0, 0, 0, n_c * c["c"] - L)).view(b, H_kv, n_c, c["c"], d)
        st["landmarks"] = torch.empty((b, H_kv, n_c, d), dtype=dt, device="cuda")
        for i in range(b):
            st["landmarks"][i] = full[i].float().mean(2).to(dt)
    elif c["kind"] == "weights":
        st["q"] = randn(b, H_q, d).to(dt)
        st["weights"] = randn(b, H_kv, L).mul(2.0).exp() / L
    else:
        # heavy tails, and rows that nothing ever looked at
        w = randn(b, H_kv, L).mul(2.0).exp()
        st["weights"] = torch.where(torch.rand((b, H_kv, L), generator=g, device="cuda") < 0.05, 0.0, w)
        st["K_out"], st["V_out"] = (torch.zeros((b, H_kv, c["k"], d), dtype=dt, device="cuda") for _ in "KV")
    return st


# ------------------------------------------------------------------------------------------------------------ a pass
def run(st):
    kind = st["c"]["kind"]
    if own:
        return {"tree": _own_tree, "block": _own_block, "weights": _own_weights, "evict": _own_evict}[kind](st)
    return {"tree": _tree, "block": _block, "weights": _weights, "evict": _evict}[kind](st)


def _kept(st):
    """The binding, and what a program keeps between calls: the shape, a workspace, buffers for results."""
    from paper_2503_18893_amd import binding as xb
    c = st["c"]
    if "shape" not in st:
        s = xb.Shape(1, c["H_kv"], c["H_q"], c["d_h"], 1, 1, c["L"], c.get("k", 1), c["batch"], c["dtype"])
        st["ws"] = torch.empty(xb.xkv_cache_workspace_bytes(s, c.get("N", 1), c.get("c", 0)), dtype=torch.uint8, device="cuda")
        if c["kind"] != "evict":
            lead = (c["batch"], c["N"]) if "N" in c else (c["batch"],)
            st["out"] = torch.empty((*lead, c["H_q"], c["d_h"]), dtype=_dtype(c), device="cuda")
        else:
            rows = (c["batch"], c["H_kv"], c["k"])
            st["weights_out"] = torch.zeros(rows, dtype=torch.float32, device="cuda")
            st["rows_out"] = torch.empty(rows, dtype=torch.int32, device="cuda")
            st["lengths_out"] = torch.empty_like(st["lengths"])
        st["shape"] = s
    return xb, c, st["shape"]


def _own_tree(st):
    xb, c, s = _kept(st)
    xb.xkv_tree_decode(s, st["K"], st["V"], st["lengths"], st["q"], st["K_draft"], st["V_draft"], st["tree"], c["N"], st["out"], st["ws"])
    return st["out"]


def _own_block(st):
    xb, c, s = _kept(st)
    xb.xkv_block_decode(s, st["K"], st["V"], st["visible"], st["q"], c["N"], st["landmarks"], c["c"], st["out"], None, st["ws"])
    return st["out"]


def _own_weights(st):
    xb, c, s = _kept(st)
    xb.xkv_dense_decode_weights(s, st["K"], st["V"], st["lengths"], st["q"], st["out"], st["weights"], st["ws"])
    return {"out": st["out"], "weights": st["weights"]}


def _own_evict(st):
    xb, c, s = _kept(st)
    xb.xkv_evict(s, st["K"], st["V"], st["weights"], st["lengths"], c["sink"], c["recent"], c["k"], st["K_out"], st["V_out"],
                 st["weights_out"], st["rows_out"], st["lengths_out"], st["ws"])
    return {"K": st["K_out"], "V": st["V_out"], "weights": st["weights_out"], "rows": st["rows_out"], "lengths": st["lengths_out"]}


# the plain forms
def _softmax(z):
    """Softmax over the last axis; a row that sees nothing gets zeros."""
    m = z.amax(-1, keepdim=True)
    p = torch.exp(z - torch.where(m == -math.inf, torch.zeros_like(m), m))
    s = p.sum(-1, keepdim=True)
    return p / torch.where(s > 0, s, torch.ones_like(s))


def _heads(c, q):
    """q [batch][N][H_q][d_h] as single-precision rows of each KV head, [batch][H_kv][N n_rep][d_h]."""
    b, N, H_q, d = q.shape
    return q.float().view(b, N, c["H_kv"], H_q // c["H_kv"], d).transpose(1, 2).reshape(b, c["H_kv"], -1, d)


def _back(c, o, dt):
    """... and back."""
    b, H_kv, rows, d = o.shape
    r = c["H_q"] // H_kv
    return o.view(b, H_kv, rows // r, r, d).transpose(1, 2).reshape(b, rows // r, H_kv * r, d).to(dt)


def _tree(st):
    c, K, N = st["c"], st["K"], st["c"]["N"]
    r, pos = c["H_q"] // c["H_kv"], torch.arange(c["L"], device="cuda")
    q = _heads(c, st["q"]) * (1.0 / math.sqrt(c["d_h"]))
    z = q @ K.float().transpose(-1, -2)
    z.masked_fill_(pos >= st["lengths"][:, None, None, None], -math.inf)
    sees = (st["tree"][..., None] >> torch.arange(32, device="cuda", dtype=torch.int32) & 1).flatten(2)[:, :, :N] > 0
    y = (q @ st["K_draft"].float().transpose(-1, -2)).masked_fill(~sees.repeat_interleave(r, 1)[:, None], -math.inf)
    p = _softmax(torch.cat((z, y), -1))
    o = p[..., :c["L"]] @ st["V"].float() + p[..., c["L"]:] @ st["V_draft"].float()
    return _back(c, o, K.dtype)


def _block(st):
    c, K, V, v = st["c"], st["K"], st["V"], st["visible"]
    b, N, H_kv, r, n_c = c["batch"], c["N"], c["H_kv"], c["H_q"] // c["H_kv"], st["landmarks"].shape[2]
    q = _heads(c, st["q"])
    # values next to the border of the selection: sums in 64 bits, rounded once
    S = (q.double() @ st["landmarks"].double().transpose(-1, -2)).float().view(b, H_kv, N, r, n_c).amax(3)
    last = torch.div(v - 1, c["c"], rounding_mode="floor")[:, None, :, None]
    j = torch.arange(n_c, device="cuda")
    S = S.masked_fill(j == last, math.inf).masked_fill(j > last, -math.inf)
    ids = torch.sort(S, dim=-1, descending=True, stable=True).indices[..., :_blocks(c)]
    rows = (ids[..., None] * c["c"] + torch.arange(c["c"], device="cuda")).flatten(3)
    ok = rows < v[:, None, :, None]
    rows = rows.clamp_max(c["L"] - 1)
    at = torch.arange(b, device="cuda")[:, None, None, None], torch.arange(H_kv, device="cuda")[None, :, None, None], rows
    z = (q.view(b, H_kv, N, r, -1) * (1.0 / math.sqrt(c["d_h"]))) @ K[at].float().transpose(-1, -2)
    p = _softmax(z.masked_fill(~ok[:, :, :, None], -math.inf))
    return _back(c, (p @ V[at].float()).flatten(2, 3), K.dtype)


def _weights(st):
    c, K = st["c"], st["K"]
    q = _heads(c, st["q"][:, None]) * (1.0 / math.sqrt(c["d_h"]))
    z = q @ K.float().transpose(-1, -2)
    unused = torch.arange(c["L"], device="cuda") >= st["lengths"][:, None, None, None]
    p = _softmax(z.masked_fill(unused, -math.inf))
    st["weights"] += p.sum(2)
    return {"out": _back(c, p @ st["V"].float(), K.dtype)[:, 0], "weights": st["weights"]}


def _evict(st):
    c, n, k = st["c"], st["lengths"][:, None, None], st["c"]["k"]
    t = torch.arange(c["L"], device="cuda")
    w = st["weights"]
    w = w.masked_fill((t < c["sink"]) | (t >= n - c["recent"]), math.inf).masked_fill(t >= n, -math.inf)
    rows = torch.sort(w, dim=-1, descending=True, stable=True).indices[..., :k].sort(-1).values
    ok = rows < n
    take = lambda x, y: torch.where(ok[..., None], x.gather(2, rows[..., None].expand(-1, -1, -1, x.shape[-1])), y)  # noqa: E731
    weights = torch.where(ok, st["weights"].gather(2, rows), 0.0)
    return {"K": take(st["K"], st["K_out"]), "V": take(st["V"], st["V_out"]), "weights": weights,
            "rows": torch.where(ok, rows, -1).to(torch.int32), "lengths": st["lengths"].clamp_max(k)}


# -------------------------------------------------------------------------------------------------------- what is due
def work(case):
    c, n = case, _lengths(case)
    b, H_kv, H_q, d, e = c["batch"], c["H_kv"], c["H_q"], c["d_h"], 4 if c["dtype"] == "f32" else 2
    row, N = H_kv * d * e, c.get("N", 1)
    qo = 2 * b * N * H_q * d * e
    if c["kind"] == "tree":
        return {"bytes": 2 * row * (sum(n) + b * N) + qo + b * N * (-(-N // 32)) * 4, "flops": 4 * d * H_q * N * (sum(n) + b * N)}
    if c["kind"] == "block":
        picked = [min(_blocks(c) * c["c"], x) for x in n]
        means = [-(-x // c["c"]) for x in n]
        return {"bytes": row * (sum(means) + 2 * sum(min(N * p, x) for p, x in zip(picked, n))) + qo + 4 * b * N,
                "flops": d * H_q * N * (4 * sum(picked) + 2 * sum(means))}
    if c["kind"] == "weights":
        return {"bytes": sum(n) * (2 * row + 8 * H_kv) + qo, "flops": 4 * d * H_q * sum(n)}
    m = sum(min(x, c["k"]) for x in n)
    return {"bytes": 4 * H_kv * sum(n) + m * (4 * row + 8 * H_kv), "flops": 0}


# ---------------------------------------------------------------------------------------------- the same, in 64 bits
def exact(case, seed):
    if case["kind"] == "evict":
        return None  # copies: nothing is computed
    st = prepare(case, seed)
    c, K, V, n = st["c"], st["K"], st["V"], _lengths(case)
    b, H_kv, r, d = c["batch"], c["H_kv"], c["H_q"] // c["H_kv"], c["d_h"]
    q = st["q"].double()
    out = torch.zeros(q.shape, dtype=torch.float64, device="cuda")
    if c["kind"] == "weights":
        total = st["weights"].double()
        for i in range(b):
            for h in range(c["H_q"]):
                g = h // r
                z = K[i, g, : n[i]].double() @ q[i, h] / math.sqrt(d)
                p = torch.softmax(z, 0)
                out[i, h] = p @ V[i, g, : n[i]].double()
                total[i, g, : n[i]] += p
        return {"out": out, "weights": total}
    for i in range(b):
        for g in range(H_kv):
            k_all, v_all = K[i, g, : n[i]].double(), V[i, g, : n[i]].double()
            heads = slice(g * r, (g + 1) * r)
            if c["kind"] == "tree":
                kd, vd = st["K_draft"][i, g].double(), st["V_draft"][i, g].double()
                keys, values = torch.cat((k_all, kd)), torch.cat((v_all, vd))
                x = torch.arange(c["N"], device="cuda")
                bit = (st["tree"][i].long()[:, x // 32] >> (x % 32)) & 1
                hidden = torch.cat((torch.zeros((c["N"], n[i]), dtype=torch.bool, device="cuda"), bit == 0), 1)
                for h in range(g * r, (g + 1) * r):
                    z = (q[i, :, h] @ keys.T / math.sqrt(d)).masked_fill(hidden, -math.inf)
                    out[i, :, h] = torch.softmax(z, 1) @ values
                continue
            marks = st["landmarks"][i, g].double()
            seen = st["visible"][i].tolist()
            for j in range(c["N"]):
                if seen[j] < 1:
                    continue
                mine = (seen[j] - 1) // c["c"]
                score = (marks[:mine] @ q[i, j, heads].T).float().amax(1) if mine else torch.empty(0, device="cuda")
                best = torch.sort(score, dim=0, descending=True, stable=True).indices[: _blocks(c) - 1]
                taken = torch.zeros(seen[j], dtype=torch.bool, device="cuda")
                taken[mine * c["c"]:] = True
                taken[(best[:, None] * c["c"] + torch.arange(c["c"], device="cuda")).flatten()] = True
                kk, vv = k_all[: seen[j]][taken], v_all[: seen[j]][taken]
                out[i, j, heads] = torch.softmax(q[i, j, heads] @ kk.T / math.sqrt(d), 1) @ vv
    return out
