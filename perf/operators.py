"""Performance cases of two operators that stand beside the tree-verification calls: attention over a whole prompt, and the
paged cache held in 4 bits (written, read back, attended over, appended to).

Kinds (``case["kind"]``):

  prompt       causal attention of packed prompts of different lengths, grouped heads: what lays down a prefix
  attention    one tree_verify_attention call over a cache in 4 bits; trees of one node are plain decoding
  write        a prefill's K/V rows into the 4-bit cache and back out of it
  step         the accepted path appended to the 4-bit cache, then attention of the next tree over the longer prefix

A row of 32 consecutive head dims of one token shares a scale 2^(s - 127) (a byte s) and holds 32 E2M1 values
(0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives; code bit 3 is the sign), low nibble first.  Bytes of one
(block, kv head) page, bs slots of D head dims:

  K:  element (slot, d) in byte ((d / 32) bs + slot) 16 + (d % 32) / 2;               scale in bs D / 2 + slot (D / 32) + d / 32
  V:  element (slot, d) in byte ((slot / 8) (D / 4) + d / 4) 16 + (slot % 8) 2 + (d % 4) / 2;  scale in bs D / 2 + (d / 32) bs + slot

Lengths and tree sizes of a case come from ``case["shape_seed"]`` alone (they are the case's work); values, tree shapes and
the block permutation come from the seed that prepare() gets.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
BLOCK = 32                                   # elements that share a scale
_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
_handle = None


def _lib():
    """The one library handle a program keeps per device."""
    global _handle
    if _handle is None:
        from paper_2604_09731_amd import binding as B
        _handle = B.SmartTree(0)
    return _handle


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _prompt(name, prompts, tokens, heads, dtype="bf16", head_dim=128, lse=False, shape_seed=0):
    c = dict(kind="prompt", prompts=prompts, tokens_min=tokens[0], tokens_max=tokens[1], q_heads=heads[0],
             kv_heads=heads[1], dtype=dtype, head_dim=head_dim, lse=lse, shape_seed=shape_seed)
    if name:
        c["name"] = name
    return c


def _cached(kind, name, batch, heads, prefix, nodes, dtype="bf16", head_dim=128, block_size=16, lse=False, shape_seed=0):
    c = dict(kind=kind, batch=batch, q_heads=heads[0], kv_heads=heads[1], prefix_min=prefix[0], prefix_max=prefix[1],
             nodes_min=nodes[0], nodes_max=nodes[1], dtype=dtype, head_dim=head_dim, block_size=block_size, lse=lse,
             shape_seed=shape_seed)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user's short question: latency
        _prompt("prompt_one_short", 1, (37, 37), (32, 8), shape_seed=1),
        # an admission batch of a server: ragged prompts of an 8B model, log-sum-exp kept for a later merge
        _prompt("prompt_batch_ragged", 5, (300, 3000), (32, 8), lse=True, shape_seed=2),
        # many short requests of a small model packed into one call
        _prompt("prompt_many_short", 64, (1, 300), (8, 2), head_dim=64, shape_seed=3),
        # a document at 70B shapes: the most arithmetic
        _prompt("prompt_long", 1, (16384, 16384), (64, 8), shape_seed=4),
        # fp32 prefill of a small model
        _prompt("prompt_f32", 8, (128, 1536), (8, 2), dtype="f32", head_dim=64, lse=True, shape_seed=5),
        # one interactive user early in a conversation: a small tree on a short odd prefix; latency
        _cached("attention", "fp4_one_short", 1, (32, 8), (517, 517), (7, 7), shape_seed=6),
        # a loaded server, trees cut small by the cost rule
        _cached("attention", "fp4_batch32_small_trees", 32, (32, 8), (2048, 4096), (4, 7), shape_seed=7),
        # the same server with cheap verification, trees of all sizes
        _cached("attention", "fp4_batch32_wide_trees", 32, (32, 8), (2048, 4096), (4, 64), lse=True, shape_seed=8),
        # plain decoding at 70B shapes and long contexts, one token a sequence: the most bytes
        _cached("attention", "fp4_batch64_long_single_token", 64, (64, 8), (16384, 16384), (1, 1), shape_seed=9),
        # fp32 verification of a small model, other block size
        _cached("attention", "fp4_f32_batch8", 8, (8, 2), (128, 1536), (15, 15), dtype="f32", head_dim=64, block_size=32,
                lse=True, shape_seed=10),
        # prefill of ragged prompts into the 4-bit cache and its rows back (to hand a sequence to another cache)
        dict(name="fp4_write_read_prefill", kind="write", prompts=5, tokens=8190, kv_heads=8, dtype="bf16", head_dim=128,
             block_size=16),
        # the end of a step and the next one's attention for a few users
        _cached("step", "fp4_step_batch4", 4, (32, 8), (2048, 2048), (40, 48), shape_seed=11),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    caps = {c["name"]: work(c) for c in listed()}
    kind = rng.choices(["prompt", "attention", "write", "step"], [5, 5, 1, 2])[0]
    shape_seed = rng.randrange(1, 1 << 30)
    heads = rng.choice([(8, 2), (32, 8), (32, 8), (28, 4), (64, 8), (8, 8)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    head_dim = rng.choice([64, 128, 128])
    if kind == "prompt":
        cap = caps["prompt_f32" if dtype == "f32" else "prompt_long"]
        while True:
            hi = _log_int(rng, 1, 1536 if dtype == "f32" else 16384)
            lo = rng.choice([hi, max(1, hi // 2), max(1, hi // 30)])
            c = _prompt(None, _log_int(rng, 1, 64), (lo, hi), heads, dtype, head_dim, rng.random() < 0.4, shape_seed)
            w = work(c)
            if w["flops"] <= cap["flops"] and w["bytes"] <= 4 * cap["bytes"]:
                return c
    if kind == "write":
        return dict(kind=kind, prompts=rng.randrange(1, 7), tokens=_log_int(rng, 1, 8190), kv_heads=rng.choice([2, 4, 8]),
                    dtype=dtype, head_dim=head_dim, block_size=rng.choice([8, 16, 16, 32, 64]))
    if kind == "step":
        hi = _log_int(rng, 100, 4096)
        n_hi = rng.choice([1, 7, 10, 24, 48, 64])
        return _cached(kind, None, _log_int(rng, 1, 32), heads, (max(1, hi // 2), hi), (max(1, n_hi // 2), n_hi),
                       shape_seed=shape_seed)
    cap = caps["fp4_f32_batch8" if dtype == "f32" else "fp4_batch64_long_single_token"]
    other = caps["fp4_batch32_wide_trees"]
    while True:
        hi = _log_int(rng, 1, 1536 if dtype == "f32" else 16384)
        lo = rng.choice([hi, max(1, hi // 2), max(1, hi // 8)])
        n_hi = rng.choice([1, 1, 7, 10, 24, 48, 64, 128])
        n_lo = rng.choice([n_hi, max(1, n_hi // 2), max(1, n_hi // 12)])
        c = _cached(kind, None, _log_int(rng, 1, 96), heads, (lo, hi), (n_lo, n_hi), dtype, head_dim,
                    rng.choice([8, 16, 16, 16, 32, 64]), rng.random() < 0.4, shape_seed)
        w = work(c)
        if w["bytes"] <= cap["bytes"] and w["flops"] <= max(cap["flops"], other["flops"] if dtype == "bf16" else 0):
            return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _spread(case, salt, lo, hi, count):
    return np.random.default_rng([case["shape_seed"], salt]).integers(lo, hi + 1, count)


def _lengths(case):
    if case["kind"] == "prompt":
        return _spread(case, 1, case["tokens_min"], case["tokens_max"], case["prompts"])
    return _spread(case, 1, case["prefix_min"], case["prefix_max"], case["batch"])


def _nodes(case):
    return _spread(case, 2, case["nodes_min"], case["nodes_max"], case["batch"])


def _offsets(n):
    return np.concatenate([[0], np.cumsum(n)]).astype(np.int32)


def _gen(seed, stream):
    return torch.Generator(device=DEV).manual_seed(seed * 64 + stream)


def _normal(seed, stream, shape, dtype):
    return torch.randn(shape, generator=_gen(seed, stream), device=DEV, dtype=torch.float32).to(dtype)


def _keys(seed, stream, shape, dtype):
    """Normal values with a few strong head dims, as the keys of trained models have them."""
    x = torch.randn(shape, generator=_gen(seed, stream), device=DEV, dtype=torch.float32)
    x[..., 5::37] *= 3.0
    return x.to(dtype)


def _dev(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).to(DEV)


def _quantise(x):
    """fp32 [..., D] -> E2M1 codes (uint8) and scale bytes (uint8) [..., D / 32], by the nearest value, ties to the even code."""
    blocks = x.unflatten(-1, (-1, BLOCK))
    top = blocks.abs().amax(-1, keepdim=True)
    bits = top.view(torch.int32)
    s = (bits >> 23) - 127 - 2 + ((bits & 0x7FFFFF) > 0x600000).int()    # above 1.75 2^e: one more, so that nothing is cut
    s = s.clamp(-125, 125)
    y = blocks.abs() * torch.ldexp(torch.ones_like(top), -s)
    code = torch.zeros_like(blocks, dtype=torch.uint8)
    for edge, closed in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (y >= edge if closed else y > edge).to(torch.uint8)
    code |= torch.signbit(blocks).to(torch.uint8) << 3
    return code.flatten(-2), (s + 127).to(torch.uint8).squeeze(-1)


def _pages(codes, scales, bs, values):
    """codes [nb, H, bs, D], scales [nb, H, bs, D / 32] -> pages [nb, H, bytes]."""
    nb, H, _, D = codes.shape
    pairs = codes[..., 0::2] | (codes[..., 1::2] << 4)                   # [nb, H, bs, D / 2]
    if values:
        body = pairs.view(nb, H, bs // 8, 8, D // 4, 2).permute(0, 1, 2, 4, 3, 5)
        scales = scales.transpose(2, 3)
    else:
        body = pairs.view(nb, H, bs, D // 32, 16).permute(0, 1, 3, 2, 4)
    return torch.cat([body.reshape(nb, H, -1), scales.reshape(nb, H, -1)], -1)


def _cache(case, seed, stream, num_blocks, values):
    bs, D, H = case["block_size"], case["head_dim"], case["kv_heads"]
    out = torch.empty((num_blocks, H, bs * D // 2 + bs * D // 32), dtype=torch.uint8, device=DEV)
    step = max(1, (1 << 25) // (H * bs * D))
    for i, at in enumerate(range(0, num_blocks, step)):
        n = min(step, num_blocks - at)
        make = _normal if values else _keys
        x = make(seed * 4096 + i, stream, (n, H, bs, D), torch.float32)
        out[at:at + n] = _pages(*_quantise(x), bs, values)
    return out


def _trees(seed, n):
    """Parent arrays (local indices) of random trees, concatenated."""
    g = np.random.default_rng([seed, 4])
    return np.concatenate([np.array([-1] + [int(g.integers(max(0, i - 8), i)) for i in range(1, m)], np.int32) for m in n])


def _ancestors(cu, parent):
    """anc[i]: the ancestors-or-self of node i (local ids) as a bit set; and the 64-bit words of it."""
    sets, cu, parent = [0] * len(parent), cu.tolist(), parent.tolist()
    for lo, hi in zip(cu, cu[1:]):
        for i in range(lo, hi):
            sets[i] = (1 << (i - lo)) | (sets[lo + parent[i]] if parent[i] >= 0 else 0)
    words = np.array([[s & (2 ** 64 - 1), s >> 64] for s in sets], np.uint64).view(np.int64)
    return sets, words


def _prepare_prompt(case, seed):
    cu = _offsets(_lengths(case))
    T, D, dt = int(cu[-1]), case["head_dim"], _TORCH[case["dtype"]]
    return dict(case=case, cu=_dev(cu), h_cu=cu, q=_normal(seed, 1, (T, case["q_heads"], D), dt),
                k=_keys(seed, 2, (T, case["kv_heads"], D), dt), v=_normal(seed, 3, (T, case["kv_heads"], D), dt))


def _prepare_cached(case, seed):
    L, n = _lengths(case), _nodes(case)
    cu, parent = _offsets(n), _trees(seed, n)
    N, D, bs, dt = int(cu[-1]), case["head_dim"], case["block_size"], _TORCH[case["dtype"]]
    room = 9 if case["kind"] == "step" else 0
    blocks = (L + room + bs - 1) // bs
    num_blocks = int(blocks.sum()) + 3
    perm = np.random.default_rng([seed, 5]).permutation(num_blocks).astype(np.int32)
    table = np.full((case["batch"], int(blocks.max()) + 1), -1, np.int32)
    for b, at in enumerate(np.cumsum(blocks) - blocks):
        table[b, :blocks[b]] = perm[at:at + blocks[b]]
    sets, words = _ancestors(cu, parent)
    visible = np.zeros((N, int(n.max())), bool)
    for i, s in enumerate(sets):
        visible[i] = [(s >> j) & 1 for j in range(visible.shape[1])]
    s = dict(case=case, q=_normal(seed, 1, (N, case["q_heads"], D), dt), kt=_keys(seed, 2, (N, case["kv_heads"], D), dt),
             vt=_normal(seed, 3, (N, case["kv_heads"], D), dt), kc=_cache(case, seed, 4, num_blocks, False),
             vc=_cache(case, seed, 5, num_blocks, True), table=_dev(table), len=_dev(L, np.int32), cu=_dev(cu),
             mask=_dev(words), visible=_dev(visible), h_cu=cu, h_len=L)
    if case["kind"] == "step":
        done = _spread(case, 3, 0, 8, case["batch"])                      # drafts accepted in the step before
        path = np.full((case["batch"], 9), -1, np.int32)
        for b, a in enumerate(done):
            path[b, :a + 1] = np.arange(a + 1)
        old = _offsets(np.full(case["batch"], 9))
        slots = np.concatenate([table[b, (L[b] + np.arange(a + 1)) // bs].astype(np.int64) * bs + (L[b] + np.arange(a + 1)) % bs
                                for b, a in enumerate(done)])
        rows = np.concatenate([old[b] + np.arange(a + 1) for b, a in enumerate(done)])
        M = int(old[-1])
        s.update(old_cu=_dev(old), done=_dev(done, np.int32), path=_dev(path), slots=_dev(slots), rows=_dev(rows),
                 h_done=done, k_old=_keys(seed, 6, (M, case["kv_heads"], D), dt),
                 v_old=_normal(seed, 7, (M, case["kv_heads"], D), dt))
    return s


def _prepare_write(case, seed):
    T, bs, H, D = case["tokens"], case["block_size"], case["kv_heads"], case["head_dim"]
    cuts = np.sort(np.random.default_rng(T).integers(0, T + 1, case["prompts"] - 1))
    lens = np.diff(np.concatenate([[0], cuts, [T]]))
    blocks = (lens + bs - 1) // bs
    num_blocks = int(blocks.sum()) + 3
    perm = np.random.default_rng([seed, 6]).permutation(num_blocks)
    slots = [perm[at + np.arange(m) // bs] * bs + np.arange(m) % bs for m, at in zip(lens, np.cumsum(blocks) - blocks)]
    dt = _TORCH[case["dtype"]]
    kc, vc = (torch.zeros((num_blocks, H, bs * D // 2 + bs * D // 32), dtype=torch.uint8, device=DEV) for _ in range(2))
    return dict(case=case, k=_keys(seed, 1, (T, H, D), dt), v=_normal(seed, 2, (T, H, D), dt), kc=kc, vc=vc,
                slots=_dev(np.concatenate(slots), np.int64))


def prepare(case, seed):
    return dict(prompt=_prepare_prompt, attention=_prepare_cached, step=_prepare_cached,
                write=_prepare_write)[case["kind"]](case, seed)


# ---------------------------------------------------------------------------
# one pass, in elementary operations
# ---------------------------------------------------------------------------
def _plain_decode(pages, bs, D, values):
    """Pages [n, H, bytes] -> the fp32 values [n, bs, H, D] they stand for."""
    n, H, _ = pages.shape
    body, scale = pages[..., :bs * D // 2], pages[..., bs * D // 2:]
    code = torch.stack([body & 15, body >> 4], -1)
    if values:
        code = code.view(n, H, bs // 8, D // 4, 8, 4).permute(0, 2, 4, 1, 3, 5).reshape(n, bs, H, D)
        scale = scale.view(n, H, D // BLOCK, bs).permute(0, 3, 1, 2)
    else:
        code = code.view(n, H, D // BLOCK, bs, BLOCK).permute(0, 3, 1, 2, 4).reshape(n, bs, H, D)
        scale = scale.view(n, H, bs, D // BLOCK).permute(0, 2, 1, 3)
    lut = torch.tensor(_VALUES + tuple(-v for v in _VALUES), device=pages.device)
    size = torch.exp2(scale.float() - 127.0)
    return (lut[code.long()].unflatten(-1, (-1, BLOCK)) * size.unsqueeze(-1)).flatten(-2)


def _softmax_rows(s):
    """exp(s - max) and its sum, along the last dimension."""
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    return p, total, (top + torch.log(total)).squeeze(-1)


def _plain_prompt(s):
    c = s["case"]
    q, k, v, Hkv, G = s["q"], s["k"], s["v"], c["kv_heads"], c["q_heads"] // c["kv_heads"]
    scale = 1.0 / math.sqrt(c["head_dim"])
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    for lo, hi in zip(s["h_cu"][:-1].tolist(), s["h_cu"][1:].tolist()):
        rows = max(1, (1 << 28) // (c["q_heads"] * (hi - lo)))               # of a piece: its scores are one array
        key, value = (x[lo:hi].float().transpose(0, 1).contiguous() for x in (k, v))
        for r0 in range(0, hi - lo, rows):
            r1 = min(hi - lo, r0 + rows)
            qs = q[lo + r0:lo + r1].float().unflatten(1, (Hkv, G)).permute(1, 2, 0, 3).flatten(1, 2)     # [Hkv, G rows, D]
            score = (torch.matmul(qs, key[:, :r1].transpose(1, 2).contiguous()) * scale).unflatten(1, (G, r1 - r0))
            later = torch.arange(r1, device=q.device) > torch.arange(r0, r1, device=q.device).unsqueeze(1)
            p, total, row = _softmax_rows(score.masked_fill(later, -math.inf))
            o = torch.matmul(p.flatten(1, 2), value[:, :r1]).unflatten(1, (G, r1 - r0)) / total
            out[lo + r0:lo + r1] = o.permute(2, 0, 1, 3).flatten(1, 2).to(out.dtype)
            lse[lo + r0:lo + r1] = row.permute(2, 0, 1).flatten(1, 2)
    return (out, lse) if c["lse"] else out


def _plain_attention(s, lengths):
    c = s["case"]
    bs, D, Hkv, G = c["block_size"], c["head_dim"], c["kv_heads"], c["q_heads"] // c["kv_heads"]
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=out.device)
    for b, L in enumerate(lengths):
        lo, hi = int(s["h_cu"][b]), int(s["h_cu"][b + 1])
        n, pages = hi - lo, s["table"][b, :(L + bs - 1) // bs].long()
        key = torch.cat([_plain_decode(s["kc"][pages], bs, D, False).flatten(0, 1)[:L], s["kt"][lo:hi].float()])
        value = torch.cat([_plain_decode(s["vc"][pages], bs, D, True).flatten(0, 1)[:L], s["vt"][lo:hi].float()])
        q = s["q"][lo:hi].float().view(n, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, n * G, D)
        score = torch.matmul(q, key.permute(1, 2, 0).contiguous()) / math.sqrt(D)
        hidden = torch.cat([torch.zeros((n, L), dtype=torch.bool, device=q.device), ~s["visible"][lo:hi, :n]], 1)
        score = score.masked_fill(hidden.repeat_interleave(G, 0), -math.inf)
        p, total, row = _softmax_rows(score)
        o = torch.matmul(p, value.transpose(0, 1).contiguous()) / total
        out[lo:hi] = o.view(Hkv, n, G, D).permute(1, 0, 2, 3).reshape(n, Hkv * G, D).to(out.dtype)
        lse[lo:hi] = row.view(Hkv, n, G).permute(1, 0, 2).reshape(n, Hkv * G)
    return (out, lse) if c["lse"] else out


def _plain_put(pages, codes, scales, slots, bs, values):
    """Rows [T, H, D] of codes and [T, H, D / 32] of scales into their slots of the pages."""
    T, H, D = codes.shape
    pairs = codes[..., 0::2] | (codes[..., 1::2] << 4)
    block, slot = (slots // bs).view(T, 1, 1), (slots % bs).view(T, 1, 1)
    head = torch.arange(H, device=pages.device).view(1, H, 1)
    i, j = (torch.arange(m, device=pages.device).view(1, 1, m) for m in (D // 2, D // BLOCK))
    if values:
        pages[block, head, ((slot // 8) * (D // 4) + i // 2) * 16 + slot % 8 * 2 + i % 2] = pairs
        pages[block, head, bs * D // 2 + j * bs + slot] = scales
    else:
        pages[block, head, ((i // 16) * bs + slot) * 16 + i % 16] = pairs
        pages[block, head, bs * D // 2 + slot * (D // BLOCK) + j] = scales


def _plain_get(pages, slots, bs, D, values, dtype):
    """The rows of the slots, as values."""
    used, where = torch.unique(slots // bs, return_inverse=True)
    return _plain_decode(pages[used], bs, D, values)[where, slots % bs].to(dtype)


def _plain_write(s):
    c, dt = s["case"], s["k"].dtype
    bs, D = c["block_size"], c["head_dim"]
    _plain_put(s["kc"], *_quantise(s["k"].float()), s["slots"], bs, False)
    _plain_put(s["vc"], *_quantise(s["v"].float()), s["slots"], bs, True)
    return _plain_get(s["kc"], s["slots"], bs, D, False, dt), _plain_get(s["vc"], s["slots"], bs, D, True, dt)


def _plain_step(s):
    c, dt = s["case"], s["q"].dtype
    bs, D = c["block_size"], c["head_dim"]
    _plain_put(s["kc"], *_quantise(s["k_old"][s["rows"]].float()), s["slots"], bs, False)
    _plain_put(s["vc"], *_quantise(s["v_old"][s["rows"]].float()), s["slots"], bs, True)
    out = _plain_attention(s, s["h_len"] + s["h_done"] + 1)
    return (s["len"] + s["done"] + 1, out, _plain_get(s["kc"], s["slots"], bs, D, False, dt),
            _plain_get(s["vc"], s["slots"], bs, D, True, dt))


# ---------------------------------------------------------------------------
# one pass, by the framework's calls
# ---------------------------------------------------------------------------
def _own_prompt(s):
    return _lib().prompt_attention(s["q"], s["k"], s["v"], s["cu"], 1.0 / math.sqrt(s["case"]["head_dim"]),
                                     want_lse=s["case"]["lse"])


def _own_attention(s, lengths):
    from paper_2604_09731_amd import binding as B
    c = s["case"]
    return _lib().tree_verify_attention(s["q"], s["kt"], s["vt"], s["kc"], s["vc"], s["table"], lengths, s["cu"], s["mask"],
                                          1.0 / math.sqrt(c["head_dim"]), B.SMART_KV_INTERLEAVED, block_size=c["block_size"],
                                          want_lse=c["lse"], kv_cache_dtype=B.SMART_FP4_E2M1)


def _own_write(s):
    c = s["case"]
    _lib().kv_cache_write_fp4(s["k"], s["v"], s["slots"], s["kc"], s["vc"], c["block_size"])
    return _lib().kv_cache_read_fp4(s["slots"], s["kc"], s["vc"], c["head_dim"], c["block_size"], s["k"].dtype)


def _own_step(s):
    c = s["case"]
    lengths, _ = _lib().tree_commit_fp4(s["old_cu"], s["done"], s["path"], s["k_old"], s["v_old"], s["kc"], s["vc"],
                                          s["table"], s["len"], c["block_size"])
    out = _own_attention(s, lengths)
    k, v = _lib().kv_cache_read_fp4(s["slots"], s["kc"], s["vc"], c["head_dim"], c["block_size"], s["q"].dtype)
    return lengths, out, k, v


def run(state):
    kind = state["case"]["kind"]
    if own:
        return (_own_attention(state, state["len"]) if kind == "attention" else
                dict(prompt=_own_prompt, write=_own_write, step=_own_step)[kind](state))
    return (_plain_attention(state, state["h_len"]) if kind == "attention" else
            dict(prompt=_plain_prompt, write=_plain_write, step=_plain_step)[kind](state))


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    e, D, H = 4 if case["dtype"] == "f32" else 2, case["head_dim"], case["kv_heads"]
    row4 = 2 * (D // 2 + D // BLOCK)                       # K and V of one token and head in 4 bits
    if case["kind"] == "write":
        return {"bytes": case["tokens"] * (H * (2 * 2 * D * e + row4) + 8), "flops": 0}
    Hq, L = case["q_heads"], _lengths(case).astype(np.int64)
    if case["kind"] == "prompt":
        T = int(L.sum())
        return {"bytes": T * D * e * 2 * (Hq + H) + (T * Hq * 4 if case["lse"] else 0),
                "flops": 4 * D * Hq * int((L * (L + 1) // 2).sum())}
    n = _nodes(case).astype(np.int64)
    N = int(n.sum())
    table = int(((L + case["block_size"] - 1) // case["block_size"]).sum()) * 4
    byts = int(L.sum()) * H * row4 + N * 2 * (Hq + H) * D * e + N * 16 + table + (N * Hq * 4 if case["lse"] else 0)
    if case["kind"] == "step":
        byts += 5 * case["batch"] * H * (2 * 2 * D * e + row4)     # five rows a sequence on average, written and read back
    return {"bytes": byts, "flops": 4 * D * Hq * int((n * L).sum() + N)}


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def _exact_page_rows(pages, block, slot, bs, D, values):
    """float64 [T, H, D]: the rows (block[t], slot[t]), element by element through the offset formulas."""
    d = torch.arange(D, device=pages.device)
    slot = slot.view(-1, 1)
    if values:
        byte = ((slot // 8) * (D // 4) + d // 4) * 16 + (slot % 8) * 2 + (d % 4) // 2
        scale = bs * D // 2 + (d // 32) * bs + slot
    else:
        byte = ((d // 32) * bs + slot) * 16 + (d % 32) // 2
        scale = bs * D // 2 + slot * (D // 32) + d // 32
    row = pages[block]                                                     # [T, H, bytes]
    pick = lambda at: row.gather(2, at.unsqueeze(1).expand(-1, row.shape[1], -1)).long()
    code = (pick(byte) >> ((d % 2) * 4)) & 15
    size = code & 7
    # E2M1: exponent in bits 2 .. 1 (bias 1), mantissa in bit 0
    mag = torch.where(size < 2, size.double() * 0.5, (1.0 + (size & 1) * 0.5).double() * torch.exp2(((size >> 1) - 1).double()))
    return torch.where(code >= 8, -mag, mag) * torch.exp2(pick(scale).double() - 127.0)


def _exact_stored(x):
    """float64 values that rows x [..., D] are stored as: the nearest of each block's grid, ties to the even code."""
    b = x.double().unflatten(-1, (-1, 32))
    top = b.abs().amax(-1, keepdim=True)
    e = torch.floor(torch.log2(torch.where(top > 0, top, torch.ones_like(top))))
    s = torch.where(top > 1.75 * torch.exp2(e), e - 1, e - 2)
    s = torch.where(top > 0, s, torch.full_like(s, -125.0)).clamp(-125, 125)
    grid = torch.tensor(_VALUES, dtype=torch.float64, device=x.device)
    far = (b.abs().unsqueeze(-1) / torch.exp2(s).unsqueeze(-1) - grid).abs()
    # ties to the even code: an odd one is pushed off by less than any other difference of two distances
    pick = (far + 1e-9 * (torch.arange(8, device=x.device) % 2)).argmin(-1)
    return (torch.copysign(grid[pick], b) * torch.exp2(s)).flatten(-2)


def _exact_rows(q, key, value, hidden, scale):
    """q [H, R, D], key / value [H, K, D], hidden [R, K]: float64 softmax average and log-sum-exp."""
    s = torch.matmul(q, key.transpose(1, 2).contiguous()) * scale
    s = torch.where(hidden, torch.full_like(s, -math.inf), s)
    lse = torch.logsumexp(s, -1)
    return torch.matmul(torch.exp(s - lse.unsqueeze(-1)), value), lse


def _exact_prompt(case, s):
    Hkv, Hq, D = case["kv_heads"], case["q_heads"], case["head_dim"]
    G, scale = Hq // Hkv, 1.0 / math.sqrt(D)
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    cu = np.concatenate([[0], np.cumsum(_lengths(case))])
    for b in range(case["prompts"]):
        lo, hi = int(cu[b]), int(cu[b + 1])
        at = torch.arange(hi - lo, device=DEV)
        for h in range(Hq):
            k, v = (s[x][lo:hi, h // G].double().unsqueeze(0) for x in "kv")
            for r in at.split(1024):
                last = int(r[-1]) + 1
                o, l = _exact_rows(s["q"][lo + r, h].double().unsqueeze(0), k[:, :last], v[:, :last],
                                   at[:last].unsqueeze(0) > r.unsqueeze(1), scale)
                out[lo + r, h], lse[lo + r, h] = o[0], l[0]
    return (out, lse) if case["lse"] else out


def _exact_attention(case, s, appended=None):
    """``appended``: per sequence (K rows, V rows) in float64 that follow the cached prefix."""
    Hkv, Hq, D, bs = case["kv_heads"], case["q_heads"], case["head_dim"], case["block_size"]
    G, scale, L = Hq // Hkv, 1.0 / math.sqrt(D), _lengths(case)
    cu = np.concatenate([[0], np.cumsum(_nodes(case))])
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    for b in range(case["batch"]):
        lo, hi = int(cu[b]), int(cu[b + 1])
        t = torch.arange(int(L[b]), device=DEV)
        block = s["table"][b].long()[t // bs]
        k, v = ([_exact_page_rows(s[c], block, t % bs, bs, D, c == "vc")] for c in ("kc", "vc"))
        if appended:
            k.append(appended[b][0])
            v.append(appended[b][1])
        k, v = (torch.cat(x + [s[y][lo:hi].double()]) for x, y in ((k, "kt"), (v, "vt")))
        hidden = torch.zeros((hi - lo, k.shape[0]), dtype=torch.bool, device=DEV)
        for i in range(lo, hi):
            w = s["mask"][i].tolist()
            bits = (w[0] & (2 ** 64 - 1)) | ((w[1] & (2 ** 64 - 1)) << 64)
            hidden[i - lo, k.shape[0] - (hi - lo):] = torch.tensor([not (bits >> j) & 1 for j in range(hi - lo)], device=DEV)
        for h in range(Hkv):
            q = s["q"][lo:hi, h * G:(h + 1) * G].double().transpose(0, 1)           # [G, n, D]
            o, l = _exact_rows(q, k[:, h].unsqueeze(0).expand(G, -1, -1).contiguous(),
                               v[:, h].unsqueeze(0).expand(G, -1, -1).contiguous(), hidden, scale)
            out[lo:hi, h * G:(h + 1) * G], lse[lo:hi, h * G:(h + 1) * G] = o.transpose(0, 1), l.t()
    return (out, lse) if case["lse"] else out


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "prompt":
        return _exact_prompt(case, s)
    if case["kind"] == "attention":
        return _exact_attention(case, s)
    if case["kind"] == "write":
        return _exact_stored(s["k"]), _exact_stored(s["v"])
    done = s["done"].tolist()
    first = np.concatenate([[0], np.cumsum(np.array(done) + 1)])
    k, v = _exact_stored(s["k_old"][s["rows"]]), _exact_stored(s["v_old"][s["rows"]])
    parts = [(k[first[b]:first[b + 1]], v[first[b]:first[b + 1]]) for b in range(case["batch"])]
    return s["len"] + s["done"] + 1, _exact_attention(case, s, parts), k, v
