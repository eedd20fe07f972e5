"""Performance cases of the operators of a target model's layer with a sliding window, from its projections to its attention:

  prompt       causal attention of packed prompts in which a token sees the last ``window`` tokens, its own among them, and the
               first ``sinks`` tokens of its prompt
  tree         the same window for draft trees over a paged cache whose pages behind the window have been given back; trees of
               one node are plain decoding
  norm         each head of the queries and keys of one projection divided by its root mean square, weighted, and rotated by
               its token's position
  blocks       the page bookkeeping between two steps: pages that the window has left and those of finished sequences go back
               to the list of free ones, then block tables and slot maps of the tokens that come next

A node at depth d of a tree over a prefix of L tokens has position L + d, a cached token its index; a query at position p sees
the keys at positions k <= p with p - k < window or k < sinks (of its tree's nodes, its ancestors and itself).

Lengths and tree sizes of a case come from ``case["shape_seed"]`` alone (they are the case's work); values, tree shapes and
block permutations come from the seed that prepare() gets.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DEV = "cuda:0"
_TORCH = {"bf16": torch.bfloat16, "f32": torch.float32}
_K_SCALE, _V_SCALE = 0.0625, 0.03125                  # of fp8 caches: powers of two, the largest stored values well inside 448
_EPS, _BASE = 1e-6, 500000.0
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
def _prompt(name, prompts, tokens, heads, window, sinks, dtype="bf16", head_dim=128, lse=False, shape_seed=0):
    c = dict(kind="prompt", prompts=prompts, tokens_min=tokens[0], tokens_max=tokens[1], q_heads=heads[0], kv_heads=heads[1],
             window=window, sinks=sinks, dtype=dtype, head_dim=head_dim, lse=lse, shape_seed=shape_seed)
    if name:
        c["name"] = name
    return c


def _tree(name, batch, heads, prefix, nodes, window, sinks, dtype="bf16", cache="same", layout="interleaved", head_dim=128,
          block_size=16, lse=False, shape_seed=0):
    c = dict(kind="tree", batch=batch, q_heads=heads[0], kv_heads=heads[1], prefix_min=prefix[0], prefix_max=prefix[1],
             nodes_min=nodes[0], nodes_max=nodes[1], window=window, sinks=sinks, dtype=dtype, cache=cache, layout=layout,
             head_dim=head_dim, block_size=block_size, lse=lse, shape_seed=shape_seed)
    if name:
        c["name"] = name
    return c


def _norm(name, tokens, heads, dtype="bf16", head_dim=128, rotary_dim=128, pairing="half", shape_seed=0):
    c = dict(kind="norm", tokens=tokens, q_heads=heads[0], kv_heads=heads[1], dtype=dtype, head_dim=head_dim,
             rotary_dim=rotary_dim, pairing=pairing, shape_seed=shape_seed)
    if name:
        c["name"] = name
    return c


def _blocks(name, running, finished, fresh, prefix, step, prompt, window, sinks, block_size=16, slack=0, short=False, shape_seed=0):
    c = dict(kind="blocks", running=running, finished=finished, fresh=fresh, prefix_min=prefix[0], prefix_max=prefix[1], step=step,
             prompt_min=prompt[0], prompt_max=prompt[1], window=window, sinks=sinks, block_size=block_size, slack=slack,
             short=short, shape_seed=shape_seed)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one user's message, little longer than the window: latency
        _prompt("prompt_one_short", 1, (301, 301), (32, 8), 128, 4, shape_seed=1),
        # an admission batch of a server: ragged prompts of an 8B model, log-sum-exp kept for a later merge
        _prompt("prompt_batch_ragged", 5, (300, 5000), (32, 8), 1024, 4, lse=True, shape_seed=2),
        # a document at 70B shapes: the most arithmetic
        _prompt("prompt_long", 1, (16384, 16384), (64, 8), 4096, 0, shape_seed=3),
        # fp32 prefill of a small model with a narrow window
        _prompt("prompt_f32", 8, (128, 1536), (8, 2), 200, 3, dtype="f32", head_dim=64, lse=True, shape_seed=4),
        # one interactive user well into a conversation: a small tree; latency
        _tree("tree_one", 1, (32, 8), (5003, 5003), (7, 7), 512, 4, shape_seed=5),
        # a loaded server, trees of all sizes over conversations of all lengths
        _tree("tree_batch32_wide_trees", 32, (32, 8), (100, 8192), (4, 64), 1024, 4, lse=True, shape_seed=6),
        # plain decoding at 70B shapes and long contexts, one token a sequence: the most bytes
        _tree("tree_batch64_single_token", 64, (64, 8), (16384, 16384), (1, 1), 4096, 0, shape_seed=7),
        # a small server with an fp8 cache in plain pages
        _tree("tree_batch12_fp8_plain", 12, (28, 4), (1500, 8192), (10, 24), 2000, 64, cache="fp8", layout="plain", shape_seed=8),
        # the tree of one verification step
        _norm("norm_step", 41, (32, 8), shape_seed=9),
        # a prefill chunk
        _norm("norm_prefill", 16384, (32, 8), shape_seed=10),
        # a server between two verification steps: room for the deepest accepted path, a few sequences done
        _blocks("blocks_step", 64, 3, 0, (500, 16384), 9, (1, 1), 4096, 4, shape_seed=11),
        # the same with an admission batch of ragged prompts
        _blocks("blocks_admission", 200, 20, 48, (100, 16384), 9, (1, 8192), 1024, 4, slack=1000, shape_seed=12),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    caps = {c["name"]: work(c) for c in listed()}
    kind = rng.choices(["prompt", "tree", "norm", "blocks"], [4, 5, 2, 2])[0]
    shape_seed = rng.randrange(1, 1 << 30)
    heads = rng.choice([(8, 2), (32, 8), (32, 8), (28, 4), (64, 8), (8, 8)])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    head_dim = rng.choice([64, 128, 128])
    sinks = rng.choice([0, 1, 4, 4, 17, 64, 200])
    if kind == "norm":
        dim = rng.choice([head_dim, head_dim, 80, 96])
        return _norm(None, _log_int(rng, 1, 16384 if dtype == "bf16" else 8192), rng.choice([(8, 2), (32, 8), (28, 4), (8, 8)]),
                     dtype, dim, rng.choice([dim, dim, dim // 2, 32]), rng.choice(["half", "half", "interleaved"]), shape_seed)
    if kind == "blocks":
        running = _log_int(rng, 1, 256)
        hi = _log_int(rng, 1, 16384)
        return _blocks(None, running, rng.randrange(0, running // 4 + 1), rng.choice([0, 1, 7, 48]), (max(1, hi // 20), hi),
                       rng.choice([1, 5, 9, 17]), (1, _log_int(rng, 1, 8192)), _log_int(rng, 16, 8192), sinks,
                       rng.choice([8, 16, 16, 32, 64]), rng.choice([0, 0, 333]), rng.random() < 0.2, shape_seed)
    if kind == "prompt":
        cap = caps["prompt_f32" if dtype == "f32" else "prompt_long"]
        while True:
            hi = _log_int(rng, 1, 1536 if dtype == "f32" else 16384)
            lo = rng.choice([hi, max(1, hi // 2), max(1, hi // 30)])
            c = _prompt(None, _log_int(rng, 1, 64), (lo, hi), heads, _log_int(rng, 1, 2 * hi), sinks, dtype, head_dim,
                        rng.random() < 0.4, shape_seed)
            w = work(c)
            if w["flops"] <= cap["flops"] and w["bytes"] <= 4 * cap["bytes"]:
                return c
    cap, other = caps["tree_batch64_single_token"], caps["tree_batch32_wide_trees"]
    while True:
        hi = _log_int(rng, 1, 1536 if dtype == "f32" else 16384)
        lo = rng.choice([hi, max(1, hi // 2), max(1, hi // 8)])
        n_hi = rng.choice([1, 1, 7, 10, 24, 48, 64, 128])
        n_lo = rng.choice([n_hi, max(1, n_hi // 2), max(1, n_hi // 12)])
        c = _tree(None, _log_int(rng, 1, 96 if dtype == "bf16" else 24), heads, (lo, hi), (n_lo, n_hi), _log_int(rng, 1, 8192), sinks,
                  dtype, rng.choice(["same", "same", "fp8"]), rng.choice(["interleaved", "plain"]), head_dim,
                  rng.choice([8, 16, 16, 16, 32, 64]), rng.random() < 0.4, shape_seed)
        w = work(c)
        if w["bytes"] <= cap["bytes"] and w["flops"] <= max(cap["flops"], other["flops"]):
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


def _normal(seed, stream, shape, dtype):
    g = torch.Generator(device=DEV).manual_seed(seed * 64 + stream)
    return torch.randn(shape, generator=g, device=DEV, dtype=torch.float32).to(dtype)


def _keys(seed, stream, shape, dtype):
    """Normal values with a few strong head dims, as the keys of trained models have them."""
    g = torch.Generator(device=DEV).manual_seed(seed * 64 + stream)
    x = torch.randn(shape, generator=g, device=DEV, dtype=torch.float32)
    x[..., 5::37] *= 3.0
    return x.to(dtype)


def _dev(a, dtype=None):
    return torch.from_numpy(np.ascontiguousarray(a, dtype)).to(DEV)


def _trees(seed, n):
    """Parent arrays (local indices) of random trees, concatenated."""
    g = np.random.default_rng([seed, 4])
    return np.concatenate([np.array([-1] + [int(g.integers(max(0, i - 8), i)) for i in range(1, m)], np.int32) for m in n])


def _ancestors(cu, parent):
    """The ancestors-or-self of every node (local ids): bit sets, and the two 64-bit words of each."""
    sets, cu, parent = [0] * len(parent), cu.tolist(), parent.tolist()
    for lo, hi in zip(cu, cu[1:]):
        for i in range(lo, hi):
            sets[i] = (1 << (i - lo)) | (sets[lo + parent[i]] if parent[i] >= 0 else 0)
    return sets, np.array([[s & (2 ** 64 - 1), s >> 64] for s in sets], np.uint64).view(np.int64)


def _prepare_prompt(case, seed):
    cu = _offsets(_lengths(case))
    T, D, dt = int(cu[-1]), case["head_dim"], _TORCH[case["dtype"]]
    return dict(case=case, cu=_dev(cu), h_cu=cu, q=_normal(seed, 1, (T, case["q_heads"], D), dt),
                k=_keys(seed, 2, (T, case["kv_heads"], D), dt), v=_normal(seed, 3, (T, case["kv_heads"], D), dt))


def _seen_tokens(case, L):
    """The cached tokens that some node of a tree over L tokens sees (its root sees the most)."""
    return np.concatenate([np.arange(min(case["sinks"], L)), np.arange(max(min(case["sinks"], L), L - case["window"] + 1), L)])


def _prepare_tree(case, seed):
    L, n = _lengths(case), _nodes(case)
    cu, parent = _offsets(n), _trees(seed, n)
    N, D, H, bs, dt = int(cu[-1]), case["head_dim"], case["kv_heads"], case["block_size"], _TORCH[case["dtype"]]
    # pages that nobody sees have been given back, and their entries hold anything
    live = [np.unique(_seen_tokens(case, int(x)) // bs) for x in L]
    num_blocks = sum(len(x) for x in live) + 3
    g = np.random.default_rng([seed, 5])
    perm, at = g.permutation(num_blocks).astype(np.int32), 0
    table = g.integers(-5, num_blocks + 5, (case["batch"], (int(L.max()) + bs - 1) // bs + 1)).astype(np.int32)
    for b, x in enumerate(live):
        table[b, x] = perm[at:at + len(x)]
        at += len(x)
    sets, words = _ancestors(cu, parent)
    ancestor = np.zeros((N, int(n.max())), bool)
    for i, s in enumerate(sets):
        ancestor[i] = [(s >> j) & 1 for j in range(ancestor.shape[1])]
    kc, vc = _keys(seed, 4, (num_blocks, H, bs, D), torch.float32), _normal(seed, 5, (num_blocks, H, bs, D), torch.float32)
    if case["cache"] == "fp8":
        kc, vc = ((x / s).to(torch.float8_e4m3fn).view(torch.uint8) for x, s in ((kc, _K_SCALE), (vc, _V_SCALE)))
    else:
        kc, vc = kc.to(dt), vc.to(dt)
    if case["layout"] == "interleaved":
        kc = kc.view(num_blocks, H, bs, D // 8, 8).permute(0, 1, 3, 2, 4).contiguous()
        vc = vc.view(num_blocks, H, bs // 8, 8, D).permute(0, 1, 2, 4, 3).contiguous()
    return dict(case=case, q=_normal(seed, 1, (N, case["q_heads"], D), dt), kt=_keys(seed, 2, (N, H, D), dt),
                vt=_normal(seed, 3, (N, H, D), dt), kc=kc, vc=vc, table=_dev(table), len=_dev(L, np.int32), cu=_dev(cu),
                mask=_dev(words), ancestor=_dev(ancestor), h_cu=cu, h_len=L)


def _prepare_norm(case, seed):
    N, Hq, H, D, dt = case["tokens"], case["q_heads"], case["kv_heads"], case["head_dim"], _TORCH[case["dtype"]]
    proj = _keys(seed, 1, (N, Hq + 2 * H, D), dt)          # one projection's output: queries, keys, values of a token
    g = np.random.default_rng([seed, 7])
    position = (g.integers(0, 131072, N) if N < 1000 else np.arange(N) + g.integers(0, 100000)).astype(np.int32)
    weight = [1.0 + 0.2 * torch.randn(D, generator=torch.Generator(device=DEV).manual_seed(seed * 64 + x), device=DEV) for x in (2, 3)]
    return dict(case=case, q=proj[:, :Hq], k=proj[:, Hq:Hq + H], position=_dev(position), wq=weight[0].to(dt), wk=weight[1].to(dt))


def _block_sizes(case):
    """Lengths, tokens to come and a flag for sequences that are done: running sequences (the done ones among them), then fresh."""
    running, fresh = case["running"], case["fresh"]
    length = np.concatenate([_spread(case, 1, case["prefix_min"], case["prefix_max"], running), np.zeros(fresh, np.int64)])
    done = np.zeros(running + fresh, np.int64)
    done[np.random.default_rng([case["shape_seed"], 3]).permutation(running)[:case["finished"]]] = 1
    new = np.concatenate([np.full(running, case["step"]), _spread(case, 2, case["prompt_min"], case["prompt_max"], fresh)])
    return length, np.where(done == 1, 0, new), done


def _prepare_blocks(case, seed):
    bs, S = case["block_size"], case["sinks"]
    length, new, done = _block_sizes(case)
    ceil = lambda x: (x + bs - 1) // bs
    held = ceil(length + np.where(length > 0, case["step"] // 2, 0))        # room that the step before did not fill
    # the step before gave back what its window had left
    left = np.maximum(0, np.maximum(0, length - case["step"] - case["window"] + 1) // bs)
    released = np.where(left > ceil(S), left, 0)
    kept = held - np.maximum(0, released - ceil(S))
    need = int(np.maximum(0, ceil(np.where(done == 1, 0, length) + new) - held).sum())
    spare = need // 2 if case["short"] else need + 16                        # some servers run short of pages
    num_blocks = int(kept.sum()) + spare
    g = np.random.default_rng([seed, 8])
    perm, at = g.permutation(num_blocks).astype(np.int32), 0
    width = int(ceil(max((length + new).max(), 1)) + case["step"] + 1)
    table = g.integers(-5, num_blocks + 5, (len(length), width)).astype(np.int32)
    for b in range(len(length)):
        pages = [j for j in range(held[b]) if j < ceil(S) or j >= released[b]]
        table[b, pages] = perm[at:at + len(pages)]
        at += len(pages)
    free = np.full(num_blocks, -1, np.int32)
    free[:spare] = perm[at:at + spare]
    i32 = lambda x: _dev(x, np.int32)
    return dict(case=case, length=i32(length), new=i32(new), held=i32(held), released=i32(released), done=i32(done),
                table=i32(table), free=i32(free), count=i32([spare]), num_blocks=num_blocks, cap=int(new.sum()) + case["slack"])


def prepare(case, seed):
    return dict(prompt=_prepare_prompt, tree=_prepare_tree, norm=_prepare_norm, blocks=_prepare_blocks)[case["kind"]](case, seed)


# ---------------------------------------------------------------------------
# one pass, in elementary operations
# ---------------------------------------------------------------------------
def _softmax_rows(s):
    """exp(s - max) and its sum, along the last dimension, and the logarithm of the sum of exp(s)."""
    top = s.amax(-1, keepdim=True)
    p = torch.exp(s - top)
    total = p.sum(-1, keepdim=True)
    return p, total, (top + torch.log(total)).squeeze(-1)


def _seen(query, key, window, sinks):
    """query [.., 1] and key [K] positions."""
    return (key <= query) & ((query - key < window) | (key < sinks))


def _plain_prompt(s):
    c = s["case"]
    q, k, v, Hkv, G = s["q"], s["k"], s["v"], c["kv_heads"], c["q_heads"] // c["kv_heads"]
    W, S, scale = c["window"], c["sinks"], 1.0 / math.sqrt(c["head_dim"])
    out = torch.empty_like(q)
    lse = torch.empty(q.shape[:2], dtype=torch.float32, device=q.device)
    for lo, hi in zip(s["h_cu"][:-1].tolist(), s["h_cu"][1:].tolist()):
        rows = max(1, min(2048, (1 << 28) // (c["q_heads"] * (hi - lo))))     # of a piece: its scores are one array
        key, value = (x[lo:hi].float().transpose(0, 1).contiguous() for x in (k, v))
        for r0 in range(0, hi - lo, rows):
            r1 = min(hi - lo, r0 + rows)
            first = max(0, r0 - W + 1)
            at = torch.arange(first, r1, device=q.device)
            if S and first:
                at = torch.cat([torch.arange(min(S, first), device=q.device), at])
            qs = q[lo + r0:lo + r1].float().unflatten(1, (Hkv, G)).permute(1, 2, 0, 3).flatten(1, 2)     # [Hkv, G rows, D]
            score = (torch.matmul(qs, key[:, at].transpose(1, 2).contiguous()) * scale).unflatten(1, (G, r1 - r0))
            hidden = ~_seen(torch.arange(r0, r1, device=q.device).unsqueeze(1), at, W, S)
            p, total, row = _softmax_rows(score.masked_fill(hidden, -math.inf))
            o = torch.matmul(p.flatten(1, 2), value[:, at]).unflatten(1, (G, r1 - r0)) / total
            out[lo + r0:lo + r1] = o.permute(2, 0, 1, 3).flatten(1, 2).to(out.dtype)
            lse[lo + r0:lo + r1] = row.permute(2, 0, 1).flatten(1, 2)
    return (out, lse) if c["lse"] else out


def _plain_pages(pages, c, values):
    """Pages of the cache -> the fp32 values [pages, bs, H, D] they hold."""
    x = pages.view(torch.float8_e4m3fn).float() * (_V_SCALE if values else _K_SCALE) if c["cache"] == "fp8" else pages.float()
    if c["layout"] == "plain":
        return x.permute(0, 2, 1, 3)
    return (x.permute(0, 2, 4, 1, 3) if values else x.permute(0, 3, 1, 2, 4)).reshape(len(x), c["block_size"], c["kv_heads"], c["head_dim"])


def _plain_tree(s):
    c = s["case"]
    bs, D, Hkv, G, W, S = c["block_size"], c["head_dim"], c["kv_heads"], c["q_heads"] // c["kv_heads"], c["window"], c["sinks"]
    out = torch.empty_like(s["q"])
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float32, device=out.device)
    for b, L in enumerate(s["h_len"].tolist()):
        lo, hi = int(s["h_cu"][b]), int(s["h_cu"][b + 1])
        n, tokens = hi - lo, _dev(_seen_tokens(c, L))
        used, where = torch.unique(tokens // bs, return_inverse=True)
        pages = s["table"][b, used].long()
        key = torch.cat([_plain_pages(s["kc"][pages], c, False)[where, tokens % bs], s["kt"][lo:hi].float()])
        value = torch.cat([_plain_pages(s["vc"][pages], c, True)[where, tokens % bs], s["vt"][lo:hi].float()])
        ancestor = s["ancestor"][lo:hi, :n]
        position = L + ancestor.sum(1) - 1
        q = s["q"][lo:hi].float().view(n, Hkv, G, D).permute(1, 0, 2, 3).reshape(Hkv, n * G, D)
        score = torch.matmul(q, key.permute(1, 2, 0).contiguous()) / math.sqrt(D)
        seen = torch.cat([_seen(position.unsqueeze(1), tokens, W, S), ancestor & _seen(position.unsqueeze(1), position, W, S)], 1)
        score = score.masked_fill(~seen.repeat_interleave(G, 0), -math.inf)
        p, total, row = _softmax_rows(score)
        o = torch.matmul(p, value.transpose(0, 1).contiguous()) / total
        out[lo:hi] = o.view(Hkv, n, G, D).permute(1, 0, 2, 3).reshape(n, Hkv * G, D).to(out.dtype)
        lse[lo:hi] = row.view(Hkv, n, G).permute(1, 0, 2).reshape(n, Hkv * G)
    return (out, lse) if c["lse"] else out


def _plain_norm(s):
    c = s["case"]
    rot, half = c["rotary_dim"], c["rotary_dim"] // 2
    rate = torch.exp2(torch.arange(half, device=s["q"].device, dtype=torch.float64) * (-2.0 / rot * math.log2(_BASE)))
    angle = (s["position"].double().unsqueeze(1) * rate).unsqueeze(1)                    # [N, 1, rot / 2]
    cos, sin = torch.cos(angle).float(), torch.sin(angle).float()
    out = []
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
        y = x.float()
        y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + _EPS) * w.float()
        a, b = (y[..., :half], y[..., half:rot]) if c["pairing"] == "half" else (y[..., 0:rot:2], y[..., 1:rot:2])
        turned = (a * cos - b * sin, a * sin + b * cos)
        turned = torch.cat(turned, -1) if c["pairing"] == "half" else torch.stack(turned, -1).flatten(-2)
        out.append(torch.cat([turned, y[..., rot:]], -1).to(x.dtype))
    return tuple(out)


def _within(count, first):
    """For rows count[b] behind one another: each row's b, and its number within b plus first[b]."""
    b = torch.repeat_interleave(torch.arange(len(count), device=count.device), count)
    start = torch.cumsum(count, 0) - count
    return b, torch.arange(len(b), device=count.device) - start[b] + first[b]


def _plain_blocks(s):
    c = s["case"]
    bs, W, table, free = c["block_size"], c["window"], s["table"], s["free"]
    length, new, held, released, done, have = (s[x].long() for x in ("length", "new", "held", "released", "done", "count"))
    done, width, dev = done != 0, table.shape[1], table.device
    zero = torch.zeros_like(length)
    sink = torch.minimum(held, torch.full_like(held, (c["sinks"] + bs - 1) // bs))
    # pages back to the list: behind the window, or all that a finished sequence still has
    first = torch.maximum(sink, released)
    end = torch.where(done, held, torch.minimum((length - W + 1).clamp(min=0) // bs, held))
    tail = (end - first).clamp(min=0)
    give = tail + torch.where(done, sink, zero)
    given = torch.cumsum(give, 0)
    fits = (given <= len(free) - have) | (give == 0)
    give = torch.where(fits, give, zero)
    b, i = _within(give, zero)
    at = torch.where(done[b], torch.where(i < sink[b], i, first[b] + i - sink[b]), first[b] + i)
    free[(have + (given - give)[b] + i).long()] = table[b, at]
    have = have + give.sum()
    back = torch.where(fits, zero, zero - 3)
    gone = done & fits
    length, held = torch.where(gone, zero, length), torch.where(gone, zero, held)
    released = torch.where(gone, zero, torch.where(fits & (tail > 0), end, released))
    left = (length.int(), held.int(), released.int())
    # room for the tokens that come
    rows = torch.cumsum(new, 0)
    room = (rows <= s["cap"]) & (length + new <= width * bs)
    want = torch.where(room, ((length + new + bs - 1) // bs - held).clamp(min=0), zero)
    wanted = torch.cumsum(want, 0)
    served = room & ((wanted <= have) | (want == 0))
    want = torch.where(served, want, zero)
    b, j = _within(want, held)
    table[b, j] = free[have - 1 - ((wanted - want)[b] + j - held[b])]
    slots = torch.full((s["cap"],), -1, dtype=torch.int64, device=dev)
    take = torch.where(served, new, zero)
    b, t = _within(take, length)
    page = table[b, t // bs].long()
    page = torch.where((page < 0) | (page >= s["num_blocks"]), torch.full_like(page, -1), page)
    slots[(rows - new)[b] + t - length[b]] = torch.where(page < 0, page, page * bs + t % bs)
    cu = torch.cat([zero[:1], rows]).clamp(max=s["cap"]).int()
    return left, back.int(), dict(cu=cu, slots=slots, length=(length + take).int(), held=(held + want).int(),
                                  count=(have - want.sum()).int().view(1), status=torch.where(served, zero, zero - 3).int(),
                                  table=table, free=free)


# ---------------------------------------------------------------------------
# one pass, by the framework's calls
# ---------------------------------------------------------------------------
def _own_prompt(s):
    c = s["case"]
    return _lib().prompt_attention(s["q"], s["k"], s["v"], s["cu"], 1.0 / math.sqrt(c["head_dim"]), want_lse=c["lse"],
                                   window=c["window"], sinks=c["sinks"])


def _own_tree(s):
    from paper_2604_09731_amd import binding as B
    c = s["case"]
    fp8 = dict(k_scale=_K_SCALE, v_scale=_V_SCALE) if c["cache"] == "fp8" else {}
    layout = B.SMART_KV_PLAIN if c["layout"] == "plain" else B.SMART_KV_INTERLEAVED
    return _lib().tree_verify_attention(s["q"], s["kt"], s["vt"], s["kc"], s["vc"], s["table"], s["len"], s["cu"], s["mask"],
                                        1.0 / math.sqrt(c["head_dim"]), layout, block_size=c["block_size"], want_lse=c["lse"],
                                        window=c["window"], sinks=c["sinks"], **fp8)


def _own_norm(s):
    from paper_2604_09731_amd import binding as B
    c = s["case"]
    pairing = B.SMART_ROPE_HALF_SPLIT if c["pairing"] == "half" else B.SMART_ROPE_INTERLEAVED
    return _lib().tree_norm_rope(s["position"], s["q"], s["k"], s["wq"], s["wk"], eps=_EPS, base=_BASE, rotary_dim=c["rotary_dim"],
                                 pairing=pairing)


def _own_blocks(s):
    c, lib = s["case"], _lib()
    length, held, released, count, back = lib.kv_cache_release(s["length"], s["held"], s["released"], s["table"], s["free"], s["count"],
                                                               c["block_size"], finished=s["done"], window=c["window"],
                                                               sinks=c["sinks"])
    cu, slots, new_length, new_held, new_count, status = lib.kv_cache_extend(length, s["new"], held, s["table"], s["free"], count,
                                                                             c["block_size"], s["num_blocks"], s["cap"])
    return (length, held, released), back, dict(cu=cu, slots=slots, length=new_length, held=new_held, count=new_count, status=status,
                                                table=s["table"], free=s["free"])


def run(state):
    kind = state["case"]["kind"]
    if own:
        return dict(prompt=_own_prompt, tree=_own_tree, norm=_own_norm, blocks=_own_blocks)[kind](state)
    return dict(prompt=_plain_prompt, tree=_plain_tree, norm=_plain_norm, blocks=_plain_blocks)[kind](state)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------
def work(case):
    if case["kind"] == "blocks":
        bs = case["block_size"]
        length, new, done = _block_sizes(case)
        taken = int(np.maximum(0, -(-(length + new) // bs) - -(-length // bs)).sum())
        back = int((done * -(-np.minimum(length, case["window"] + case["sinks"]) // bs)).sum()) + case["running"] // 2
        # five numbers a sequence in and seven out, a table entry of its last page; free-list and table entries; slots
        return {"bytes": len(length) * (12 + 1) * 4 + (taken + back) * 8 + (int(new.sum()) + case["slack"]) * 8, "flops": 0}
    e, D, H, Hq = 4 if case["dtype"] == "f32" else 2, case["head_dim"], case["kv_heads"], case["q_heads"]
    if case["kind"] == "norm":
        n = case["tokens"] * (Hq + H) * D
        return {"bytes": 2 * n * e + case["tokens"] * 4 + 2 * D * e, "flops": 8 * n}
    L = _lengths(case).astype(np.int64)
    span = case["window"] + case["sinks"]
    if case["kind"] == "prompt":
        T = int(L.sum())
        full = np.minimum(L, span)                        # tokens that see all that came before them
        return {"bytes": T * D * e * 2 * (Hq + H) + (T * Hq * 4 if case["lse"] else 0),
                "flops": 4 * D * Hq * int((full * (full + 1) // 2 + (L - full) * span).sum())}
    n, keys = _nodes(case).astype(np.int64), np.minimum(L, span - 1)
    N = int(n.sum())
    row = 2 * D * (1 if case["cache"] == "fp8" else e)    # K and V of one token and head
    table = int(((keys + case["block_size"] - 1) // case["block_size"]).sum()) * 4
    return {"bytes": int(keys.sum()) * H * row + N * 2 * (Hq + H) * D * e + N * 16 + table + (N * Hq * 4 if case["lse"] else 0),
            "flops": 4 * D * Hq * int((n * keys).sum() + N)}


# ---------------------------------------------------------------------------
# the definition in 64 bits
# ---------------------------------------------------------------------------
def _exact_rows(q, key, value, seen, scale):
    """q [R, D], key / value [K, D], seen [R, K]: float64 softmax average and log-sum-exp."""
    score = torch.where(seen, torch.matmul(q, key.t().contiguous()) * scale, torch.full((), -math.inf, dtype=torch.float64, device=DEV))
    lse = torch.logsumexp(score, -1)
    return torch.matmul(torch.exp(score - lse.unsqueeze(-1)), value), lse


def _exact_prompt(case, s):
    Hq, G, W, S = case["q_heads"], case["q_heads"] // case["kv_heads"], case["window"], case["sinks"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    at = 0
    for L in _lengths(case).tolist():
        for r in torch.arange(L, device=DEV).split(1024):
            p0, p1 = int(r[0]), int(r[-1])
            u = torch.arange(p1 + 1, device=DEV)
            u = u[(u < S) | (u > p0 - W)]
            back = r.unsqueeze(1) - u.unsqueeze(0)                             # how far behind its query a key lies
            seen = (back >= 0) & ((back < W) | (u < S).unsqueeze(0))
            for h in range(Hq):
                k, v = s["k"][at + u, h // G].double(), s["v"][at + u, h // G].double()
                out[at + r, h], lse[at + r, h] = _exact_rows(s["q"][at + r, h].double(), k, v, seen, case["head_dim"] ** -0.5)
        at += L
    return (out, lse) if case["lse"] else out


def _exact_cached(case, s, table, t, values):
    """float64 [tokens, H, D] of the cached tokens t, element by element through the layouts' offsets."""
    bs, D, pages = case["block_size"], case["head_dim"], s["vc" if values else "kc"]
    d, slot = torch.arange(D, device=DEV), (t % bs).unsqueeze(1)
    if case["layout"] == "plain":
        at = slot * D + d
    else:
        at = ((slot // 8) * D + d) * 8 + slot % 8 if values else ((d // 8) * bs + slot) * 8 + d % 8
    page = pages.flatten(2)[table.long()[t // bs]]                             # [tokens, H, bs D]
    x = page.gather(2, at.unsqueeze(1).expand(-1, page.shape[1], -1))
    if case["cache"] != "fp8":
        return x.double()
    x = x.long()                                                               # E4M3: bias 7, subnormals at exponent 0
    e, m = (x >> 3) & 15, (x & 7).double()
    size = torch.where(e == 0, m * 2.0 ** -9, (1 + m / 8) * torch.exp2((e - 7).double()))
    return torch.where(x >= 128, -size, size) * (_V_SCALE if values else _K_SCALE)


def _exact_tree(case, s):
    Hq, G, W, S, D = case["q_heads"], case["q_heads"] // case["kv_heads"], case["window"], case["sinks"], case["head_dim"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=DEV)
    lse = torch.empty(s["q"].shape[:2], dtype=torch.float64, device=DEV)
    cu = np.concatenate([[0], np.cumsum(_nodes(case))]).tolist()
    for b, L in enumerate(_lengths(case).tolist()):
        lo, hi = cu[b], cu[b + 1]
        line = []                                                              # local ids from the root to each node
        for i in range(lo, hi):
            w = s["mask"][i].tolist()
            bits = (w[0] & (2 ** 64 - 1)) | ((w[1] & (2 ** 64 - 1)) << 64)
            line.append([j for j in range(hi - lo) if (bits >> j) & 1])
        t = torch.arange(L, device=DEV)
        t = t[(t < S) | (t > L - W)]
        seen = torch.zeros((hi - lo, len(t) + hi - lo), dtype=torch.bool, device=DEV)
        for i, nodes in enumerate(line):
            p = L + len(nodes) - 1
            seen[i, :len(t)] = (t > p - W) | (t < S)
            seen[i, [len(t) + j for d, j in enumerate(nodes) if L + d > p - W or L + d < S]] = True
        k, v = (torch.cat([_exact_cached(case, s, s["table"][b], t, x == "vt"), s[x][lo:hi].double()]) for x in ("kt", "vt"))
        for h in range(Hq):
            out[lo:hi, h], lse[lo:hi, h] = _exact_rows(s["q"][lo:hi, h].double(), k[:, h // G], v[:, h // G], seen, D ** -0.5)
    return (out, lse) if case["lse"] else out


def _exact_norm(case, s):
    rot = case["rotary_dim"]
    i = torch.arange(rot, device=DEV)
    half = case["pairing"] == "half"
    pair = i % (rot // 2) if half else i // 2
    low = i < rot // 2 if half else i % 2 == 0
    other = (i + rot // 2) % rot if half else i + 1 - 2 * (i % 2)
    turn = s["position"].double().unsqueeze(1) * torch.pow(torch.tensor(_BASE, dtype=torch.float64, device=DEV), -2.0 * pair.double() / rot)
    cos, sin = torch.cos(turn).unsqueeze(1), torch.sin(turn).unsqueeze(1) * torch.where(low, -1.0, 1.0)
    out = []
    for x, w in ((s["q"], s["wq"]), (s["k"], s["wk"])):
        y = x.double()
        y = y / torch.sqrt(torch.linalg.vecdot(y, y).unsqueeze(-1) / y.shape[-1] + _EPS) * w.double()
        z = y[..., :rot]
        out.append(torch.cat([z * cos + z[..., other] * sin, y[..., rot:]], -1))
    return tuple(out)


def exact(case, seed):
    if case["kind"] == "blocks":
        return None
    return dict(prompt=_exact_prompt, tree=_exact_tree, norm=_exact_norm)[case["kind"]](case, prepare(case, seed))
