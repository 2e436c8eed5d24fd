"""Performance cases of the operators around a prompt and its reuse: rotary positions of several axes, the prompt's rows on
their way into the key/value cache, and the attention of a batch whose sequences share a long prefix.

Three kinds of pass:

    rope     rotary embedding of packed q and k rows by one to three position axes (text, images, video)
    append   the same rotation with the k and v rows placed in the cache, contiguous or paged, of a ragged batch
    prefix   tree (or single-token) attention over a paged cache of sequences that share their first blocks

Each has a plain form in elementary torch operations and, where ``own`` is set, the call of the framework.
Heads, prefix lengths and tree sizes are those of the package's synthetic workloads; q, k, v are N(0,1) in bf16.
"""
import math

import numpy as np
import torch

DEV = "cuda"
own = False


# ------------------------------------------------------------------------------------------------ listed cases

def _rope(name, T, heads, D, axes, theta, layout="text", interleaved=False, fused=False):
    named = {"name": name} if name else {}
    return {**named, "op": "rope", "T": T, "Hq": heads[0], "Hkv": heads[1], "D": D, "axes": axes, "theta": theta,
            "layout": layout, "interleaved": interleaved, "fused": fused}


def _append(name, B, new, old, heads, D, axes, theta, layout="text", interleaved=False, fused=False, page_rows=0,
            token_major=False):
    named = {"name": name} if name else {}
    return {**named, "op": "append", "B": B, "new_lo": new[0], "new_hi": new[1], "old_lo": old[0], "old_hi": old[1],
            "Hq": heads[0], "Hkv": heads[1], "D": D, "axes": axes, "theta": theta, "layout": layout,
            "interleaved": interleaved, "fused": fused, "page_rows": page_rows, "token_major": token_major}


def _prefix(name, B, N, P, tail, heads, page_rows, token_major=False, lse=True):
    named = {"name": name} if name else {}
    return {**named, "op": "prefix", "B": B, "N": N, "P": P, "tail_lo": tail[0], "tail_hi": tail[1], "Hq": heads[0],
            "Hkv": heads[1], "D": 128, "page_rows": page_rows, "token_major": token_major, "lse": lse}


def listed():
    return [
        # one decoding step of eight sequences: eight rows, a call's latency
        _rope("rope_8_tokens", 8, (28, 4), 128, "16,24,24", 1e6),
        # the prompt of Qwen2.5-VL 7B with its image, q and k still inside the rows of the fused projection
        _rope("rope_image_prompt", 3344, (28, 4), 128, "16,24,24", 1e6, "image", fused=True),
        # a long video of Qwen2.5-VL 3B, axes dealt in turn
        _rope("rope_video", 32768, (16, 2), 128, "24,20,20", 1e6, "video", interleaved=True),
        # one new token for each of 32 running sequences, pool of 16-slot blocks
        _append("append_tokens_b32", 32, (1, 1), (3000, 5000), (40, 40), 128, "64", 1e4, page_rows=16, token_major=True),
        # one image prompt into an empty sequence of the pool
        _append("append_image_prompt", 1, (3344, 3344), (0, 0), (28, 4), 128, "16,24,24", 1e6, "image", fused=True,
                page_rows=16),
        # a ragged batch of LLaVA-1.6 13B prompts into the contiguous cache, one axis
        _append("append_ragged_b4", 4, (3000, 5000), (0, 0), (40, 40), 128, "64", 1e4),
        # the follow-up turns of eight running video chats of Qwen2.5-VL 3B, large blocks
        _append("append_chunks_b8", 8, (301, 2048), (1000, 16384), (16, 2), 128, "16,24,24", 1e6, "video", fused=True,
                page_rows=128, token_major=True),
        # eight samples on one image, one token each: latency
        _prefix("prefix_decode_b8", 8, 1, 3344, (46, 354), (28, 4), 16),
        # 32 answers on one image, multi-head: one row per sequence and head
        _prefix("prefix_decode_mha_b32", 32, 1, 2880, (46, 354), (40, 40), 32, token_major=True),
        # eight samples on one image with full draft trees, LLaVA-1.6 7B
        _prefix("prefix_tree_llava7b_b8", 8, 60, 3904, (46, 354), (32, 32), 16, token_major=True),
        # four questions on one image with Qwen2.5-VL 7B's grouped heads
        _prefix("prefix_tree_qwen7b_b4", 4, 60, 3344, (46, 354), (28, 4), 64),
        # the largest: eight full-size trees behind one very long video
        _prefix("prefix_tree_S32768_b8", 8, 128, 32768, (300, 2048), (16, 2), 128),
    ]


# ------------------------------------------------------------------------------------------------ drawn cases

_HEADS = [(32, 32), (28, 4), (40, 40), (16, 2), (32, 8)]
_SECTIONS = {128: ["64", "16,24,24", "32,32", "24,20,20"], 64: ["32", "8,12,12", "16,16"]}


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    """One more case of the same ranges: sizes spread over their logarithm, odd ones among them."""
    op = rng.choice(["rope", "append", "append", "prefix", "prefix", "prefix"])
    heads = rng.choice(_HEADS)
    if op == "prefix":
        # at most the largest listed case's row-key pairs and rows of keys
        B, N = _log_int(rng, 2, 48), rng.choice([1, 1, 8, 16, 31, 60, 128, rng.randint(2, 127)])
        P, tail_hi = _log_int(rng, 100, 32768), _log_int(rng, 1, 2048)
        while B * N * heads[0] * (P + tail_hi + N) > 5.0e8 or heads[1] * (P + B * (tail_hi + N)) > 1.0e6:
            P, tail_hi = max(100, P // 2), max(1, tail_hi // 2)
            B = max(2, B // 2) if P == 100 or tail_hi == 1 else B
        tail_lo = rng.choice([0, tail_hi, rng.randint(0, tail_hi)])
        return _prefix(None, B, N, P, (tail_lo, tail_hi), heads, rng.choice([16, 32, 64, 128]), rng.random() < 0.5,
                       rng.random() < 0.7)
    D = rng.choice([128, 128, 128, 64])
    axes = rng.choice(_SECTIONS[D])
    # sections may be dealt in turn where every axis gets its share that way
    inter = axes in ("24,20,20", "32,32", "16,16") and rng.random() < 0.6
    layout = rng.choice(["image", "video"]) if "," in axes else "text"
    theta, fused = rng.choice([1e4, 1e6]), rng.random() < 0.5
    if op == "rope":
        T = _log_int(rng, 1, 32768 if heads[0] < 28 else 12000)
        return _rope(None, T, heads, D, axes, theta, layout, inter, fused)
    B = _log_int(rng, 1, 32)
    most = (200000 if heads[0] < 28 else 60000 if heads[1] < 28 else 20000) // B
    hi = _log_int(rng, 1, min(most, 8192))
    old = _log_int(rng, 1, max(2, min(most, 8192)))
    lo = rng.choice([hi, rng.randint(0, hi), 0])
    return _append(None, B, (lo, hi), (rng.randint(0, old), old), heads, D, axes, theta, layout, inter, fused,
                   rng.choice([0, 0, 16, 32, 64, 128]) if D == 128 else 0, rng.random() < 0.5)


# ------------------------------------------------------------------------------------------------ inputs

def _i32(a):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.int32)).to(DEV)


def _normal(shape, gen):
    return torch.randn(shape, generator=gen, device=DEV, dtype=torch.bfloat16)


def _tokens(case):
    """All new tokens of an append: the middle of its lengths' range per sequence."""
    return max(1, case["B"] * (case["new_lo"] + case["new_hi"]) // 2)


def _lengths(case, rng):
    """New tokens per sequence, spread over the range, with the sum that every seed has."""
    new = rng.integers(case["new_lo"], case["new_hi"] + 1, size=case["B"])
    while (off := _tokens(case) - int(new.sum())) != 0:
        b = int(rng.integers(case["B"]))
        new[b] = min(max(int(new[b]) + off, case["new_lo"]), case["new_hi"])
    return new


def _sections(case):
    return [int(x) for x in case["axes"].split(",")]


def _positions(n_axes, n, start, layout, rng):
    """Positions [n_axes, n] of n tokens that follow `start`: text, then one image or a video's frames, then text."""
    flat = np.tile(np.arange(n, dtype=np.int64), (3, 1))
    if layout != "text" and n >= 16:
        head = int(rng.integers(1, max(2, n // 8)))
        body = int((n - head) * rng.uniform(0.5, 0.95))
        frames = int(rng.integers(2, 9)) if layout == "video" else 1
        w = max(1, int(math.sqrt(body / frames)))
        h = max(1, body // (frames * w))
        body = frames * h * w
        i = np.arange(body)
        flat[0, head:head + body] = head + 2 * (i // (h * w))
        flat[1, head:head + body] = head + (i // w) % h
        flat[2, head:head + body] = head + i % w
        rest = n - head - body
        flat[:, head + body:] = flat[:, :head + body].max() + 1 + np.arange(rest)
    return start + flat[:n_axes]


def _tree(N, rng):
    """Visible nodes of a random draft tree, [N, N] truth values (each node, its ancestors)."""
    seen = np.zeros((N, N), dtype=bool)
    seen[0, 0] = True
    for i in range(1, N):
        seen[i] = seen[int(rng.integers(max(0, i - 12), i))]
        seen[i, i] = True
    return seen


def _rows(case, T, gen):
    """q, k (and v) rows of T tokens: separate tensors, or slices of the fused projection's rows."""
    Hq, Hkv, D = case["Hq"], case["Hkv"], case["D"]
    if case["fused"]:
        x = _normal((T, Hq + 2 * Hkv, D), gen)
        return x[:, :Hq], x[:, Hq:Hq + Hkv], x[:, Hq + Hkv:]
    return _normal((T, Hq, D), gen), _normal((T, Hkv, D), gen), _normal((T, Hkv, D), gen)


def _pool(case, blocks, gen):
    pr, Hkv, D = case["page_rows"], case["Hkv"], case["D"]
    shape = (blocks, pr, Hkv, D) if case["token_major"] else (blocks, Hkv, pr, D)
    return _normal(shape, gen), _normal(shape, gen)


def prepare(case, seed):
    c = dict(case)
    rng = np.random.Generator(np.random.SFC64(seed))
    gen = torch.Generator(device=DEV).manual_seed(seed)
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    s = {"c": c}
    if c["op"] == "prefix":
        B, N, P, pr = c["B"], c["N"], c["P"], c["page_rows"]
        kv_len = P + rng.integers(c["tail_lo"], c["tail_hi"] + 1, size=B)
        per, shared = (P + c["tail_hi"] + N + pr - 1) // pr, P // pr
        blocks = shared + B * (per - shared)
        perm = rng.permutation(blocks)
        table = np.concatenate([np.tile(perm[:shared], (B, 1)), perm[shared:].reshape(B, per - shared)], axis=1)
        seen = np.stack([_tree(N, rng) for _ in range(B)])
        W = (N + 63) // 64
        words = np.zeros((B, N, W), dtype=np.uint64)
        for t in range(N):
            words[:, :, t // 64] |= seen[:, :, t].astype(np.uint64) << np.uint64(t % 64)
        s["k"], s["v"] = _pool(c, blocks, gen)
        s["q"] = _normal((B, N, Hq, D), gen)
        s["kv_len"], s["table"] = _i32(kv_len), _i32(table)
        s["mask"] = torch.from_numpy(words.view(np.int64)).to(DEV)
        s["scale"] = 1.0 / math.sqrt(D)
        s["out"] = torch.zeros_like(s["q"])
        s["lse"] = torch.zeros((B, Hq, N), dtype=torch.float32, device=DEV) if c["lse"] else None
        if own:
            from paper_2509_15235_b200 import binding
            s["ctx"] = binding.VerifyContext(B, N, Hq, Hkv, D, per * pr, 1)
            s["ctx"].cache_register_paged(0, s["k"], s["v"], c["token_major"])
            s["scratch"] = s["ctx"].prefix_scratch(B, N)
        return s

    sections = _sections(c)
    if c["op"] == "rope":
        T = c["T"]
        start = int(rng.integers(0, 4096)) if c["layout"] == "text" else 0
        pos = _positions(len(sections), T, start, c["layout"], rng)
        s["q"], s["k"], _ = _rows(c, T, gen)
        B, S_max = 1, 256
    else:
        B, pr = c["B"], c["page_rows"]
        new = _lengths(c, rng)
        old = rng.integers(c["old_lo"], c["old_hi"] + 1, size=B)
        T = int(new.sum())
        pos = np.concatenate([_positions(len(sections), int(n), int(o), c["layout"], rng) for n, o in zip(new, old)], axis=1)
        S_max = (c["old_hi"] + c["new_hi"] + 1 + 127) // 128 * 128
        if pr:
            per = S_max // pr
            s["table"] = _i32(rng.permutation(B * per).reshape(B, per))
            s["k_cache"], s["v_cache"] = _pool(c, B * per, gen)
        else:
            s["k_cache"], s["v_cache"] = _normal((B, Hkv, S_max, D), gen), _normal((B, Hkv, S_max, D), gen)
        s["q"], s["k"], s["v"] = _rows(c, T, gen)
        s["kv_len"], s["cu_len"] = _i32(old), _i32(np.concatenate([[0], np.cumsum(new)]))
        s["kv_len_out"] = torch.zeros(B, dtype=torch.int32, device=DEV)
    s["positions"] = _i32(pos)
    s["q_out"] = torch.zeros((T, Hq, D), dtype=torch.bfloat16, device=DEV)
    if c["op"] == "rope":
        s["k_out"] = torch.zeros((T, Hkv, D), dtype=torch.bfloat16, device=DEV)
    if own:
        from paper_2509_15235_b200 import binding
        s["axes"] = binding.RopeAxes(sections, c["theta"], c["interleaved"])
        s["ctx"] = binding.VerifyContext(B, 1, Hq, Hkv, D, S_max, 1)
        if c["op"] == "append" and c["page_rows"]:
            s["ctx"].cache_register_paged(0, s["k_cache"], s["v_cache"], c["token_major"])
        elif c["op"] == "append":
            s["ctx"].cache_register(0, s["k_cache"], s["v_cache"])
    return s


# ------------------------------------------------------------------------------------------------ plain forms

def _axis_of(case):
    """The position axis of each of the D/2 frequencies: blocks of the sections' sizes, or dealt in turn (frequency j to
    axis j mod n as long as that axis has fewer than its share, to axis 0 otherwise)."""
    sec = _sections(case)
    n = len(sec)
    if not case["interleaved"]:
        return [a for a in range(n) for _ in range(sec[a])]
    return [j % n if j < n * sec[j % n] else 0 for j in range(sum(sec))]


def _plain_rotate(x, cos, sin):
    half = x.shape[-1] // 2
    lo, hi = x[..., :half].float(), x[..., half:].float()
    return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], dim=-1).to(torch.bfloat16)


def _plain_angles(s):
    c = s["c"]
    axis = torch.tensor(_axis_of(c), device=DEV)
    freq = c["theta"] ** (-2.0 * torch.arange(c["D"] // 2, device=DEV, dtype=torch.float64) / c["D"])
    angle = s["positions"][axis].t().double() * freq                      # [T, D/2]
    return torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]


def _plain_append(s):
    c = s["c"]
    cos, sin = _plain_angles(s)
    q, k = _plain_rotate(s["q"], cos, sin), _plain_rotate(s["k"], cos, sin)
    cu, kv_len = s["cu_len"].long(), s["kv_len"].long()
    t = torch.arange(s["k"].shape[0], device=DEV)
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True)
    slot = kv_len[b] + t - cu[b]
    for cache, rows in ((s["k_cache"], k), (s["v_cache"], s["v"])):
        if not c["page_rows"]:
            cache[b, :, slot] = rows
            continue
        block, row = s["table"].long()[b, slot // c["page_rows"]], slot % c["page_rows"]
        if c["token_major"]:
            cache[block, row] = rows
        else:
            cache[block, :, row] = rows
    return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"], "kv_len": (kv_len + cu[1:] - cu[:-1]).int()}


def _plain_prefix(s):
    c = s["c"]
    B, N, Hq, Hkv, D, pr = (c[k] for k in ("B", "N", "Hq", "Hkv", "D", "page_rows"))
    G, slots = Hq // Hkv, s["table"].shape[1] * pr
    outs, lses = [], []
    step = max(1, int(1.5e9) // (4 * slots * (Hq * N + 2 * Hkv * D)))     # sequences at a time
    bit = torch.arange(N, device=DEV)
    j = torch.arange(slots, device=DEV)
    for b0 in range(0, B, step):
        b1 = min(B, b0 + step)
        n = b1 - b0
        k, v = s["k"][s["table"][b0:b1].long()], s["v"][s["table"][b0:b1].long()]
        order = (0, 3, 1, 2, 4) if c["token_major"] else (0, 2, 1, 3, 4)
        k = k.permute(*order).reshape(n, Hkv, slots, D).float()
        v = v.permute(*order).reshape(n, Hkv, slots, D).float()
        tree = (s["mask"][b0:b1][:, :, bit // 64] >> (bit % 64)) & 1      # [n, N, N]
        rel = j[None] - s["kv_len"][b0:b1, None]                          # [n, slots]
        node = torch.gather(tree, 2, rel.clamp(0, N - 1)[:, None].expand(n, N, slots)) > 0
        allowed = (rel[:, None] < 0) | ((rel[:, None] < N) & node)        # [n, N, slots]
        q = s["q"][b0:b1].float().reshape(n, N, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(n, Hkv, N * G, D)
        x = (q @ k.transpose(2, 3)).mul_(s["scale"]).reshape(n, Hkv, N, G, slots)
        x.masked_fill_(~allowed[:, None, :, None], -math.inf)
        top = x.amax(dim=-1, keepdim=True)
        x.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
        total = x.sum(dim=-1, keepdim=True)
        o = (x.reshape(n, Hkv, N * G, slots) @ v).reshape(n, Hkv, N, G, D) / torch.where(total == 0, torch.ones_like(total), total)
        outs.append(o.permute(0, 2, 1, 3, 4).reshape(n, N, Hq, D).to(torch.bfloat16))
        lses.append((top + torch.log(total))[..., 0].permute(0, 1, 3, 2).reshape(n, Hq, N))
    res = {"out": torch.cat(outs)}
    return {**res, "lse": torch.cat(lses)} if c["lse"] else res


# ------------------------------------------------------------------------------------------------ the pass

def run(s):
    c = s["c"]
    if not own:
        if c["op"] == "rope":
            cos, sin = _plain_angles(s)
            return {"q": _plain_rotate(s["q"], cos, sin), "k": _plain_rotate(s["k"], cos, sin)}
        return _plain_append(s) if c["op"] == "append" else _plain_prefix(s)
    ctx = s["ctx"]
    if c["op"] == "rope":
        ctx.rope_axes_rows(s["q"], s["k"], s["positions"], s["axes"], s["q_out"], s["k_out"])
        return {"q": s["q_out"], "k": s["k_out"]}
    if c["op"] == "append":
        if c["page_rows"]:
            ctx.kv_append_paged(0, s["q"], s["k"], s["v"], s["positions"], s["axes"], s["cu_len"], s["kv_len"], s["table"],
                                s["q_out"], s["kv_len_out"])
        else:
            ctx.kv_append(0, s["q"], s["k"], s["v"], s["positions"], s["axes"], s["cu_len"], s["kv_len"], s["q_out"],
                          s["kv_len_out"])
        return {"q": s["q_out"], "k_cache": s["k_cache"], "v_cache": s["v_cache"], "kv_len": s["kv_len_out"]}
    ctx.tree_verify_attn_prefix_paged(0, s["q"], s["kv_len"], s["table"], c["P"], s["mask"], s["scale"], s["scratch"],
                                      s["out"], s["lse"])
    return {"out": s["out"], "lse": s["lse"]} if c["lse"] else {"out": s["out"]}


# ------------------------------------------------------------------------------------------------ work, exact results

def work(case):
    """Bytes that have to be read and written once and the operations of one pass.  Lengths drawn per sequence count at
    their mean."""
    c = case
    Hq, Hkv, D = c["Hq"], c["Hkv"], c["D"]
    if c["op"] == "prefix":
        B, N = c["B"], c["N"]
        tail = 0.5 * (c["tail_lo"] + c["tail_hi"])
        kv = 4.0 * Hkv * D * (c["P"] + B * (tail + N))
        return {"bytes": kv + 4.0 * B * N * Hq * D + (4.0 * B * N * Hq if c["lse"] else 0.0) + 8.0 * B * N * ((N + 63) // 64),
                "flops": 4.0 * D * Hq * N * B * (c["P"] + tail + N)}
    axes = len(_sections(c))
    T = c["T"] if c["op"] == "rope" else _tokens(c)
    rows = T * (Hq + Hkv)
    return {"bytes": 4.0 * rows * D + 4.0 * axes * T + (4.0 * T * Hkv * D + 16.0 * c["B"] if c["op"] == "append" else 0.0),
            "flops": 3.0 * rows * D}


def _exact_rotation(x, positions, case):
    """Every pair (x[j], x[j + D/2]) as a complex number times exp(i angle), in 64 bits."""
    T, H, D = x.shape
    half, sec = D // 2, _sections(case)
    angle = torch.empty((T, half), dtype=torch.float64, device=DEV)
    left, first = list(sec), [sum(sec[:a]) for a in range(len(sec))]
    for j in range(half):
        if case["interleaved"]:
            a = j % len(sec)
            a = a if a == 0 or left[a] > 0 else 0
            left[a] -= 1
        else:
            a = max(i for i in range(len(sec)) if first[i] <= j)
        angle[:, j] = positions[a].double() * math.exp(-2.0 * j / D * math.log(case["theta"]))
    z = torch.complex(x[..., :half].double(), x[..., half:].double()) * torch.polar(torch.ones_like(angle), angle)[:, None]
    return torch.cat([z.real, z.imag], dim=-1)


def exact(case, seed):
    s = prepare(case, seed)
    c = s["c"]
    if c["op"] == "rope":
        return {"q": _exact_rotation(s["q"], s["positions"], c), "k": _exact_rotation(s["k"], s["positions"], c)}
    if c["op"] == "append":
        k = _exact_rotation(s["k"], s["positions"], c)
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        cu, old, pr = s["cu_len"].tolist(), s["kv_len"].tolist(), c["page_rows"]
        for b in range(c["B"]):
            t, n = cu[b], cu[b + 1] - cu[b]
            while n > 0:
                at = old[b] + t - cu[b]
                m = min(n, pr - at % pr) if pr else n                     # rows that lie in one block
                if pr:
                    e, r = int(s["table"][b, at // pr]), at % pr
                    dst = [x[e, r:r + m] if c["token_major"] else x[e, :, r:r + m].transpose(0, 1) for x in (kc, vc)]
                else:
                    dst = [x[b, :, at:at + m].transpose(0, 1) for x in (kc, vc)]
                dst[0].copy_(k[t:t + m])
                dst[1].copy_(s["v"][t:t + m].double())
                t, n = t + m, n - m
        new = torch.tensor([old[b] + cu[b + 1] - cu[b] for b in range(c["B"])], dtype=torch.int32, device=DEV)
        return {"q": _exact_rotation(s["q"], s["positions"], c), "k_cache": kc, "v_cache": vc, "kv_len": new}
    B, N, Hq, Hkv, D, pr = (c[x] for x in ("B", "N", "Hq", "Hkv", "D", "page_rows"))
    out = torch.zeros((B, N, Hq, D), dtype=torch.float64, device=DEV)
    lse = torch.full((B, Hq, N), -math.inf, dtype=torch.float64, device=DEV)
    words = s["mask"].cpu().numpy().view(np.uint64)
    for b, S in enumerate(s["kv_len"].tolist()):
        need = s["table"][b, :(S + N + pr - 1) // pr].long()
        k, v = s["k"][need], s["v"][need]
        if not c["token_major"]:
            k, v = k.transpose(1, 2), v.transpose(1, 2)
        k, v = (x.reshape(-1, Hkv, D)[:S + N].double() for x in (k, v))
        sees = np.array([[(int(words[b, i, t // 64]) >> (t % 64)) & 1 for t in range(N)] for i in range(N)], dtype=bool)
        shut = torch.zeros((N, S + N), dtype=torch.bool, device=DEV)
        shut[:, S:] = ~torch.from_numpy(sees).to(DEV)
        for h in range(Hq):
            x = s["scale"] * (s["q"][b, :, h].double() @ k[:, h * Hkv // Hq].T)
            x = x.masked_fill(shut, -math.inf)
            lse[b, h] = torch.logsumexp(x, dim=-1)
            out[b, :, h] = torch.nan_to_num(torch.exp(x - lse[b, h][:, None])) @ v[:, h * Hkv // Hq]
    return {"out": out, "lse": lse} if c["lse"] else {"out": out}
