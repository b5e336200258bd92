"""Performance cases of the paged cache's second set of calls: positions of several axes (``kv_append`` with positions,
``rotate``), trees of drafted tokens (``tree_mask``, ``forward_paged`` with one), tokens and pages moved in the cache
(``kv_compact``, ``kv_copy``), and attention whose scores are capped, biased by distance, windowed or given a prefix
(``forward_paged``), with inputs, minimal work, a plain form in elementary torch operations and a 64-bit reference.

A case is a dict of plain values:
  op       "tree_append", "append", "rotate", "attend", "compact" or "copy"
  new      new tokens of each sequence, "1x64" for 64 sequences of one token, or a comma-separated list of such items
  keys     keys of each sequence after the append, likewise
  Hq, Hkv, dqk, dv, page   heads, head dimensions and tokens per page
  cache    attend: "bf16", or "fp8" for e4m3 with a scale per key/value head
  rot, begin, inter        rotation: rotated dims, the first of them, and whether a pair is two neighbouring dims (else dim
           c goes with dim c + rot / 2)
  axes     rotation: pairs of each axis, "16,24,24" in a row, or with "cyclic" dealt in turn while they last
  causal, lse              attend: options (lse: the call also returns the log-sum-exp)
  cap, slopes, window, prefix, tree   attend: cap of the scores (0: none), whether they get a bias by distance, window (0:
           none), keys of each sequence that all its tokens see ("": none), whether the new tokens are a tree of drafted ones
  kept, layers             compact: new tokens that each sequence keeps, layers whose caches lie in one buffer
  B, S     rotate: batch and tokens
  pages    copy: pages copied
Activations are i.i.d. N(0, 1), as in ``workloads``; queries of capped scores are 4 times that, so that the cap acts. The
pages of a sequence lie anywhere in the cache, in no order.
"""

from __future__ import annotations

import math

import torch

own = False

HEAD_DIMS = ((64, 64), (128, 128), (192, 128))
FP8_MAX = 448.0
WORDS = 2  # 32-bit words of a tree's mask: up to 64 drafted tokens


def _attend(name, new, keys, Hq, Hkv, dqk, dv, page, cache, causal=True, lse=False, cap=0.0, slopes=False, window=0, prefix="",
            tree=False):
    return {"name": name, "op": "attend", "new": new, "keys": keys, "Hq": Hq, "Hkv": Hkv, "dqk": dqk, "dv": dv, "page": page,
            "cache": cache, "causal": causal, "lse": lse, "cap": cap, "slopes": slopes, "window": window, "prefix": prefix,
            "tree": tree}


def listed():
    return [
        # One request's drafted tree: mask and positions from the parents, then its keys into the cache. The smallest
        # call, where launch and host latency count.
        {"name": "append_tree_b1", "op": "tree_append", "new": "26", "keys": "1026", "Hq": 32, "Hkv": 8, "dqk": 128, "dv": 128,
         "page": 16, "rot": 128, "begin": 0, "inter": False},
        # Prompts of a model that sees video: time, height and width have sections of the angles; one request is text.
        {"name": "append_video_8k", "op": "append", "new": "8192,777,1", "keys": "8192,1500,501", "Hq": 32, "Hkv": 8, "dqk": 128,
         "dv": 128, "page": 64, "rot": 128, "begin": 0, "inter": False, "axes": "16,24,24", "cyclic": False},
        # An encoder of video frames: queries turned in front of attention without a cache, and the gradient on the way back.
        {"name": "rotate_frames", "op": "rotate", "B": 2, "H": 16, "S": 9999, "d": 64, "rot": 64, "begin": 0, "inter": True,
         "axes": "8,12,12", "cyclic": False},
        # One request's tree over a short cache: latency.
        _attend("tree_b1_2k", "26", "2026", 32, 8, 128, 128, 16, "bf16", tree=True),
        # A serving step that checks trees of 60 drafted tokens of 16 requests of very different lengths.
        _attend("tree_b16_ragged", "60x16", "9000x4,4099x6,1200x6", 32, 8, 128, 128, 16, "bf16", tree=True),
        # The decode step of 32 requests of a model with capped scores.
        _attend("capped_tokens_b32", "1x32", "8000x8,3001x12,700x12", 32, 8, 128, 128, 16, "bf16", cap=50.0),
        # Long conversations of a model with a window that keeps the first tokens visible, from an 8-bit cache.
        _attend("window_tokens_fp8", "1x48", "60001x24,9000x24", 32, 8, 128, 128, 32, "fp8", window=4096, prefix="4x48"),
        # Prompts in a layer with a window and capped scores.
        _attend("capped_window_prompts", "8192,3001", "8192,3001", 16, 8, 128, 128, 16, "bf16", cap=50.0, window=1024),
        # A prompt and a chunk of one with a bias by distance instead of positions.
        _attend("slopes_prompts", "4096,777", "4096,3000", 32, 32, 64, 64, 16, "bf16", lse=True, slopes=True),
        # Two pictures with a question each: all tokens of a prompt see its picture, the question's are causal.
        _attend("prefix_prompts", "2500,1357", "2500,1357", 16, 4, 128, 128, 64, "bf16", prefix="2048,1024"),
        # After the check: the accepted path of every tree closes up, in all layers at once.
        {"name": "compact_b64", "op": "compact", "new": "60x64", "keys": "1000x32,333x32", "kept": "5x40,2x12,9x12", "layers": 32,
         "Hkv": 8, "dqk": 128, "dv": 128, "page": 16},
        # Forked sequences (beams, several answers to one prompt) copy the pages that they are going to write to.
        {"name": "copy_pages", "op": "copy", "pages": 500, "layers": 32, "Hkv": 8, "dqk": 128, "dv": 128, "page": 16},
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], uniform over its logarithm (so odd and even alike)."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def _text(values):
    return ",".join(map(str, values))


def _sections(rng, pairs):
    """Three axes' shares of the pairs."""
    a = max(1, round(pairs * rng.choice([0.25, 0.34, 0.5])))
    b = (pairs - a) // 2
    return _text([a, b, pairs - a - b])


def draw(rng):
    """One more case of the listed ranges: the operator, head dimensions, group, pages, cache type, batch and lengths
    at random, shortened until it costs no more than the largest listed ones."""
    dqk, dv = rng.choice(HEAD_DIMS)
    hkv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 7, 8])
    c = {"Hq": hkv * group, "Hkv": hkv, "dqk": dqk, "dv": dv, "page": rng.choice([16, 32, 64, 128])}
    kind = rng.choice(["turn", "tree", "tree", "tokens", "tokens", "prompts", "prompts", "move"])
    if kind == "turn":
        rot = rng.choice([32, 64, dqk])
        turn = {"rot": rot, "inter": rng.random() < 0.4}
        which = rng.choice(["tree_append", "append", "rotate"])
        if which == "rotate":
            d = rng.choice([64, 128, 192])
            rot = min(rot, d)
            return {"op": "rotate", "B": rng.choice([1, 1, 2, 3]), "H": c["Hq"], "S": _log(rng, 1, 9000), "d": d, "rot": rot,
                    "begin": rng.choice([0, d - rot]), "inter": turn["inter"], "axes": _sections(rng, rot // 2),
                    "cyclic": rng.random() < 0.4}
        c.update(turn, op=which, begin=rng.choice([0, dqk - rot]))
        if which == "append":
            new = [_log(rng, 1, 4000) for _ in range(rng.choice([1, 2, 3]))]
            c.update(axes=_sections(rng, rot // 2), cyclic=rng.random() < 0.4)
        else:
            new = [_log(rng, 1, 64) for _ in range(_log(rng, 1, 64))]
        keys = [n + (0 if rng.random() < 0.3 else _log(rng, 1, 500)) for n in new]
    elif kind == "move":
        c["layers"] = rng.choice([1, 5, 32])
        if rng.random() < 0.5:
            c.update(op="copy", pages=max(1, _log(rng, 1, 2000) * 256 // (c["layers"] * hkv * c["page"])))
            return c
        new = [_log(rng, 3, 64) for _ in range(_log(rng, 1, 64))]
        keys = [n + _log(rng, 1, 500) for n in new]
        c.update(op="compact", kept=_text(rng.randint(1, min(9, n - 1)) for n in new))
    else:
        c.update(op="attend", cache=rng.choice(["bf16", "bf16", "fp8"]), causal=True, lse=rng.random() < 0.4, cap=0.0,
                 slopes=False, window=0, prefix="", tree=kind == "tree")
        if rng.random() < (0.3 if kind == "tree" else 0.5):
            c["cap"] = rng.choice([20.0, 30.0, 50.0])
        if kind == "tree":
            new = [_log(rng, 2, 64) for _ in range(_log(rng, 1, 24))]
        elif kind == "tokens":
            new = [rng.choice([1, 1, 1, 2, 5])] * _log(rng, 1, 64)
        else:
            new = [_log(rng, 33, 4000) for _ in range(rng.choice([1, 1, 2, 3]))]
            c["causal"] = rng.random() < 0.85
        if kind == "prompts":
            keys = [n + (0 if rng.random() < 0.5 else _log(rng, 1, 4000)) for n in new]
            while max(new) * max(keys) * len(new) * c["Hq"] > 1_000_000_000:
                new = [max(1, n // 2) for n in new]
        else:
            longest = _log(rng, 200, 60001)
            keys = [n + _log(rng, max(1, longest // 20), longest) for n in new]
            while sum(keys) * hkv > 2_400_000 or sum(new) * max(keys) * c["Hq"] > 400_000_000:
                keys = [max(n, k // 2) for n, k in zip(new, keys)]
        if kind != "tree":
            c["slopes"] = rng.random() < 0.35
            if rng.random() < 0.4:
                c["window"] = _log(rng, 1, 4096)
            if rng.random() < 0.35:
                c["prefix"] = _text(rng.choice([0, 4, k // 3, k]) for k in keys)
    c["new"], c["keys"] = _text(new), _text(keys)
    return c


def _list(text):
    out = []
    for item in filter(None, text.split(",")):
        n, _, times = item.partition("x")
        out += [int(n)] * int(times or 1)
    return out


def _seen(case):
    """Pairs of token and visible key (of a tree: with its cached keys and itself), and keys that some token sees."""
    new, keys = _list(case["new"]), _list(case["keys"])
    prefix, w = _list(case["prefix"]) or [0] * len(new), case["window"] or 1 << 40
    pairs = seen = 0
    for n, kv, pre in zip(new, keys, prefix):
        if case["tree"]:
            pairs, seen = pairs + n * (kv - n + 1), seen + kv
            continue
        pre, p = min(pre, kv), torch.arange(kv - n, kv)
        first = (p - w + 1).clamp_min(0)
        last = p if case["causal"] else (p + w - 1).clamp_max(kv - 1)
        both = (torch.minimum(last + 1, torch.full_like(p, pre)) - first).clamp_min(0)  # in the prefix too
        pairs += int((last + 1 - first + pre - both).sum())
        # Keys [0, pre) and [first of the first token, last of the last one].
        lo, hi = int(first[0]), int(last[-1]) + 1
        seen += pre + hi - max(lo, min(pre, hi))
    return pairs, seen


def work(case):
    op = case["op"]
    if op == "rotate":
        n = case["B"] * case["S"]
        # The rows of angles of all positions of an image are read by many tokens; each token has its three positions.
        return {"bytes": n * (case["H"] * case["d"] * 8 + 12), "flops": 6 * n * case["H"] * case["rot"]}
    Hkv, dqk, dv = case["Hkv"], case["dqk"], case["dv"]
    if op == "copy":
        return {"bytes": 4 * case["pages"] * case["layers"] * Hkv * case["page"] * (dqk + dv), "flops": 0}
    new, keys = _list(case["new"]), _list(case["keys"])
    T = sum(new)
    if op == "compact":
        moved = sum(_list(case["kept"])) - len(new)  # the first one stays
        return {"bytes": 4 * moved * case["layers"] * Hkv * (dqk + dv) + 4 * (sum(_list(case["kept"])) + 5 * len(new)), "flops": 0}
    Hq = case["Hq"]
    if op in ("append", "tree_append"):
        extra = T * (4 + 4 + 4 * WORDS) if op == "tree_append" else 12 * T
        return {"bytes": T * (2 * Hq * dqk + 2 * Hkv * (dqk + dv)) * 2 + extra, "flops": 3 * T * (Hq + Hkv) * case["rot"]}
    size = 1 if case["cache"] == "fp8" else 2
    pairs, seen = _seen(case)
    moved = seen * Hkv * (dqk + dv) * size + T * Hq * (dqk + dv) * 2 + (T * Hq * 4 if case["lse"] else 0)
    return {"bytes": moved + (T * 4 * WORDS if case["tree"] else 0), "flops": 2 * Hq * (dqk + dv) * pairs}


def _generator(seed):
    g = torch.Generator(device="cuda:0")
    g.manual_seed(seed)
    return g


def _pair_axes(case, dev):
    """The axis of each pair: sections in a row, or dealt in turn."""
    left = _list(case["axes"])
    if not case["cyclic"]:
        out = [a for a, n in enumerate(left) for _ in range(n)]
    else:
        out, a = [], 0
        while any(left):
            if left[a % len(left)]:
                left[a % len(left)] -= 1
                out.append(a % len(left))
            a += 1
    return torch.tensor(out, dtype=torch.uint8, device=dev)


def _video(n, start):
    """Positions of n tokens: frames of 12 x 17 patches from `start` on, the last third text behind them, on all axes."""
    video = n - n // 3
    i = torch.arange(video)
    p = torch.stack([i // 204, i // 17 % 12, i % 17], dim=1)
    text = (int(p.max()) + 1 if video else 0) + torch.arange(n // 3)[:, None].expand(-1, 3)
    return start + torch.cat([p, text])


def _table(positions, rot, dev):
    """The program's rotation table: cos and sin of every position's angles, base 500000."""
    freq = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=dev) / rot)
    angle = torch.arange(positions, dtype=torch.float64, device=dev)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def prepare(case, seed):
    dev, g, op = torch.device("cuda:0"), _generator(seed), case["op"]
    s = {"case": case}

    def randn(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32).to(torch.bfloat16)

    if op == "rotate":
        s["x"], s["dy"] = randn(case["B"], case["H"], case["S"], case["d"]), randn(case["B"], case["H"], case["S"], case["d"])
        s["positions"] = _video(case["S"], 0).expand(case["B"], -1, -1).contiguous().to(torch.int32).to(dev)
        s["pair_axes"], s["cos_sin"] = _pair_axes(case, dev), _table(case["S"] + 64, case["rot"], dev)
        return s
    page, Hkv, dqk, dv = case["page"], case["Hkv"], case["dqk"], case["dv"]
    if op == "copy":
        n, heads = case["pages"], case["layers"] * Hkv
        order = torch.randperm(2 * n + 3, generator=g, device=dev).to(torch.int32)
        s["src"], s["dst"] = order[:n].contiguous(), order[n:2 * n].contiguous()
        s["k_cache"], s["v_cache"] = randn(2 * n + 3, heads, page, dqk), randn(2 * n + 3, heads, page, dv)
        return s
    new, keys = _list(case["new"]), _list(case["keys"])
    blocks = [-(-k // page) for k in keys]
    n_pages = sum(blocks) + 3
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    table = torch.full((len(keys), max(blocks)), -1, dtype=torch.int32, device=dev)  # -1 behind a sequence's pages
    held = torch.arange(max(blocks), device=dev)[None] < torch.tensor(blocks, device=dev)[:, None]
    table[held] = order[: sum(blocks)]
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s.update(table=table, kv_lens=torch.tensor(keys, dtype=torch.int32, device=dev),
             q_starts=torch.tensor(starts, dtype=torch.int32, device=dev), max_q=max(new), T=starts[-1])
    heads = Hkv * case.get("layers", 1)
    k_cache, v_cache = randn(n_pages, heads, page, dqk), randn(n_pages, heads, page, dv)
    if op == "compact":
        # Of every sequence's new tokens the first, in its place, and others behind the next one.
        kept, most = _list(case["kept"]), max(_list(case["kept"]))
        s["kept"] = torch.full((len(new), most), -1, dtype=torch.int32, device=dev)
        for b, (n, m) in enumerate(zip(new, kept)):
            s["kept"][b, 0] = 0
            if m > 1:
                s["kept"][b, 1:m] = torch.randperm(n - 2, generator=g, device=dev)[: m - 1].sort().values.to(torch.int32) + 2
        s.update(n_kept=torch.tensor(kept, dtype=torch.int32, device=dev), k_cache=k_cache, v_cache=v_cache)
        return s
    if case.get("tree") or op == "tree_append":
        # A node's parent is some token drafted before it, more often a late one; the first is the root.
        i = torch.arange(starts[-1], device=dev) - torch.repeat_interleave(s["q_starts"][:-1].long(), s["q_starts"].diff().long())
        r = torch.rand(starts[-1], generator=g, device=dev).sqrt()
        s["parents"] = torch.where(i == 0, -1, (r * i).long().clamp_max(i - 1)).to(torch.int32)
        s["tree_mask"] = _tree(s)[0] if op == "attend" else None
    s["q"] = randn(starts[-1], case["Hq"], dqk)
    if op in ("append", "tree_append"):
        s["k"], s["v"] = randn(starts[-1], Hkv, dqk), randn(starts[-1], Hkv, dv)
        s["cos_sin"] = _table(max(keys) + 64, case["rot"], dev)
        if op == "append":
            s["pair_axes"] = _pair_axes(case, dev)
            s["positions"] = torch.cat([_video(n, k - n) for n, k in zip(new, keys)]).to(torch.int32).to(dev)
        s.update(k_cache=k_cache, v_cache=v_cache)
        return s
    if case["cap"]:
        s["q"] = s["q"] * 4
    s["k_scale"] = s["v_scale"] = s["slopes"] = s["prefix"] = None
    if case["cache"] == "fp8":
        s["k_scale"], s["v_scale"] = (0.008 + 0.006 * torch.rand(Hkv, generator=g, device=dev) for _ in range(2))
        k_cache = (k_cache.float() / s["k_scale"][:, None, None]).clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn)
        v_cache = (v_cache.float() / s["v_scale"][:, None, None]).clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn)
    s["k_cache"], s["v_cache"] = k_cache, v_cache
    if case["slopes"]:
        s["slopes"] = 2.0 ** (-8.0 * (torch.arange(case["Hq"], device=dev) + 1) / case["Hq"])
    if case["prefix"]:
        s["prefix"] = torch.tensor(_list(case["prefix"]), dtype=torch.int32, device=dev)
    return s


def run(s):
    if own:
        return _own(s)
    return {"rotate": _plain_rotate, "copy": _plain_copy, "compact": _plain_compact, "append": _plain_append,
            "tree_append": _plain_append, "attend": _plain_attend}[s["case"]["op"]](s)


def _own(s):
    import paper_2609_21264_amd as fa

    c = s["case"]
    if c["op"] == "rotate":
        how = {"positions": s["positions"], "pair_axes": s["pair_axes"], "rot_begin": c["begin"], "interleaved": c["inter"]}
        return {"y": fa.rotate(s["x"], s["cos_sin"], **how), "dx": fa.rotate(s["dy"], s["cos_sin"], inverse=True, **how)}
    if c["op"] == "copy":
        fa.kv_copy(s["k_cache"], s["v_cache"], s["src"], s["dst"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if c["op"] == "compact":
        lens = fa.kv_compact(s["k_cache"], s["v_cache"], s["table"], s["kv_lens"], s["q_starts"], s["kept"], s["n_kept"])
        return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "kv_lens": lens}
    if c["op"] in ("append", "tree_append"):
        out = {}
        if c["op"] == "tree_append":
            out["tree_mask"], positions = fa.tree_mask(s["parents"], s["q_starts"], s["kv_lens"], words=WORDS)
            out["positions"], pair_axes = positions, None
        else:
            positions, pair_axes = s["positions"], s["pair_axes"]
        q = fa.kv_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["kv_lens"], s["q_starts"], q=s["q"],
                         cos_sin=s["cos_sin"], rot_begin=c["begin"], interleaved=c["inter"], positions=positions,
                         pair_axes=pair_axes)
        return {**out, "q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    r = fa.forward_paged(s["q"], s["k_cache"], s["v_cache"], s["table"], s["kv_lens"], s["q_starts"], max_q=s["max_q"],
                         causal=c["causal"], return_lse=c["lse"], k_scale=s["k_scale"], v_scale=s["v_scale"],
                         softcap=c["cap"] or None, slopes=s["slopes"], window=c["window"] or None, prefix_lens=s["prefix"],
                         tree_mask=s["tree_mask"] if c["tree"] else None)
    return {"o": r[0], "lse": r[1]} if c["lse"] else {"o": r}


def _tokens(s):
    """The sequence of every new token, its number in it and its place among the sequence's keys."""
    t = torch.arange(s["T"], device=s["table"].device)
    starts, lens = s["q_starts"].long(), s["kv_lens"].long()
    seq = torch.searchsorted(starts[1:].contiguous(), t, right=True)
    return seq, t - starts[seq], t - starts[1:][seq] + lens[seq]


def _tree(s):
    """Bits of every token's ancestors and itself, [T, WORDS] int32, and its position: the cached keys and its depth."""
    seq, i, _ = _tokens(s)
    starts, parents = s["q_starts"].long(), s["parents"].long()
    bits = torch.zeros(s["T"], 32 * WORDS, dtype=torch.bool, device=i.device)
    rows = torch.arange(s["T"], device=i.device)
    at = i.clone()
    for _ in range(s["max_q"]):
        live = at >= 0
        bits[rows, at.clamp_min(0)] |= live
        at = torch.where(live, parents[starts[seq] + at.clamp_min(0)], at)
    words = (bits.view(-1, WORDS, 32).long() << torch.arange(32, device=i.device)).sum(dim=2)
    base = s["kv_lens"].long()[seq] - s["q_starts"].diff().long()[seq]
    return torch.where(words >= 1 << 31, words - (1 << 32), words).to(torch.int32), (base + bits.sum(dim=1) - 1).to(torch.int32)


def _turned(x, cos, sin, begin, inter):
    """x [..., d] with dims begin .. begin + rot - 1 turned by cos, sin [..., rot / 2]."""
    half = cos.shape[-1]
    part = x[..., begin:begin + 2 * half]
    a, b = (part[..., 0::2], part[..., 1::2]) if inter else (part[..., :half], part[..., half:])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    both = torch.stack([ra, rb], dim=-1).flatten(-2) if inter else torch.cat([ra, rb], dim=-1)
    return torch.cat([x[..., :begin], both, x[..., begin + 2 * half:]], dim=-1)


def _angles(cos_sin, positions, pair_axes):
    """cos and sin [..., rot / 2] of tokens with positions [..., axes]."""
    half = cos_sin.shape[1] // 2
    row = positions.long()[..., pair_axes.long()]
    c = torch.arange(half, device=row.device)
    return cos_sin[row, c], cos_sin[row, half + c]


def _plain_rotate(s):
    c = s["case"]
    cos, sin = (t[:, None] for t in _angles(s["cos_sin"], s["positions"], s["pair_axes"]))
    return {"y": _turned(s["x"].float(), cos, sin, c["begin"], c["inter"]).to(torch.bfloat16),
            "dx": _turned(s["dy"].float(), cos, -sin, c["begin"], c["inter"]).to(torch.bfloat16)}


def _plain_copy(s):
    for cache in (s["k_cache"], s["v_cache"]):
        cache[s["dst"].long()] = cache[s["src"].long()]
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_compact(s):
    page = s["case"]["page"]
    base = s["kv_lens"].long() - s["q_starts"].diff().long()
    b, i = (torch.arange(s["kept"].shape[1], device=base.device) < s["n_kept"][:, None]).nonzero(as_tuple=True)
    frm, to = base[b] + s["kept"].long()[b, i], base[b] + i
    for cache in (s["k_cache"], s["v_cache"]):
        rows = cache[s["table"].long()[b, frm // page], :, frm % page]
        cache[s["table"].long()[b, to // page], :, to % page] = rows
    return {"k_cache": s["k_cache"], "v_cache": s["v_cache"], "kv_lens": (base + s["n_kept"]).to(torch.int32)}


def _plain_append(s):
    c, out = s["case"], {}
    seq, _, place = _tokens(s)
    if c["op"] == "tree_append":
        out["tree_mask"], out["positions"] = _tree(s)
        rows = s["cos_sin"][out["positions"].long()]
        cos, sin = rows.chunk(2, dim=1)
    else:
        cos, sin = _angles(s["cos_sin"], s["positions"], s["pair_axes"])
    q, k = (_turned(s[x].float(), cos[:, None], sin[:, None], c["begin"], c["inter"]).to(torch.bfloat16) for x in "qk")
    page, slot = s["table"].long()[seq, place // c["page"]], place % c["page"]
    s["k_cache"][page, :, slot], s["v_cache"][page, :, slot] = k, s["v"]
    return {**out, "q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attend(s):
    c = s["case"]
    Hq, Hkv, dqk, dv, cap = c["Hq"], c["Hkv"], c["dqk"], c["dv"], c["cap"]
    group, dev = Hq // Hkv, s["q"].device
    new, keys, at = _list(c["new"]), _list(c["keys"]), 0
    out, lse = [], []
    for b, (n, kv) in enumerate(zip(new, keys)):
        pages = s["table"][b, : -(-kv // c["page"])].long()
        k, v = (t[pages].float().transpose(0, 1).reshape(Hkv, -1, d)[:, :kv] for t, d in ((s["k_cache"], dqk), (s["v_cache"], dv)))
        if s["k_scale"] is not None:
            k, v = k * s["k_scale"][:, None, None], v * s["v_scale"][:, None, None]
        q = s["q"][at:at + n].float().view(n, Hkv, group, dqk).permute(1, 2, 0, 3).reshape(Hkv, group * n, dqk)
        x = torch.matmul(q, k.transpose(1, 2).contiguous()).view(Hkv, group, n, kv) * (1.0 / math.sqrt(dqk))
        if cap:
            x = cap * torch.tanh(x / cap)
        p, j = torch.arange(kv - n, kv, device=dev)[:, None], torch.arange(kv, device=dev)
        if s["slopes"] is not None:
            x = x - s["slopes"].view(Hkv, group, 1, 1) * (p - j).abs().float()
        seen = (j <= p) if c["causal"] else torch.ones(n, kv, dtype=torch.bool, device=dev)
        if c["window"]:
            seen = seen & ((p - j).abs() < c["window"])
        if s["prefix"] is not None:
            seen = seen | (j < s["prefix"][b])
        if c["tree"]:
            drafted = (s["tree_mask"][at:at + n, :, None] >> torch.arange(32, device=dev, dtype=torch.int32)) & 1
            seen = torch.cat([torch.ones(n, kv - n, dtype=torch.bool, device=dev), drafted.view(n, -1)[:, :n].bool()], dim=1)
        x = x.masked_fill(~seen, -math.inf)
        top = x.amax(dim=-1, keepdim=True)
        x = torch.exp(x - top)
        total = x.sum(dim=-1, keepdim=True)
        o = torch.matmul(x.view(Hkv, group * n, kv), v).view(Hkv, group, n, dv) / total
        out.append(o.permute(2, 0, 1, 3).reshape(n, Hq, dv).to(torch.bfloat16))
        lse.append((top + total.log()).permute(2, 0, 1, 3).reshape(n, Hq))
        at += n
    return {"o": torch.cat(out), "lse": torch.cat(lse)} if c["lse"] else {"o": torch.cat(out)}


def _exact_turn(x, cos_sin, rows, begin, inter, sign=1.0):
    """x [n, H, d] in 64 bits; rows [n, rot / 2]: the table row of each pair of each token. z = x + iy times the angle's unit
    number."""
    half = cos_sin.shape[1] // 2
    x = x.double()
    for c in range(half):
        unit = torch.complex(cos_sin[rows[:, c], c].double(), sign * cos_sin[rows[:, c], half + c].double())[:, None]
        i, j = (begin + 2 * c, begin + 2 * c + 1) if inter else (begin + c, begin + half + c)
        z = torch.complex(x[..., i].clone(), x[..., j].clone()) * unit
        x[..., i], x[..., j] = z.real, z.imag
    return x


def exact(case, seed):
    """The outputs of one pass in 64 bits: pair by pair for the rotation, token by token for what is moved, head by head
    for the attention; none of masks, positions and lengths, which are whole numbers."""
    s = prepare(case, seed)
    op = case["op"]
    if op == "rotate":
        out = {}
        axis = s["pair_axes"].long()
        for name, x, sign in (("y", "x", 1.0), ("dx", "dy", -1.0)):
            out[name] = torch.stack([_exact_turn(s[x][b].transpose(0, 1), s["cos_sin"], s["positions"][b].long()[:, axis],
                                                 case["begin"], case["inter"], sign).transpose(0, 1) for b in range(case["B"])])
        return out
    if op == "copy":
        src, dst = s["src"].tolist(), s["dst"].tolist()
        for cache in (s["k_cache"], s["v_cache"]):
            before = cache.clone()
            for a, b in zip(src, dst):
                cache[b] = before[a]
        return {"k_cache": s["k_cache"].double(), "v_cache": s["v_cache"].double()}
    new, keys, page = _list(case["new"]), _list(case["keys"]), case["page"]
    table = s["table"].tolist()
    if op == "compact":
        kept, n_kept = s["kept"].tolist(), s["n_kept"].tolist()
        for cache in (s["k_cache"], s["v_cache"]):
            for b, (n, kv) in enumerate(zip(new, keys)):
                for to, frm in enumerate(kept[b][: n_kept[b]]):  # downwards: what is read has not been written over
                    a, z = kv - n + frm, kv - n + to
                    cache[table[b][z // page], :, z % page] = cache[table[b][a // page], :, a % page]
        return {"k_cache": s["k_cache"].double(), "v_cache": s["v_cache"].double(), "kv_lens": None}
    parents = s["parents"].tolist() if s.get("parents") is not None else None
    paths, at = [], 0  # of every drafted token: itself and its ancestors
    for n in new:
        for i in range(n if parents else 0):
            paths.append([i] + (paths[at + parents[at + i]] if parents[at + i] >= 0 else []))
        at += n
    if op in ("append", "tree_append"):
        if op == "append":
            rows = s["positions"].long()[:, s["pair_axes"].long()]
        else:
            base = [kv - n for n, kv in zip(new, keys) for _ in range(n)]
            rows = torch.tensor([b + len(p) - 1 for b, p in zip(base, paths)], device="cuda:0")[:, None].expand(-1, case["rot"] // 2)
        q, k = (_exact_turn(s[x], s["cos_sin"], rows, case["begin"], case["inter"]) for x in "qk")
        kc, vc, at = s["k_cache"].double(), s["v_cache"].double(), 0
        for b, (n, kv) in enumerate(zip(new, keys)):
            pos = torch.arange(kv - n, kv, device="cuda:0")
            pg, slot = s["table"][b].long()[pos // page], pos % page
            kc[pg, :, slot], vc[pg, :, slot] = k[at:at + n], s["v"][at:at + n].double()
            at += n
        none = {"tree_mask": None, "positions": None} if op == "tree_append" else {}
        return {**none, "q": q, "k_cache": kc, "v_cache": vc}
    Hq, group = case["Hq"], case["Hq"] // case["Hkv"]
    o = torch.zeros(sum(new), Hq, case["dv"], dtype=torch.float64, device="cuda:0")
    lse = torch.zeros(sum(new), Hq, dtype=torch.float64, device="cuda:0")
    prefix, at = _list(case["prefix"]) or [0] * len(new), 0
    for b, (n, kv) in enumerate(zip(new, keys)):
        p, j = torch.arange(kv - n, kv, device="cuda:0").double()[:, None], torch.arange(kv, device="cuda:0").double()
        far = torch.where(p > j, p - j, j - p)
        hidden = (far >= (case["window"] or math.inf)) | ((j > p) & case["causal"])
        hidden &= j >= prefix[b]
        if case["tree"]:
            hidden = torch.ones(n, kv, dtype=torch.bool)
            hidden[:, : kv - n] = False
            for i in range(n):
                hidden[i, [kv - n + a for a in paths[at + i]]] = False
            hidden = hidden.to("cuda:0")
        pg = s["table"][b, : -(-kv // page)].long()
        k_b, v_b = s["k_cache"][pg], s["v_cache"][pg]  # [pages, Hkv, page, d]
        for h in range(Hq):
            g = h // group
            k, v = k_b[:, g].double().flatten(0, 1)[:kv], v_b[:, g].double().flatten(0, 1)[:kv]
            if s["k_scale"] is not None:
                k, v = k * s["k_scale"].double()[g], v * s["v_scale"].double()[g]
            x = (s["q"][at:at + n, h].double() @ k.T.contiguous()) * case["dqk"] ** -0.5
            if case["cap"]:
                x = case["cap"] * torch.tanh(x / case["cap"])
            if case["slopes"]:
                x = x - s["slopes"].double()[h] * far
            x[hidden] = -math.inf
            lse[at:at + n, h] = torch.logsumexp(x, dim=1)
            o[at:at + n, h] = torch.softmax(x, dim=1) @ v
        at += n
    return {"o": o, "lse": lse} if case["lse"] else {"o": o}
