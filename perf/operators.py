"""Performance cases of the paged key/value cache: appending new tokens to it with their position rotation
(``kv_append``) and the attention of the new tokens over it (``forward_paged``), with inputs, minimal work, a plain
form in elementary torch operations and a 64-bit reference.

A case is a dict of plain values:
  op       "append" or "attend"
  new      new tokens of each sequence, "1x64" for 64 sequences of one token, or a comma-separated list of such items
  keys     keys of each sequence after the append, likewise
  Hq, Hkv, dqk, dv, page   heads, head dimensions and tokens per page
  cache    "bf16", or "fp8" for e4m3 with a scale per key/value head
  rot, begin, inter        append: rotated dims (0: none), the first of them, and whether a pair is two neighbouring
           dims (else dim c goes with dim c + rot / 2)
  causal, lse              attend: options (lse: the call also returns the log-sum-exp)
Activations are i.i.d. N(0, 1), as in ``workloads``; the pages of a sequence lie anywhere in the cache, in no order.
"""

from __future__ import annotations

import math

import torch

own = False

HEAD_DIMS = ((64, 64), (128, 128), (192, 128))
FP8_MAX = 448.0


def _append(name, new, keys, Hq, Hkv, dqk, dv, page, cache, rot, begin=0, inter=False):
    return {"name": name, "op": "append", "new": new, "keys": keys, "Hq": Hq, "Hkv": Hkv, "dqk": dqk, "dv": dv,
            "page": page, "cache": cache, "rot": rot, "begin": begin, "inter": inter}


def _attend(name, new, keys, Hq, Hkv, dqk, dv, page, cache, causal=True, lse=False):
    return {"name": name, "op": "attend", "new": new, "keys": keys, "Hq": Hq, "Hkv": Hkv, "dqk": dqk, "dv": dv,
            "page": page, "cache": cache, "causal": causal, "lse": lse}


def listed():
    return [
        # A single request's decode step: the smallest call, where launch and host latency count.
        _append("append_one_token", "1", "1000", 32, 8, 128, 128, 16, "bf16", 128),
        # The decode step of 64 requests into an 8-bit cache.
        _append("append_b64_fp8", "1x64", "333x20,77x44", 32, 8, 128, 128, 32, "fp8", 128),
        # The prompts of three requests at once, ragged.
        _append("append_prompts_8k", "8192,4097,1", "8192,4100,501", 32, 8, 128, 128, 64, "bf16", 128),
        # Wide heads of which the last 64 dims are rotated in neighbouring pairs; a chunk behind a cached part.
        _append("append_wide_chunk", "777", "1500", 16, 16, 192, 128, 16, "bf16", 64, 128, True),
        # One token of one request against a short cache: latency.
        _attend("one_token_1k", "1", "1023", 32, 8, 128, 128, 16, "bf16"),
        # A serving step of 64 requests whose lengths differ by two orders of magnitude.
        _attend("tokens_b64_ragged", "1x64", "20000x2,9001x6,4099x16,1200x20,130x20", 32, 8, 128, 128, 16, "bf16"),
        # One token against 128K cached ones, split over the whole chip.
        _attend("one_token_128k", "1", "131072", 32, 8, 128, 128, 64, "bf16", lse=True),
        # The same step of 16 requests from an 8-bit cache.
        _attend("tokens_b16_fp8", "1x16", "16384x8,10001x8", 32, 8, 128, 128, 32, "fp8"),
        # Draft tokens of a small model (7:1 group, 64-wide heads), checked five at a time.
        _attend("draft_tokens_b8", "5x8", "3001x8", 14, 2, 64, 64, 16, "bf16"),
        # Two prompts without a cached part.
        _attend("prompts_4k", "4096,3001", "4096,3001", 32, 8, 128, 128, 16, "bf16", lse=True),
        # A chunk of a long prompt beside the decode step of 24 other requests.
        _attend("chunk_beside_tokens", "1024,1x24", "9000,2000x24", 32, 8, 128, 128, 64, "bf16"),
        # A chunk of wide heads behind a cached part.
        _attend("wide_chunk", "512", "4500", 32, 32, 192, 128, 32, "bf16"),
    ]


def _log(rng, lo, hi):
    """An integer of [lo, hi], uniform over its logarithm (so odd and even alike)."""
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case of the listed ranges: the operator, head dimensions, group, pages, cache type, batch and lengths
    at random, shortened until it costs no more than the largest listed ones."""
    dqk, dv = rng.choice(HEAD_DIMS)
    hkv, group = rng.choice([1, 2, 4, 8]), rng.choice([1, 2, 4, 7, 8])
    c = {"Hq": hkv * group, "Hkv": hkv, "dqk": dqk, "dv": dv, "page": rng.choice([16, 32, 64, 128]),
         "cache": rng.choice(["bf16", "bf16", "fp8"])}
    kind = rng.choice(["append", "tokens", "tokens", "prompts"])
    if kind == "append":
        if rng.random() < 0.5:
            new = [1] * _log(rng, 1, 128)
        else:
            new = [_log(rng, 1, 4000) for _ in range(rng.choice([1, 2, 3]))]
        keys = [n + (0 if rng.random() < 0.5 else _log(rng, 1, 500)) for n in new]
        rot = rng.choice([0, 32, 64, dqk])
        c.update(op="append", rot=rot, begin=rng.choice([0, dqk - rot]), inter=rng.random() < 0.4)
    elif kind == "tokens":
        batch, few = _log(rng, 1, 96), rng.choice([1, 1, 1, 2, 4, 7])
        new = [few] * batch
        longest = _log(rng, 200, 131072)
        keys = [max(few, _log(rng, max(1, longest // 20), longest)) for _ in new]
        while sum(keys) * hkv > 2_400_000 or max(keys) * batch * hkv > 5_000_000:
            keys = [max(few, x // 2) for x in keys]
        c.update(op="attend", causal=rng.random() < 0.8, lse=rng.random() < 0.4)
    else:
        new = [_log(rng, 33, 4000) for _ in range(rng.choice([1, 1, 2, 3]))]
        keys = [n + (0 if rng.random() < 0.5 else _log(rng, 1, 4000)) for n in new]
        while max(new) * max(keys) * len(new) * hkv * group > 1_000_000_000:
            new = [max(1, n // 2) for n in new]
        c.update(op="attend", causal=rng.random() < 0.8, lse=rng.random() < 0.4)
    c["new"], c["keys"] = ",".join(map(str, new)), ",".join(map(str, keys))
    return c


def _list(text):
    out = []
    for item in text.split(","):
        n, _, times = item.partition("x")
        out += [int(n)] * int(times or 1)
    return out


def work(case):
    new, keys = _list(case["new"]), _list(case["keys"])
    T, Hq, Hkv, dqk, dv = sum(new), case["Hq"], case["Hkv"], case["dqk"], case["dv"]
    size = 1 if case["cache"] == "fp8" else 2
    if case["op"] == "append":
        moved = T * (2 * Hq * dqk + Hkv * (dqk + dv)) * 2 + T * Hkv * (dqk + dv) * size + T * case["rot"] * 4
        return {"bytes": moved, "flops": 3 * T * (Hq + Hkv) * case["rot"]}
    pairs = sum(n * k - (n * (n - 1) // 2 if case["causal"] else 0) for n, k in zip(new, keys))
    moved = sum(keys) * Hkv * (dqk + dv) * size + T * Hq * (dqk + dv) * 2 + (T * Hq * 4 if case["lse"] else 0)
    return {"bytes": moved, "flops": 2 * Hq * (dqk + dv) * pairs}


def prepare(case, seed):
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev)
    g.manual_seed(seed)
    new, keys, page = _list(case["new"]), _list(case["keys"]), case["page"]
    Hq, Hkv, dqk, dv, fp8 = case["Hq"], case["Hkv"], case["dqk"], case["dv"], case["cache"] == "fp8"
    blocks = [-(-k // page) for k in keys]
    n_pages = sum(blocks) + 3
    order = torch.randperm(n_pages, generator=g, device=dev).to(torch.int32)
    table = torch.full((len(keys), max(blocks)), -1, dtype=torch.int32, device=dev)  # -1 behind a sequence's pages
    held = torch.arange(max(blocks), device=dev)[None] < torch.tensor(blocks, device=dev)[:, None]
    table[held] = order[: sum(blocks)]
    starts = [0]
    for n in new:
        starts.append(starts[-1] + n)
    s = {"case": case, "table": table, "kv_lens": torch.tensor(keys, dtype=torch.int32, device=dev),
         "q_starts": torch.tensor(starts, dtype=torch.int32, device=dev), "max_q": max(new), "T": starts[-1],
         "k_scale": None, "v_scale": None}

    def randn(*shape):
        return torch.randn(shape, generator=g, device=dev, dtype=torch.float32).to(torch.bfloat16)

    s["q"] = randn(starts[-1], Hq, dqk)
    k_cache, v_cache = randn(n_pages, Hkv, page, dqk), randn(n_pages, Hkv, page, dv)
    if fp8:
        s["k_scale"], s["v_scale"] = (0.008 + 0.006 * torch.rand(Hkv, generator=g, device=dev) for _ in range(2))
        k_cache = _fp8(k_cache.float() / s["k_scale"][:, None, None])
        v_cache = _fp8(v_cache.float() / s["v_scale"][:, None, None])
    s["k_cache"], s["v_cache"] = k_cache, v_cache
    if case["op"] == "append":
        s["k"], s["v"] = randn(starts[-1], Hkv, dqk), randn(starts[-1], Hkv, dv)
        # The program's rotation table: cos and sin of every position's angles, base 500000.
        s["cos_sin"] = _table(max(blocks) * page, case["rot"], dev).float() if case["rot"] else None
    return s


def _table(positions, rot, dev):
    freq = 500000.0 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=dev) / rot)
    angle = torch.arange(positions, dtype=torch.float64, device=dev)[:, None] * freq
    return torch.cat([angle.cos(), angle.sin()], dim=1)


def _fp8(x):
    return x.clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn)


def run(s):
    if own:
        return _own(s)
    return _plain_append(s) if s["case"]["op"] == "append" else _plain_attend(s)


def _own(s):
    import paper_2609_21264_amd as fa

    c = s["case"]
    scales = {"k_scale": s["k_scale"], "v_scale": s["v_scale"]}
    if c["op"] == "append":
        q = fa.kv_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["kv_lens"], s["q_starts"],
                         q=s["q"], cos_sin=s["cos_sin"], rot_begin=c["begin"], interleaved=c["inter"], **scales)
        return {"q": q, "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    r = fa.forward_paged(s["q"], s["k_cache"], s["v_cache"], s["table"], s["kv_lens"], s["q_starts"],
                         max_q=s["max_q"], causal=c["causal"], return_lse=c["lse"], **scales)
    return {"o": r[0], "lse": r[1]} if c["lse"] else {"o": r}


def _tokens(s):
    """The sequence of every new token and its position."""
    t = torch.arange(s["T"], device=s["q"].device)
    seq = torch.searchsorted(s["q_starts"][1:].long(), t, right=True)
    return seq, t - s["q_starts"][1:].long()[seq] + s["kv_lens"].long()[seq]


def _rotated(x, cos_sin, begin, inter):
    """x [T, H, d] with dims begin .. begin + rot - 1 rotated by cos_sin [T, rot], both of one type."""
    rot = cos_sin.shape[1]
    cos, sin = cos_sin[:, None, : rot // 2], cos_sin[:, None, rot // 2:]
    part = x[..., begin:begin + rot]
    a, b = (part[..., 0::2], part[..., 1::2]) if inter else (part[..., : rot // 2], part[..., rot // 2:])
    ra, rb = a * cos - b * sin, b * cos + a * sin
    both = torch.stack([ra, rb], dim=-1).flatten(-2) if inter else torch.cat([ra, rb], dim=-1)
    return torch.cat([x[..., :begin], both, x[..., begin + rot:]], dim=-1)


def _plain_append(s):
    c = s["case"]
    seq, pos = _tokens(s)
    page, slot = s["table"].long()[seq, pos // c["page"]], pos % c["page"]
    q, k, v = s["q"].float(), s["k"].float(), s["v"].float()
    if c["rot"]:
        rows = s["cos_sin"][pos]
        q, k = _rotated(q, rows, c["begin"], c["inter"]), _rotated(k, rows, c["begin"], c["inter"])
    if s["k_scale"] is not None:
        # Written as bytes: torch puts no 8-bit floats by index.
        k, v = _fp8(k / s["k_scale"][:, None]), _fp8(v / s["v_scale"][:, None])
        s["k_cache"].view(torch.uint8)[page, :, slot] = k.view(torch.uint8)
        s["v_cache"].view(torch.uint8)[page, :, slot] = v.view(torch.uint8)
    else:
        s["k_cache"][page, :, slot] = k.to(torch.bfloat16)
        s["v_cache"][page, :, slot] = v.to(torch.bfloat16)
    return {"q": q.to(torch.bfloat16), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}


def _plain_attend(s):
    c, B, most = s["case"], s["table"].shape[0], s["max_q"]
    Hq, Hkv, dqk, dv = c["Hq"], c["Hkv"], c["dqk"], c["dv"]
    group = Hq // Hkv

    def pages(cache, scale, d):  # [B, Hkv, keys, d]
        x = cache[s["table"].clamp_min(0).long()].float()
        x = x if scale is None else x * scale[:, None, None]
        return x.permute(0, 2, 1, 3, 4).reshape(B, Hkv, -1, d)

    k, v = pages(s["k_cache"], s["k_scale"], dqk), pages(s["v_cache"], s["v_scale"], dv)
    n = s["q_starts"].diff().long()
    rows = torch.arange(most, device=n.device)
    token = (s["q_starts"][:-1].long()[:, None] + rows).clamp_max(s["T"] - 1)  # [B, most]; rows past n are dropped
    q = s["q"].float()[token].reshape(B, most, Hkv, group, dqk).permute(0, 2, 3, 1, 4).reshape(B, Hkv, -1, dqk)
    x = torch.matmul(q, k.transpose(2, 3).contiguous()).view(B, Hkv, group, most, -1) * (1.0 / math.sqrt(dqk))
    key = torch.arange(k.shape[2], device=n.device)
    last = s["kv_lens"].long()[:, None] - 1 + ((rows - n[:, None] + 1) if c["causal"] else torch.zeros_like(token))
    x = x.masked_fill((key > last[:, :, None])[:, None, None], -math.inf)
    top = x.amax(dim=-1, keepdim=True)
    x = torch.exp(x - top)
    total = x.sum(dim=-1, keepdim=True)
    o = torch.matmul(x.view(B, Hkv, group * most, -1), v).view(B, Hkv, group, most, dv) / total
    seq, pos = _tokens(s)
    row = torch.arange(s["T"], device=n.device) - s["q_starts"].long()[seq]
    out = {"o": o[seq, :, :, row].reshape(s["T"], Hq, dv).to(torch.bfloat16)}
    if c["lse"]:
        out["lse"] = (top + total.log())[seq, :, :, row].reshape(s["T"], Hq)
    return out


def exact(case, seed):
    """The outputs of one pass in 64 bits: token by token for the append, sequence by sequence and head by head for
    the attention."""
    s = prepare(case, seed)
    new, keys, page = _list(case["new"]), _list(case["keys"]), case["page"]
    table, group = s["table"].cpu().long(), case["Hq"] // case["Hkv"]
    ks = s["k_scale"].double() if s["k_scale"] is not None else None
    vs = s["v_scale"].double() if s["v_scale"] is not None else None
    if case["op"] == "append":
        q, k, v = s["q"].double(), s["k"].double(), s["v"].double()
        kc, vc = s["k_cache"].double(), s["v_cache"].double()
        at = 0
        for b, (n, end) in enumerate(zip(new, keys)):
            pos = torch.arange(end - n, end)
            rows = slice(at, at + n)
            if case["rot"]:
                # z = x + iy turned by the angle's unit number, as the program's table (fp32) has it.
                half, first = case["rot"] // 2, case["begin"]
                unit = torch.complex(*s["cos_sin"].double()[pos.to(q.device)].split(half, dim=1))[:, None]
                c = torch.arange(half, device=q.device)
                x, y = (first + 2 * c, first + 2 * c + 1) if case["inter"] else (first + c, first + half + c)
                for t in (q, k):
                    z = torch.complex(t[rows][..., x], t[rows][..., y]) * unit
                    t[rows, :, x], t[rows, :, y] = z.real, z.imag
            pg, slot = table[b, pos // page].to(q.device), (pos % page).to(q.device)
            kc[pg, :, slot] = (k[rows] / ks[:, None]).clamp(-FP8_MAX, FP8_MAX) if ks is not None else k[rows]
            vc[pg, :, slot] = (v[rows] / vs[:, None]).clamp(-FP8_MAX, FP8_MAX) if vs is not None else v[rows]
            at += n
        return {"q": q, "k_cache": kc, "v_cache": vc}
    T = sum(new)
    o = torch.zeros(T, case["Hq"], case["dv"], dtype=torch.float64, device=s["q"].device)
    lse = torch.zeros(T, case["Hq"], dtype=torch.float64, device=s["q"].device)
    at = 0
    for b, (n, end) in enumerate(zip(new, keys)):
        pg = table[b, : -(-end // page)].to(o.device)
        k_b, v_b = s["k_cache"][pg], s["v_cache"][pg]  # [pages, Hkv, page, d]
        seen = torch.arange(end, device=o.device)[None] <= torch.arange(end - n, end, device=o.device)[:, None]
        for g in range(case["Hkv"]):
            k, v = k_b[:, g].double().flatten(0, 1)[:end], v_b[:, g].double().flatten(0, 1)[:end]
            k, v = (k * ks[g], v * vs[g]) if ks is not None else (k, v)
            for h in range(g * group, (g + 1) * group):
                x = (s["q"][at:at + n, h].double() @ k.T.contiguous()) * case["dqk"] ** -0.5
                x = torch.where(seen, x, -math.inf) if case["causal"] else x
                lse[at:at + n, h] = torch.logsumexp(x, dim=1)
                o[at:at + n, h] = torch.softmax(x, dim=1) @ v
        at += n
    return {"o": o, "lse": lse} if case["lse"] else {"o": o}
