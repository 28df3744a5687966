"""Performance cases of decoding over a paged key-value cache: the page tables, the preparation of Q, K and V, the attention.

Three operators, each as a serving program calls it once per step (the first and, per layer, the other two):

  pages    `attn_kv_pages`: from the lengths of the requests and the tokens each of them adds, the pages they take from the free list, the
           cache slot and the position of every token of the batch, and the new lengths
  prepare  `attn_qkv_prepare`: norms of queries and keys for each head, position rotation, K and V written to their slots (or, for a prompt
           that goes through attn_fwd, Q, K and V laid out as it takes them)
  decode   `attn_decode`: attention of one new token per request over the pages of its cache

Where `own` is false `run` computes the same in elementary torch operations.  Head counts, head dimensions and lengths are those of the
package's workloads (8, 16 and 32 heads of 64 and 128, up to 131072 keys) and generic ones: grouped heads, odd counts, ragged lengths.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16}


def _pages(R, most, most_new, page_size, release=0, short=False, pad=0):
    """R requests of up to `most` tokens that add up to `most_new` each; the first `release` of them end; pool too small if `short`."""
    return {"op": "pages", "R": R, "most": most, "most_new": most_new, "page_size": page_size, "release": release, "short": short,
            "pad": pad}


def _prepare(B, N, H, KH, d, dtype, rot=None, interleaved=False, norm=True, cache=True, heads_first=False, page_size=16, start=0, pad=0):
    return {"op": "prepare", "B": B, "N": N, "H": H, "KH": KH, "d": d, "dtype": dtype, "rot": d if rot is None else rot,
            "interleaved": interleaved, "norm": norm, "cache": cache, "heads_first": heads_first, "page_size": page_size,
            "start": start, "pad": pad}


def _decode(R, most, H, KH, d, dtype, page_size=16, ragged=False, empty=0, window=0):
    return {"op": "decode", "R": R, "most": most, "H": H, "KH": KH, "d": d, "dtype": dtype, "page_size": page_size, "ragged": ragged,
            "empty": empty, "window": window}


def listed():
    def named(name, case):
        return {"name": name, **case}
    return [
        # one step of a few conversations: nothing but latency
        named("pages_step_8", _pages(8, 4000, 1, 16)),
        # one step of a busy server, some requests ending, the batch padded to its captured size
        named("pages_step_1000", _pages(1000, 8192, 1, 16, release=37, pad=24)),
        # prompts admitted together, 64 K tokens and more of them
        named("pages_prompts_60", _pages(60, 2000, 4096, 64)),
        # a single conversation far into its context
        named("prepare_1", _prepare(1, 1, 32, 8, 128, "bf16", start=100000)),
        # one step of a batch: odd head counts, part of the head rotated, interleaved pairs, padding rows behind the last request
        named("prepare_step_200", _prepare(1, 200, 28, 4, 64, "f16", rot=32, interleaved=True, start=3000, pad=56)),
        # a prompt of the 16-head causal workload, laid out for attn_fwd
        named("prepare_prompt_16x8192", _prepare(1, 8192, 16, 16, 128, "bf16", cache=False, heads_first=True)),
        # a long prompt with grouped heads on its way into the cache
        named("prepare_prompt_32x16384", _prepare(1, 16384, 32, 8, 128, "f16", page_size=64)),
        # a single short conversation: nothing but latency
        named("decode_1x200", _decode(1, 200, 8, 8, 64, "f16")),
        # a single conversation at the longest context: few rows, a long axis
        named("decode_1x131072", _decode(1, 131072, 32, 8, 128, "bf16", page_size=64)),
        # a server's ragged batch, one padding row
        named("decode_64_ragged", _decode(64, 8192, 32, 8, 128, "bf16", ragged=True, empty=1)),
        # odd everything under a sliding window: 7 query heads to a key head, lengths that end inside pages
        named("decode_21_window", _decode(21, 30001, 28, 4, 128, "f16", page_size=32, ragged=True, window=4099)),
        # ungrouped heads, full batch at 32 K keys: the largest
        named("decode_16x32768", _decode(16, 32768, 16, 16, 128, "bf16")),
    ]


_MOST_BYTES = 2.0 * 16 * 32768 * 16 * 128 * 2       # keys and values of the largest listed case


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    """One more case of one of the operators: sizes uniform over their logarithm, redrawn while they cost more than the largest listed."""
    op = rng.choice(["pages", "prepare", "decode", "decode"])
    if op == "pages":
        while True:
            R = _log(rng, 1, 4096)
            new = 1 if rng.random() < 0.5 else _log(rng, 2, 16384)
            if R * new <= 131072:
                break
        return _pages(R, _log(rng, 1, 16384), new, rng.choice([16, 32, 64, 128]), release=rng.choice([0, 0, R // 10]),
                      short=rng.random() < 0.2, pad=rng.choice([0, rng.randint(1, 64)]))
    KH = rng.choice([1, 2, 3, 4, 5, 8, 8, 16, 32])
    d, dtype, page_size = rng.choice([64, 128]), rng.choice(["f16", "bf16"]), rng.choice([16, 16, 32, 64, 128, 256])
    if op == "prepare":
        G = rng.choice([1, 1, 2, 3, 4, 7, 8])
        while True:
            B, N = rng.choice([1, 1, 2, 3]), _log(rng, 1, 32768)
            if B * N * KH * (G + 2) * d <= 16384 * 48 * 128:
                break
        cache = rng.random() < 0.7
        return _prepare(B, N, KH * G, KH, d, dtype, rot=rng.choice([d, d, d // 2, d // 4]), interleaved=rng.random() < 0.3,
                        norm=rng.random() < 0.8, cache=cache, heads_first=not cache or rng.random() < 0.3, page_size=page_size,
                        start=rng.choice([0, rng.randint(1, 1000000)]), pad=rng.choice([0, rng.randint(1, 8)]))
    G = rng.choice([1, 1, 2, 3, 4, 4, 5, 6, 7, 8, 8, 12, 16])
    while True:
        R, most = _log(rng, 1, 256), _log(rng, 1, 131072)
        if 4.0 * R * most * KH * d <= _MOST_BYTES:
            break
    return _decode(R, most, KH * G, KH, d, dtype, page_size, ragged=rng.random() < 0.6, empty=rng.choice([0, 0, R // 8]),
                   window=rng.choice([0, 0, 0, _log(rng, 1, most)]))


# ------------------------------------------------------------------------------------------- inputs

def _spread(n, most):
    """n lengths up to `most`, evenly spaced over their logarithm from most / 64 on: the same ones for every seed."""
    low = max(1.0, most / 64.0)
    return np.array([int(round(low * (most / low) ** (i / (n - 1)))) if n > 1 else most for i in range(n)], dtype=np.int64)


def _decode_lengths(case):
    lens = _spread(case["R"], case["most"]) if case["ragged"] else np.full(case["R"], case["most"], dtype=np.int64)
    lens[:case["empty"]] = 0
    return lens


def _page_requests(case):
    """(tokens in the cache, new tokens or -1) of every request, before they are put in an order."""
    lens, new = _spread(case["R"], case["most"]), _spread(case["R"], case["most_new"])[::-1].copy()
    new[:case["release"]] = -1
    return lens, new


def _page_counts(case):
    """(pages held, pages asked for, pages given back, new tokens)"""
    lens, new = _page_requests(case)
    ps, n = case["page_size"], np.maximum(new, 0)
    held = -(-lens // ps)
    return int(held.sum()), int((-(-(lens + n) // ps) - held).sum()), int(held[new < 0].sum()), int(n.sum())


def _up(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _prepare_pages(case, seed):
    rng = np.random.default_rng(seed)
    R, ps = case["R"], case["page_size"]
    lens, new = _page_requests(case)
    order = rng.permutation(R)
    lens, new = lens[order], new[order]
    held, asked, back, tokens = _page_counts(case)
    available = asked // 2 if case["short"] else asked + 7
    ring = held + available + 5                                  # every page of the pool fits into the ring
    pages = rng.permutation(ring).astype(np.int32)
    first = int(rng.integers(0, ring))
    free = np.full(ring, -1, dtype=np.int32)
    free[(first + np.arange(available)) % ring] = pages[held:held + available]
    wide = int((-(-(lens + np.maximum(new, 0)) // ps)).max())
    table = np.zeros((R, wide), dtype=np.int32)
    at = 0
    for r in range(R):
        n = int(-(-lens[r] // ps))
        table[r, :n] = pages[at:at + n]
        at += n
    T = tokens + case["pad"]
    i32 = {"dtype": torch.int32, "device": "cuda"}
    return {"op": "pages", "page_size": ps, "lengths": _up(lens.astype(np.int32)), "new": _up(new.astype(np.int32)),
            "table": _up(table), "free": _up(free), "state": _up(np.array([first, available], dtype=np.int32)),
            "lengths_out": torch.zeros(R, **i32), "granted": torch.zeros(R, **i32), "offsets": torch.zeros(R + 1, **i32),
            "state_out": torch.zeros(2, **i32), "slots": torch.zeros(T, dtype=torch.int64, device="cuda"),
            "positions": torch.zeros(T, **i32)}


def _prepare_prepare(case, seed):
    rng = np.random.default_rng(seed)
    g = torch.Generator("cuda").manual_seed(int(seed))
    B, N, H, KH, d, ps = (case[k] for k in ("B", "N", "H", "KH", "d", "page_size"))
    dt, rows, rot = _DTYPE[case["dtype"]], case["N"] + case["pad"], case["rot"]

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    # one projection's output: the heads of Q, K and V of a token side by side
    qkv = normal(B, rows, H + 2 * KH, d).to(dt)
    q, k, v = qkv[:, :, :H], qkv[:, :, H:H + KH], qkv[:, :, H + KH:]

    def out(heads):
        if case["heads_first"]:
            return torch.zeros(B, heads, rows, d, dtype=dt, device="cuda").transpose(1, 2)
        return torch.zeros(B, rows, heads, d, dtype=dt, device="cuda")
    prompt = N > 256                                             # a prompt has rising positions, a step one of its own per request
    pos = np.full((B, rows), -1, dtype=np.int32)
    pos[:, :N] = case["start"] + (np.arange(N) if prompt else rng.integers(0, 1000, (B, N)))
    s = {"op": "prepare", "N": N, "rot": rot, "interleaved": case["interleaved"], "page_size": ps, "q": q, "k": k, "v": v,
         "positions": _up(pos), "eps": 1e-6,
         "frequencies": _up((1e6 ** (-np.arange(rot // 2) * 2.0 / rot)).astype(np.float64)),
         "q_weight": 1.0 + 0.1 * normal(d) if case["norm"] else None, "k_weight": 1.0 + 0.1 * normal(d) if case["norm"] else None,
         "q_out": out(H), "k_out": None, "v_out": None, "cache_k": None, "cache_v": None, "slots": None}
    if case["heads_first"]:
        s["k_out"], s["v_out"] = out(KH), out(KH)
    if case["cache"]:
        pages = -(-B * N // ps) + 3
        s["cache_k"], s["cache_v"] = normal(pages, KH, ps, d).to(dt), normal(pages, KH, ps, d).to(dt)
        if prompt:                                               # whole pages in any order, filled one after the other
            slot = rng.permutation(pages)[np.arange(B * N) // ps] * ps + np.arange(B * N) % ps
        else:
            slot = rng.permutation(pages * ps)[:B * N]
        slots = np.full((B, rows), -1, dtype=np.int64)
        slots[:, :N] = slot.reshape(B, N)
        s["slots"] = _up(slots)
    return s


def _prepare_decode(case, seed):
    rng = np.random.default_rng(seed)
    g = torch.Generator("cuda").manual_seed(int(seed))
    R, H, KH, d, ps = (case[k] for k in ("R", "H", "KH", "d", "page_size"))
    dt = _DTYPE[case["dtype"]]
    lens = rng.permutation(_decode_lengths(case))
    count = -(-lens // ps)
    total = int(count.sum()) + 3
    pages = rng.permutation(total).astype(np.int32)
    table = np.zeros((R, max(1, int(count.max()))), dtype=np.int32)
    at = 0
    for r in range(R):
        table[r, :count[r]] = pages[at:at + count[r]]
        at += int(count[r])

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)
    return {"op": "decode", "q": normal(R, H, d), "cache_k": normal(total, KH, ps, d), "cache_v": normal(total, KH, ps, d),
            "table": _up(table), "lengths": _up(lens.astype(np.int32)), "o": torch.zeros(R, H, d, dtype=dt, device="cuda"),
            "scale": 1.0 / math.sqrt(d), "window": case["window"]}


def _handles(s):
    """What a program keeps beside the tensors: the description of its cache and, for the attention, the workspace."""
    from paper_2601_16032_amd import binding
    s["binding"] = binding
    if s.get("cache_k") is not None:
        s["cache"] = binding.KVCache(s["cache_k"], s["cache_v"])
    if s["op"] == "decode":
        need = binding.attn_decode_workspace_bytes(s["q"].shape[0], s["q"].shape[1], s["cache"], s["table"].shape[1])
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    s = {"pages": _prepare_pages, "prepare": _prepare_prepare, "decode": _prepare_decode}[case["op"]](case, seed)
    if own:
        _handles(s)
    return s


# ------------------------------------------------------------------------------------------- one pass

def _plain_pages(s):
    ps, F = s["page_size"], s["free"].numel()
    table, R = s["table"], s["lengths"].numel()
    lens, new = s["lengths"].long(), s["new"].long()
    first, available = s["state"][0].long(), s["state"][1].long()
    n = new.clamp(min=0)
    end, held = lens + n, (lens + ps - 1) // ps
    fits = (n > 0) & (end <= table.shape[1] * ps)
    need = torch.where(fits, (end + ps - 1) // ps - held, 0)
    upto = need.cumsum(0)
    granted = fits & ((need == 0) | (upto <= available))
    used = torch.where(upto <= available, upto, 0).max()
    gone = new < 0
    back = torch.where(gone, held, 0)
    back_upto = back.cumsum(0)
    j = torch.arange(table.shape[1], device=table.device)[None, :]
    taken = granted[:, None] & (j >= held[:, None]) & (j < (held + need)[:, None])
    source = (first + (upto - need - held)[:, None] + j) % F
    s["table"].copy_(torch.where(taken, s["free"][source], table))
    target = torch.where(gone[:, None] & (j < held[:, None]), (first + available + (back_upto - back)[:, None] + j) % F, F)
    ring = torch.cat([s["free"], s["free"][:1]])                 # one place more, for what is not given back
    s["free"].copy_(ring.scatter_(0, target.reshape(-1), table.reshape(-1))[:F])
    s["state_out"].copy_(torch.stack([(first + used) % F, available - used + back_upto[-1]]))
    s["lengths_out"].copy_(torch.where(gone, 0, torch.where(granted, end, lens)))
    s["granted"].copy_(torch.where(granted, n, 0))
    s["offsets"].copy_(torch.cat([torch.zeros_like(n[:1]), n.cumsum(0)]))
    t = torch.arange(s["slots"].numel(), device=table.device)
    behind = n.cumsum(0)
    r = torch.searchsorted(behind, t, right=True).clamp(max=R - 1)
    position = lens[r] + t - (behind - n)[r]
    valid = (t < behind[-1]) & granted[r]
    page = table[r, torch.where(valid, position // ps, 0)].long()
    s["slots"].copy_(torch.where(valid, page * ps + position % ps, -1))
    s["positions"].copy_(torch.where(valid, position, -1))


def _plain_rows(s, x, weight):
    """Norm of each head and rotation, in 32 bits, the angles in 64."""
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + s["eps"]) * weight
    rot = s["rot"]
    angle = s["positions"][:, :s["N"], None].double() * s["frequencies"]
    cos, sin = angle.cos().float()[:, :, None], angle.sin().float()[:, :, None]
    turned = x[..., :rot]
    a, b = (turned[..., 0::2], turned[..., 1::2]) if s["interleaved"] else (turned[..., :rot // 2], turned[..., rot // 2:])
    a, b = a * cos - b * sin, a * sin + b * cos
    turned = torch.stack([a, b], -1).flatten(-2) if s["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _plain_prepare(s):
    N = s["N"]                                                   # rows behind these are padding
    k = _plain_rows(s, s["k"][:, :N], s["k_weight"]).to(s["k"].dtype)
    v = s["v"][:, :N]
    s["q_out"][:, :N] = _plain_rows(s, s["q"][:, :N], s["q_weight"]).to(s["q"].dtype)
    if s["k_out"] is not None:
        s["k_out"][:, :N], s["v_out"][:, :N] = k, v
    if s["cache_k"] is not None:
        slots = s["slots"][:, :N].reshape(-1)
        page, row = slots // s["page_size"], slots % s["page_size"]
        s["cache_k"][page, :, row] = k.reshape(-1, *k.shape[2:])
        s["cache_v"][page, :, row] = v.reshape(-1, *v.shape[2:])


def _plain_decode(s):
    (R, H, d), (_, KH, ps, _) = s["q"].shape, s["cache_k"].shape
    wide = s["table"].shape[1]
    G, L = H // KH, wide * ps
    step = max(1, (1 << 28) // (KH * L * d))                     # as many requests at a time as leave the copies below 1 GiB each
    key = torch.arange(L, device=s["q"].device)
    for r in range(0, R, step):
        pages, n = s["table"][r:r + step].long(), s["lengths"][r:r + step, None]
        k = s["cache_k"][pages].float().transpose(1, 2).reshape(-1, KH, L, d)
        q = s["q"][r:r + step].float().reshape(-1, KH, G, d).transpose(2, 3).contiguous()
        p = torch.matmul(k, q).mul_(s["scale"])                  # [requests, key heads, keys, queries of the group]
        del k
        hidden = key[None] >= n
        if s["window"]:
            hidden = hidden | (key[None] < n - s["window"])
        p.masked_fill_(hidden[:, None, :, None], -math.inf)
        most = p.amax(2, keepdim=True)
        p = torch.exp(p - torch.where(most == -math.inf, 0.0, most))
        total = p.sum(2)
        v = s["cache_v"][pages].float().transpose(1, 2).reshape(-1, KH, L, d)
        o = torch.matmul(p.transpose(2, 3).contiguous(), v)
        o = o / torch.where(total == 0, 1.0, total)[..., None]
        s["o"][r:r + step] = o.reshape(-1, H, d).to(s["o"].dtype)


def _own_pages(s):
    s["binding"].attn_kv_pages(s["lengths"], s["new"], s["table"], s["free"], s["state"], page_size=s["page_size"],
                               lengths_out=s["lengths_out"], granted=s["granted"], token_offsets=s["offsets"],
                               free_state_out=s["state_out"], slots=s["slots"], positions=s["positions"])


def _own_prepare(s):
    s["binding"].attn_qkv_prepare(s["q"], s["k"], s["v"], positions=s["positions"], frequencies=s["frequencies"],
                                  interleaved=s["interleaved"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=s["eps"],
                                  q_out=s["q_out"], k_out=s["k_out"], v_out=s["v_out"], cache=s.get("cache"), slots=s["slots"])


def _own_decode(s):
    s["binding"].attn_decode(s["q"], s["cache"], s["table"], s["lengths"], s["o"], scale=s["scale"], window=s["window"],
                             workspace=s["workspace"])


_PLAIN = {"pages": _plain_pages, "prepare": _plain_prepare, "decode": _plain_decode}
_OWN = {"pages": _own_pages, "prepare": _own_prepare, "decode": _own_decode}
_OUT = {"pages": ("table", "free", "lengths_out", "granted", "offsets", "state_out", "slots", "positions"),
        "prepare": ("q_out", "k_out", "v_out", "cache_k", "cache_v"), "decode": ("o",)}


def run(state):
    if own and "binding" not in state:
        _handles(state)
    (_OWN if own else _PLAIN)[state["op"]](state)
    return {name: state[name] for name in _OUT[state["op"]] if state[name] is not None}


def work(case):
    if case["op"] == "pages":
        _, asked, back, tokens = _page_counts(case)
        # lengths and counts in; lengths, counts, offsets out; a page from the list into the table or back; slot and position per token
        return {"bytes": 20.0 * case["R"] + 8 * (asked + back) + 12 * (tokens + case["pad"]), "flops": 4.0 * tokens}
    d = case["d"]
    if case["op"] == "prepare":
        tokens, H, KH = case["B"] * case["N"], case["H"], case["KH"]
        written = H + 2 * KH * (int(case["cache"]) + int(case["heads_first"]))
        return {"bytes": 2.0 * tokens * d * (H + 2 * KH + written) + tokens * (12 if case["cache"] else 4),
                "flops": 8.0 * tokens * d * (H + KH)}
    lens = _decode_lengths(case)
    seen = float((np.minimum(lens, case["window"]) if case["window"] else lens).sum())
    return {"bytes": 4.0 * seen * case["KH"] * d + 4.0 * case["R"] * case["H"] * d + 4.0 * seen / case["page_size"],
            "flops": 4.0 * seen * case["H"] * d}


# ------------------------------------------------------------------------------------------- the definition, in 64 bits

def _exact_pages(s):
    """Request by request, as the definition reads, on the host."""
    ps = s["page_size"]
    lens, new, free = s["lengths"].tolist(), s["new"].tolist(), s["free"].tolist()
    first, available = s["state"].tolist()
    table = s["table"].cpu().numpy().copy()
    F, asked, used, back = len(free), 0, 0, 0
    out_len, granted, offsets, slots, positions = [], [], [0], [], []
    ring = list(free)
    for r, (length, n) in enumerate(zip(lens, new)):
        held = -(-length // ps)
        offsets.append(offsets[-1] + max(n, 0))
        if n < 0:                                                # ends: its pages go behind the last free one
            for j in range(held):
                ring[(first + available + back + j) % F] = int(table[r, j])
            back += held
            out_len.append(0)
            granted.append(0)
            continue
        ok = n > 0 and length + n <= table.shape[1] * ps
        need = -(-(length + n) // ps) - held if ok else 0
        asked += need
        if need and asked > available:
            ok = False
        elif need:
            table[r, held:held + need] = [free[(first + used + j) % F] for j in range(need)]
            used += need
        out_len.append(length + n if ok else length)
        granted.append(n if ok else 0)
        at = np.arange(length, length + n)
        positions.append(at if ok else np.full(n, -1))
        slots.append(table[r, at // ps].astype(np.int64) * ps + at % ps if ok else np.full(n, -1))

    def whole(parts, like):
        x = np.concatenate([np.zeros(0, dtype=np.int64)] + parts)
        return torch.from_numpy(np.concatenate([x, np.full(like.numel() - x.size, -1)])).to(like)

    def ints(x, like):
        return torch.tensor(x).to(like)
    return {"table": ints(table, s["table"]), "free": ints(ring, s["free"]), "lengths_out": ints(out_len, s["lengths_out"]),
            "granted": ints(granted, s["granted"]), "offsets": ints(offsets, s["offsets"]),
            "state_out": ints([(first + used) % F, available - used + back], s["state_out"]),
            "slots": whole(slots, s["slots"]), "positions": whole(positions, s["positions"])}


def _exact_prepare(s):
    N, rot = s["N"], s["rot"]
    half = torch.arange(rot // 2, device="cuda")
    ia, ib = (2 * half, 2 * half + 1) if s["interleaved"] else (half, half + rot // 2)
    angle = s["positions"][:, :N].double()[:, :, None, None] * s["frequencies"]
    turn = torch.complex(angle.cos(), angle.sin())

    def rows(x, weight):
        x = x[:, :N].double()
        if weight is not None:
            x = x / torch.sqrt(x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + s["eps"]) * weight.double()
        z = torch.complex(x[..., ia], x[..., ib]) * turn
        x[..., ia], x[..., ib] = z.real, z.imag
        return x
    q, k, v = rows(s["q"].clone(), s["q_weight"]), rows(s["k"].clone(), s["k_weight"]), s["v"][:, :N].double()
    out = {"q_out": s["q_out"].double()}
    out["q_out"][:, :N] = q
    if s["k_out"] is not None:
        out["k_out"], out["v_out"] = s["k_out"].double(), s["v_out"].double()
        out["k_out"][:, :N], out["v_out"][:, :N] = k, v
    if s["cache_k"] is not None:
        flat = s["slots"][:, :N].reshape(-1)
        for name, x in (("cache_k", k), ("cache_v", v)):
            rows_of = s[name].double().transpose(1, 2).reshape(-1, *x.shape[2:])          # [slots, heads, d]
            rows_of[flat] = x.reshape(-1, *x.shape[2:])
            pages, heads, ps, d = s[name].shape
            out[name] = rows_of.reshape(pages, ps, heads, d).transpose(1, 2).contiguous()
    return out


def _exact_decode(s):
    (R, H, d), (_, KH, ps, _) = s["q"].shape, s["cache_k"].shape
    out = torch.zeros(R, H, d, dtype=torch.float64, device="cuda")
    for r, n in enumerate(s["lengths"].tolist()):
        low = max(0, n - s["window"]) if s["window"] else 0
        if n == 0:
            continue
        pages = s["table"][r, low // ps:-(-n // ps)].long()
        for h in range(KH):
            k, v = (s[c][pages, h].double().reshape(-1, d)[low % ps:n - low // ps * ps] for c in ("cache_k", "cache_v"))
            q = s["q"][r, h * (H // KH):(h + 1) * (H // KH)].double()
            w = torch.softmax(torch.mm(q, k.t().contiguous()) * s["scale"], dim=1)
            out[r, h * (H // KH):(h + 1) * (H // KH)] = torch.mm(w, v)
    return {"o": out}


def exact(case, seed):
    s = {"pages": _prepare_pages, "prepare": _prepare_prepare, "decode": _prepare_decode}[case["op"]](case, seed)
    out = {"pages": _exact_pages, "prepare": _exact_prepare, "decode": _exact_decode}[case["op"]](s)
    return {name: out[name] for name in _OUT[case["op"]] if name in out}
