"""Performance cases of requests that share pages of a paged key-value cache: forks, page copies, common rows, attention.

Four operators, as a program calls them that searches with beams, samples several answers to a prompt or keeps prompts for later requests:

  fork    `attn_kv_fork`, once per step: every request of the new batch goes on from one of the old batch, whole pages are shared, pages that
          nobody holds any more go back to the free list, and the part-filled pages to be copied are named
  copy    `attn_kv_copy`, once per fork: those pages are copied, in all layers
  rows    `attn_kv_shared_rows`, once per fork: how many leading rows the requests of a group have in the same pages
  shared  `attn_decode_shared`, per layer and step: attention of one new token per request, the rows that a group shares read once for all of it

Where `own` is false `run` computes the same in elementary torch operations.  Head counts, head dimensions and lengths are those of the
package's workloads (8, 16 and 32 heads of 64 and 128, up to 32768 keys) and generic ones: grouped heads, odd counts, ragged lengths.
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

_DTYPE = {"f16": torch.float16, "bf16": torch.bfloat16}


def _fork(groups, old, new, most, page_size, end=0, cut=False, short=False):
    """`groups` families of `old` requests of up to `most` rows each that become `new` each, the first `end` of the batch ending; some of
    the new ones cut short if `cut`; fewer free pages than are asked for if `short`."""
    return {"op": "fork", "groups": groups, "old": old, "new": new, "most": most, "page_size": page_size, "end": end, "cut": cut, "short": short}


def _copy(n, real, layers, heads, d, dtype, page_size):
    """A list of `n` copies, `real` of them to be made, in each of `layers` caches."""
    return {"op": "copy", "n": n, "real": real, "layers": layers, "heads": heads, "d": d, "dtype": dtype, "page_size": page_size}


def _rows(groups, size, most, page_size, empty=0):
    return {"op": "rows", "groups": groups, "size": size, "most": most, "page_size": page_size, "empty": empty}


def _shared(groups, size, prefix, tail, H, KH, d, dtype, page_size=16, ragged=False, pad=0, alone=0):
    """`groups` groups of `size` requests, `prefix` rows in common (ragged: up to as many), up to `tail` rows of their own; then `alone` requests in
    no group and `pad` empty ones."""
    return {"op": "shared", "groups": groups, "size": size, "prefix": prefix, "tail": tail, "H": H, "KH": KH, "d": d, "dtype": dtype,
            "page_size": page_size, "ragged": ragged, "pad": pad, "alone": alone}


def listed():
    def named(name, case):
        return {"name": name, **case}
    return [
        # one step of a search with eight beams over one prompt: nothing but latency
        named("fork_step_8", _fork(1, 8, 8, 2000, 16)),
        # one step of a busy server with beams, some requests ending, some cut back to what a check has accepted
        named("fork_step_1000", _fork(125, 8, 8, 8192, 16, end=31, cut=True)),
        # many answers to each of a hundred prompts begin: the largest batch, long tables
        named("fork_prompts_4000", _fork(100, 1, 40, 16384, 16, cut=True)),
        # the pages that eight beams have to copy, in two layers: latency
        named("copy_8_2_layers", _copy(8, 3, 2, 8, 64, "f16", 16)),
        # those of a full batch, in all layers of a small model
        named("copy_200_16_layers", _copy(200, 121, 16, 8, 128, "bf16", 64)),
        # eight beams over one prompt
        named("rows_8", _rows(1, 8, 4000, 16)),
        # a full batch in groups, long prompts, some requests ended
        named("rows_1000", _rows(40, 25, 16384, 16, empty=3)),
        # four beams over a short prompt: nothing but latency
        named("shared_4_beams", _shared(1, 4, 500, 40, 8, 8, 64, "f16")),
        # searches with four beams over sixteen prompts
        named("shared_16x4_beams", _shared(16, 4, 4096, 200, 32, 8, 128, "bf16", ragged=True)),
        # a server's batch behind one long instruction, one padding row
        named("shared_64", _shared(1, 64, 8192, 1000, 32, 8, 128, "bf16", page_size=64, pad=1)),
        # odd everything: 7 query heads to a key head, 21 requests to a group, some requests on their own
        named("shared_5x21_odd", _shared(5, 21, 7001, 333, 28, 4, 128, "f16", page_size=32, ragged=True, alone=3)),
        # the largest: a full batch behind a prompt of 32 K
        named("shared_256", _shared(1, 256, 32768, 2000, 32, 8, 128, "bf16", page_size=64)),
    ]


def _log(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


_MOST_SEEN = 256.0 * (32768 + 600) * 32 * 128       # flops / 4 of the largest listed case
_MOST_BYTES = 256.0 * 600 * 8 * 128                 # bytes / 4 of its requests' own rows


def draw(rng):
    """One more case of one of the operators: sizes uniform over their logarithm, redrawn while they cost more than the largest listed."""
    op = rng.choice(["fork", "copy", "rows", "shared", "shared", "shared"])
    page_size = rng.choice([16, 16, 32, 64, 128])
    if op == "fork":
        while True:
            groups, old, new, most = _log(rng, 1, 512), _log(rng, 1, 64), _log(rng, 1, 64), _log(rng, 1, 16384)
            if groups * max(old, new) <= 4096 and groups * max(old, new) * most / page_size <= 2e6:
                break
        return _fork(groups, old, new, most, page_size, end=rng.choice([0, 0, groups * new // 10]), cut=rng.random() < 0.4, short=rng.random() < 0.2)
    if op == "rows":
        while True:
            groups, size, most = _log(rng, 1, 256), _log(rng, 2, 256), _log(rng, 64 * page_size, 32768)
            if groups * size <= 4096 and groups * size * most / page_size <= 2e6:
                break
        return _rows(groups, size, most, page_size, empty=rng.choice([0, 0, groups * size // 10]))
    KH = rng.choice([1, 2, 3, 4, 5, 8, 8, 16, 32])
    d, dtype = rng.choice([64, 128]), rng.choice(["f16", "bf16"])
    if op == "copy":
        while True:
            n, layers = _log(rng, 1, 1024), _log(rng, 1, 40)
            if (n + 10.0) * layers * KH * page_size * d <= 200 * 16 * 8 * 64 * 128:
                break
        return _copy(n, rng.randint(0, n), layers, KH, d, dtype, page_size)
    G = rng.choice([1, 1, 2, 3, 4, 4, 5, 6, 7, 8, 8, 12, 16])
    while True:
        groups, size, prefix, tail = _log(rng, 1, 32), _log(rng, 1, 256), _log(rng, 1, 65536), _log(rng, 1, 4096)
        n = groups * size
        if n <= 1024 and n * (prefix + tail) * KH * G * d <= _MOST_SEEN and groups * prefix * KH * d <= 32768 * 32 * 128 and n * tail * KH * d <= _MOST_BYTES * 2:
            break
    return _shared(groups, size, prefix, tail, KH * G, KH, d, dtype, page_size, ragged=rng.random() < 0.5, pad=rng.choice([0, 0, rng.randint(1, 8)]),
                   alone=rng.choice([0, 0, 0, rng.randint(1, 3)]))


# ------------------------------------------------------------------------------------------- inputs

def _spread(n, most):
    """n lengths up to `most`, evenly spaced over their logarithm from most / 64 on: the same ones for every seed."""
    low = max(1.0, most / 64.0)
    return np.array([int(round(low * (most / low) ** (i / (n - 1)))) if n > 1 else most for i in range(n)], dtype=np.int64)


def _up(x):
    return torch.from_numpy(np.ascontiguousarray(x)).cuda()


def _fork_requests(case):
    """(rows of a request of each family, their common whole pages, most rows that each new request keeps)"""
    ps, new = case["page_size"], case["new"]
    lens = _spread(case["groups"], case["most"])
    common = lens * 9 // 10 // ps
    keep = np.repeat(lens, new)
    if case["cut"]:                                              # every third goes back by up to seven rows, every twelfth by half
        i = np.arange(keep.size)
        keep = np.where(i % 3 == 1, keep - i % 8, np.where(i % 12 == 5, keep // 2, keep)).clip(min=0)
    return lens, common, keep


def _fork_entries(case):
    """(entries of the old tables, entries of the new ones)"""
    lens, _, keep = _fork_requests(case)
    ps = case["page_size"]
    return int((-(-lens // ps)).sum()) * case["old"], int((-(-keep[case["end"]:] // ps)).sum())


def _prepare_fork(case, seed):
    rng = np.random.default_rng(seed)
    groups, old, new, ps = (case[k] for k in ("groups", "old", "new", "page_size"))
    lens, common, keep = _fork_requests(case)
    R, N = groups * old, groups * new
    count = -(-lens // ps)
    held = int((common + (count - common) * old).sum())
    available = max(1, N // 4) if case["short"] else N + 3
    total = held + available + 5
    pages = rng.permutation(total).astype(np.int32)
    wide = int(count.max())
    table = np.zeros((R, wide), dtype=np.int32)
    at = 0
    for g in range(groups):
        c, n = int(common[g]), int(count[g])
        table[g * old:(g + 1) * old, :c] = pages[at:at + c]
        at += c
        table[g * old:(g + 1) * old, c:n] = pages[at:at + (n - c) * old].reshape(old, n - c)
        at += (n - c) * old
    source = (np.repeat(np.arange(groups), new) * old + rng.integers(0, old, N)).astype(np.int32)
    source[:case["end"]] = -1
    first = int(rng.integers(0, total))
    free = np.full(total, -1, dtype=np.int32)
    free[(first + np.arange(available)) % total] = pages[held:held + available]
    i32 = {"dtype": torch.int32, "device": "cuda"}
    return {"op": "fork", "page_size": ps, "pages": total, "lengths": _up(np.repeat(lens, old).astype(np.int32)), "source": _up(source),
            "rows": _up(keep.astype(np.int32)) if case["cut"] else None, "table": _up(table), "free": _up(free),
            "state": _up(np.array([first, available], dtype=np.int32)), "table_out": torch.zeros(N, wide, **i32),
            "lengths_out": torch.zeros(N, **i32), "copies": torch.zeros(N, 3, **i32), "state_out": torch.zeros(2, **i32)}


def _copied_rows(case):
    return _spread(case["real"], case["page_size"]) if case["real"] else np.zeros(0, dtype=np.int64)


def _prepare_copy(case, seed):
    rng = np.random.default_rng(seed)
    g = torch.Generator("cuda").manual_seed(int(seed))
    n, real, ps = case["n"], case["real"], case["page_size"]
    total = 2 * real + 3
    pages = rng.permutation(total)
    copies = np.full((n, 3), -1, dtype=np.int32)
    copies[:, 2] = 0
    where = rng.permutation(n)[:real]
    copies[where, 0], copies[where, 1], copies[where, 2] = pages[:real], pages[real:2 * real], rng.permutation(_copied_rows(case))
    caches = [[torch.randn(total, case["heads"], ps, case["d"], generator=g, device="cuda", dtype=_DTYPE[case["dtype"]]) for _ in range(2)]
              for _ in range(case["layers"])]
    return {"op": "copy", "copies": _up(copies), "caches": caches}


def _rows_common(case):
    """(lengths, whole pages in common at most) of every group, before some requests end"""
    lens = _spread(case["groups"], case["most"])
    return lens, lens * 7 // 8 // case["page_size"]


def _prepare_rows(case, seed):
    rng = np.random.default_rng(seed)
    groups, size, ps = case["groups"], case["size"], case["page_size"]
    lens, common = _rows_common(case)
    common -= rng.integers(0, common // 8 + 1)
    count = -(-lens // ps)
    table = rng.integers(0, 1 << 20, (groups * size, int(count.max()))).astype(np.int32)
    for g in range(groups):
        table[g * size:(g + 1) * size, :common[g]] = table[g * size, :common[g]]
        if size > 1 and common[g] < table.shape[1]:              # they do differ in the page behind
            table[g * size + 1, common[g]] = table[g * size, common[g]] ^ 1
    lengths = np.repeat(lens, size)
    lengths[rng.permutation(groups * size)[:case["empty"]]] = 0
    return {"op": "rows", "page_size": ps, "groups": groups, "size": size, "table": _up(table), "lengths": _up(lengths.astype(np.int32)),
            "offsets": _up(np.arange(groups + 1, dtype=np.int32) * size), "shared": torch.zeros(groups, dtype=torch.int32, device="cuda")}


def _shared_lengths(case):
    """(rows in common of each group, rows of each request of its own: of the groups, then of those in none)"""
    groups = case["groups"]
    prefix = _spread(groups, case["prefix"]) if case["ragged"] else np.full(groups, case["prefix"], dtype=np.int64)
    return prefix, _spread(groups * case["size"] + case["alone"], case["tail"])


def _prepare_shared(case, seed):
    rng = np.random.default_rng(seed)
    g = torch.Generator("cuda").manual_seed(int(seed))
    groups, size, H, KH, d, ps = (case[k] for k in ("groups", "size", "H", "KH", "d", "page_size"))
    dt = _DTYPE[case["dtype"]]
    prefix, tail = _shared_lengths(case)
    n = groups * size
    R = n + case["alone"] + case["pad"]
    lens = np.zeros(R, dtype=np.int64)
    lens[:n + case["alone"]] = rng.permutation(tail)
    lens[:n] += np.repeat(prefix, size)
    whole = np.zeros(R, dtype=np.int64)                          # pages in common: the part-filled last one of the prefix is everyone's own
    whole[:n] = np.repeat(prefix // ps, size)
    count = -(-lens // ps)
    total = int((count - whole).sum() + (prefix // ps).sum()) + 3
    pages = rng.permutation(total).astype(np.int32)
    table = np.zeros((R, int(count.max())), dtype=np.int32)
    at = 0
    for r in range(R):
        if r < n and r % size == 0:
            table[r:r + size, :whole[r]] = pages[at:at + whole[r]]
            at += int(whole[r])
        mine = int(count[r] - whole[r])
        table[r, whole[r]:count[r]] = pages[at:at + mine]
        at += mine

    def normal(*shape):
        return torch.randn(shape, generator=g, device="cuda", dtype=dt)
    return {"op": "shared", "q": normal(R, H, d), "cache_k": normal(total, KH, ps, d), "cache_v": normal(total, KH, ps, d), "table": _up(table),
            "lengths": _up(lens.astype(np.int32)), "offsets": _up(np.arange(groups + 1, dtype=np.int32) * size),
            "shared": _up(prefix.astype(np.int32)), "o": torch.zeros(R, H, d, dtype=dt, device="cuda"), "scale": 1.0 / math.sqrt(d),
            # what a plain program knows of its requests: first, behind the last, pages in common, most pages
            "groups": [(i * size, (i + 1) * size, int(p) // ps, int(count[i * size:(i + 1) * size].max())) for i, p in enumerate(prefix)],
            "others": [(n, R, 0, int(count[n:].max()))] if R > n else []}


_PREPARE = {"fork": _prepare_fork, "copy": _prepare_copy, "rows": _prepare_rows, "shared": _prepare_shared}


def _handles(s):
    """What a program keeps beside the tensors: the descriptions of its caches, the workspaces."""
    from paper_2601_16032_amd import binding
    s["binding"] = binding
    if s["op"] == "fork":
        need = binding.attn_kv_fork_workspace_bytes(s["lengths"].numel(), s["source"].numel(), s["pages"])
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")
    elif s["op"] == "copy":
        s["layers"] = binding.KVLayers([binding.KVCache(k, v) for k, v in s["caches"]])
    elif s["op"] == "shared":
        s["cache"] = binding.KVCache(s["cache_k"], s["cache_v"])
        need = binding.attn_decode_shared_workspace_bytes(s["q"].shape[0], s["q"].shape[1], s["shared"].numel(), s["cache"], s["table"].shape[1])
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")


def prepare(case, seed):
    s = _PREPARE[case["op"]](case, seed)
    if own:
        _handles(s)
    return s


# ------------------------------------------------------------------------------------------- one pass

def _plain_fork(s):
    ps, F, P = s["page_size"], s["free"].numel(), s["pages"]
    table = s["table"]
    (R, wide), N = table.shape, s["source"].numel()
    lens = s["lengths"].long()
    source = s["source"].long()
    first, available = s["state"][0].long(), s["state"][1].long()
    valid = (source >= 0) & (source < R)
    source = torch.where(valid, source, 0)
    n = torch.where(valid, lens[source], 0)
    if s["rows"] is not None:
        n = torch.minimum(n, s["rows"].long())
    full, part = n // ps, n % ps > 0
    last = part & (full == lens[source] // ps)                   # ends in the part-filled page of its source: the first such takes it over
    r = torch.arange(N, device=table.device)
    winner = torch.full((R + 1,), N, device=table.device).scatter_reduce_(0, torch.where(last, source, R), r, "amin")
    takes = last & (winner[source] == r)
    missing = part & ~takes
    upto = missing.long().cumsum(0)
    ok = ~missing | (upto <= available)
    used = torch.minimum(upto[-1], available)
    fresh = s["free"][(first + upto - 1) % F].long()
    j = torch.arange(wide, device=table.device)[None, :]
    old = table[source]
    same = ok[:, None] & (j < (full + takes)[:, None])
    new = torch.where(same, old, s["table_out"])
    s["table_out"].copy_(torch.where((missing & ok)[:, None] & (j == full[:, None]), fresh[:, None], new))
    s["lengths_out"].copy_(torch.where(ok, n, 0))
    torn = old.gather(1, torch.clamp(full, max=wide - 1)[:, None])[:, 0].long()
    s["copies"].copy_(torch.stack([torch.where(missing, torn, -1), torch.where(missing & ok, fresh, -1), torch.where(missing, n % ps, 0)], 1))
    kept = torch.zeros(P + 1, dtype=torch.bool, device=table.device)
    kept[torch.where(same, old, P).long()] = True
    held = torch.zeros(P + 1, dtype=torch.bool, device=table.device)
    held[torch.where(j < ((lens + ps - 1) // ps)[:, None], table, P).long()] = True
    freed = held[:P] & ~kept[:P]
    at = freed.long().cumsum(0)
    ring = torch.cat([s["free"], s["free"][:1]])                 # one place more, for what is not given back
    page = torch.arange(P, dtype=torch.int32, device=table.device)
    s["free"].copy_(ring.scatter_(0, torch.where(freed, (first + available + at - 1) % F, F), page)[:F])
    s["state_out"].copy_(torch.stack([(first + used) % F, available - used + at[-1]]))


def _plain_copy(s):
    copies = s["copies"].long()
    total, _, ps, _ = s["caches"][0][0].shape
    real = (copies[:, 0] >= 0) & (copies[:, 1] >= 0)
    written = torch.zeros(total + 1, device=copies.device).index_fill_(0, torch.where(real, copies[:, 1], total), 1.0)
    spare = written.argmin()                                     # a page that no copy writes: entries that are none copy it to itself
    source, target = torch.where(real, copies[:, 0], spare), torch.where(real, copies[:, 1], spare)
    row = torch.arange(ps, device=copies.device)[None, :] < copies[:, 2, None]
    for pair in s["caches"]:
        for x in pair:
            x[target] = torch.where(row[:, None, :, None], x[source], x[target])


def _plain_rows(s):
    ps, groups, size = s["page_size"], s["groups"], s["size"]
    table = s["table"].view(groups, size, -1)
    lens = s["lengths"].view(groups, size).long()
    some = lens > 0
    first = some.int().argmax(1)                                 # the first request that is not empty
    lead = table.gather(1, first[:, None, None].expand(-1, 1, table.shape[2]))
    j = torch.arange(table.shape[2], device=table.device)
    equal = ((table == lead) & (j < (lens // ps)[:, :, None])) | ~some[:, :, None]
    common = equal.all(1).int().cumprod(1).sum(1)
    s["shared"].copy_(torch.where(some.any(1), common * ps, 0))


def _plain_part(q, k, v, scale, hidden=None):
    """(maxima, sums, weighted sums) of q [.., columns, d] over k, v [.., keys, d]"""
    p = torch.matmul(q, k.transpose(-1, -2).contiguous()).mul_(scale)
    if hidden is not None:
        p.masked_fill_(hidden, -math.inf)
    most = p.amax(-1, keepdim=True)
    p = p.sub_(torch.where(most == -math.inf, 0.0, most)).exp_()
    return most, p.sum(-1, keepdim=True), torch.matmul(p, v)


def _plain_shared(s):
    (R, H, d), (_, KH, ps, _), scale = s["q"].shape, s["cache_k"].shape, s["scale"]
    G = H // KH
    q = s["q"].float().view(R, KH, G, d)
    most = torch.full((R, KH, G, 1), -math.inf, device=q.device)
    total, o = torch.zeros_like(most), torch.zeros_like(q)

    def whole(cache, pages):                                     # the rows of some pages: [key heads, rows, d]
        return cache[pages.long()].float().transpose(0, 1).reshape(KH, -1, d)
    for a, b, pages, _ in s["groups"]:
        if pages:
            k, v = (whole(s[c], s["table"][a, :pages]) for c in ("cache_k", "cache_v"))
            parts = _plain_part(q[a:b].transpose(0, 1).reshape(KH, -1, d), k, v, scale)
            most[a:b], total[a:b], o[a:b] = (x.view(KH, b - a, G, -1).transpose(0, 1) for x in parts)
    for a, b, pages, wide in s["groups"] + s["others"]:
        if pages == wide:
            continue
        step = max(1, (1 << 28) // (KH * (wide - pages) * ps * d))   # as many requests at a time as leave the copies below 1 GiB each
        for r in range(a, b, step):
            e = min(b, r + step)
            table, n = s["table"][r:e, pages:wide].long(), s["lengths"][r:e, None] - pages * ps
            k, v = (s[c][table].float().transpose(1, 2).reshape(e - r, KH, -1, d) for c in ("cache_k", "cache_v"))
            hidden = torch.arange(k.shape[2], device=q.device)[None] >= n
            m, t, x = _plain_part(q[r:e], k, v, scale, hidden[:, None, None, :])
            both = torch.maximum(most[r:e], m)
            safe = torch.where(both == -math.inf, 0.0, both)
            f, g = torch.exp(most[r:e] - safe), torch.exp(m - safe)
            total[r:e] = total[r:e] * f + t * g
            o[r:e] = o[r:e] * f + x * g
    empty = (s["lengths"] <= 0)[:, None, None, None]
    o = torch.where(empty, 0.0, o / torch.where(empty, 1.0, total))
    s["o"].copy_(o.view(R, H, d))


def _own_fork(s):
    s["binding"].attn_kv_fork(s["lengths"], s["source"], s["table"], s["free"], s["state"], page_size=s["page_size"], pages=s["pages"], rows=s["rows"],
                              table_out=s["table_out"], lengths_out=s["lengths_out"], copies=s["copies"], free_state_out=s["state_out"],
                              workspace=s["workspace"])


def _own_copy(s):
    s["binding"].attn_kv_copy(s["layers"], s["copies"])


def _own_rows(s):
    s["binding"].attn_kv_shared_rows(s["table"], s["lengths"], s["offsets"], page_size=s["page_size"], shared=s["shared"])


def _own_shared(s):
    s["binding"].attn_decode_shared(s["q"], s["cache"], s["table"], s["lengths"], s["offsets"], s["shared"], s["o"], scale=s["scale"],
                                    workspace=s["workspace"])


_PLAIN = {"fork": _plain_fork, "copy": _plain_copy, "rows": _plain_rows, "shared": _plain_shared}
_OWN = {"fork": _own_fork, "copy": _own_copy, "rows": _own_rows, "shared": _own_shared}
_OUT = {"fork": ("table_out", "lengths_out", "copies", "free", "state_out"), "copy": ("caches",), "rows": ("shared",), "shared": ("o",)}


def run(state):
    if own and "binding" not in state:
        _handles(state)
    (_OWN if own else _PLAIN)[state["op"]](state)
    return {name: state[name] for name in _OUT[state["op"]]}


def work(case):
    if case["op"] == "fork":
        old, new = _fork_entries(case)
        # tables in and out; lengths, sources and bounds in; lengths and copies out
        return {"bytes": 4.0 * (old + new) + 4.0 * case["groups"] * (case["old"] + case["new"] * (5 + int(case["cut"]))), "flops": float(old + new)}
    if case["op"] == "copy":
        rows = float(_copied_rows(case).sum())
        return {"bytes": 8.0 * rows * case["layers"] * case["heads"] * case["d"] + 12.0 * case["n"], "flops": float(case["n"])}
    if case["op"] == "rows":
        n = 4.0 * float(_rows_common(case)[1].sum() + case["groups"]) * case["size"]
        return {"bytes": n + 4.0 * case["groups"] * (case["size"] + 2), "flops": n / 4}
    prefix, tail = _shared_lengths(case)
    H, KH, d = case["H"], case["KH"], case["d"]
    rows = float(prefix.sum() + tail.sum())                      # of K and of V, each once
    seen = float(prefix.sum() * case["size"] + tail.sum())
    return {"bytes": 4.0 * rows * KH * d + 4.0 * tail.size * H * d + 4.0 * rows / case["page_size"], "flops": 4.0 * seen * H * d}


# ------------------------------------------------------------------------------------------- the definition, in 64 bits

def _exact_fork(s):
    """Request by request, as the definition reads, on the host."""
    ps = s["page_size"]
    lens, source, free = s["lengths"].tolist(), s["source"].tolist(), s["free"].tolist()
    first, available = s["state"].tolist()
    rows = s["rows"].tolist() if s["rows"] is not None else None
    table = s["table"].cpu().numpy()
    out = s["table_out"].cpu().numpy().copy()
    F, asked, used, taken, kept = len(free), 0, 0, set(), set()
    out_len, copies = [], []
    for r, parent in enumerate(source):
        n = lens[parent] if 0 <= parent < len(lens) else 0
        n = min(n, rows[r]) if rows is not None else n
        whole, rest = divmod(n, ps)
        copies.append((-1, -1, 0))
        if rest and whole == lens[parent] // ps and parent not in taken:
            taken.add(parent)
            whole += 1                                           # the part-filled page goes on as it is
        elif rest:
            asked += 1
            if asked > available:
                copies[r] = (int(table[parent, whole]), -1, rest)
                out_len.append(0)
                continue
            out[r, whole] = free[(first + used) % F]
            copies[r] = (int(table[parent, whole]), int(out[r, whole]), rest)
            used += 1
        if whole:
            out[r, :whole] = table[parent, :whole]
            kept.update(table[parent, :whole].tolist())
        out_len.append(n)
    held = set()
    for r, n in enumerate(lens):
        held.update(table[r, :-(-n // ps)].tolist())
    back = sorted(held - kept)
    for i, page in enumerate(back):
        free[(first + available + i) % F] = page

    def ints(x, like):
        return torch.tensor(x).to(like)
    return {"table_out": torch.from_numpy(out).to(s["table_out"]), "lengths_out": ints(out_len, s["lengths_out"]), "copies": ints(copies, s["copies"]),
            "free": ints(free, s["free"]), "state_out": ints([(first + used) % F, available - used + len(back)], s["state_out"])}


def _exact_copy(s):
    caches = [[x.double() for x in pair] for pair in s["caches"]]
    for source, target, rows in s["copies"].tolist():
        if source >= 0 and target >= 0:
            for pair in caches:
                for x in pair:
                    x[target, :, :rows] = x[source, :, :rows]
    return {"caches": caches}


def _exact_rows(s):
    table, lens = s["table"].cpu().numpy(), s["lengths"].cpu().numpy()
    out = []
    for g in range(s["groups"]):
        mine = [table[r, :lens[r] // s["page_size"]] for r in range(g * s["size"], (g + 1) * s["size"]) if lens[r] > 0]
        n = min((len(x) for x in mine), default=0)
        differ = np.zeros(n, dtype=bool)
        for x in mine:
            differ |= x[:n] != mine[0][:n]
        out.append((int(differ.argmax()) if differ.any() else n) * s["page_size"])
    return {"shared": torch.tensor(out).to(s["shared"])}


def _exact_shared(s):
    """Every request over all of its own table, shared or not."""
    (R, H, d), (_, KH, ps, _) = s["q"].shape, s["cache_k"].shape
    out = torch.zeros(R, H, d, dtype=torch.float64, device="cuda")
    for r, n in enumerate(s["lengths"].tolist()):
        if n == 0:
            continue
        pages = s["table"][r, :-(-n // ps)].long()
        for h in range(KH):
            k, v = (s[c][pages, h].double().reshape(-1, d)[:n] for c in ("cache_k", "cache_v"))
            q = s["q"][r, h * (H // KH):(h + 1) * (H // KH)].double()
            w = torch.softmax(torch.mm(q, k.t().contiguous()) * s["scale"], dim=1)
            out[r, h * (H // KH):(h + 1) * (H // KH)] = torch.mm(w, v)
    return {"o": out}


def exact(case, seed):
    s = _PREPARE[case["op"]](case, seed)
    return {"fork": _exact_fork, "copy": _exact_copy, "rows": _exact_rows, "shared": _exact_shared}[case["op"]](s)
