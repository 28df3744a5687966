"""Decoding over a paged key-value cache: page tables, preparation of Q, K and V, attention of one token, and a step of all three."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2601_16032_amd import binding

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
POISON = -0x70000000


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def smallest(dtype):
    """Half the distance of subnormal numbers: what rounding costs where a value is tiny."""
    return torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps / 2


def f64(t):
    return t.detach().cpu().double().numpy()


# ------------------------------------------------------------------------------------------- refusals, without a GPU

def refused(rc, want, text):
    assert rc == want and text in binding.attn_last_error(), (rc, binding.attn_last_error())


def test_pages_refusals():
    L = binding.lib()
    at = [0x100000 * (i + 1) for i in range(11)]
    base = dict(lengths=at[0], new=at[1], R=4, table=at[2], stride=8, wide=8, ps=16, free=at[3], ring=32, state=at[4], out=at[5],
                granted=at[6], offsets=at[7], state_out=at[8], slots=at[9], positions=at[10], tokens=100)

    def call(**kw):
        return L.attn_kv_pages(*dict(base, **kw).values(), None)
    bad, no = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
    for name in ("lengths", "new", "table", "free", "state", "out", "granted", "offsets", "state_out", "slots", "positions"):
        refused(call(**{name: None}), bad, "null")
        refused(call(**{name: base[name] + 2}), bad, "aligned")
    refused(call(slots=base["slots"] + 4), bad, "aligned")
    for name in ("R", "wide", "ring"):
        refused(call(**{name: 0}), bad, "positive")
    refused(call(tokens=-1), bad, "not negative")
    refused(call(tokens=2 ** 31 - 2 ** 20), bad, "below")
    refused(call(R=4097), no, "SAWATTN_MOST_REQUESTS")
    for ps in (0, 8, 24, 2 ** 21, -16):
        refused(call(ps=ps), no, "page size")
    refused(call(wide=2 ** 27, stride=2 ** 27), bad, "below 2^31")
    refused(call(R=4096, wide=2 ** 19, stride=2 ** 19, ps=16), bad, "below 2^31")
    refused(call(stride=7), bad, "table_stride")
    refused(call(out=base["lengths"]), bad, "overlaps an input")
    refused(call(state_out=base["state"] + 4), bad, "overlaps an input")
    refused(call(granted=base["out"] + 12), bad, "two outputs")
    refused(call(slots=base["table"] + 4 * 31 + 4 - 8), bad, "two outputs")


def cache_struct(**kw):
    a = dict(k=0x10000000, v=0x20000000, k_page=16 * 128 * 2, k_head=16 * 128, k_row=128, v_page=16 * 128 * 2, v_head=16 * 128, v_row=128,
             pages=10, page_size=16, heads=2, d=128, dtype=0)
    a.update(kw)
    return binding._CacheStruct(*a.values())


BAD_CACHES = [(dict(k=None), 1, "non-null"), (dict(v=0x20000008), 1, "aligned"), (dict(pages=0), 1, "positive"), (dict(heads=-1), 1, "positive"),
              (dict(d=96), 2, "head dimension"), (dict(page_size=24), 2, "page size"), (dict(page_size=8), 2, "page size"),
              (dict(dtype=2), 1, "dtype"), (dict(k_row=100), 1, "row strides"), (dict(v_page=-8), 1, "page strides"),
              (dict(v_head=4), 1, "head strides"), (dict(k_page=2 ** 60), 1, "page strides")]


def test_prepare_refusals():
    L = binding.lib()
    rows = (ctypes.c_int64 * 24)(*[x for i in range(6) for x in (0x1000000 * (i + 1), 4096, 512, 128)])
    where = ctypes.addressof(rows)
    cache = cache_struct()
    base = dict(rows=where, cache=ctypes.addressof(cache), slots=0x9000000, positions=0x9100000, qw=0x9200000, kw=0x9300000, eps=1e-6,
                f=0x9400000, rotated=128, inter=0, B=2, N=8, H=4, KH=2, d=128, dtype=0)

    def call(**kw):
        return L.attn_qkv_prepare(*dict(base, **kw).values(), None)
    bad, no = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
    for name in ("rows", "positions", "f"):
        refused(call(**{name: None}), bad, "non-null")
    for name in ("cache", "slots"):
        refused(call(**{name: None}), bad, "given together")
    for name in ("B", "N", "H", "KH", "d"):
        refused(call(**{name: 0}), bad, "positive")
    refused(call(d=96), no, "head dimension")
    refused(call(dtype=2), bad, "dtype")
    refused(call(B=2 ** 16, N=2 ** 10), bad, "B*N")
    refused(call(H=2 ** 16 - 1, KH=1), bad, "at most 2^16")
    for rotated in (-8, 4, 136):
        refused(call(rotated=rotated), bad, "rotated")
    for eps in (-1.0, math.nan, math.inf):
        refused(call(eps=eps), bad, "eps")
    for name in ("qw", "kw", "f"):
        refused(call(**{name: base[name] + 8}), bad, "16-byte")
    refused(call(positions=0x9100002), bad, "aligned")
    refused(call(slots=0x9000004), bad, "aligned")
    for i, value, text in ((0, 0, "non-null"), (4, 0, "non-null"), (8, 0, "non-null"), (12, 0, "non-null"), (16, 0, "given together"),
                           (20, 0, "given together"), (0, 0x1000008, "16-byte"), (9, 4097, "strides of rows"), (14, -512, "strides of rows"),
                           (7, 4, "strides of rows"), (13, 0, "at least d"), (15, 64, "at least d"), (22, 64, "at least d")):
        kept, rows[i] = rows[i], value
        refused(call(), bad, text)
        rows[i] = kept
    for change, code, text in BAD_CACHES + [(dict(heads=1), 1, "the cache's heads"), (dict(d=64), 1, "the cache's heads"),
                                            (dict(dtype=1), 1, "the cache's heads"), (dict(k_row=0), 1, "at least d"),
                                            (dict(v_page=0), 1, "at least d"), (dict(k_head=64), 1, "at least d")]:
        other = cache_struct(**change)
        refused(call(cache=ctypes.addressof(other)), code, text)


def test_decode_refusals():
    L = binding.lib()
    cache = cache_struct()
    n = ctypes.c_size_t(0)
    assert L.attn_decode_workspace_bytes(ctypes.addressof(cache), 3, 8, 10, ctypes.byref(n)) == 0 and n.value == 0      # short tables
    assert L.attn_decode_workspace_bytes(ctypes.addressof(cache), 3, 8, 100, ctypes.byref(n)) == 0 and n.value > 0
    base = dict(Q=0x1000000, qr=1024, qh=128, O=0x2000000, orow=1024, oh=128, odt=0, cache=ctypes.addressof(cache), table=0x3000000,
                stride=100, wide=100, lengths=0x4000000, R=3, H=8, scale=0.1, window=0, ws=0x5000000, bytes=n.value)

    def call(**kw):
        return L.attn_decode(*dict(base, **kw).values(), None)
    bad = binding.ERR_INVALID_ARG
    for name in ("Q", "O", "table", "lengths", "ws"):
        refused(call(**{name: None}), bad, "non-null")
        refused(call(**{name: base[name] + 2}), bad, "aligned")
    refused(call(cache=None), bad, "non-null")
    for name in ("R", "H", "wide"):
        refused(call(**{name: 0}), bad, "positive")
    refused(call(H=7), bad, "multiple of the cache's heads")
    refused(call(R=2 ** 20, H=8), bad, "R*H")
    refused(call(wide=2 ** 27, stride=2 ** 27), bad, "at most 2^30")
    refused(call(R=2 ** 18, wide=2 ** 16, stride=2 ** 16), bad, "2^31 - 2048")
    refused(call(odt=3), bad, "o_dtype")
    for scale in (math.nan, math.inf):
        refused(call(scale=scale), bad, "scale")
    refused(call(window=-1), bad, "window")
    refused(call(stride=99), bad, "table_stride")
    for name, value in (("qr", -8), ("qh", 100), ("orow", 1020), ("oh", -128)):
        refused(call(**{name: value}), bad, "strides of Q and O")
    refused(call(oh=64), bad, "at least d")
    refused(call(bytes=n.value - 1), bad, "smaller than")
    for name, value in (("O", 0x1000000 + 2 * 1024), ("ws", 0x10000000), ("O", 0x20000010), ("ws", 0x1000000), ("O", 0x3000000)):
        refused(call(**{name: value}), bad, "overlap")
    refused(call(O=0x5000000), bad, "must not overlap the workspace")
    for change, code, text in BAD_CACHES:
        other = cache_struct(**change)
        refused(call(cache=ctypes.addressof(other)), code, text)
        if "k" not in change and "v" not in change and not any(x in text for x in ("strides", "aligned")):
            refused(L.attn_decode_workspace_bytes(ctypes.addressof(other), 3, 8, 10, ctypes.byref(n)), code, text)
    refused(L.attn_decode_workspace_bytes(ctypes.addressof(cache), 3, 8, 10, None), bad, "non-null")
    refused(L.attn_decode_workspace_bytes(ctypes.addressof(cache), 3, 7, 10, ctypes.byref(n)), bad, "multiple")


def test_binding_refuses_host_tensors():
    x = torch.zeros(4, 1, 16, 64, dtype=torch.float16)
    with pytest.raises(ValueError, match="device tensor"):
        binding.KVCache(x, x)
    with pytest.raises(ValueError, match="device tensor"):
        binding.attn_qkv_prepare(x[0], x[0], x[0], positions=torch.zeros(1, dtype=torch.int32))


# ------------------------------------------------------------------------------------------- page tables

def pages_case(rng, R, ps, most, most_new, ends=0.1, idle=0.1, pool="enough", room=3, tokens=None):
    lengths = rng.integers(0, most + 1, R)
    new = rng.integers(1, most_new + 1, R)
    new[rng.random(R) < idle] = 0
    new[rng.random(R) < ends] = -1
    held = -(-lengths // ps)
    wide = int(max(1, held.max() + room))
    missing = int((-(-(lengths + np.maximum(new, 0)) // ps) - held).sum())
    available = {"enough": missing + 2, "exact": missing, "half": missing // 2, "none": 0}[pool]
    F = int(held.sum()) + available + 1
    ids = rng.permutation(F)
    first = int(rng.integers(0, F))
    ring = np.full(F, -5)
    ring[(first + np.arange(available)) % F] = ids[held.sum():held.sum() + available]
    table = np.full((R, wide), -7)
    at = 0
    for r in range(R):
        table[r, :held[r]] = ids[at:at + held[r]]
        at += held[r]
    total = int(np.maximum(new, 0).sum())
    return lengths, new, table, ring, [first, available], ps, total + 5 if tokens is None else tokens(total)


def run_pages(lengths, new, table, ring, state, ps, tokens, stride=0):
    def up(x, dtype=torch.int32):
        return torch.tensor(np.asarray(x)).to(dtype).cuda()
    R, wide = table.shape
    whole = torch.full((R, wide + stride), 99, dtype=torch.int32, device="cuda")
    whole[:, :wide] = up(table)
    ring_t, T = up(ring), {"dtype": torch.int32, "device": "cuda"}
    guarded = [torch.full((n + 2,), POISON, dtype=dt, device="cuda") for n, dt in (
        (R, torch.int32), (R, torch.int32), (R + 1, torch.int32), (2, torch.int32), (tokens, torch.int64), (tokens, torch.int32))]
    out = [g[:-2] for g in guarded]
    step = binding.attn_kv_pages(up(lengths), up(new), whole[:, :wide], ring_t, torch.tensor(state, **T), page_size=ps, lengths_out=out[0],
                                 granted=out[1], token_offsets=out[2], free_state_out=out[3], slots=out[4], positions=out[5])
    torch.cuda.synchronize()
    assert step.slots is out[4]
    assert all((g[-2:] == POISON).all() for g in guarded) and (whole[:, wide:] == 99).all()
    return [o.cpu().numpy() for o in out] + [whole[:, :wide].cpu().numpy(), ring_t.cpu().numpy()]


NAMES = ("lengths", "granted", "offsets", "state", "slots", "positions", "table", "ring")


def check_pages(*case, stride=0):
    got, want = run_pages(*case, stride=stride), po.kv_pages(*case)
    for name, g, w in zip(NAMES, got, want):
        assert np.array_equal(g, np.asarray(w, dtype=g.dtype).reshape(g.shape)), name


@pytest.mark.gpu
@pytest.mark.parametrize("R,ps,most,most_new", [(1, 16, 0, 1), (1, 16, 7, 1), (1, 16, 16, 5000), (2, 64, 100, 1), (63, 16, 40, 1), (64, 16, 9, 30),
                                                (65, 1024, 3000, 700), (257, 16, 600, 1), (1000, 32, 900, 40), (4096, 16, 64, 3)])
@pytest.mark.parametrize("pool", ["enough", "exact", "half", "none"])
def test_pages(R, ps, most, most_new, pool):
    rng = np.random.default_rng(R + most)
    check_pages(*pages_case(rng, R, ps, most, most_new, pool=pool), stride=0 if R % 2 else 3)


@pytest.mark.gpu
def test_pages_refuses_requests_not_calls():
    rng = np.random.default_rng(5)
    # table rows too short for some; tokens behind the batch's end; no tokens at all; everything ends; nothing happens
    check_pages(*pages_case(rng, 90, 16, 200, 100, room=1))
    check_pages(*pages_case(rng, 90, 16, 200, 100, tokens=lambda total: total // 2))
    check_pages(*pages_case(rng, 90, 16, 200, 100, tokens=lambda total: 0))
    check_pages(*pages_case(rng, 300, 16, 500, 1, ends=1.1))
    check_pages(*pages_case(rng, 300, 16, 500, 1, ends=0, idle=1.1))


@pytest.mark.gpu
def test_pages_whatever_the_numbers():
    """Lengths, counts and ring states that no program should pass stay inside the tables: the oracle's rules, clamped, hold."""
    big = 2 ** 31 - 1
    table, ring = np.arange(20).reshape(5, 4), np.arange(100, 130)
    lengths, new = np.array([-3, big, 10, big, 5]), np.array([4, 1, big, -9, 2])
    got = run_pages(lengths, new, table, ring, [3, 8], 16, 12)
    want = po.kv_pages(lengths, new, table, ring, [3, 8], 16, 12)
    want[2][:] = np.minimum(want[2], big)
    for name, g, w in zip(NAMES, got, want):
        assert np.array_equal(g, np.asarray(w, dtype=g.dtype).reshape(g.shape)), name
    for state in ([-1, 500], [30, 8], [big, big], [2, -4]):
        g = run_pages(np.array([0, 16, 40]), np.array([64, -1, 2]), table[:3], ring, state, 16, 70)
        want = po.kv_pages(np.array([0, 16, 40]), np.array([64, -1, 2]), table[:3], ring, [state[0] if 0 <= state[0] < 30 else 0, min(max(state[1], 0), 30)], 16, 70)
        want[3][1] = min(want[3][1], 30)
        for i in (0, 1, 2, 3, 5):      # (with more pages given back than the ring has room for, which page a slot is in is left open)
            assert np.array_equal(g[i], np.asarray(want[i], dtype=g[i].dtype)), (NAMES[i], state)


# ------------------------------------------------------------------------------------------- preparation of Q, K, V

def check_rows(got, exact, size, dtype):
    """Rounded once (half a step), and before that: 12 roundings of the sum of squares count half, root, quotient, two products, cosine and
    sine within 2^-21 (2 units in the last place, and the angle's own rounding), two products and a sum: below 2^-19 of |a| + |b|."""
    got = f64(got)
    bound = half_step(dtype) * np.abs(exact) * (1 + 2.0 ** -10) + 2.0 ** -19 * size + smallest(dtype)
    off = np.abs(got - exact)
    assert np.isfinite(got).all() and (off <= bound).all(), float((off / bound).max())


def frequencies(rot, base=10000.0):
    return torch.tensor([base ** (-2.0 * i / rot) for i in range(rot // 2)], dtype=torch.float64, device="cuda") if rot else None


def prepare_inputs(B, N, H, KH, d, dtype, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    qkv = torch.randn(B, N, H + 2 * KH, d, generator=g, device="cuda").to(DTYPES[dtype])
    weights = [1 + 0.2 * torch.randn(d, generator=g, device="cuda") for _ in range(2)]
    return qkv[:, :, :H], qkv[:, :, H:H + KH], qkv[:, :, H + KH:], weights


@pytest.mark.gpu
@pytest.mark.parametrize("d,rot", [(64, 64), (64, 16), (64, 8), (64, 0), (128, 128), (128, 64), (128, 40), (128, 0)])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("norm", ["both", "q", "none"])
def test_prepare_rows(d, rot, dtype, interleaved, norm):
    for B, N, H, KH in ((1, 1, 1, 1), (2, 3, 5, 5), (1, 70, 12, 3), (3, 1, 33, 11)):
        q, k, v, (wq, wk) = prepare_inputs(B, N, H, KH, d, dtype, seed=B * N * H + d + rot)
        wq, wk = (wq if norm != "none" else None), (wk if norm == "both" else None)
        rng = np.random.default_rng(N)
        pos = rng.integers(0, 2 ** 31 - 1, (B, N)).astype(np.int32)
        pos[0, 0] = 0
        f = frequencies(rot)
        qo, ko, vo = binding.attn_qkv_prepare(q, k, v, positions=torch.from_numpy(pos).cuda(), frequencies=f, interleaved=interleaved,
                                              q_weight=wq, k_weight=wk, eps=1e-5)
        for got, x, w in ((qo, q, wq), (ko, k, wk)):
            exact, size = po.rows(f64(x), None if w is None else f64(w), 1e-5, pos, None if f is None else f64(f), interleaved)
            check_rows(got, exact, size, DTYPES[dtype])
        assert torch.equal(vo, v)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,d", [("f16", 64), ("bf16", 128)])
@pytest.mark.parametrize("page_first", [False, True])
def test_prepare_fills_the_cache(dtype, d, page_first):
    """Rows go to their slots and nowhere else; padding and slots outside the cache are left out; the copies for attn_fwd are the same rows."""
    B, N, H, KH, ps, pages = 2, 21, 6, 3, 16, 5
    q, k, v, (wq, wk) = prepare_inputs(B, N, H, KH, d, dtype, seed=3)
    rng = np.random.default_rng(8)
    pos, slots = rng.integers(0, 5000, (B, N)), rng.permutation(pages * ps)[:B * N].reshape(B, N)
    pos[0, 4] = pos[1, 20] = -1
    slots[0, 7], slots[0, 8], slots[1, 0] = -1, pages * ps, 2 ** 62
    shape = (pages, ps, KH, d) if page_first else (pages, KH, ps, d)
    caches = [torch.full(shape, 7.0, dtype=DTYPES[dtype], device="cuda") for _ in range(2)]
    views = [c.transpose(1, 2) if page_first else c for c in caches]
    outs = [torch.full((B, n, N, d), 5.0, dtype=DTYPES[dtype], device="cuda").transpose(1, 2) for n in (H, KH, KH)]
    kw = dict(positions=torch.tensor(pos, dtype=torch.int32, device="cuda"), frequencies=frequencies(d), q_weight=wq, k_weight=wk)
    plain = binding.attn_qkv_prepare(q, k, v, **kw)
    binding.attn_qkv_prepare(q, k, v, q_out=outs[0], k_out=outs[1], v_out=outs[2], cache=binding.KVCache(*views),
                             slots=torch.tensor(slots, device="cuda"), **kw)
    torch.cuda.synchronize()
    padding = torch.tensor(pos < 0, device="cuda")
    for got, want in zip(outs, plain):
        assert torch.equal(got[~padding], want[~padding]) and (got[padding] == 5.0).all()
    want = [torch.full((pages * ps, KH, d), 7.0, dtype=DTYPES[dtype], device="cuda") for _ in range(2)]
    for b in range(B):
        for n in range(N):
            if pos[b, n] >= 0 and 0 <= slots[b, n] < pages * ps:
                want[0][slots[b, n]], want[1][slots[b, n]] = plain[1][b, n], v[b, n]
    for view, w in zip(views, want):
        assert torch.equal(view.transpose(1, 2).reshape(pages * ps, KH, d), w)


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
def test_prepare_in_place_and_by_rows(interleaved):
    """In place, [N, heads, d] and rows far apart give the same bits; a head that is no number stays alone."""
    q, k, v, (wq, wk) = prepare_inputs(1, 50, 7, 7, 128, "f16", seed=12)
    q[0, 9, 3, 100] = float("nan")
    q[0, 9, 4, 5] = float("inf")
    kw = dict(positions=torch.arange(50, dtype=torch.int32, device="cuda"), frequencies=frequencies(64), interleaved=interleaved, q_weight=wq,
              k_weight=wk)
    want = binding.attn_qkv_prepare(q, k, v, **kw)
    assert want[0][0, 9, 3].isnan().all()
    others = torch.ones(50, 7, dtype=torch.bool, device="cuda")
    others[9, 3] = others[9, 4] = False
    assert want[0][0][others].isfinite().all()
    rows = binding.attn_qkv_prepare(q[0], k[0], v[0], **kw)
    far = [torch.zeros(50, 9, 256, dtype=torch.float16, device="cuda")[:, 1:8, 64:192] for _ in range(3)]
    binding.attn_qkv_prepare(q[0], k[0], v[0], q_out=far[0], k_out=far[1], v_out=far[2], **kw)
    binding.attn_qkv_prepare(q, k, v, q_out=q, k_out=k, v_out=v, **kw)
    for w, r, f, inplace in zip(want, rows, far, (q, k, v)):
        bits = w.contiguous().view(torch.int16)
        assert torch.equal(bits[0], r.view(torch.int16)) and torch.equal(bits[0], f.contiguous().view(torch.int16))
        assert torch.equal(bits, inplace.contiguous().view(torch.int16))


@pytest.mark.gpu
@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("d,H,KH", [(128, 7, 2), (64, 13, 5)])
def test_prepare_several_trips(d, H, KH, interleaved):
    """Enough tokens for a wavefront to take a token's rows in several trips, the last not full; in place, with padding among them, into a cache."""
    N, ps = 5000, 32
    q, k, v, (wq, wk) = prepare_inputs(1, N, H, KH, d, "bf16", seed=6)
    pos = torch.arange(N, dtype=torch.int32, device="cuda")
    pos[[3, 77, 4999]] = -1
    slots = torch.randperm((N // ps + 2) * ps, generator=torch.Generator().manual_seed(5))[:N].cuda()
    kw = dict(positions=pos, frequencies=frequencies(d // 2), interleaved=interleaved, q_weight=wq, k_weight=wk)
    pages = [torch.zeros(N // ps + 2, KH, ps, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    outs = [torch.zeros_like(x, memory_format=torch.contiguous_format) for x in (q, k, v)]
    binding.attn_qkv_prepare(q, k, v, q_out=outs[0], k_out=outs[1], v_out=outs[2], cache=binding.KVCache(*pages), slots=slots, **kw)
    real = (pos >= 0).cpu().numpy()
    for got, x, w in ((outs[0], q, wq), (outs[1], k, wk)):
        exact, size = po.rows(f64(x), f64(w), 1e-6, pos.cpu().numpy(), f64(kw["frequencies"]), interleaved)
        check_rows(got[:, real], exact[:, real], size[:, real], torch.bfloat16)
        assert (got[:, ~real] == 0).all()
    for page, out in zip(pages, outs[1:]):
        assert torch.equal(page.transpose(1, 2).reshape(-1, KH, d)[slots], out[0])
    untouched = [x[:, ~real].clone() for x in (q, k, v)]
    binding.attn_qkv_prepare(q, k, v, q_out=q, k_out=k, v_out=v, **kw)
    for x, out, kept in zip((q, k, v), outs, untouched):
        assert torch.equal(x[:, real], out[:, real]) and torch.equal(x[:, ~real], kept)


@pytest.mark.gpu
def test_prepare_many_tokens():
    """More tokens than one round of wavefronts, and offsets that pass 32 bits (the last row at 2^32 bytes and more)."""
    B, N, H, KH, d = 2, 3001, 6, 2, 64
    q, k, v, (wq, wk) = prepare_inputs(B, N, H, KH, d, "bf16", seed=4)
    pos = torch.arange(B * N, dtype=torch.int32, device="cuda").reshape(B, N)
    kw = dict(positions=pos, frequencies=frequencies(d), q_weight=wq, k_weight=wk, eps=0.0)
    qo, ko, _ = binding.attn_qkv_prepare(q, k, v, **kw)
    for got, x, w in ((qo, q, wq), (ko, k, wk)):
        exact, size = po.rows(f64(x), f64(w), 0.0, pos.cpu().numpy(), f64(kw["frequencies"]), False)
        check_rows(got, exact, size, torch.bfloat16)
    row = ((1 << 31) // N // 64 + 10) * 64
    assert (N - 1) * row * 2 > 2 ** 32
    out = torch.zeros(N * row, dtype=torch.bfloat16, device="cuda").as_strided((N, H, d), (row, d, 1))
    binding.attn_qkv_prepare(q[0], k[0], v[0], q_out=out, positions=pos[0], frequencies=kw["frequencies"], q_weight=wq, k_weight=wk, eps=0.0,
                             k_out=torch.empty_like(ko[0]), v_out=torch.empty_like(ko[0]))
    assert torch.equal(out, qo[0])


# ------------------------------------------------------------------------------------------- attention of one token

def fill_cache(lengths, KH, d, ps, dtype, seed, extra=2, page_first=False, garbage=float("nan")):
    """Keys and values of requests in pages of any order; whatever no request holds is `garbage`, table entries behind the last page too."""
    rng = np.random.default_rng(seed)
    g = torch.Generator("cuda").manual_seed(seed)
    count = [-(-max(n, 0) // ps) for n in lengths]
    pages = sum(count) + extra
    shape = (pages, ps, KH, d) if page_first else (pages, KH, ps, d)
    caches = [torch.full(shape, garbage, dtype=DTYPES[dtype], device="cuda") for _ in range(2)]
    views = [c.transpose(1, 2) if page_first else c for c in caches]
    table = np.full((len(lengths), max(max(count), 1)), POISON)
    ids = rng.permutation(pages)
    keys, at = ([], []), 0
    for r, n in enumerate(lengths):
        table[r, :count[r]] = ids[at:at + count[r]]
        at += count[r]
        for view, kept in zip(views, keys):
            x = torch.randn(max(n, 0), KH, d, generator=g, device="cuda").to(DTYPES[dtype])
            for j in range(count[r]):
                part = x[j * ps:(j + 1) * ps]
                view[int(table[r, j]), :, :part.shape[0]] = part.transpose(0, 1)
            kept.append(x)
    return binding.KVCache(*views), torch.tensor(table, dtype=torch.int32, device="cuda"), keys


def check_decode(got, q, keys, scale, lengths, window=0, skip=()):
    """|error| <= half a step of the output + (error of probabilities) * sum p |v|.  A score is a 32-bit sum of exact products, each addition
    off by up to 2^-23 of the sum of |q k|; twice that (the score's and the reference's, which is a score too) is the relative error of a
    probability, plus exp2 and its operand (2^-19 at scores up to 16), plus one addition of 2^-23 per tile of 32 and for the joining."""
    q, dtype = f64(q), got.dtype
    keys = [[f64(x) for x in side] for side in keys]
    exact, size, score = po.decode(q, *keys, scale, lengths, window)
    got = f64(got)
    n = max(max(lengths), 1)
    relative = 2 * (q.shape[2] + 4) * 2.0 ** -23 * score * abs(scale) + 2.0 ** -19 + (n / 32 + 64) * 2.0 ** -23
    bound = half_step(dtype) * np.abs(exact) * (1 + 2.0 ** -9) + (relative[..., None] * 2 + 2.0 ** -24) * size + smallest(dtype)
    rows = [r for r in range(len(lengths)) if r not in skip]
    off = np.abs(got - exact)[rows]
    assert np.isfinite(got[rows]).all() and (off <= bound[rows]).all(), float((off / bound[rows]).max())


def queries(R, H, d, dtype, seed):
    return torch.randn(R, H, d, generator=torch.Generator("cuda").manual_seed(seed), device="cuda").to(DTYPES[dtype])


LENGTHS = [0, 1, 7, 8, 9, 31, 32, 33, 63, 64, 65, 127, 129, 255, 257, 1000, 0, 1023, 2049]


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("G,KH", [(1, 1), (1, 5), (3, 2), (4, 2), (8, 1), (16, 1), (17, 1), (40, 2)])
def test_decode(d, dtype, G, KH):
    ps = {1: 16, 3: 16, 4: 32, 8: 64, 16: 1024, 17: 16, 40: 128}[G]
    cache, table, keys = fill_cache(LENGTHS, KH, d, ps, dtype, seed=G * d, page_first=G == 4)
    q = queries(len(LENGTHS), G * KH, d, dtype, seed=1)
    lengths = torch.tensor(LENGTHS, dtype=torch.int32, device="cuda")
    got = binding.attn_decode(q, cache, table, lengths, scale=d ** -0.5)
    check_decode(got, q, keys, d ** -0.5, LENGTHS)
    assert (got[0] == 0).all() and (got[16] == 0).all()
    # the same bits whatever the table's rows and the strides of Q and O are
    wide_table = torch.full((len(LENGTHS), table.shape[1] + 3), POISON, dtype=torch.int32, device="cuda")
    wide_table[:, :table.shape[1]] = table
    qs = torch.full((G * KH, len(LENGTHS), d + 8), float("nan"), dtype=q.dtype, device="cuda")[:, :, :d].transpose(0, 1)
    qs.copy_(q)
    os_ = torch.full((len(LENGTHS), G * KH + 1, d), 3.0, dtype=q.dtype, device="cuda")
    binding.attn_decode(qs, cache, wide_table[:, :table.shape[1]], lengths, os_[:, :-1], scale=d ** -0.5)
    assert torch.equal(os_[:, :-1], got) and (os_[:, -1] == 3.0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [("f16", "f32"), ("bf16", "f32"), ("bf16", "f16"), ("f16", "bf16")])
@pytest.mark.parametrize("scale", [0.0, -0.11, 1.0])
def test_decode_outputs_and_scales(dtype, out, scale):
    lengths = [5, 0, 700, 64]
    cache, table, keys = fill_cache(lengths, 2, 64, 16, dtype, seed=2)
    q = queries(4, 6, 64, dtype, seed=3)
    got = binding.attn_decode(q, cache, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), scale=scale, o_dtype=DTYPES[out])
    assert got.dtype == DTYPES[out]
    check_decode(got, q, keys, scale, lengths)


@pytest.mark.gpu
@pytest.mark.parametrize("window", [1, 8, 31, 32, 100, 1000, 5000])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "f16")])
def test_decode_window(window, d, dtype):
    """Rows in front of the window take no part, whatever their pages are: their table entries are poisoned too."""
    cache, table, keys = fill_cache(LENGTHS, 2, d, 16, dtype, seed=window)
    for r, n in enumerate(LENGTHS):
        table[r, :max(0, n - window) // 16] = POISON
    q = queries(len(LENGTHS), 4, d, dtype, seed=1)
    got = binding.attn_decode(q, cache, table, torch.tensor(LENGTHS, dtype=torch.int32, device="cuda"), scale=d ** -0.5, window=window)
    check_decode(got, q, keys, d ** -0.5, LENGTHS, window)


@pytest.mark.gpu
@pytest.mark.parametrize("lengths,KH,G,d", [([200001], 1, 2, 128), ([70000, 3, 0, 33], 2, 1, 64), ([1] * 700, 4, 2, 128), ([97] * 300, 8, 1, 64),
                                            (list(range(0, 2100, 7)), 1, 4, 64), ([40000] + [2] * 200, 2, 3, 128),
                                            ([3000, 9001, 0, 77], 2, 35, 64)])
def test_decode_lengths(lengths, KH, G, d):
    """One long request, many short ones, both: units spread over many workgroups, and many units to a workgroup."""
    cache, table, keys = fill_cache(lengths, KH, d, 64, "bf16", seed=9)
    q = queries(len(lengths), KH * G, d, "bf16", seed=1)
    got = binding.attn_decode(q, cache, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), scale=d ** -0.5, o_dtype=torch.float32)
    check_decode(got, q, keys, d ** -0.5, lengths)
    again = binding.attn_decode(q, cache, table, torch.tensor(lengths, dtype=torch.int32, device="cuda"), scale=d ** -0.5, o_dtype=torch.float32)
    assert torch.equal(got, again)


@pytest.mark.gpu
@pytest.mark.parametrize("most", [1, 16, 32, 47, 64, 100, 128, 200, 256, 300, 512])
@pytest.mark.parametrize("R,KH,G", [(5, 2, 3), (150, 8, 1), (9, 1, 33)])
def test_decode_short_tables(most, R, KH, G):
    """Tables of few rows: one, two, four and eight wavefronts to a unit, with few units and with more than a thousand; what lies behind
    the lengths, and in front of a window, is NaN."""
    lengths = [(7 * i) % (most + 1) for i in range(R)]
    lengths[0] = most
    for d, dtype in ((64, "f16"), (128, "bf16")):
        cache, table, keys = fill_cache(lengths, KH, d, 16, dtype, seed=most)
        q, lens = queries(R, KH * G, d, dtype, seed=2), torch.tensor(lengths, dtype=torch.int32, device="cuda")
        assert binding.attn_decode_workspace_bytes(R, KH * G, cache, table.shape[1]) == 0
        check_decode(binding.attn_decode(q, cache, table, lens, scale=d ** -0.5), q, keys, d ** -0.5, lengths)
        window = most // 2 + 1
        check_decode(binding.attn_decode(q, cache, table, lens, scale=d ** -0.5, window=window), q, keys, d ** -0.5, lengths, window)


@pytest.mark.gpu
def test_binding_refusals():
    """What the calls refuse before they reach the library: types, shapes, sizes."""
    cache, table, _ = fill_cache([20, 40], 2, 64, 16, "f16", seed=1)
    q, lens = queries(2, 4, 64, "f16", seed=1), torch.tensor([20, 40], dtype=torch.int32, device="cuda")
    pos = torch.zeros(2, dtype=torch.int32, device="cuda")
    ok = dict(scale=0.1)
    for args, kw in (((q.float(), cache, table, lens), ok), ((q[0], cache, table, lens), ok), ((q[:, :, :32], cache, table, lens), ok),
                     ((q.cpu(), cache, table, lens), ok), ((q, cache, table.long(), lens), ok), ((q, cache, table[:1], lens), ok),
                     ((q, cache, table.t().contiguous().t(), lens), ok), ((q, cache, table, lens.long()), ok), ((q, cache, table, lens[:1]), ok),
                     ((q, cache, table, lens.cpu()), ok), ((q, cache, table, lens, q.double()), ok), ((q, cache, table, lens, q[:1]), ok),
                     ((q, cache, table, lens), dict(scale=0.1, workspace=torch.zeros(9)))):
        with pytest.raises(ValueError):
            binding.attn_decode(*args, **kw)
    with pytest.raises(binding.SawattnError, match="multiple"):
        binding.attn_decode(q[:, :3], cache, table, lens, scale=0.1)
    with pytest.raises(binding.SawattnError, match="scale"):
        binding.attn_decode(q, cache, table, lens, scale=math.nan)
    with pytest.raises(binding.SawattnError, match="smaller"):
        long = torch.zeros(2, 600, dtype=torch.int32, device="cuda")
        binding.attn_decode(q, cache, long, lens, scale=0.1, workspace=torch.zeros(64, device="cuda"))
    for k, v in ((cache.k, cache.v[:, :1]), (cache.k.float(), cache.v.float()), (cache.k, cache.v.bfloat16()), (cache.k[0], cache.v[0]),
                 (cache.k.transpose(2, 3), cache.v.transpose(2, 3)), (cache.k, cache.v.cpu())):
        with pytest.raises(ValueError):
            binding.KVCache(k, v)
    k, slots, f, w = q[:, :2], torch.zeros(2, dtype=torch.int64, device="cuda"), frequencies(64), torch.ones(64, device="cuda")
    good = dict(positions=pos, frequencies=f, cache=cache, slots=slots, q_weight=w)
    binding.attn_qkv_prepare(q, k, k, **{**good, "slots": slots - 1})
    for change in (dict(positions=pos.long()), dict(positions=pos[:1]), dict(slots=None), dict(slots=pos), dict(q_weight=w.half()), dict(q_weight=w[:8]),
                   dict(frequencies=f.float()), dict(k_out=k), dict(k_out=k, v_out=k.float()), dict(q_out=q[:, :2]), dict(positions=pos.cpu())):
        with pytest.raises(ValueError):
            binding.attn_qkv_prepare(q, k, k, **{**good, **change})
    for args in ((q, k.float(), k), (q, k, k[:1]), (q, k[:, :, :32], k), (q.float(), k, k), (q, k.cpu(), k), (q[0], k, k)):
        with pytest.raises(ValueError):
            binding.attn_qkv_prepare(*args, **good)
    with pytest.raises(binding.SawattnError, match="rotated"):
        binding.attn_qkv_prepare(q, k, k, **{**good, "frequencies": f[:3]})
    ring, state = torch.arange(8, dtype=torch.int32, device="cuda"), torch.tensor([0, 8], dtype=torch.int32, device="cuda")
    call = lambda **kw: binding.attn_kv_pages(*[kw.pop(n, x) for n, x in (("lengths", lens), ("new", pos), ("table", table), ("ring", ring), ("state", state))],
                                              **{"page_size": 16, "tokens": 4, **kw})
    call()
    for change in (dict(lengths=lens.long()), dict(new=pos[:1]), dict(table=table.long()), dict(ring=ring.float()), dict(state=ring), dict(tokens=None),
                   dict(slots=slots), dict(slots=pos, tokens=2), dict(positions=pos), dict(granted=pos[:1]), dict(free_state_out=ring), dict(new=pos.cpu()),
                   dict(token_offsets=pos), dict(lengths=lens.cpu())):
        with pytest.raises(ValueError):
            call(**change)
    with pytest.raises(binding.SawattnError, match="overlap"):
        call(lengths_out=lens)


@pytest.mark.gpu
def test_decode_peaks_and_tiny_weights():
    """One row that outweighs a hundred thousand others, first, last and in the middle; and others that together outweigh it."""
    n, d = 100000, 64
    cache, table, keys = fill_cache([n] * 4, 1, d, 256, "f16", seed=5)
    q = queries(4, 1, d, "f16", seed=6)
    for r, at in enumerate((0, n - 1, n // 2)):
        x = q[r, 0].float()
        k = (x * (14.0 / 0.125 / (x @ x))).half()      # a score of 14
        keys[0][r][at, 0] = k
        cache.k[int(table[r, at // 256]), 0, at % 256] = k
    lengths = torch.full((4,), n, dtype=torch.int32, device="cuda")
    got = binding.attn_decode(q, cache, table, lengths, scale=0.125, o_dtype=torch.float32)
    check_decode(got, q, keys, 0.125, [n] * 4)


@pytest.mark.gpu
def test_decode_whatever_the_tables_hold():
    """Lengths outside the tables count as their ends; a page outside the cache among the visible ones makes its request NaN, and no other."""
    given = [-5, 2 ** 31 - 1, 40, 100, 64]
    real = [0, 128, 40, 100, 64]
    cache, table, keys = fill_cache(real, 2, 64, 16, "f16", seed=7)
    assert table.shape[1] == 8
    table[3, 5], table[4, 3] = cache.pages, -1
    q = queries(5, 4, 64, "f16", seed=6)
    lengths = torch.tensor(given, dtype=torch.int32, device="cuda")
    got = binding.attn_decode(q, cache, table, lengths, scale=0.125)
    check_decode(got, q, keys, 0.125, real, skip=(3, 4))
    assert got[3].isnan().all() and got[4].isnan().all()
    # outside the window the same entries do not matter
    got = binding.attn_decode(q, cache, table, lengths, scale=0.125, window=4)
    check_decode(got, q, keys, 0.125, real, 4, skip=(4,))
    assert got[4].isnan().all()


@pytest.mark.gpu
def test_decode_long_tables():
    """Tables long enough for units in parts: nothing in them at all, a page outside the cache, lengths outside the table."""
    for lengths in ([0] * 9, [0, 9000, 0]):
        cache, table, keys = fill_cache(lengths, 2, 64, 16, "bf16", seed=3)
        table = torch.cat([table, torch.full((len(lengths), 700 - table.shape[1]), POISON, dtype=torch.int32, device="cuda")], 1)
        q, o = queries(len(lengths), 6, 64, "bf16", seed=1), torch.full((len(lengths), 6, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
        binding.attn_decode(q, cache, table, torch.tensor(lengths, dtype=torch.int32, device="cuda") - 4 * (torch.tensor(lengths, device="cuda") == 0).int(), o,
                            scale=0.125)
        check_decode(o, q, keys, 0.125, lengths)
    real = [9008, 9008, 5, 9008]
    cache, table, keys = fill_cache(real, 2, 64, 16, "f16", seed=4)
    table[1, 77], table[3, 562] = 2 ** 31 - 1, cache.pages
    given = torch.tensor([2 ** 31 - 1, 9008, 5, 9008], dtype=torch.int32, device="cuda")
    q = queries(4, 6, 64, "f16", seed=1)
    got = binding.attn_decode(q, cache, table, given, scale=0.125)
    check_decode(got, q, keys, 0.125, real, skip=(1, 3))
    assert got[1].isnan().all() and got[3].isnan().all()
    got = binding.attn_decode(q, cache, table, given, scale=0.125, window=3000)
    check_decode(got, q, keys, 0.125, real, 3000, skip=(3,))
    assert got[3].isnan().all()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("length", [300, 6000])
def test_decode_keeps_what_is_no_number_to_itself(d, length):
    """NaN among the visible rows reaches the heads that see it and no others."""
    lengths = [length] * 3
    cache, table, keys = fill_cache(lengths, 2, d, 16, "bf16", seed=8)
    cache.k[int(table[1, 3]), 0, 5, 11] = float("nan")      # request 1, key head 0
    cache.v[int(table[2, 18]), 1, 2, 7] = float("nan")      # request 2, key head 1, element 7
    q = queries(3, 4, d, "bf16", seed=6)
    lens = torch.tensor(lengths, dtype=torch.int32, device="cuda")
    got = binding.attn_decode(q, cache, table, lens, scale=d ** -0.5)
    assert got[1, :2].isnan().all() and got[2, 2:, 7].isnan().all()
    ok = got.clone()
    ok[1, :2], ok[2, 2:, 7] = 0, 0
    exact, _, _ = po.decode(f64(q), *[[f64(x) for x in side] for side in keys], d ** -0.5, lengths)
    exact[1, :2], exact[2, 2:, 7] = 0, 0
    assert np.abs(f64(ok) - exact).max() <= 2.0 ** -8 * np.abs(exact).max()


@pytest.mark.gpu
def test_decode_far_into_a_large_cache():
    """Pages whose elements lie behind the 2^31st and whose bytes lie behind the 2^32nd."""
    pages, KH, ps, d = 2 ** 31 // (16 * 128) + 40, 1, 16, 128
    k = torch.zeros(pages, KH, ps, d, dtype=torch.float16, device="cuda")
    v = torch.zeros_like(k)
    cache = binding.KVCache(k, v)
    lengths = [500, 130]
    small, table, keys = fill_cache(lengths, KH, d, ps, "f16", seed=3, garbage=0.0)
    k[-small.pages:], v[-small.pages:] = small.k, small.v
    far = torch.where(table >= 0, table + (pages - small.pages), table)
    q = queries(2, 4, d, "f16", seed=6)
    got = binding.attn_decode(q, cache, far, torch.tensor(lengths, dtype=torch.int32, device="cuda"), scale=d ** -0.5)
    check_decode(got, q, keys, d ** -0.5, lengths)
    # and written there
    binding.attn_qkv_prepare(q[:, :1], small.k[:2, 0, :1], small.v[:2, 0, :1], positions=torch.zeros(2, dtype=torch.int32, device="cuda"),
                             cache=cache, slots=torch.tensor([pages * 16 - 1, pages * 16 - 18], device="cuda"))
    assert torch.equal(v[-1, 0, 15], small.v[0, 0, 0]) and torch.equal(v[-2, 0, 14], small.v[1, 0, 0])


# ------------------------------------------------------------------------------------------- together

class Server:
    """A few requests of one layer, stepped as a program would: tables, preparation, attention; and the same on the host in 64 bits."""

    def __init__(self, R=6, H=6, KH=2, d=64, ps=16, wide=12, dtype="bf16", seed=1):
        self.R, self.H, self.KH, self.d, self.ps, self.dtype = R, H, KH, d, ps, dtype
        i32 = {"dtype": torch.int32, "device": "cuda"}
        pages = R * wide
        self.cache = binding.KVCache(*[torch.full((pages, KH, ps, d), float("nan"), dtype=DTYPES[dtype], device="cuda") for _ in range(2)])
        self.table = torch.full((R, wide), POISON, **i32)
        self.ring = torch.randperm(pages, generator=torch.Generator().manual_seed(seed)).int().cuda()
        self.state = torch.tensor([5, pages], **i32)
        self.lengths = torch.zeros(R, **i32)
        self.new = torch.zeros(R, **i32)
        self.f = frequencies(d)
        self.weights = [torch.linspace(0.5, 1.5, d, device="cuda"), torch.linspace(1.2, 0.7, d, device="cuda")]
        self.keys = [[np.zeros((0, KH, d)) for _ in range(R)] for _ in range(2)]
        self.workspace = torch.empty(binding.attn_decode_workspace_bytes(R, H, self.cache, wide), dtype=torch.uint8, device="cuda")

    def step(self, qkv, tokens):
        """All three operators; the last token of every request attends."""
        got = binding.attn_kv_pages(self.lengths, self.new, self.table, self.ring, self.state, page_size=self.ps, tokens=tokens)
        q, k, v = qkv[:, :self.H], qkv[:, self.H:self.H + self.KH], qkv[:, self.H + self.KH:]
        q, _, _ = binding.attn_qkv_prepare(q, k, v, positions=got.positions, frequencies=self.f, q_weight=self.weights[0],
                                           k_weight=self.weights[1], cache=self.cache, slots=got.slots,
                                           q_out=torch.zeros_like(q, memory_format=torch.contiguous_format))
        last = q[(got.token_offsets[1:].long() - 1).clamp(min=0)]
        o = binding.attn_decode(last, self.cache, self.table, got.lengths, scale=self.d ** -0.5, workspace=self.workspace)
        self.lengths.copy_(got.lengths)
        self.state.copy_(got.free_state)
        return o, last

    def host(self, qkv, new):
        """The same rows appended on the host, rounded to the cache's type."""
        at, kept = 0, f64(qkv)
        for r, n in enumerate(new):
            if n < 0:
                for side in self.keys:
                    side[r] = np.zeros((0, self.KH, self.d))
            if n > 0:
                start = len(self.keys[0][r])
                k, _ = po.rows(kept[at:at + n, self.H:self.H + self.KH], f64(self.weights[1]), 1e-6, np.arange(start, start + n), f64(self.f), False)
                self.keys[0][r] = np.concatenate([self.keys[0][r], f64(torch.tensor(k).to(DTYPES[self.dtype]))])
                self.keys[1][r] = np.concatenate([self.keys[1][r], kept[at:at + n, self.H + self.KH:]])
                at += n
        return [len(x) for x in self.keys[0]]

    def check(self, o, last, lengths):
        q, got = f64(last), f64(o)
        exact, size, score = po.decode(q, *self.keys, self.d ** -0.5, lengths)
        # as in check_decode, and keys that are rounded the other way here and there: half a step of bfloat16 on every product
        relative = 2 * score * self.d ** -0.5 * (2 * half_step(torch.bfloat16)) + 2.0 ** -18
        bound = half_step(o.dtype) * np.abs(exact) * 1.01 + relative[..., None] * size + smallest(o.dtype)
        assert np.isfinite(got).all() and (np.abs(got - exact) <= bound).all()


PLAN = [[20, 1, 0, 33, 8, 7], [1, 1, 5, 1, 1, 1], [1, 1, 1, -1, 1, 1], [1, 0, 1, 40, 1, 1], [1, 1, 1, 1, -1, 1], [1, 1, 1, 1, 9, 1]]


@pytest.mark.gpu
def test_steps_of_a_server():
    s = Server()
    for i, new in enumerate(PLAN):
        s.new.copy_(torch.tensor(new, dtype=torch.int32))
        tokens = sum(max(n, 0) for n in new) + 2
        qkv = queries(tokens, s.H + 2 * s.KH, s.d, s.dtype, seed=100 + i)
        o, last = s.step(qkv, tokens)
        torch.cuda.synchronize()
        lengths = s.host(qkv, new)
        assert s.lengths.tolist() == lengths
        s.check(o, last, lengths)
    first, available = s.state.tolist()
    held = [int(p) for r in range(s.R) for p in s.table[r, :-(-lengths[r] // s.ps)]]
    free = [int(s.ring[(first + j) % s.ring.numel()]) for j in range(available)]
    assert sorted(held + free) == list(range(s.ring.numel()))      # no page lost, none twice


@pytest.mark.gpu
def test_steps_captured():
    """A step captured once and replayed while the requests grow, with eager work in between, gives the eager results bit by bit."""
    a, b = Server(), Server()
    plan = [[12, 3, 5, 9, 1, 8]] + [[1] * 6] * 3
    n = 6 * 16
    qkv = torch.zeros(n, a.H + 2 * a.KH, a.d, dtype=torch.bfloat16, device="cuda")
    a.step(qkv, n)      # loads everything, adds nothing
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        o, _ = a.step(qkv, n)
    for i, new in enumerate(plan):
        for s in (a, b):
            s.new.copy_(torch.tensor(new, dtype=torch.int32))
        qkv.copy_(queries(n, a.H + 2 * a.KH, a.d, "bf16", seed=i))
        graph.replay()
        torch.cuda.synchronize()
        want, last = b.step(qkv, n)
        torch.cuda.synchronize()
        assert torch.equal(o, want) and a.lengths.tolist() == b.lengths.tolist(), i
        lengths = b.host(qkv, new)
        b.check(want, last, lengths)


@pytest.mark.gpu
def test_streams_of_their_own():
    """Two steps at once on two streams, each with its own workspace, and the stream argument."""
    servers, streams, plain = [Server(seed=1), Server(seed=2)], [torch.cuda.Stream(), torch.cuda.Stream()], [Server(seed=1), Server(seed=2)]
    inputs = [queries(40, 10, 64, "bf16", seed=i) for i in range(2)]
    for s in servers + plain:
        s.new.copy_(torch.tensor([12, 3, 0, 9, 1, 8], dtype=torch.int32))
    want = [s.step(x, 40)[0] for s, x in zip(plain, inputs)]
    torch.cuda.synchronize()
    got = []
    for _ in range(2):
        for s, stream, x in zip(servers, streams, inputs):
            with torch.cuda.stream(stream):
                s.lengths.zero_()
                s.state.copy_(torch.tensor([5, 72], dtype=torch.int32))
                got.append(s.step(x, 40)[0])
    torch.cuda.synchronize()
    assert torch.equal(got[2], want[0]) and torch.equal(got[3], want[1])
    s = plain[0]
    q = queries(6, 6, 64, "bf16", seed=9)
    eager = binding.attn_decode(q, s.cache, s.table, s.lengths, scale=0.1)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    o = torch.zeros_like(eager)
    torch.cuda.synchronize()
    binding.attn_decode(q, s.cache, s.table, s.lengths, o, scale=0.1, workspace=s.workspace, stream=other)
    other.synchronize()
    assert torch.equal(o, eager)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_decode_agrees_with_the_prompts_attention(dtype):
    """The newest token of a prompt: attn_fwd's last causal row and attn_decode over the cache that the same call has filled."""
    B, N, H, d, ps = 2, 333, 4, 128, 16
    q, k, v, (wq, wk) = prepare_inputs(B, N, H, H, d, dtype, seed=21)
    wide = -(-N // ps)
    caches = [torch.full((B * wide, H, ps, d), float("nan"), dtype=DTYPES[dtype], device="cuda") for _ in range(2)]
    cache = binding.KVCache(*caches)
    outs = [torch.empty(B, H, N, d, dtype=DTYPES[dtype], device="cuda") for _ in range(3)]
    table = torch.arange(B * wide, dtype=torch.int32, device="cuda").flip(0).reshape(B, wide)
    rows = torch.arange(N, device="cuda")
    slots = table[:, rows // ps].long() * ps + rows % ps
    binding.attn_qkv_prepare(q, k, v, positions=rows.int().repeat(B, 1), frequencies=frequencies(d), q_weight=wq, k_weight=wk,
                             q_out=outs[0].transpose(1, 2), k_out=outs[1].transpose(1, 2), v_out=outs[2].transpose(1, 2), cache=cache, slots=slots)
    whole = binding.attn_fwd(*outs, scale=d ** -0.5, causal=True, o_dtype=torch.float32)
    one = binding.attn_decode(outs[0][:, :, -1], cache, table, torch.full((B,), N, dtype=torch.int32, device="cuda"), scale=d ** -0.5,
                              o_dtype=torch.float32)
    # attn_fwd rounds probabilities to binary16: half a step of each
    size = (outs[2].float().abs().amax(2))
    assert ((whole[:, :, -1] - one).abs() <= 2.0 ** -11 * size + 2.0 ** -16 * size).all()


def test_built_kernels(tmp_path):
    """The kernels as built: none has scratch memory, and none reads K from LDS before the direct loads that bring it have landed."""
    import re
    from .util import device_code, device_listing, kernel_bodies, llvm_tool
    notes = llvm_tool("llvm-readelf", "--notes", device_code(tmp_path))
    found = dict(re.findall(r"\.name:\s+(_ZN7sawattn\d+(?:kv_pages|qkv_prepare|decode|decode_join)_kernel\S+)\s+\.private_segment_fixed_size:\s+(\d+)", notes, re.S))
    assert len(found) >= 2 + 12 + 20 + 2 and set(found.values()) == {"0"}, found
    (tmp_path / "listing").mkdir()
    seen = 0
    for kernel, body in kernel_bodies(device_listing(tmp_path / "listing")).items():
        if "sawattn::decode_kernel<" not in kernel:
            continue
        flying, straight, behind, loads, waits = False, True, 0, 0, 0
        for text, _ in body:
            wait = re.match(r"s_waitcnt .*vmcnt\((\d+)\)", text)
            if text.startswith("global_load_lds_"):
                flying, straight, behind, loads = True, True, 0, loads + 1
            elif text.startswith("global_load_"):
                behind += 1
            elif text.startswith(("s_cbranch", "s_branch")):
                straight = False
            elif wait and (wait.group(1) == "0" or straight and int(wait.group(1)) <= behind):      # so many, of the loads behind, may still be on their way
                flying, waits = False, waits + 1
            assert not (flying and text.startswith("ds_")), (kernel, text)
        assert loads >= 4 and waits and not flying, kernel
        seen += 1
    assert seen == 20


def test_steps_study_lists_its_points(capsys):
    from paper_2601_16032_amd import sweeps
    assert sweeps.main(["--study", "steps", "--list"]) == 0
    assert len(capsys.readouterr().out.splitlines()) == len(sweeps.study_points("steps")) == 21


@pytest.mark.gpu
def test_steps_study_runs(capsys):
    """A point of the study `steps`: every operator timed, and the step right."""
    import json
    from paper_2601_16032_amd import sweeps
    assert sweeps.main(["--study", "steps", "--points", "0,17", "--launches", "2"]) == 0
    lines = [json.loads(x) for x in capsys.readouterr().out.splitlines() if x.startswith("{")]
    assert [x["point"] for x in lines] == [0, 17] and all(x[n + "_us"] > 0 for x in lines for n in ("attn_kv_pages", "attn_qkv_prepare", "attn_decode"))
    pt = {"R": 3, "length": 128, "H": 6, "KH": 3, "d": 64}
    calls, held = sweeps.decode_step(pt, dtype="f16", seed=3)
    for _ in range(2):
        for _, call in calls:
            call()
    torch.cuda.synchronize()
    cache, lengths = held["cache"], held["step"].lengths.tolist()
    assert lengths == [129] * 3 and (held["table"].cpu().sort().values.diff() != 0).all()
    keys = [[x[t.long()].transpose(1, 2).reshape(-1, 3, 64) for t in held["table"]] for x in (cache.k, cache.v)]
    check_decode(held["o"], held["q"], keys, 0.125, lengths)
    exact, size = po.rows(f64(held["qkv"][:, 6:9]), np.ones(64), 1e-6, np.full(3, 128), f64(held["frequencies"]), False)
    check_rows(torch.stack([k[128] for k in keys[0]]), exact, size, torch.float16)
    assert all(torch.equal(v[128], held["qkv"][r, 9:]) for r, v in enumerate(keys[1]))


# ------------------------------------------------------------------------------------------- what a probability holds

def weighed(R, d, dtype, wide):
    """R requests of two keys and one head: scores 0 and -x, values 0 and 1, x every number of `dtype` in turn from 1/4 on, below 2.
    O = p / (1 + p), p = exp(-x)."""
    step = torch.finfo(DTYPES[dtype]).eps
    per = int(1 / step)
    i = np.linspace(0, 3 * per - 1, R).astype(np.int64)
    x = 2.0 ** (i // per - 2) * (1 + i % per * step)
    k, v = (torch.zeros(R, 1, 16, d, dtype=DTYPES[dtype], device="cuda") for _ in range(2))
    k[:, 0, 1, 3] = -torch.tensor(x, device="cuda").to(DTYPES[dtype])
    assert np.array_equal(-f64(k[:, 0, 1, 3]), x)
    v[:, 0, 1] = 1.0
    q = torch.zeros(R, 1, d, dtype=DTYPES[dtype], device="cuda")
    q[:, :, 3] = 1.0
    table = torch.full((R, wide), POISON, dtype=torch.int32, device="cuda")
    table[:, 0] = torch.arange(R, dtype=torch.int32, device="cuda")
    return q, binding.KVCache(k, v), table, np.exp(-x)


@pytest.mark.gpu
@pytest.mark.parametrize("wide", [1, 400])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_decode_probabilities_in_32_bits(dtype, d, wide):
    """Off by 2^-20 at most, relative: the operand of exp2 is 2.9 at most and rounded twice (constant and product, 2^-24 each: 2^-22 of the
    probability), exp2 one unit in the last place (2^-23), the second product three additions (2^-23 each), the sum and the quotient one unit and a
    half: 7.5 x 2^-23.  Binary16 adds 15 to the operand, which is rounded to 2^-21 then (2^-21.5 of the probability): 10.4 x 2^-23.
    Probabilities in 16 bits are off by 2^-17."""
    R = 384
    q, cache, table, p = weighed(R, d, dtype, wide)
    assert (binding.attn_decode_workspace_bytes(R, 1, cache, wide) > 0) == (wide == 400)
    got = f64(binding.attn_decode(q, cache, table, torch.full((R,), 2, dtype=torch.int32, device="cuda"), scale=1.0, o_dtype=torch.float32))
    want = (p / (1 + p))[:, None, None]
    off = np.abs(got - want) / want
    assert off.max() <= (1.5 if dtype == "f16" else 1) * 2.0 ** -20, math.log2(off.max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d,length", [(64, 300), (128, 300), (64, 6000), (128, 6000)])
def test_decode_infinite_values(dtype, d, length):
    """An infinity among the visible values makes the elements it meets infinite; one of either sign makes them NaN; no other element changes."""
    inf, lengths = float("inf"), [length] * 4
    cache, table, keys = fill_cache(lengths, 2, d, 16, dtype, seed=length + d)
    for r, at, head, e, x in ((0, 0, 0, 3, inf), (0, 150, 1, 60, -inf), (1, length - 1, 0, 5, -inf), (1, 7, 0, 5, -inf), (2, 40, 0, 9, inf),
                              (2, 290, 0, 9, -inf), (2, 33, 1, 0, inf), (2, 34, 1, 1, -inf)):
        cache.v[int(table[r, at // 16]), head, at % 16, e] = keys[1][r][at, head, e] = x
    q, lens = queries(4, 6, d, dtype, seed=4), torch.tensor(lengths, dtype=torch.int32, device="cuda")
    for out in (q.dtype, torch.float32):
        got = binding.attn_decode(q, cache, table, lens, scale=d ** -0.5, o_dtype=out)
        with np.errstate(invalid="ignore"):
            exact, _, _ = po.decode(f64(q), *[[f64(x) for x in side] for side in keys], d ** -0.5, lengths)
        assert np.isinf(exact).sum() == 5 * 3 and np.isnan(exact).sum() == 3
        odd = ~np.isfinite(exact)
        assert np.array_equal(f64(got)[odd], exact[odd], equal_nan=True)
        plain = [[torch.where(x.isinf(), 0, x) for x in side] for side in keys]
        without = torch.where(torch.tensor(odd, device="cuda"), 0, got)
        bound_by = binding.KVCache(cache.k, torch.where(cache.v.isinf(), 0, cache.v))
        same = binding.attn_decode(q, bound_by, table, lens, scale=d ** -0.5, o_dtype=out)
        assert torch.equal(torch.where(torch.tensor(odd, device="cuda"), 0, same), without)
        check_decode(same, q, plain, d ** -0.5, lengths)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("wide", [1, 400])
def test_decode_infinite_values_of_small_weight(dtype, wide):
    """Probabilities down to 2^-38 of the largest: e^-26 = 2^-37.5."""
    q, cache, table, _ = weighed(300, 128, dtype, wide)
    cache.k[:, 0, 1, 3] = -torch.linspace(0, 26, 300, device="cuda").to(q.dtype)
    cache.v[:, 0, 1], cache.v[150:, 0, 1] = float("inf"), float("-inf")
    got = binding.attn_decode(q, cache, table, torch.full((300,), 2, dtype=torch.int32, device="cuda"), scale=1.0)
    assert (got[:150] == float("inf")).all() and (got[150:] == float("-inf")).all()


# ------------------------------------------------------------------------------------------- workspaces

def workspace_bytes(cache, R, H, pages):
    n = ctypes.c_size_t(0)
    assert binding.lib().attn_decode_workspace_bytes(ctypes.addressof(cache), R, H, pages, ctypes.byref(n)) == 0, binding.attn_last_error()
    return n.value


@pytest.mark.parametrize("d,KH,H,ps", [(128, 8, 32, 16), (64, 8, 8, 64), (128, 2, 96, 16), (64, 1, 1, 16), (128, 1, 260, 32)])
def test_decode_workspace_of_the_largest_batch(d, KH, H, ps):
    """What is reported for a batch and a table does for every smaller batch and table, at any window.  The calls name the same memory for O and
    Q: they are refused for that once they have found the workspace large enough."""
    cache = cache_struct(d=d, heads=KH, page_size=ps, k=0x100000000, v=0x200000000, k_page=KH * ps * d, k_head=ps * d, k_row=d, v_page=KH * ps * d,
                         v_head=ps * d, v_row=d)
    L, batches, tables = binding.lib(), (1, 2, 7, 31, 32, 33, 63, 255, 256, 300), (1, 17, 128, 200, 1000)
    for R in batches:
        for pages in tables:
            most = workspace_bytes(cache, R, H, pages)
            for fewer in (r for r in batches if r <= R):
                for narrower in (p for p in tables if p <= pages):
                    assert workspace_bytes(cache, fewer, H, narrower) <= most
                    for window in (0, 300):
                        rc = L.attn_decode(0x1000000, H * d, d, 0x1000000, H * d, d, 0, ctypes.addressof(cache), 0x3000000, narrower, narrower,
                                           0x4000000, fewer, H, 0.1, window, 0x5000000, most, None)
                        refused(rc, binding.ERR_INVALID_ARG, "must not overlap what is read")


class LongServer(Server):
    """A server whose tables are long enough for units in parts: shares, records of begun units and the second kernel.  Before each step the
    workspace, made for the largest batch, is filled with bytes that are no number, no request and no place."""

    def __init__(self, **kw):
        super().__init__(**{"wide": 128, "H": 40, "d": 128, "dtype": "bf16", **kw})      # 20 query heads to a key head: two sets of workgroups
        assert self.workspace.numel() > 0

    def step(self, qkv, tokens):
        self.workspace.fill_(0xff)
        return super().step(qkv, tokens)


LONG_PLAN = [[700, 1, 0, 1290, 128, 127], [1, 1, 600, 1, 1, 1], [1, 1, 1, -1, 129, 1], [1, 0, 1, 1500, 1, -1], [1, 1, 1, 1, -1, 0]]


@pytest.mark.gpu
def test_long_steps_of_a_server():
    """Requests that start, grow over several steps of 128 rows, end and start anew, in parts, against 64 bits."""
    s = LongServer()
    for i, new in enumerate(LONG_PLAN):
        s.new.copy_(torch.tensor(new, dtype=torch.int32))
        tokens = sum(max(n, 0) for n in new) + 2
        qkv = queries(tokens, s.H + 2 * s.KH, s.d, s.dtype, seed=200 + i)
        o, last = s.step(qkv, tokens)
        torch.cuda.synchronize()
        lengths = s.host(qkv, new)
        assert s.lengths.tolist() == lengths
        s.check(o, last, lengths)


@pytest.mark.gpu
def test_long_steps_captured():
    """A step in parts captured once and replayed while shares change with the lengths, with eager work in between: the eager results bit by bit."""
    a, b = LongServer(), LongServer()
    n = 6 * 300
    qkv = torch.zeros(n, a.H + 2 * a.KH, a.d, dtype=torch.bfloat16, device="cuda")
    a.step(qkv, n)      # loads everything, adds nothing
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        o, _ = a.step(qkv, n)
    for i, new in enumerate([[300, 3, 129, 255, 1, 600], [1] * 6, [300] * 6, [1, -1, 1, 300, 0, -1], [300] * 6, [1] * 6]):
        for s in (a, b):
            s.new.copy_(torch.tensor(new, dtype=torch.int32))
        qkv.copy_(queries(n, a.H + 2 * a.KH, a.d, "bf16", seed=i))
        graph.replay()
        torch.cuda.synchronize()
        want, last = b.step(qkv, n)
        torch.cuda.synchronize()
        assert torch.equal(o, want) and a.lengths.tolist() == b.lengths.tolist(), i
        b.check(want, last, b.host(qkv, new))
    assert max(b.lengths.tolist()) > 1000


@pytest.mark.gpu
def test_long_steps_on_streams_of_their_own():
    """Steps in parts on two streams at once, each with its own workspace, and the stream argument: the results of one after the other."""
    servers, plain = [LongServer(seed=i) for i in (1, 2)], [LongServer(seed=i) for i in (1, 2)]
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    inputs = [queries(4000, 44, 128, "bf16", seed=i) for i in range(2)]
    new = torch.tensor([900, 3, 0, 1299, 1, 1700], dtype=torch.int32, device="cuda")
    for s in servers + plain:
        s.new.copy_(new)
    want = [s.step(x, 4000) for s, x in zip(plain, inputs)]
    torch.cuda.synchronize()
    assert all(s.lengths.tolist() == new.tolist() for s in plain)
    got = []
    for _ in range(4):
        for s, stream, x in zip(servers, streams, inputs):
            with torch.cuda.stream(stream):
                s.lengths.zero_()
                s.state.copy_(torch.tensor([5, s.ring.numel()], dtype=torch.int32))
                got.append(s.step(x, 4000)[0])
    torch.cuda.synchronize()
    for i, o in enumerate(got):
        assert torch.equal(o, want[i % 2][0]), i
    # calls given their streams, queued beside each other
    outs = [[torch.zeros_like(want[0][0]) for _ in range(4)] for _ in range(2)]
    for s in servers:
        s.workspace.fill_(0xff)
    torch.cuda.synchronize()
    for j in range(4):
        for i, s in enumerate(servers):
            binding.attn_decode(want[i][1], s.cache, s.table, s.lengths, outs[i][j], scale=128 ** -0.5, workspace=s.workspace, stream=streams[i])
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(o, want[i][0]) for o in outs[i])


@pytest.mark.gpu
def test_decode_one_workspace_for_all():
    """One workspace, made for the largest batch, used in turn by smaller ones, narrower tables, windows and other numbers of heads, each
    finding what the one before left: the bits of a call with a workspace of its own."""
    lengths = [5000, 0, 130, 2048, 1, 4097, 900, 3333] + [37 * i % 300 for i in range(32)]
    cache, table, keys = fill_cache(lengths, 8, 128, 64, "f16", seed=31)
    assert binding.attn_decode_workspace_bytes(40, 32, cache, 32) >= binding.attn_decode_workspace_bytes(31, 32, cache, 32) > 0
    workspace = torch.full((max(binding.attn_decode_workspace_bytes(40, H, cache, table.shape[1]) for H in (32, 8, 160)),), 0xff, dtype=torch.uint8, device="cuda")
    for R, H, wide, window in ((40, 32, 79, 0), (3, 32, 79, 0), (31, 32, 32, 0), (32, 32, 32, 0), (8, 160, 79, 0), (40, 8, 79, 2500), (1, 8, 79, 0), (6, 32, 79, 1)):
        q = queries(R, H, 128, "f16", seed=R)
        seen = [min(n, wide * 64) for n in lengths[:R]]
        lens = torch.tensor(lengths[:R], dtype=torch.int32, device="cuda")
        got = binding.attn_decode(q, cache, table[:R, :wide], lens, scale=0.09, window=window, workspace=workspace)
        check_decode(got, q, keys, 0.09, seen, window)
        assert torch.equal(got, binding.attn_decode(q, cache, table[:R, :wide], lens, scale=0.09, window=window))


@pytest.mark.gpu
def test_steps_study_in_parts():
    """A step of the study `steps` long enough for the shared launch, made twice: right, and the same bits."""
    from paper_2601_16032_amd import sweeps
    calls, held = sweeps.decode_step({"R": 3, "length": 4999, "H": 12, "KH": 4, "d": 128}, seed=3)
    cache, outs = held["cache"], []
    assert binding.attn_decode_workspace_bytes(3, 12, cache, held["table"].shape[1]) > 0
    for _ in range(2):
        for _, call in calls:
            call()
        outs.append(held["o"].clone())
    keys = [[x[t.long()].transpose(1, 2).reshape(-1, 4, 128) for t in held["table"]] for x in (cache.k, cache.v)]
    check_decode(outs[0], held["q"], keys, 128 ** -0.5, held["step"].lengths.tolist())
    assert torch.equal(*outs) and held["step"].lengths.tolist() == [5000] * 3


@pytest.mark.parametrize("d", [64, 128])
def test_decode_workspace_stays_in_bounds(d):
    """17 MiB, or 64 d + 136 bytes for each query head to a key head: long tables, whose need is largest, up to the most heads accepted."""
    cache = cache_struct(d=d, heads=1)
    sizes = {H: workspace_bytes(cache, 1, H, 16384) for H in [*range(1, 2100), 4111, 65536, 2 ** 20 + 16, 2 ** 22 - 1]}
    for H, n in sizes.items():
        assert n <= max(17 << 20, -(-H // 16) * 16 * (64 * d + 136)), (H, n)
        assert H >= 2100 or n <= 17 << 20
    assert max(n for H, n in sizes.items() if H <= 1024) > 10 << 20
    assert workspace_bytes(cache_struct(d=d, heads=8), 511, 8 * 1024, 16384) <= 17 << 20


@pytest.mark.gpu
def test_cache_of_too_many_pages():
    """Counts that pass 32 bits are refused, not cut off (2^32 + 10 pages would be 10)."""
    for shape, wide in (((1, 1, 16, 64), (2 ** 32 + 10, 1, 16, 64)), ((1, 1, 16, 64), (1, 2 ** 32 + 1, 16, 64)), ((1, 1, 1, 64), (1, 1, 2 ** 32 + 16, 64))):
        x = torch.empty(shape, dtype=torch.float16, device="cuda").expand(wide)
        with pytest.raises(ValueError, match="fewer than 2"):
            binding.KVCache(x, x)


@pytest.mark.gpu
@pytest.mark.parametrize("d,wide", [(64, 1), (128, 400)])
def test_decode_large_values_of_tiny_weight(d, wide):
    """Values of 2^127 with probabilities of e^-60 to e^-80: what a probability holds does not end with the largest one's last bit.  The operand of exp2 is
    116 at most and rounded twice (2^-24 each: 2^-16.6 of the probability), and at e^-80 the third number is subnormal (2^-16)."""
    R = 300
    q, cache, table, _ = weighed(R, d, "bf16", wide)
    x = torch.linspace(60, 80, R, device="cuda").bfloat16()
    cache.k[:, 0, 1, 3] = -x
    cache.v[:, 0, 1] = 2.0 ** 127
    got = f64(binding.attn_decode(q, cache, table, torch.full((R,), 2, dtype=torch.int32, device="cuda"), scale=1.0, o_dtype=torch.float32))
    want = np.exp(-f64(x))[:, None, None] * 2.0 ** 127
    assert (np.abs(got - want) <= 2.0 ** -15 * want).all(), float((np.abs(got - want) / want).max())
