"""Requests that share pages of a paged key-value cache: forks, page copies, common rows, attention by groups, and steps of all of them."""
import ctypes
import math

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from oracle import shared_oracle as so
from paper_2601_16032_amd import binding

from .test_paged import BAD_CACHES, DTYPES, POISON, cache_struct, f64, half_step, queries, refused, smallest


def up(x, dtype=torch.int32):
    return torch.tensor(np.asarray(x)).to(dtype).cuda()


# ------------------------------------------------------------------------------------------- refusals, without a GPU

def test_fork_refusals():
    L = binding.lib()
    n = ctypes.c_size_t(0)
    assert L.attn_kv_fork_workspace_bytes(4, 6, 100, ctypes.byref(n)) == 0 and n.value >= 200 + 48
    at = [0x100000 * (i + 1) for i in range(12)]
    base = dict(lengths=at[0], R=4, source=at[1], rows=at[2], N=6, table=at[3], stride=8, table_out=at[4], out_stride=9, wide=8, ps=16, pages=100,
                free=at[5], ring=100, state=at[6], out=at[7], copies=at[8], state_out=at[9], ws=at[10], bytes=n.value)

    def call(**kw):
        return L.attn_kv_fork(*dict(base, **kw).values(), None)
    bad, no = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
    for name in ("lengths", "source", "table", "table_out", "free", "state", "out", "copies", "state_out", "ws"):
        refused(call(**{name: None}), bad, "null")
        refused(call(**{name: base[name] + 2}), bad, "aligned")
    refused(call(rows=base["rows"] + 2), bad, "aligned")
    refused(call(ws=base["ws"] + 8), bad, "16-byte")
    for name in ("R", "N", "pages", "wide", "ring"):
        refused(call(**{name: 0}), bad, "positive")
    for name in ("R", "N"):
        refused(call(**{name: 4097}), no, "SAWATTN_MOST_REQUESTS")
    for ps in (0, 8, 24, 2 ** 21, -16):
        refused(call(ps=ps), no, "page size")
    refused(call(wide=2 ** 27, stride=2 ** 27, out_stride=2 ** 27), bad, "below 2^31")
    refused(call(N=4096, wide=2 ** 19, stride=2 ** 19, out_stride=2 ** 19, bytes=2 ** 20), bad, "below 2^31")
    for name in ("stride", "out_stride"):
        refused(call(**{name: 7}), bad, "strides of the tables")
    refused(call(bytes=n.value - 1), bad, "smaller than")
    for name, value in (("out", "lengths"), ("copies", "source"), ("table_out", "table"), ("state_out", "state"), ("out", "rows"), ("ws", "table")):
        refused(call(**{name: base[value]}), bad, "overlaps an input")
    refused(call(copies=base["out"] + 20), bad, "two outputs")
    refused(call(out=base["table_out"] + 4 * (9 * 5 + 7)), bad, "two outputs")
    refused(L.attn_kv_fork_workspace_bytes(4, 6, 100, None), bad, "non-null")
    refused(L.attn_kv_fork_workspace_bytes(4, 5000, 100, ctypes.byref(n)), no, "SAWATTN_MOST_REQUESTS")


def test_copy_refusals():
    L = binding.lib()
    structs = (binding._CacheStruct * 2)(cache_struct(), cache_struct(k=0x30000000, v=0x40000000, k_row=256, k_head=4096, k_page=8192))
    base = dict(caches=ctypes.addressof(structs), layers=2, copies=0x1000000, n=5)

    def call(**kw):
        return L.attn_kv_copy(*dict(base, **kw).values(), None)
    bad = binding.ERR_INVALID_ARG
    for name in ("caches", "copies"):
        refused(call(**{name: None}), bad, "non-null")
    for name in ("layers", "n"):
        refused(call(**{name: 0}), bad, "positive")
    refused(call(n=4097), binding.ERR_UNSUPPORTED, "SAWATTN_MOST_REQUESTS")
    refused(call(copies=0x1000002), bad, "aligned")
    refused(call(copies=0x40000010), bad, "must not lie in a cache")
    for name in ("pages", "page_size", "heads", "d", "dtype"):
        kept = getattr(structs[1], name)
        setattr(structs[1], name, {"pages": 11, "page_size": 32, "heads": 3, "d": 64, "dtype": 1}[name])
        refused(call(), bad, "must share")
        setattr(structs[1], name, kept)
    for change, code, text in BAD_CACHES:
        structs[1] = cache_struct(**change)
        refused(call(), code, text)
    big = cache_struct(heads=2 ** 15, page_size=2 ** 16)
    refused(call(caches=ctypes.addressof(big), layers=1), bad, "below 2^31")


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,heads,page_size", [(1, 2 ** 27 - 1, 16), (1, 2 ** 27 - 3, 16)])
def test_copy_refuses_rows_that_do_not_round_up(n, heads, page_size, d):
    """n*heads*page_size below 2^31, but not what the pieces count that the rows are dealt out in.  (Heads that all lie in the same place.)"""
    cache = cache_struct(d=d, heads=heads, page_size=page_size, k_head=0, v_head=0)
    assert n * heads * page_size < 2 ** 31
    refused(binding.lib().attn_kv_copy(ctypes.addressof(cache), 1, 0x1000000, n, None), binding.ERR_INVALID_ARG, "below 2^31")


def test_copy_wants_caches_of_its_own_kinds():
    """Caches of several layers come as a KVLayers; anything else is refused as such, before a tensor is looked at."""
    for caches in ([], [1], (object(), object()), None, torch.zeros(3)):
        with pytest.raises(ValueError, match="KVLayers"):
            binding.attn_kv_copy(caches, torch.zeros(1, 3, dtype=torch.int32))


def test_shared_rows_refusals():
    L = binding.lib()
    base = dict(lengths=0x100000, R=4, table=0x200000, stride=8, wide=8, ps=16, offsets=0x300000, groups=2, shared=0x400000)

    def call(**kw):
        return L.attn_kv_shared_rows(*dict(base, **kw).values(), None)
    bad, no = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
    for name in ("lengths", "table", "offsets", "shared"):
        refused(call(**{name: None}), bad, "null")
        refused(call(**{name: base[name] + 1}), bad, "aligned")
    for name in ("R", "wide", "groups"):
        refused(call(**{name: 0}), bad, "positive")
    for name in ("R", "groups"):
        refused(call(**{name: 4097}), no, "SAWATTN_MOST_REQUESTS")
    refused(call(ps=17), no, "page size")
    refused(call(wide=2 ** 27, stride=2 ** 27), bad, "below 2^31")
    refused(call(stride=7), bad, "table_stride")
    for name in ("lengths", "table", "offsets"):
        refused(call(shared=base[name] + 4), bad, "overlaps an input")


def test_decode_shared_refusals():
    L = binding.lib()
    cache = cache_struct()
    n = ctypes.c_size_t(0)
    assert L.attn_decode_shared_workspace_bytes(ctypes.addressof(cache), 3, 8, 2, 100, ctypes.byref(n)) == 0 and n.value > 0
    base = dict(Q=0x1000000, qr=1024, qh=128, O=0x2000000, orow=1024, oh=128, odt=0, cache=ctypes.addressof(cache), table=0x3000000,
                stride=100, wide=100, lengths=0x4000000, offsets=0x4100000, shared=0x4200000, groups=2, R=3, H=8, scale=0.1, ws=0x50000000, bytes=n.value)

    def call(**kw):
        return L.attn_decode_shared(*dict(base, **kw).values(), None)
    bad, no = binding.ERR_INVALID_ARG, binding.ERR_UNSUPPORTED
    for name in ("Q", "O", "table", "lengths", "offsets", "shared", "ws"):
        refused(call(**{name: None}), bad, "non-null")
        refused(call(**{name: base[name] + 2}), bad, "aligned")
    refused(call(cache=None), bad, "non-null")
    for name in ("R", "H", "wide", "groups"):
        refused(call(**{name: 0}), bad, "positive")
    refused(call(H=7), bad, "multiple of the cache's heads")
    refused(call(R=5000), no, "SAWATTN_MOST_REQUESTS")
    refused(call(groups=5000), no, "SAWATTN_MOST_REQUESTS")
    refused(call(R=4096, H=512, wide=2 ** 13, stride=2 ** 13), bad, "2^31 - 8192")
    refused(call(odt=3), bad, "o_dtype")
    refused(call(scale=math.nan), bad, "scale")
    refused(call(stride=99), bad, "table_stride")
    for name, value in (("qr", -8), ("qh", 100), ("orow", 1020), ("oh", -128)):
        refused(call(**{name: value}), bad, "strides of Q and O")
    refused(call(oh=64), bad, "at least d")
    refused(call(bytes=n.value - 1), bad, "smaller than")
    for name, value in (("O", 0x1000000 + 2 * 1024), ("ws", 0x10000000), ("O", 0x20000010), ("ws", 0x1000000), ("O", 0x3000000), ("O", 0x4100000), ("ws", 0x4200000 - 16)):
        refused(call(**{name: value}), bad, "overlap")
    refused(call(O=0x50000000), bad, "must not overlap the workspace")
    for change, code, text in BAD_CACHES:
        other = cache_struct(**change)
        refused(call(cache=ctypes.addressof(other)), code, text)
    refused(L.attn_decode_shared_workspace_bytes(ctypes.addressof(cache), 3, 8, 2, 10, None), bad, "non-null")
    refused(L.attn_decode_shared_workspace_bytes(ctypes.addressof(cache), 3, 7, 2, 10, ctypes.byref(n)), bad, "multiple")


@pytest.mark.parametrize("d,KH,H,ps", [(128, 8, 32, 16), (64, 8, 8, 64), (128, 2, 96, 16), (64, 1, 1, 16)])
def test_workspaces_do_for_smaller_calls(d, KH, H, ps):
    cache = cache_struct(d=d, heads=KH, page_size=ps)
    n = ctypes.c_size_t(0)

    def need(R, groups, pages):
        assert binding.lib().attn_decode_shared_workspace_bytes(ctypes.addressof(cache), R, H, groups, pages, ctypes.byref(n)) == 0
        return n.value
    sizes = (1, 2, 3, 16, 17, 64, 255, 1000)
    for R in sizes:
        for groups in sizes:
            assert need(R, groups, 10) <= need(R + 1, groups, 10) and need(R, groups, 10) <= need(R, groups + 1, 10) and need(R, groups, 10) <= need(R, groups, 700)
        assert need(R, 1, 700) <= 8 * d * R * H + 8 * R * H + 16 * R + 110 * 2 ** 20 + 24 * R * H
    def fork(*a):
        assert binding.lib().attn_kv_fork_workspace_bytes(*a, ctypes.byref(n)) == 0
        return n.value
    for R in sizes:
        assert fork(R, R, 1000) <= fork(R + 1, R + 1, 1000) and fork(R, R, 1000) <= fork(R, R, 1001) <= 2 * 1016 + 16 * R + 64


# ------------------------------------------------------------------------------------------- forks

def fork_case(rng, R, N, ps, most, cut=0.5, none=0.1, pool="enough", room=1):
    """Requests of a consistent server: whole pages shared by neighbours here and there, part-filled ones nobody else's."""
    lengths = rng.integers(0, most + 1, R)
    held = -(-lengths // ps)
    wide = int(max(1, held.max() + room))
    F = int(held.sum()) + 3 * N + 7
    ids = rng.permutation(F).tolist()
    table = np.full((R, wide), -7)
    for r in range(R):
        like = r - 1 if r and rng.random() < 0.6 else None
        share = int(rng.integers(0, 1 + min(lengths[r] // ps, lengths[like] // ps))) if like is not None else 0
        if share:
            table[r, :share] = table[like, :share]
        for j in range(share, held[r]):
            table[r, j] = ids.pop()
    source = rng.integers(0, R, N)
    source[rng.random(N) < none] = rng.choice([-1, R, 2 ** 31 - 1, -2 ** 31])
    rows = np.full(N, 2 ** 31 - 1)
    if cut:
        which = rng.random(N) < cut
        rows[which] = (lengths[np.clip(source, 0, R - 1)] - rng.integers(0, 2 * ps + 1, N))[which]
    missing = sum(c[0] >= 0 for c in so.kv_fork(lengths, source, rows, table, [0], [0, 0], ps, F, np.zeros((N, wide), dtype=np.int64))[2])
    available = {"enough": missing + 2, "exact": missing, "half": missing // 2, "none": 0}[pool]
    first = int(rng.integers(0, F))
    ring = np.full(F, -5)
    ring[(first + np.arange(available)) % F] = [ids.pop() for _ in range(available)]
    return lengths, source, rows if cut else None, table, ring, [first, available], ps, F


def run_fork(lengths, source, rows, table, ring, state, ps, pages, stride=0):
    """What attn_kv_fork writes, into poisoned tensors with guards around them, over a workspace that holds anything."""
    (R, wide), N = table.shape, len(source)
    old = torch.full((R, wide + stride), 99, dtype=torch.int32, device="cuda")
    old[:, :wide] = up(table)
    new = torch.full((N, wide + stride), 99, dtype=torch.int32, device="cuda")
    new[:, :wide] = POISON
    guarded = [torch.full((n + 2,), POISON, dtype=torch.int32, device="cuda") for n in (N, 3 * N, 2)]
    out = [g[:-2] for g in guarded]
    ring_t = up(ring)
    need = binding.attn_kv_fork_workspace_bytes(R, N, pages)
    workspace = torch.full((need + 64,), 0xa5, dtype=torch.uint8, device="cuda")
    step = binding.attn_kv_fork(up(lengths), up(source), old[:, :wide], ring_t, up(state), page_size=ps, pages=pages, rows=None if rows is None else up(rows),
                                table_out=new[:, :wide], lengths_out=out[0], copies=out[1], free_state_out=out[2], workspace=workspace[:need])
    torch.cuda.synchronize()
    assert step.copies is out[1]
    assert all((g[-2:] == POISON).all() for g in guarded) and (new[:, wide:] == 99).all() and (workspace[need:] == 0xa5).all()
    assert torch.equal(old[:, :wide].cpu(), torch.tensor(np.asarray(table)).int())
    return new[:, :wide].cpu().numpy(), out[0].cpu().numpy(), out[1].cpu().numpy(), ring_t.cpu().numpy(), out[2].cpu().numpy()


def check_fork(*case, stride=0):
    lengths, source, rows, table, ring, state, ps, pages = case
    got = run_fork(*case, stride=stride)
    want = so.kv_fork(lengths, source, rows, table, ring, state, ps, pages, np.full((len(source), table.shape[1]), POISON))
    for name, g, w in zip(("table", "lengths", "copies", "ring", "state"), got, want):
        assert np.array_equal(g, np.asarray(w, dtype=np.int64).astype(np.int32).reshape(g.shape)), name


@pytest.mark.gpu
@pytest.mark.parametrize("R,N,ps,most", [(1, 1, 16, 0), (1, 1, 16, 16), (1, 8, 16, 100), (8, 8, 16, 1000), (63, 64, 32, 300), (65, 257, 16, 40), (1024, 1025, 16, 500),
                                         (4096, 4096, 64, 2000), (3, 4096, 16, 5000), (4096, 2, 16, 33), (5, 7, 1024, 5000), (2, 40, 16, 40000)])
@pytest.mark.parametrize("pool", ["enough", "exact", "half", "none"])
def test_fork(R, N, ps, most, pool):
    rng = np.random.default_rng(R + N + most)
    check_fork(*fork_case(rng, R, N, ps, most, pool=pool), stride=0 if R % 2 else 3)
    check_fork(*fork_case(rng, R, N, ps, most, pool=pool, cut=0, none=0))


@pytest.mark.gpu
def test_fork_everything_ends():
    rng = np.random.default_rng(5)
    check_fork(*fork_case(rng, 300, 20, 16, 500, none=1.1))
    check_fork(*fork_case(rng, 20, 300, 16, 0))


@pytest.mark.gpu
def test_fork_many_pages():
    """More pages than one workgroup looks at, in any order, those given back among all of them."""
    rng = np.random.default_rng(11)
    for pages in (16384, 16385, 50000, 131072, 131072 + 7, 256 * 16384 + 5, 3 * 256 * 16384 - 7):
        lengths = np.array([16 * 900, 16 * 800 + 3, 16 * 700])
        table = np.zeros((3, 901), dtype=np.int64)
        ids = rng.permutation(pages)
        table[0, :900], table[1, :801], table[2, :700] = ids[:900], ids[900:1701], ids[1701:2401]
        table[1, :400] = table[0, :400]
        ring = np.full(pages, -5)
        ring[:50] = ids[3000:3050]
        check_fork(lengths, np.array([1, 1, 0]), np.array([16 * 500 + 1, 16 * 800 + 2, 16 * 300]), table, ring, [0, 50], 16, pages)
        check_fork(lengths, np.array([-1]), None, table, ring, [0, 50], 16, pages)


@pytest.mark.gpu
def test_fork_into_a_ring_too_small():
    """Pages given back that the ring has no room for are lost, and none of those in use is counted as free in their place."""
    rng = np.random.default_rng(12)
    for wide in (8, 800):
        lengths, table = np.full(30, 16 * wide - 3), np.arange(30 * wide).reshape(30, wide)
        ring = np.arange(30 * wide, 30 * wide + 40)
        for state in ([0, 32], [37, 40], [20, 0], [39, 39]):
            check_fork(lengths, rng.integers(0, 30, 12), rng.integers(1, 16 * wide, 12), table, ring, state, 16, 31 * wide + 40)
            check_fork(lengths, np.array([3, 3]), np.array([17, 18]), table, ring, state, 16, 31 * wide + 40)


@pytest.mark.gpu
def test_fork_whatever_the_numbers():
    """Lengths, sources, bounds, pages and ring states that no program should pass stay inside the tensors: the oracle's rules, clamped, hold."""
    big = 2 ** 31 - 1
    table = np.arange(20).reshape(5, 4)
    table[2, 1], table[4, 0], table[0, 3] = big, -big - 1, 20
    ring = np.arange(100, 130)
    lengths = np.array([big, -3, 40, 64, 20])
    source, rows = np.array([0, 0, 1, 2, 2, 4, 3, 3, 77, -5]), np.array([big, 33, 5, 39, 17, -4, 64, 0, 3, 3])
    for state in ([3, 8], [-1, 500], [30, 8], [big, big], [2, -4], [29, 2]):
        check_fork(lengths, source, rows, table, ring, state, 16, 20)


@pytest.mark.gpu
@pytest.mark.parametrize("wide,N", [(1100, 10), (2100, 7), (40, 1030)])
@pytest.mark.parametrize("room", [30, 20000])
def test_fork_whatever_the_numbers_of_long_tables(wide, N, room):
    """The same where three launches share the work (tables of more than 16384 entries in all, or more than 1024 requests)."""
    big, rng = 2 ** 31 - 1, np.random.default_rng(wide)
    assert (5 + N) * wide > 16384
    pages = 5 * wide - 70                                             # the last ones of the last request are outside, as are
    table = np.arange(5 * wide).reshape(5, wide)
    table[2, 1], table[4, 0], table[0, 3], table[3, wide - 1], table[1, 30], table[0, 17] = big, -big - 1, pages, -1, pages + 5, 7
    ring = np.arange(room) - 10
    lengths = np.array([big, -3, 16 * wide - 5, 16 * wide, 20 * 16])
    source = np.resize([0, 0, 1, 2, 2, 4, 3, 3, 77, -5], N)
    rows = np.resize([big, 33, 5, 16 * wide - 7, 17, -4, 16 * wide - 9, 0, 3, 3, big, 16 * 20 + 1], N)
    for first, free in ((3, 8), (-1, 50000), (room, 8), (big, big), (2, -4), (room - 1, 2)):
        check_fork(lengths, source, rows, table, ring, [first, free], 16, pages, stride=5)
        check_fork(lengths, rng.permutation(source), None, table, ring, [first, free], 16, pages)


@pytest.mark.gpu
def test_forks_and_appends_lose_no_page():
    """Some dozen steps of a server that branches, cuts short, ends and appends: pages held and pages free are all pages, every page once, and a page that
    is written on is one request's."""
    rng = np.random.default_rng(3)
    R, ps, wide, pages = 24, 16, 12, 400
    lengths, table = torch.zeros(R, dtype=torch.int32, device="cuda"), torch.zeros(R, wide, dtype=torch.int32, device="cuda")
    ring, state = torch.randperm(pages, generator=torch.Generator().manual_seed(1)).int().cuda(), up([0, pages])
    for step in range(40):
        source = np.arange(R)
        change = rng.random(R) < 0.3
        source[change] = rng.integers(-1, R, R)[change]
        rows = np.where(rng.random(R) < 0.2, np.maximum(lengths.cpu().numpy()[source] - rng.integers(0, 40, R), 0), 2 ** 31 - 1)
        fork = binding.attn_kv_fork(lengths, up(source), table, ring, state, page_size=ps, pages=pages, rows=up(rows))
        table, lengths = fork.table, fork.lengths
        new = np.where(lengths.cpu().numpy() > 150, 0, rng.integers(0, 21, R))
        more = binding.attn_kv_pages(lengths, up(new), table, ring, fork.free_state, page_size=ps, tokens=500)
        lengths, state = more.lengths, more.free_state
        n, t, (first, free) = lengths.tolist(), table.tolist(), state.tolist()
        assert more.granted.tolist() == new.tolist()
        held = {p for r in range(R) for p in t[r][:-(-n[r] // ps)]}
        loose = [ring.tolist()[(first + i) % pages] for i in range(free)]
        assert len(set(loose)) == free and not held & set(loose) and len(held) + free == pages
        part = [t[r][n[r] // ps] for r in range(R) if n[r] % ps]
        assert all(sum(p in t[r][:-(-n[r] // ps)] for r in range(R)) == 1 for p in part)


# ------------------------------------------------------------------------------------------- copies

@pytest.mark.gpu
@pytest.mark.parametrize("d,dtype,heads,ps,layers,n", [(64, "f16", 1, 16, 1, 1), (128, "bf16", 3, 16, 2, 7), (64, "bf16", 8, 64, 3, 100), (128, "f16", 2, 128, 33, 20),
                                                     (128, "bf16", 5, 32, 70, 3), (64, "f16", 2, 16, 1, 4096), (128, "f16", 1, 1024, 1, 5)])
@pytest.mark.parametrize("page_first", [False, True])
def test_copy(d, dtype, heads, ps, layers, n, page_first):
    rng = np.random.default_rng(d + n + layers)
    real = max(1, n * 2 // 3)
    pages = 2 * real + 2
    ids = rng.permutation(pages)
    copies = np.full((n, 3), -1)
    copies[:, 2] = rng.integers(0, ps + 1, n)
    where = rng.permutation(n)[:real]
    copies[where, 0], copies[where, 1], copies[where, 2] = ids[:real], ids[real:2 * real], rng.integers(0, ps + 1, real)
    for i, wrong in zip([i for i in range(n) if i not in set(where.tolist())], ((pages, 0, 5), (0, pages, 5), (int(ids[-1]), int(ids[-1]), ps), (3, -1, 4), (2 ** 31 - 1, 1, 1))):
        copies[i] = wrong
    if real > 3:
        copies[where[0], 2], copies[where[1], 2], copies[where[2], 2] = ps, -4, 2 ** 31 - 1
    g = torch.Generator("cuda").manual_seed(1)
    shape = (pages, ps, heads, d + 8) if page_first else (pages, heads, ps, d)
    tensors = [torch.randn(shape, generator=g, device="cuda").to(DTYPES[dtype]) for _ in range(2 * layers)]
    views = [t[..., :d].transpose(1, 2) if page_first else t for t in tensors]
    before = [t.clone() for t in tensors]
    for b in before:
        x = b[..., :d].transpose(1, 2) if page_first else b
        for i in where:
            a, z, rows = (int(c) for c in copies[i])
            rows = min(max(rows, 0), ps)
            x[z, :, :rows] = x[a, :, :rows].clone()
    caches = [binding.KVCache(views[2 * i], views[2 * i + 1]) for i in range(layers)]
    binding.attn_kv_copy(binding.KVLayers(caches) if layers > 1 else caches[0], up(copies))
    torch.cuda.synchronize()
    assert all(torch.equal(t, b) for t, b in zip(tensors, before))


@pytest.mark.gpu
def test_copy_far_into_a_large_cache():
    """Pages more than 2^32 bytes from the front."""
    heads, ps, d = 8, 64, 128
    pages = 2 ** 32 // (heads * ps * d * 2) + 20
    k, v = (torch.zeros(pages, heads, ps, d, dtype=torch.float16, device="cuda") for _ in range(2))
    k[pages - 1], v[3] = 1.5, 2.5
    binding.attn_kv_copy(binding.KVCache(k, v), up([[pages - 1, pages - 3, 40], [3, pages - 5, 64]]))
    assert (k[pages - 3, :, :40] == 1.5).all() and (k[pages - 3, :, 40:] == 0).all() and (v[pages - 5] == 2.5).all()
    assert float(k.sum(dtype=torch.float64)) == 1.5 * heads * d * (ps + 40) and float(v.sum(dtype=torch.float64)) == 2.5 * heads * d * 2 * ps


# ------------------------------------------------------------------------------------------- common rows

@pytest.mark.gpu
@pytest.mark.parametrize("sizes,ps,wide", [([1], 16, 1), ([2], 16, 5), ([8], 16, 250), ([3, 0, 7, 1, 0], 32, 70), ([300], 16, 40), ([2, 2, 2], 16, 1024), ([5, 4], 16, 1025),
                                           ([17, 9], 64, 3000), ([1] * 4096, 16, 3), ([4096], 16, 2),
                                           ([1000], 16, 512), ([300, 2], 32, 1500), ([4090, 0, 6], 16, 100), ([1], 16, 140000), ([2, 1], 16, 200000), ([129], 64, 1017), ([100], 16, 65)])
def test_shared_rows(sizes, ps, wide):
    rng = np.random.default_rng(sum(sizes) + wide)
    R = sum(sizes)
    offsets = np.concatenate([[0], np.cumsum(sizes)])
    for trial in range(4):
        table = rng.integers(0, 1000, (R, wide))
        lengths = rng.integers(wide * ps // 2, wide * ps + 1, R)
        for g, size in enumerate(sizes):
            if size:
                a, common = offsets[g], (0, wide, wide // 2, int(rng.integers(0, wide + 1)))[trial]
                table[a:a + size, :common] = table[a, :common]
                if trial == 3 and size > 1:      # one entry that differs, of any request
                    table[a + int(rng.integers(0, size)), int(rng.integers(0, wide))] += 1
        lengths[rng.random(R) < 0.2] = rng.choice([0, -3])
        if trial == 1:
            lengths[:] = np.where(lengths > 0, wide * ps, lengths)
        whole = torch.full((R, wide + trial), -9, dtype=torch.int32, device="cuda")
        whole[:, :wide] = up(table)
        out = torch.full((len(sizes) + 1,), POISON, dtype=torch.int32, device="cuda")
        binding.attn_kv_shared_rows(whole[:, :wide], up(lengths), up(offsets), page_size=ps, shared=out[:-1])
        assert out[:-1].tolist() == so.shared_rows(table, lengths, offsets, ps) and int(out[-1]) == POISON, trial


@pytest.mark.gpu
def test_shared_rows_whatever_the_offsets():
    table, lengths = np.zeros((6, 4), dtype=np.int64), np.array([64, 2 ** 31 - 1, 60, 0, 64, 33])
    for offsets in ([0, 6], [-5, 2, 99], [3, 3, 4], [5, 2, 6], [2 ** 31 - 1, -2 ** 31, 5]):
        got = binding.attn_kv_shared_rows(up(table), up(lengths), up(offsets), page_size=16)
        assert got.tolist() == so.shared_rows(table, lengths, offsets, 16), offsets


# ------------------------------------------------------------------------------------------- attention

def fill_groups(groups, alone, KH, d, ps, dtype, seed, page_first=False, spare=2):
    """groups: (rows in common, rows of its own of each request); alone: rows of requests in no group, behind them.  Whole pages of common rows
    are the group's, all others a request's own; what no request holds is NaN, table entries behind the last page are POISON."""
    rng = np.random.default_rng(seed)
    g = torch.Generator("cuda").manual_seed(seed)
    lengths, lead, prefix, sizes = [], [], [], []
    for common, tails in groups:
        sizes.append(len(tails))
        lead += [len(lengths)] * len(tails)
        prefix += [common] * len(tails)
        lengths += [common + t if t >= 0 else 0 for t in tails]
    lead += list(range(len(lengths), len(lengths) + len(alone)))
    prefix += [0] * len(alone)
    lengths += list(alone)
    count = [-(-n // ps) for n in lengths]
    total = sum(count) + spare
    shape = (total, ps, KH, d) if page_first else (total, KH, ps, d)
    caches = [torch.full(shape, float("nan"), dtype=DTYPES[dtype], device="cuda") for _ in range(2)]
    views = [c.transpose(1, 2) if page_first else c for c in caches]
    table = np.full((len(lengths), max(max(count), 1)), POISON)
    ids = rng.permutation(total).tolist()
    keys, first_of = ([], []), {}
    for r, n in enumerate(lengths):
        if lead[r] not in first_of and n:
            first_of[lead[r]] = r
        f = first_of.get(lead[r], r)
        whole = prefix[r] // ps if n and f != r else 0
        table[r, :whole] = table[f, :whole]
        for j in range(whole, count[r]):
            table[r, j] = ids.pop()
        for view, kept in zip(views, keys):
            x = torch.randn(n, KH, d, generator=g, device="cuda").to(DTYPES[dtype])
            if n and f != r:
                x[:prefix[r]] = kept[f][:prefix[r]]
            for j in range(whole, count[r]):
                part = x[j * ps:(j + 1) * ps]
                view[int(table[r, j]), :, :part.shape[0]] = part.transpose(0, 1)
            kept.append(x)
    offsets = np.concatenate([[0], np.cumsum(sizes)])
    return binding.KVCache(*views), up(table), lengths, up(offsets), up([c for c, _ in groups]), keys


def check_shared(got, q, keys, scale, lengths, cache_dtype, skip=()):
    """|error| <= half a step of the output + (error of probabilities) * sum p |v|.  Scores, exp2 and additions as for attn_decode: a score is off by up to
    2^-23 of the sum of |q k| for each addition, twice that is the relative error of a probability, exp2 and its operand add 2^-19, every tile of 32 rows and
    every joining one addition.  Of a shared row's probability two 16-bit numbers enter the second product: bfloat16: the first leaves less than
    2^-7 of it, of which the second keeps all but 2^-9, and 2^-20 more: 2^-15 covers both.  Binary16: 2^-10, of which cutting off loses 2^-10 at most: 2^-20, and,
    where that is a subnormal, 2^-24 of numbers scaled by 2^11, 2^-35 of the reference, which is not above the largest probability, for every row."""
    q, dtype = f64(q), got.dtype
    keys = [[f64(x) for x in side] for side in keys]
    exact, size, score = po.decode(q, *keys, scale, lengths)
    got = f64(got)
    n = max(max(lengths), 1)
    relative = 2 * (q.shape[2] + 4) * 2.0 ** -23 * score * abs(scale) + 2.0 ** -19 + (n / 32 + 64) * 2.0 ** -23 + (2.0 ** -15 if cache_dtype == "bf16" else 2.0 ** -20)
    most = max((float(np.abs(x).max()) for x in keys[1] if x.size), default=0.0)
    bound = half_step(dtype) * np.abs(exact) * (1 + 2.0 ** -9) + (relative[..., None] * 2 + 2.0 ** -24) * size + smallest(dtype) + n * 2.0 ** -35 * most
    rows = [r for r in range(len(lengths)) if r not in skip]
    off = np.abs(got - exact)[rows]
    assert np.isfinite(got[rows]).all() and (off <= bound[rows]).all(), float((off / bound[rows]).max())


def widened(cache, table):
    """The table in one so wide that its rows, if they were all held, would be more than attn_decode's kernels are left with (192 MiB): what is read once for
    a group is read by kernels of its own then."""
    pages = 2 ** 28 // (table.shape[0] * cache.heads * cache.page_size * 4 * cache.d) + 1
    wide = torch.full((table.shape[0], max(pages, table.shape[1])), POISON, dtype=torch.int32, device="cuda")
    wide[:, :table.shape[1]] = table
    return wide


def attend(case, q, scale, **kw):
    cache, table, lengths, offsets, shared, _ = case
    return binding.attn_decode_shared(q, cache, widened(cache, table), up(lengths), offsets, shared, scale=scale, **kw)


GROUPS = [(0, [5, 9]), (15, [1, 0, 3]), (16, [0, 0]), (16, [1, 40]), (47, [20]), (64, [-1, 3, -1, 200, 0]), (127, [1] * 9), (128, [0, 130]), (129, [2, 300]), (1000, [0, 7, 33, -1]),
          (2049, [31, 32, 33, 500])]


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("G,KH", [(1, 1), (1, 5), (3, 2), (4, 2), (8, 1), (16, 1), (17, 1), (40, 2)])
def test_decode_shared(d, dtype, G, KH):
    ps = {1: 16, 3: 16, 4: 32, 8: 64, 16: 16, 17: 16, 40: 128}[G]
    case = fill_groups(GROUPS, [0, 1, 77, 2000], KH, d, ps, dtype, seed=G * d, page_first=G == 4)
    cache, table, lengths, offsets, shared, keys = case
    R = len(lengths)
    q = queries(R, G * KH, d, dtype, seed=1)
    got = attend(case, q, d ** -0.5)
    check_shared(got, q, keys, d ** -0.5, lengths, dtype)
    assert all((got[r] == 0).all() for r in range(R) if lengths[r] == 0)
    check_shared(binding.attn_decode_shared(q, cache, table, up(lengths), offsets, shared, scale=d ** -0.5), q, keys, d ** -0.5, lengths, dtype)
    # the same bits whatever the table's rows and the strides of Q and O are
    table = widened(cache, table)
    wide_table = torch.full((R, table.shape[1] + 3), POISON, dtype=torch.int32, device="cuda")
    wide_table[:, :table.shape[1]] = table
    qs = torch.full((G * KH, R, d + 8), float("nan"), dtype=q.dtype, device="cuda")[:, :, :d].transpose(0, 1)
    qs.copy_(q)
    os_ = torch.full((R, G * KH + 1, d), 3.0, dtype=q.dtype, device="cuda")
    need = binding.attn_decode_shared_workspace_bytes(R, G * KH, shared.numel(), cache, table.shape[1])
    workspace = torch.full((need + 64,), 0xff, dtype=torch.uint8, device="cuda")
    binding.attn_decode_shared(qs, cache, wide_table[:, :table.shape[1]], up(lengths), offsets, shared, os_[:, :-1], scale=d ** -0.5, workspace=workspace[:need])
    assert torch.equal(os_[:, :-1], got) and (os_[:, -1] == 3.0).all() and (workspace[need:] == 0xff).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,out", [("f16", "f32"), ("bf16", "f32"), ("bf16", "f16"), ("f16", "bf16")])
@pytest.mark.parametrize("scale", [0.0, -0.11, 1.0])
def test_decode_shared_outputs_and_scales(dtype, out, scale):
    case = fill_groups(GROUPS, [33], 2, 128, 16, dtype, seed=2)
    q = queries(len(case[2]), 6, 128, dtype, seed=3)
    check_shared(attend(case, q, scale, o_dtype=DTYPES[out]), q, case[5], scale, case[2], dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("groups,KH,G,d", [([(16, [0] * 2)], 1, 1, 64), ([(200, [1] * 100)], 2, 4, 128), ([(4096, [100] * 70)], 1, 8, 64), ([(30000, [5, 1000, 77, 0])], 2, 4, 128),
                                          ([(64 * i, [i, 2 * i, 0]) for i in range(1, 60)], 1, 2, 64), ([(100000, [3, 3])], 1, 1, 128), ([(33, [2])] * 300, 1, 3, 64),
                                          ([(160, [1, 2])] * 1500, 1, 1, 64), ([(0, [20] * 4)] * 3, 8, 4, 128), ([(700, [1] * 5)] * 40, 8, 7, 128),
                                          ([(64, [1] * 64)] * 64, 1, 1, 128), ([(0, [1])] * 4096, 1, 1, 64), ([(32, [5, 9] * 20)] * 3, 2, 33, 128), ([(1500, [700] * 90)], 1, 2, 64),
                                          ([(0, [1])] * 4094 + [(48, [1, 2])], 1, 40, 128),
                                          ([(1000, [1] * 40), (900, [5, 0]), (1500, [9] * 6), (0, [700]), (1200, [3] * 11)] * 6, 2, 4, 128)])
def test_decode_shared_sizes(groups, KH, G, d):
    """One step to a workgroup and many, one unit and thousands, groups that a unit holds and groups of many units."""
    case = fill_groups(groups, [], KH, d, 16, "bf16", seed=len(groups))
    q = queries(len(case[2]), G * KH, d, "bf16", seed=1)
    got = attend(case, q, d ** -0.5)
    check_shared(got, q, case[5], d ** -0.5, case[2], "bf16")
    for _ in range(3):
        assert torch.equal(attend(case, q, d ** -0.5), got)


@pytest.mark.gpu
@pytest.mark.parametrize("lengths,KH,G,d", [([300, 310, 0, 299], 8, 4, 64), ([1], 1, 1, 128), ([2000] * 4, 8, 4, 128), ([500] * 40, 8, 4, 128)])
def test_decode_shared_of_little(lengths, KH, G, d):
    """What is not worth kernels of its own: the bits of attn_decode, over a workspace made for more."""
    case = fill_groups([(290 if n > 290 else 0, [max(x - 290, -1) for x in lengths]) for n in lengths[:1]], [], KH, d, 16, "bf16", seed=3)
    cache, table, lengths, offsets, shared, _ = case
    q = queries(len(lengths), G * KH, d, "bf16", seed=4)
    workspace = torch.full((binding.attn_decode_shared_workspace_bytes(64, G * KH, 8, cache, 4096),), 0xff, dtype=torch.uint8, device="cuda")
    got = binding.attn_decode_shared(q, cache, table, up(lengths), offsets, shared, scale=0.1, workspace=workspace)
    assert torch.equal(got, binding.attn_decode(q, cache, table, up(lengths), scale=0.1))


@pytest.mark.gpu
def test_decode_shared_takes_less_than_there_is():
    """Any number up to what is shared, any groups within the groups, and offsets that are none: the same result up to rounding."""
    case = fill_groups([(500, [3, 40, 0, 9, 200, -1, 1]), (300, [10] * 6)], [70], 2, 64, 16, "f16", seed=4)
    cache, table, lengths, offsets, shared, keys = case
    R = len(lengths)
    q = queries(R, 8, 64, "f16", seed=5)
    for off, sh in (([0, 7, 13], [0, 0]), ([0, 7, 13], [17, 299]), ([0, 7, 13], [2 ** 31 - 1, -5]), ([0, 3, 5, 7, 7, 11, 13], [500, 400, 30, 9, 300, 100]), ([2, 6], [496]),
                    ([0, 7, 5, 13], [500, 500, 300]), ([-4, 7, 99], [500, 300]), ([13, 14], [64]), ([0, 0], [3])):
        got = binding.attn_decode_shared(q, cache, widened(cache, table), up(lengths), up(off), up(sh), scale=0.125)
        skip = (13,) if off == [-4, 7, 99] else ()      # (that group takes in the request behind it, which shares nothing with it)
        check_shared(got, q, keys, 0.125, lengths, "f16", skip=skip)


@pytest.mark.gpu
def test_decode_shared_whatever_the_tables_hold():
    """Lengths outside the tables count as their ends; a page outside the cache makes those NaN that see it, and no others.  (Tables that are full, and long enough.)"""
    n = 2 ** 28 // (16 * 8 * 4 * 64) // 16 * 16
    case = fill_groups([(n - 32, [32] * 6 + [9]), (n - 32, [0, 20])], [n, n - 5, 0, 0, n, 1, 2], 8, 64, 16, "f16", seed=7)
    cache, table, lengths, offsets, shared, keys = case
    assert table.shape[1] * 16 == n
    q = queries(16, 16, 64, "f16", seed=8)
    given = up([2 ** 31 - 1 if x == n else -9 if x == 0 else x for x in lengths])
    table[0, n // 16 - 1], table[7, 5] = cache.pages, -1      # behind the rows in common of the first group; among those of the second
    got = binding.attn_decode_shared(q, cache, table, given, offsets, shared, scale=0.125)
    check_shared(got, q, keys, 0.125, lengths, "f16", skip=(0, 7, 8))
    assert got[0].isnan().all() and got[7].isnan().all()
    assert (got[11] == 0).all()
    empty = binding.attn_decode_shared(q, cache, table, up([-1, 0, 0, -2 ** 31] * 4), offsets, shared, scale=0.125)
    assert (empty == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("common", [64, 5008])
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_decode_shared_keeps_what_is_no_number_to_itself(d, common, dtype):
    """NaN and infinities among the visible rows reach those that see them and no others; queries that are none, their own row only."""
    case = fill_groups([(common, [5, 20, 7]), (common, [5, 20, 7])], [], 2, d, 16, dtype, seed=8)
    cache, table, lengths, offsets, shared, keys = case
    q = queries(6, 4, d, dtype, seed=6)
    q[5, 1] = float("nan")
    cache.k[int(table[0, 3]), 0, 5, 11] = float("nan")                     # first group, key head 0
    cache.v[int(table[3, 2]), 1, 2, 7] = float("nan")                      # second group, key head 1, element 7
    cache.v[int(table[3, 1]), 0, 3, 9] = float("inf")                      # second group, key head 0, element 9
    cache.v[int(table[4, (common + 1) // 16]), 1, (common + 1) % 16, 5] = float("-inf")      # request 4's own row
    got = attend(case, q, d ** -0.5)
    assert got[:3, :2].isnan().all() and got[3:, 2:, 7].isnan().all() and got[5, 1].isnan().all()
    assert (got[3:5, :2, 9] == math.inf).all() and got[5, 0, 9] == math.inf and (got[4, 2:, 5] == -math.inf).all()
    ok, clean = got.clone(), q.clone()
    clean[5, 1] = 0
    exact, _, _ = po.decode(f64(clean), *[[f64(x) for x in side] for side in keys], d ** -0.5, lengths)
    for x in (ok, exact):
        x[:3, :2], x[3:, 2:, 7], x[5, 1], x[3:, :2, 9], x[4, 2:, 5] = 0, 0, 0, 0, 0
    assert np.abs(f64(ok) - exact).max() <= half_step(DTYPES[dtype]) * 2 * np.abs(exact).max()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_decode_shared_peaks(dtype):
    """A row that outweighs all others, in the common rows or behind them, and references that rise from tile to tile."""
    d, n = 64, 3008
    case = fill_groups([(n, [40, 40, 40, 40])], [], 1, d, 16, dtype, seed=9)
    cache, table, lengths, offsets, shared, keys = case
    q = queries(4, 1, d, dtype, seed=6)
    for r, at in ((0, 5), (1, n - 1), (2, n + 30), (3, 1500)):
        x = q[r, 0].float()
        k = (x * (14.0 / 0.125 / (x @ x))).to(q.dtype)      # a score of 14
        for s in range(4):
            if at < n or s == r:
                keys[0][s][at, 0] = k
        cache.k[int(table[r, at // 16]), 0, at % 16] = k
    got = attend(case, q, 0.125, o_dtype=torch.float32)
    check_shared(got, q, keys, 0.125, lengths, dtype)


@pytest.mark.gpu
def test_decode_shared_far_into_a_large_cache():
    """Common and own pages more than 2^32 bytes from the front, beside the same in a small cache: the same bits."""
    KH, ps, d = 8, 64, 128
    small = fill_groups([(700, [10, 90, 0, 200])], [300], KH, d, ps, "bf16", seed=10)
    cache, table, lengths, offsets, shared, _ = small
    far = 2 ** 32 // (KH * ps * d * 2) + 3
    k, v = (torch.zeros(far + cache.pages, KH, ps, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    k[far:], v[far:] = cache.k, cache.v
    q = queries(len(lengths), 32, d, "bf16", seed=1)
    want = attend(small, q, 0.1)
    got = binding.attn_decode_shared(q, binding.KVCache(k, v), widened(cache, table + far), up(lengths), offsets, shared, scale=0.1)
    assert torch.equal(got, want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,below", [("f16", 30), ("bf16", 30), ("bf16", 60)])
@pytest.mark.parametrize("G", [1, 9])
def test_decode_shared_infinite_values_of_small_weight(dtype, below, G):
    """An infinite value whose probability is 2^-30 of the largest (bfloat16: 2^-60) makes its element infinite, among the rows in common and behind them."""
    d, n = 128, 1024
    case = fill_groups([(n, [40, 50, 60, 70])], [], 1, d, 16, dtype, seed=9)
    cache, table, lengths, offsets, shared, _ = case
    q = torch.zeros(4, G, d, dtype=DTYPES[dtype], device="cuda")
    q[:, :, 3] = 1.0
    cache.k[:, :, :, 3] = 0.0
    scale = math.log(2.0) / 8      # a key of 8 x in element 3 has a score of x in powers of two
    cache.k[int(table[0, 10]), 0, 7, 3], cache.v[int(table[0, 10]), 0, 7, 5] = -8.0 * below, math.inf
    cache.k[int(table[1, n // 16 + 1]), 0, 2, 3], cache.v[int(table[1, n // 16 + 1]), 0, 2, 6] = -8.0 * below, -math.inf
    got = attend(case, q, scale)
    assert (got[:, :, 5] == math.inf).all() and (got[1, :, 6] == -math.inf).all()
    got[:, :, 5], got[1, :, 6] = 0, 0
    assert got.isfinite().all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("G", [1, 5, 40])
def test_decode_shared_rising_scores(dtype, G):
    """Scores that rise from tile to tile by less and by more than what a reference is raised for, and fall again."""
    d, n = 64, 2048
    case = fill_groups([(n, [100, 100, 3])], [], 1, d, 16, dtype, seed=11)
    cache, table, lengths, offsets, shared, keys = case
    q = queries(3, G, d, dtype, seed=12)
    q[:, :, 0] = 1.0
    level = 10.0 * torch.sin(torch.arange(n + 100, device="cuda") / 300.0) + 6.0 * torch.sin(torch.arange(n + 100, device="cuda") / 7.0)
    for r in range(3):
        m = lengths[r]
        keys[0][r][:, 0, 0] = level[:m].to(q.dtype)
        rows = torch.arange(m, device="cuda")
        cache.k[table[r, rows // 16].long(), 0, rows % 16, 0] = keys[0][r][:, 0, 0]
    check_shared(attend(case, q, 1.0, o_dtype=torch.float32), q, keys, 1.0, lengths, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 6, 12, 32])      # 4, 24, 48 and 128 columns to a unit: every kind of it
def test_decode_shared_rows_of_no_weight(dtype, d, G):
    """One row of small values that has all of the weight, in front of thousands of large ones of one sign whose probabilities are e^-4096 and less: 0 in 32 bits, and
    0 in what enters the second product.  The result is that row.

    |error| <= |row| * (error of its probability in 16-bit parts, as in check_shared: 2^-20 at binary16, 2^-15 at bfloat16, and what a sum of two parts may be raised by, 2^-35;
    sums, factors of at most three joins and the quotient: fewer than 16 roundings of 2^-24)."""
    case = fill_groups([(9008, [700, 20, 5, 40])], [9000], 1, d, 16, dtype, seed=13)
    cache, table, lengths, offsets, shared, _ = case
    q = torch.full((5, G, d), 4096.0 / d / 8, dtype=DTYPES[dtype], device="cuda")
    row = queries(1, 1, d, dtype, seed=14)[0, 0] / 1024
    cache.k.zero_()
    cache.v.fill_(60000.0 if dtype == "f16" else 2.0 ** 100)
    for r in (0, 4):      # all of a group have the first page in common
        cache.k[int(table[r, 0]), 0, 3], cache.v[int(table[r, 0]), 0, 3] = 8.0, row
    got = f64(attend(case, q, 1.0, o_dtype=torch.float32))
    off = np.abs(got - f64(row)) / np.abs(f64(row))
    assert (off <= (2.0 ** -20 if dtype == "f16" else 2.0 ** -15) + 2.0 ** -35 + 2.0 ** -20).all(), off.max()


@pytest.mark.gpu
@pytest.mark.parametrize("G", [1, 12])
@pytest.mark.parametrize("scale", [0.0, 1e-36, -1e-36, 3e-34])
def test_decode_shared_scales_next_to_nothing(scale, G):
    """Scales so small that only products of queries and keys next to the largest numbers of 32 bits make a difference (none at scale 0): as in attn_decode."""
    d = 64
    case = fill_groups([(3008, [100, 5, 40, 0, 7, 9]), (160, [3, 8])], [500], 1, d, 16, "bf16", seed=15)
    cache, table, lengths, offsets, shared, keys = case
    R = len(lengths)
    q = torch.zeros(R, G, d, dtype=torch.bfloat16, device="cuda")
    q[:, :, 5] = 2.0 ** 62
    cache.k *= 2.0 ** 61      # (a product is up to 2^126)
    for x in keys[0]:
        x *= 2.0 ** 61
    got = attend(case, q, scale, o_dtype=torch.float32)
    check_shared(got, q, keys, scale, lengths, "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 12, 24, 40])      # 2, 24, 48 and 80 columns to a unit: every kind of it
def test_decode_shared_values_next_to_the_largest(G, d):
    """bfloat16 values that may not grow by the weight of their rows: of 100000 rows some have scores above those of the rows in front of them, by less than what a
    reference is raised for, and values next to the largest there are.  Each has an element to itself, where O is their value times their probability.

    |error| <= relative error of a probability, as in check_shared: 2^-15 for its parts, 2^-19 for exp2, one addition for every 32 rows and joining; the
    scores are exact."""
    n, own, most = 100032, 4000, 1.5 * 2.0 ** 126
    case = fill_groups([(n, [own, 0])], [n], 1, d, 64, "bf16", seed=16)
    cache, table, lengths, offsets, shared, _ = case
    q = torch.zeros(3, G, d, dtype=torch.bfloat16, device="cuda")
    q[:, :, 3] = 1.0
    cache.k.zero_()
    cache.v.zero_()
    heavy = [(0, n * i // 20 + 77, 8 + i) for i in range(20)] + [(0, n + 2000 + 300 * i, 30 + i) for i in range(3)] + [(2, n * i // 20 + 77, 8 + i) for i in range(20)]
    for r, at, element in heavy:
        cache.k[int(table[r, at // 64]), 0, at % 64, 3], cache.v[int(table[r, at // 64]), 0, at % 64, element] = 56.0, most
    got = f64(attend(case, q, math.log(2.0) / 8, o_dtype=torch.float32))      # a key of 56 in element 3: a score of 7 in powers of two
    for r in range(3):
        seen = {element for s, at, element in heavy if (s, r) in ((0, 0), (0, 1), (2, 2)) and at < lengths[r]}
        want = np.zeros(d)
        want[sorted(seen)] = most * 128.0 / (128 * len(seen) + lengths[r] - len(seen))
        assert (np.abs(got[r] - want) <= (2.0 ** -15 + 2.0 ** -19 + (n / 32 + 64) * 2.0 ** -23) * want).all(), (r, got[r, 0], want)


@pytest.mark.gpu
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("G", [1, 6, 12, 32])
def test_decode_shared_keys_of_the_lowest_value(G, d):
    """Rows masked by the lowest number there is in their keys, whole tiles and units of them, at a scale at which their scores are no numbers of 32 bits: they have no weight."""
    n, hidden = 5008, 3000
    case = fill_groups([(n, [700, 20, 5, 400])], [6000], 1, d, 16, "bf16", seed=17)
    cache, table, lengths, offsets, shared, keys = case
    q = queries(5, G, d, "bf16", seed=18) / 8
    q[:, :, 3] = 1.0
    lowest = torch.finfo(torch.bfloat16).min
    for r, low, high in ((0, 0, hidden), (0, n, n + 500), (3, n, n + 400), (4, 700, 6000 - 100)):
        for at in range(low, high):
            cache.k[int(table[r, at // 16]), 0, at % 16] = 0.0
            cache.k[int(table[r, at // 16]), 0, at % 16, 3] = lowest
    seen = [np.r_[hidden:n, n + 500:n + 700], np.r_[hidden:n + 20], np.r_[hidden:n + 5], np.r_[hidden:n], np.r_[0:700, 5900:6000]]
    kept = [[x[torch.as_tensor(rows, device=x.device)] for x, rows in zip(side, seen)] for side in keys]
    check_shared(attend(case, q, 1.0, o_dtype=torch.float32), q, kept, 1.0, [len(rows) for rows in seen], "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("scale", [0.125, 0.0884, 0.7, -0.31])
@pytest.mark.parametrize("d,G", [(64, 1), (128, 6), (64, 12), (128, 32)])
def test_decode_shared_keys_of_the_lowest_value_at_other_scales(d, G, scale):
    """The same where the masked rows' scores are numbers, of which the last bit is more than any exponent: they have no weight beside others, and all of it, alike, in a request
    that sees nothing else."""
    n, hidden = 5008, 3000
    case = fill_groups([(n, [700, 20, 5, 400])], [6000, 4000], 1, d, 16, "bf16", seed=19)
    cache, table, lengths, offsets, shared, keys = case
    q = queries(6, G, d, "bf16", seed=20)
    q[:, :, 3] = (1.0 + torch.arange(G, device="cuda") / 64).bfloat16() * 0.6
    masked = torch.finfo(torch.bfloat16).min * (1 if scale > 0 else -1)
    for r, low, high in ((0, 0, hidden), (0, n, n + 500), (3, n, n + 400), (4, 700, 6000 - 100), (5, 0, 4000)):
        for at in range(low, high):
            cache.k[int(table[r, at // 16]), 0, at % 16] = 0.0
            cache.k[int(table[r, at // 16]), 0, at % 16, 3] = masked
    seen = [np.r_[hidden:n, n + 500:n + 700], np.r_[hidden:n + 20], np.r_[hidden:n + 5], np.r_[hidden:n], np.r_[0:700, 5900:6000], np.r_[0:4000]]
    kept = [[x[torch.as_tensor(rows, device=x.device)] for x, rows in zip(side, seen)] for side in keys]
    kept[0][5] = torch.zeros_like(kept[0][5])      # rows of the same score, whatever it is
    check_shared(attend(case, q, scale, o_dtype=torch.float32), q, kept, scale, [len(rows) for rows in seen], "bf16")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("scale", [1.0, 0.3, 11.0, -0.7])
@pytest.mark.parametrize("d,G", [(64, 1), (128, 6), (64, 12), (128, 32)])
def test_decode_shared_scores_beyond_all_exponents(dtype, scale, d, G):
    """Scores of two sizes, both so large that the last bit of a scaled one is more than any exponent.  The rows of the larger have all of the weight and share it, so O is the
    mean of their values.  |error| as in check_shared, without that of the scores, which are alike."""
    n = 5008
    case = fill_groups([(n, [700, 20, 5, 400])], [6000], 1, d, 16, dtype, seed=21)
    cache, table, lengths, offsets, shared, keys = case
    q = torch.zeros(5, G, d, dtype=DTYPES[dtype], device="cuda")
    q[:, :, 3] = 24576.0 if dtype == "f16" else 3.0 * 2.0 ** 55
    more, less = (27648.0, 26624.0) if dtype == "f16" else (27.0 * 2.0 ** 55, 26.0 * 2.0 ** 55)
    rng, large = np.random.default_rng(1), []
    for r in range(5):
        which = rng.random(lengths[r]) < 0.3
        which[:200] = False
        if 0 < r < 4:
            which[:n] = large[0][:n]
        large.append(which)
        at = torch.arange(0 if r in (0, 4) else n, lengths[r], device="cuda")
        cache.k[table[r, at // 16].long(), 0, at % 16, 3] = torch.tensor(np.where(which, more, less)[at.cpu()], device="cuda").to(q.dtype)
    got = f64(attend(case, q, scale, o_dtype=torch.float32))
    for r in range(5):
        v = f64(keys[1][r])[large[r] if scale > 0 else ~large[r], 0]
        bound = (2.0 ** -15 if dtype == "bf16" else 2.0 ** -20) + 2.0 ** -19 + (n / 32 + 64) * 2.0 ** -23
        assert (np.abs(got[r] - v.mean(0)) <= 2 * bound * np.abs(v).mean(0)).all(), (r, got[r, 0, :4], v.mean(0)[:4])


# ------------------------------------------------------------------------------------------- all of them together

class Beams:
    """A search as a program runs it: prompts, beams that branch off them, and per step a fork by given sources, copies, a token each, attention; and what
    every beam's keys and values are, on the host."""

    def __init__(self, prompts, beams, H, KH, d, ps, dtype, seed, wide):
        self.H, self.KH, self.d, self.ps, self.beams, self.wide = H, KH, d, ps, beams, wide
        self.R = R = len(prompts) * beams
        self.pages = 4 * R + sum(-(-(n + 400) // ps) for n in prompts) * 2 + R * 8
        g = torch.Generator("cuda").manual_seed(seed)
        dt = DTYPES[dtype]
        self.layers = [binding.KVCache(*(torch.full((self.pages, KH, ps, d), float("nan"), dtype=dt, device="cuda") for _ in range(2))) for _ in range(2)]
        self.both = binding.KVLayers(self.layers)
        self.ring, state = torch.randperm(self.pages, generator=g, device="cuda").int(), up([0, self.pages])
        # the prompts, in every layer
        table, lengths, n = torch.full((len(prompts), wide), POISON, dtype=torch.int32, device="cuda"), up([0] * len(prompts)), sum(prompts)
        page = binding.attn_kv_pages(lengths, up(prompts), table, self.ring, state, page_size=ps, tokens=n)
        self.history = [[None] * R for _ in self.layers]
        for cache, kept in zip(self.layers, self.history):
            qkv = torch.randn(n, H + 2 * KH, d, generator=g, device="cuda").to(dt)
            q, k, v = qkv.split((H, KH, KH), 1)
            binding.attn_qkv_prepare(q, k, v, positions=page.positions, cache=cache, slots=page.slots)
            at = np.concatenate([[0], np.cumsum(prompts)])
            for r in range(R):
                p = r // beams
                kept[r] = (k[at[p]:at[p + 1]].clone(), v[at[p]:at[p + 1]].clone())
        self.offsets = up(np.arange(len(prompts) + 1) * beams)
        # two sets of what a fork writes beside what it reads
        self.sets = [dict(table=torch.full((R, wide), POISON, dtype=torch.int32, device="cuda"), lengths=up([0] * R), state=up([0, 0])) for _ in range(2)]
        start = binding.attn_kv_fork(page.lengths, up(np.repeat(np.arange(len(prompts)), beams)), table, self.ring, page.free_state, page_size=ps, pages=self.pages,
                                     table_out=self.sets[0]["table"], lengths_out=self.sets[0]["lengths"], free_state_out=self.sets[0]["state"])
        binding.attn_kv_copy(self.both, start.copies)
        self.workspace = [torch.full((binding.attn_decode_shared_workspace_bytes(R, H, len(prompts), self.layers[0], wide),), 0xff, dtype=torch.uint8, device="cuda"),
                          torch.full((binding.attn_kv_fork_workspace_bytes(R, R, self.pages),), 0xff, dtype=torch.uint8, device="cuda")]
        self.one = up([1] * R)

    def step(self, which, source, qkv):
        """A step from set `which` into the other one: O of each layer."""
        old, new = self.sets[which], self.sets[1 - which]
        fork = binding.attn_kv_fork(old["lengths"], source, old["table"], self.ring, old["state"], page_size=self.ps, pages=self.pages, table_out=new["table"], workspace=self.workspace[1])
        binding.attn_kv_copy(self.both, fork.copies)
        page = binding.attn_kv_pages(fork.lengths, self.one, new["table"], self.ring, fork.free_state, page_size=self.ps, tokens=self.R, lengths_out=new["lengths"],
                                     free_state_out=new["state"])
        shared = binding.attn_kv_shared_rows(new["table"], new["lengths"], self.offsets, page_size=self.ps)
        out = []
        for cache, x in zip(self.layers, qkv):
            q, k, v = x.split((self.H, self.KH, self.KH), 1)
            q, _, _ = binding.attn_qkv_prepare(q, k, v, positions=page.positions, cache=cache, slots=page.slots)
            out.append(binding.attn_decode_shared(q, cache, new["table"], new["lengths"], self.offsets, shared, scale=self.d ** -0.5, workspace=self.workspace[0]))
        return out, shared

    def follow(self, source, qkv):
        """The same on the host's side."""
        for i, x in enumerate(qkv):
            k, v = x[:, self.H:self.H + self.KH], x[:, self.H + self.KH:]
            self.history[i] = [tuple(torch.cat([a, b[r:r + 1]]) for a, b in zip(self.history[i][s], (k, v))) for r, s in enumerate(source)]

    def inputs(self, rng, g):
        source = np.concatenate([p * self.beams + rng.integers(0, self.beams, self.beams) for p in range(self.R // self.beams)])
        return source, [torch.randn(self.R, self.H + 2 * self.KH, self.d, generator=g, device="cuda").to(self.layers[0].dtype) for _ in self.layers]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,prompts,beams,H,KH,d,ps,wide", [("bf16", [77, 300], 4, 6, 2, 64, 16, 40), ("f16", [500, 16, 1], 16, 16, 8, 128, 32, 300),
                                                               ("bf16", [1300, 900], 20, 32, 8, 128, 16, 100)])
def test_a_search(dtype, prompts, beams, H, KH, d, ps, wide):
    """Beams that branch, go on and end for some pages: every step's attention against each beam's own keys and values, kept apart; no page lost."""
    rng, g = np.random.default_rng(1), torch.Generator("cuda").manual_seed(2)
    b = Beams(prompts, beams, H, KH, d, ps, dtype, seed=3, wide=wide)
    for i in range(2 * ps + 6):
        source, qkv = b.inputs(rng, g)
        out, shared = b.step(i % 2, up(source), qkv)
        b.follow(source, qkv)
        now = b.sets[1 - i % 2]
        lengths = now["lengths"].tolist()
        assert lengths == [prompts[r // beams] + i + 1 for r in range(b.R)]
        assert all(s >= n // ps * ps for s, n in zip(shared.tolist(), prompts))
        if i in (0, 1, ps - 1, ps, 2 * ps + 4, 2 * ps + 5):
            for layer, o in enumerate(out):
                check_shared(o, qkv[layer][:, :H], [[kv[j] for kv in b.history[layer]] for j in range(2)], d ** -0.5, lengths, dtype)
        held = {p for r in range(b.R) for p in now["table"][r, :-(-lengths[r] // ps)].tolist()}
        assert len(held) + int(now["state"][1]) == b.pages


@pytest.mark.gpu
def test_a_search_captured():
    """Two steps captured into a graph, replayed with new sources and tokens, eager work and synchronizations between; every replay against a search that
    makes the calls one by one."""
    a, b = (Beams([1500, 700], 16, 32, 8, 128, 16, "bf16", seed=3, wide=110) for _ in range(2))
    rng, g = np.random.default_rng(4), torch.Generator("cuda").manual_seed(5)
    sources = [up([0] * a.R) for _ in range(2)]
    first = [a.inputs(rng, g) for _ in range(2)]
    qkv = [[x.clone() for x in f[1]] for f in first]
    for s, f in zip(sources, first):
        s.copy_(up(f[0]))
    out = [b.step(i, sources[i], qkv[i])[0] for i in range(2)]      # (eagerly once, so that everything is loaded; on `a` it is the graph that steps)
    kept = [{n: t.clone() for n, t in s.items()} for s in a.sets], a.ring.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = [a.step(i, sources[i], qkv[i])[0] for i in range(2)]
    assert torch.equal(kept[1], a.ring)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for o, p in zip(outs, out) for x, y in zip(o, p))
    for _ in range(12):
        for i in range(2):
            s, x = a.inputs(rng, g)
            sources[i].copy_(up(s))
            for t, y in zip(qkv[i], x):
                t.copy_(y)
        want = [b.step(i, sources[i], qkv[i])[0] for i in range(2)]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(x, y) for o, p in zip(outs, want) for x, y in zip(o, p))
        assert all(torch.equal(x[n], y[n]) for x, y in zip(a.sets, b.sets) for n in ("lengths", "state")) and torch.equal(a.ring, b.ring)


@pytest.mark.gpu
def test_many_requests_captured():
    """Forks and common rows that take several launches, captured, replayed with new inputs and with eager work between, against the calls made one by one."""
    rng = np.random.default_rng(9)
    R, wide = 1100, 130
    lengths, source, rows, table, ring, state, ps, pages = fork_case(rng, R, R, 16, 16 * wide - 20)
    wide = table.shape[1]
    assert R * wide > 2 ** 17
    given = {"lengths": up(lengths), "source": up(source), "rows": up(rows), "table": up(table), "ring": up(ring), "state": up(state), "groups": up([0, R])}

    def calls(x, out):
        fork = binding.attn_kv_fork(x["lengths"], x["source"], x["table"], x["ring"], x["state"], page_size=ps, pages=pages, rows=x["rows"], table_out=out["table"],
                                    lengths_out=out["lengths"], copies=out["copies"], free_state_out=out["state"], workspace=out["workspace"])
        binding.attn_kv_shared_rows(x["table"], x["lengths"], x["groups"], page_size=ps, shared=out["shared"])
        return fork

    def outputs():
        i32 = {"dtype": torch.int32, "device": "cuda"}
        return {"table": torch.full((R, wide), POISON, **i32), "lengths": torch.full((R,), POISON, **i32), "copies": torch.full((R, 3), POISON, **i32), "state": torch.full((2,), POISON, **i32),
                "shared": torch.full((1,), POISON, **i32), "workspace": torch.full((binding.attn_kv_fork_workspace_bytes(R, R, pages),), 0xff, dtype=torch.uint8, device="cuda")}
    mine, apart = {n: t.clone() for n, t in given.items()}, outputs()
    calls(mine, outputs())      # (so that everything is loaded)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls(mine, apart)
    for trial in range(6):
        same = (0, 50, wide, 1, 17, 0)[trial]
        changed = {n: t.clone() for n, t in given.items()}
        changed["table"][:, :same] = changed["table"][0, :same]
        changed["lengths"].copy_(torch.where(changed["lengths"] > 0, 16 * (wide - 1) + 3, 0) if trial % 2 else given["lengths"].roll(trial))
        changed["source"].copy_(given["source"].roll(7 * trial))
        for n, t in changed.items():
            mine[n].copy_(t)
        for t in apart.values():
            t.fill_(POISON if t.dtype == torch.int32 else 0xff)
        graph.replay()
        want = outputs()
        calls(changed, want)
        torch.cuda.synchronize()
        assert all(torch.equal(apart[n], want[n]) for n in want if n != "workspace") and torch.equal(mine["ring"], changed["ring"]), trial
        assert want["shared"].tolist() == so.shared_rows(changed["table"].cpu().numpy(), changed["lengths"].tolist(), [0, R], ps), trial


@pytest.mark.gpu
def test_searches_on_streams_of_their_own():
    """Two searches at once on two streams, each with its own workspaces, and calls that are given their stream: the results of one after the other."""
    make = lambda i: Beams([1500, 700 + i], 16, 32, 8, 128, 16, "bf16", seed=3 + i, wide=110)
    at_once, plain = [make(0), make(1)], [make(0), make(1)]
    streams, rng, g = [torch.cuda.Stream(), torch.cuda.Stream()], np.random.default_rng(4), torch.Generator("cuda").manual_seed(5)
    work = [[a.inputs(rng, g) for _ in range(6)] for a in at_once]
    work = [[(up(s), x) for s, x in w] for w in work]
    want = [[p.step(i % 2, *w[i])[0] for i in range(6)] for p, w in zip(plain, work)]
    torch.cuda.synchronize()
    got = [[], []]
    for i in range(6):
        for j in range(2):
            with torch.cuda.stream(streams[j]):
                got[j].append(at_once[j].step(i % 2, *work[j][i])[0])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for a, b in zip(got, want) for o, p in zip(a, b) for x, y in zip(o, p))
    b, old = plain[0], plain[0].sets[0]
    q, shared = queries(b.R, 32, 128, "bf16", seed=1), binding.attn_kv_shared_rows(old["table"], old["lengths"], b.offsets, page_size=16)
    eager = binding.attn_decode_shared(q, b.layers[0], old["table"], old["lengths"], b.offsets, shared, scale=0.1, workspace=b.workspace[0])
    fork = binding.attn_kv_fork(old["lengths"], work[0][0][0], old["table"], b.ring.clone(), old["state"], page_size=16, pages=b.pages)
    torch.cuda.synchronize()
    other = streams[0]
    o = torch.zeros_like(eager)
    torch.cuda.synchronize()
    binding.attn_decode_shared(q, b.layers[0], old["table"], old["lengths"], b.offsets, shared, o, scale=0.1, workspace=b.workspace[0], stream=other)
    again = binding.attn_kv_fork(old["lengths"], work[0][0][0], old["table"], b.ring.clone(), old["state"], page_size=16, pages=b.pages, stream=other)
    s2 = binding.attn_kv_shared_rows(old["table"], old["lengths"], b.offsets, page_size=16, stream=other)
    binding.attn_kv_copy(b.both, torch.full((3, 3), -1, dtype=torch.int32, device="cuda"), stream=other)
    other.synchronize()
    assert torch.equal(o, eager) and torch.equal(s2, shared) and torch.equal(again.lengths, fork.lengths) and torch.equal(again.copies, fork.copies)
    assert torch.equal(again.free_state, fork.free_state)


@pytest.mark.gpu
def test_binding_refusals():
    """What the calls refuse before they reach the library: types, shapes, sizes."""
    case = fill_groups([(20, [3, 4])], [], 2, 64, 16, "f16", seed=1)
    cache, table, lengths, offsets, shared, _ = case
    lens, q = up(lengths), queries(2, 4, 64, "f16", seed=1)
    binding.attn_decode_shared(q, cache, table, lens, offsets, shared, scale=0.1)
    good = dict(q=q, cache=cache, table=table, lengths=lens, offsets=offsets, shared=shared)
    for change in (dict(q=q.float()), dict(q=q[0]), dict(q=q.cpu()), dict(q=q[:, :, :32]), dict(table=table.long()), dict(table=table[:1]), dict(lengths=lens.long()), dict(lengths=lens[:1]),
                   dict(offsets=offsets[:1]), dict(offsets=offsets.long()), dict(shared=shared.cpu()), dict(shared=shared.float()), dict(offsets=offsets.cpu())):
        with pytest.raises(ValueError):
            binding.attn_decode_shared(*{**good, **change}.values(), scale=0.1)
    for kw in (dict(O=q[:1]), dict(O=q.double()), dict(workspace=torch.zeros(9))):
        with pytest.raises(ValueError):
            binding.attn_decode_shared(*good.values(), scale=0.1, **kw)
    with pytest.raises(binding.SawattnError, match="smaller"):
        binding.attn_decode_shared(*good.values(), scale=0.1, workspace=torch.zeros(64, device="cuda"))
    ring, state, src = up(np.arange(9)), up([0, 9]), up([0, 1, 1])
    call = lambda **kw: binding.attn_kv_fork(*[kw.pop(n, x) for n, x in (("lengths", lens), ("source", src), ("table", table), ("ring", ring), ("state", state))],
                                             **{"page_size": 16, "pages": 9, **kw})
    call()
    for change in (dict(lengths=lens.long()), dict(source=src.float()), dict(table=table[:1]), dict(ring=ring.long()), dict(state=ring), dict(rows=lens), dict(table_out=table),
                   dict(table_out=torch.zeros(3, table.shape[1] + 1, dtype=torch.int32, device="cuda")), dict(lengths_out=lens), dict(copies=src), dict(free_state_out=src),
                   dict(workspace=torch.zeros(9)), dict(lengths=lens.cpu()), dict(source=src.cpu())):
        with pytest.raises(ValueError):
            call(**change)
    with pytest.raises(binding.SawattnError, match="overlap"):
        call(free_state_out=state)
    with pytest.raises(binding.SawattnError, match="smaller"):
        call(workspace=torch.zeros(4, device="cuda"))
    for copies in (src.long(), up([1, 2, 3, 4]), src.cpu()):
        with pytest.raises(ValueError):
            binding.attn_kv_copy(cache, copies)
    with pytest.raises(ValueError):
        binding.KVLayers([])
    with pytest.raises(ValueError):
        binding.KVLayers([cache, binding.KVCache(cache.k[:, :1], cache.v[:, :1])])
    for args in ((table, lens.long(), offsets), (table[:1], lens, offsets), (table, lens, offsets.long()), (table, lens.cpu(), offsets)):
        with pytest.raises(ValueError):
            binding.attn_kv_shared_rows(*args, page_size=16)
    with pytest.raises(ValueError):
        binding.attn_kv_shared_rows(table, lens, offsets, page_size=16, shared=lens)


def test_built_kernels_have_no_scratch_memory(tmp_path):
    import re
    from .util import device_code, llvm_tool
    notes = llvm_tool("llvm-readelf", "--notes", device_code(tmp_path))
    found = dict(re.findall(r"\.name:\s+(_ZN7sawattn\d+(?:kv_(?:fork|fork_table|fork_free|fork_few|copy|shared_rows)|decode_shared|decode_shared_join)_kernel\S+)\s+"
                            r"\.private_segment_fixed_size:\s+(\d+)", notes, re.S))
    assert len(found) == 7 + 4 + 4 and set(found.values()) == {"0"}, found


def test_built_wide_kernels_wait_for_what_they_send_to_lds(tmp_path):
    """Between a direct load into LDS and the barrier behind which others read what it brought there is a wait for all of them."""
    import re
    from .util import device_listing, kernel_bodies
    seen = 0
    for kernel, body in kernel_bodies(device_listing(tmp_path)).items():
        if not re.search(r"decode_shared_kernel<\d+, (true|false)>", kernel):
            continue
        flying, loads, barriers = False, 0, 0
        for text, _ in body:
            if text.startswith("global_load_lds_"):
                flying, loads = True, loads + 1
            elif re.match(r"s_waitcnt .*vmcnt\(0\)", text):
                flying = False
            elif text.startswith("s_barrier"):
                assert not flying, kernel
                barriers += 1
        assert loads >= 8 and barriers >= 6, (kernel, loads, barriers)
        seen += 1
    assert seen == 4


def test_beams_study_lists_its_points(capsys):
    from paper_2601_16032_amd import sweeps
    assert sweeps.main(["--study", "beams", "--list"]) == 0
    assert len(capsys.readouterr().out.splitlines()) == len(sweeps.study_points("beams")) == 12


@pytest.mark.gpu
def test_beams_study_runs(capsys):
    """Points of the study `beams`: every operator timed, and the step right, repeated too."""
    import json
    from paper_2601_16032_amd import sweeps
    assert sweeps.main(["--study", "beams", "--points", "0,8", "--launches", "2"]) == 0
    lines = [json.loads(x) for x in capsys.readouterr().out.splitlines() if x.startswith("{")]
    names = ("attn_kv_fork", "attn_kv_copy", "attn_kv_shared_rows", "attn_decode_shared", "attn_decode")
    assert [x["point"] for x in lines] == [0, 8] and all(x[n + "_us"] > 0 for x in lines for n in names)
    calls, held = sweeps.search_step({"prompts": 3, "beams": 20, "common": 1000, "own": 77, "H": 16, "KH": 8, "d": 128}, dtype="f16", seed=3)
    for _ in range(2):
        for _, call in calls:
            call()
    torch.cuda.synchronize()
    cache, fork = held["cache"], held["fork"]
    assert fork.lengths.tolist() == [1077] * 60 and held["shared"].tolist() == [960] * 3
    keys = [[x[t.long()].transpose(1, 2).reshape(-1, 8, 128)[:1077] for t in fork.table] for x in (cache.k, cache.v)]
    parents = [[x[held["table"][int(s)].long()].transpose(1, 2).reshape(-1, 8, 128)[:1077] for s in held["source"]] for x in (cache.k, cache.v)]
    assert all(torch.equal(a, b) for side, kept in zip(keys, parents) for a, b in zip(side, kept))
    check_shared(held["o"], held["q"], keys, 128 ** -0.5, [1077] * 60, "f16")
    check_shared(held["o_apart"], held["q"], keys, 128 ** -0.5, [1077] * 60, "f16")
