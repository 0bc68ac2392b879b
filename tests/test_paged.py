"""GPU parity of the key/value cache in pages with its float64 statements (oracle/nova_paged.py).

Page lists, slots, appended rows, means and chosen pages are exact.  Attention, element by element, with u = 2^-24 (fp32), S the
largest sum_c |q_c k_c| * scale of a query and L keys: a score is a sum of dh products and a factor, off by at most (dh + 8) u S;
2^x adds 4 u and the rounding of its argument, 2 u (S + |lse|); so every probability is off by d = (2 dh + 32) u (S + |lse| + 1) of
itself (numerator and sum), and a sum over L of them is taken in chains of at most L / 2 + 64 roundings.
  out   (2 d + (L + 128) u) w with w = sum_j p_j |v_j|; bf16: probabilities and results are rounded once each, half a step is
        2^-8: + 2^-8 w + 2^-8 |out|, and 2 % for products of the two.  fp32 ends at 2^-126: a term e^(s - max) v, its factor or
        its rescaling below that may become 0, at most 4 * 2^-126 (1 + |v|) each, L of them
  lse   d + (L + 128) u + 8 u |lse|"""
import numpy as np
import pytest
import torch

from oracle import nova_paged as P
from paper_2602_01345_amd import PagedCache

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


@pytest.fixture(scope="module")
def nova():
    import harness
    if not torch.cuda.is_available():
        pytest.fail("GPU tests need a GPU and the built libnova.so (no fallback)")
    return harness.nova()


def _np(t):
    return t.detach().cpu().to(torch.float64).numpy()


def _ints(xs):
    return None if xs is None else torch.tensor(np.asarray(xs), dtype=torch.int32, device="cuda")


# ---- page lists and slots -------------------------------------------------------------------------------------------
def _check_reserve(nova, B, p, pages, pitch, n, kv_len, now, keep, come, free_height, seed, in_place=False, raw=None):
    """now, keep, come: lists or None (as the call takes them), clamped here as the call does."""
    print(f"paged reserve B={B} p={p} pages={pages} n={n} kv_len={kv_len} in_place={in_place}", flush=True)
    g = np.random.default_rng(seed)
    clamp = lambda x, top: [min(max(v, 0), t) for v, t in zip(x, top)]
    now_r = [kv_len] * B if now is None else clamp(now, [kv_len] * B)
    keep_r = now_r if keep is None else clamp(keep, now_r)
    come_r = [n] * B if come is None else clamp(come, [n] * B)
    table = g.integers(-5, pages + 5, (B, pitch))
    ids, used = g.permutation(pages), 0
    for b, r in enumerate(now_r):
        m = -(-r // p)
        table[b, :m] = ids[used:used + m]
        used += m
    assert used <= pages and free_height <= pages - used
    free = np.full(pages, -9)
    free[:free_height] = ids[used:used + free_height]
    want = P.reserve(table, p, free, free_height, now_r, keep_r, come_r, n)
    tt, ft = _ints(table), _ints(free)
    slots = torch.full((B, n), -77, dtype=torch.int32, device="cuda")
    lens, count = _ints(now), _ints([free_height])
    nxt = lens if in_place and lens is not None else torch.full((B,), -7, dtype=torch.int32, device="cuda")
    fnx = None if in_place else torch.full((1,), -7, dtype=torch.int32, device="cuda")
    nova.paged_reserve(tt, p, n, kv_len, ft, count, nxt, fnx, slots=slots, kv_len_per_row=lens, n_per_row=_ints(come),
                       keep_per_row=_ints(keep))
    assert tt.cpu().numpy().tolist() == want[0].tolist()
    assert np.array_equal(slots.cpu().numpy(), want[1])
    assert nxt.tolist() == want[2]
    assert ft.cpu().numpy().tolist() == want[3].tolist()
    assert (count if fnx is None else fnx).item() == want[4]


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("p", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("B,n,kv_len", [(1, 1, 0), (1, 1, 16), (1, 33, 31), (3, 1, 47), (7, 5, 100), (9, 0, 300), (5, 300, 0), (70, 3, 64)])
def test_reserve(nova, in_place, p, B, n, kv_len):
    pitch = -(-(kv_len + n) // p) + 2
    g = np.random.default_rng(B * 1000 + n)
    now = [int(x) for x in g.integers(0, kv_len + 1, B)]
    keep = [int(x) for x in g.integers(-3, kv_len + 4, B)]
    come = [int(x) for x in g.integers(-2, n + 3, B)]
    most = B * pitch
    for seed, (a, k, c) in enumerate(((None, None, None), (now, None, None), (now, keep, come), (now, [0] * B, [0] * B), (None, keep, None),
                                      ([kv_len + 50] * B, None, come))):
        held = sum(-(-min(max(x, 0), kv_len) // p) for x in (a if a is not None else [kv_len] * B))
        for free in {most, 1, B // 2, 0}:
            _check_reserve(nova, B, p, held + most + 3, pitch, n, kv_len, a, k, c, free, seed, in_place)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("B,n,kv_len", [(4096, 1, 40), (4096, 2, 40), (1500, 7, 90), (3, 5000, 700), (600, 64, 64)])
def test_reserve_of_many(nova, in_place, B, n, kv_len):
    """More than one workgroup's worth of entries, images beyond one pass over them."""
    p = 16
    pitch = -(-(kv_len + n) // p)
    g = np.random.default_rng(B)
    now, keep, come = ([int(x) for x in g.integers(0, top + 1, B)] for top in (kv_len, kv_len, n))
    held = sum(-(-x // p) for x in now)
    for free in (B * pitch, B, 0):
        _check_reserve(nova, B, p, held + B * pitch, pitch, n, kv_len, now, keep, come, free, 5, in_place)


def test_reserve_with_counts_and_entries_that_are_none(nova):
    """A stack's height past its ends, pages that are no pages of the pool, stacks that would grow past the pool: nothing is written
    out of bounds, and no slot lies out of the pool."""
    for height in (-4, 99, 2 ** 31 - 1):
        table, free = _ints([[50, -3, 7], [1, -1, -1]]), _ints([4, 5, 6, 7])
        count, nxt = _ints([height]), _ints([0, 0])
        slots = torch.full((2, 20), 5, dtype=torch.int32, device="cuda")
        nova.paged_reserve(table, 16, 20, 28, free, count, nxt, None, slots=slots, kv_len_per_row=_ints([28, 3]))
        assert ((slots == -1) | ((slots >= 0) & (slots < 64))).all() and 0 <= count.item() <= 4
        got = slots.cpu().numpy()
        assert (got[0, :4] == -1).all() and got[1, :13].tolist() == list(range(16 + 3, 32))
    free, count, nxt = _ints([4, 5, 6, 7]), _ints([4]), _ints([0])
    nova.paged_reserve(_ints([[0, 1, 2]]), 16, 0, 48, free, count, nxt, None, keep_per_row=_ints([0]))
    assert free.tolist() == [4, 5, 6, 7] and count.item() == 4 and nxt.item() == 0


# ---- append ---------------------------------------------------------------------------------------------------------
def _sources(B, n, hk, dh, dtype, seed):
    g = torch.Generator().manual_seed(seed)
    joint = torch.randn((B, n, 3 * hk, dh), generator=g).to(DTYPES[dtype]).cuda()
    k, v = joint[:, :, hk:2 * hk], joint[:, :, 2 * hk:]
    pad = torch.full((B, hk, n + 3, dh), 7.0, dtype=DTYPES[dtype], device="cuda")
    padv = torch.full((B, hk, dh, n + 5), 7.0, dtype=DTYPES[dtype], device="cuda")
    pad[:, :, 1:n + 1] = k.permute(0, 2, 1, 3)
    padv[:, :, :, 3:n + 3] = v.permute(0, 2, 3, 1)
    odd = torch.full((B, n, hk, dh + 1), 7.0, dtype=DTYPES[dtype], device="cuda")     # rows that no vector load can take
    odd[..., 1:] = k
    return {"joint": (k, v), "rows": (k.contiguous(), v.contiguous()), "odd": (odd[..., 1:], v.contiguous()),
            "caches": (pad[:, :, 1:n + 1].permute(0, 2, 1, 3), padv[..., 3:n + 3].permute(0, 3, 1, 2)),
            "one row for all": (k[:1, :1].expand(B, n, hk, dh), v[:, :, :1].expand(B, n, hk, dh))}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("B,hk,n,p", [(1, 1, 1, 16), (3, 5, 1, 32), (2, 3, 70, 16), (1, 2, 257, 256), (5, 1, 19, 64)])
def test_append(nova, dtype, dh, B, hk, n, p):
    pages = -(-B * n // p) + 3
    g = np.random.default_rng(n)
    slots = g.permutation(pages * p)[:B * n].reshape(B, n)
    slots[g.random((B, n)) < 0.2] = -1
    slots.flat[0::7] = [[pages * p, -5, 2 ** 31 - 1, -2 ** 31][i % 4] for i in range(len(slots.flat[0::7]))]
    for name, (k, v) in _sources(B, n, hk, dh, dtype, 11).items():
        print(f"paged append {dtype} dh={dh} B={B} hk={hk} n={n} p={p} {name}", flush=True)
        pools = [torch.randn((pages, hk, p, dh), generator=torch.Generator().manual_seed(i)).to(DTYPES[dtype]).cuda() for i in (1, 2)]
        before = [_np(t) for t in pools]
        nova.paged_append(PagedCache(*pools), k, v, _ints(slots))
        assert np.array_equal(_np(pools[0]), P.append(before[0], _np(k), slots))
        assert np.array_equal(_np(pools[1]), P.append(before[1], _np(v), slots))


# ---- attention ------------------------------------------------------------------------------------------------------
def _fill(dtype, B, hk, p, dh, lens, pitch, seed, kscale=1.0, spare=2):
    """A pool with the images' rows in pages of no order, NaN everywhere else; the table, -1 behind an image's pages."""
    g = np.random.default_rng(seed)
    counts = [-(-L // p) for L in lens]
    pages = sum(counts) + spare
    ids, used = g.permutation(pages), 0
    table = np.full((B, pitch), -1)
    pools = [np.full((pages, hk, p, dh), np.nan, dtype=np.float32) for _ in range(2)]
    reach = np.exp(0.5 * g.standard_normal((hk, 1, dh)))
    for b, L in enumerate(lens):
        table[b, :counts[b]] = ids[used:used + counts[b]]
        used += counts[b]
        for pool in pools:
            for i in range(counts[b]):
                m = min(p, L - i * p)
                pool[table[b, i], :, :m] = kscale * reach * g.standard_normal((hk, m, dh))
    cache = PagedCache(*[torch.from_numpy(t).to(DTYPES[dtype]).cuda() for t in pools])
    return cache, table


def _bounds(ref, dtype, dh, L, vmax=2.0 ** 20):
    out, lse, w, reach = ref
    finite = np.where(np.isfinite(lse), np.abs(lse), 0.0)
    d = (2 * dh + 32) * U * (reach + finite + 1)
    t = (2 * d + (L + 128) * U)[..., None] * w + L * 4 * 2.0 ** -126 * (1 + vmax)
    if dtype == "bf16":
        t = t + 1.02 * 2.0 ** -8 * (w + np.abs(out))
    return t, d + (L + 128) * U + 8 * U * finite


def _run(nova, cache, table, q, kv_len, lens=None, counts=None, causal=False, scale=None, chosen=None):
    B, n, H, dh = q.shape
    if chosen is None:
        need = nova.paged_attention_workspace_bytes(cache, B, H, n, kv_len)
    else:
        need = nova.paged_sparse_attention_workspace_bytes(cache, B, H, n, kv_len, chosen.shape[-1])
    ws = torch.full((max(need, 16),), 255, dtype=torch.uint8, device="cuda")       # NaN wherever it is read before it is written
    out = torch.full((B, n, H, dh), float("nan"), dtype=q.dtype, device="cuda")
    lse = torch.full((B, n, H), float("nan"), device="cuda")
    kw = dict(causal=causal, scale=scale, lse=lse, n_per_row=_ints(counts), kv_len_per_row=_ints(lens))
    if chosen is None:
        nova.paged_attention(cache, _ints(table), q, out, ws, kv_len, **kw)
    else:
        nova.paged_sparse_attention(cache, _ints(table), _ints(chosen), q, out, ws, kv_len, **kw)
    torch.cuda.synchronize()
    return out, lse


def _compare(out, lse, ref, dtype, dh, L):
    t_out, t_lse = _bounds(ref, dtype, dh, L)
    got, glse = _np(out), _np(lse)
    empty = np.isneginf(ref[1])
    assert np.array_equal(np.isneginf(glse), empty)
    assert (got[empty] == 0).all()
    assert np.isfinite(got).all()
    bad = np.abs(got - ref[0]) > t_out
    assert not bad.any(), (np.argwhere(bad)[:4], np.abs(got - ref[0]).max(), t_out[bad][:4])
    with np.errstate(invalid="ignore"):
        assert (np.where(empty, 0.0, np.abs(glse - ref[1])) <= t_lse).all()


def _check(nova, dtype, B, H, hk, dh, p, n, kv_len, lens=None, counts=None, causal=False, scale=None, seed=1, kscale=1.0, q=None,
           take=0, spoil=None):
    """take > 0: over that many random pages per query and key head.  spoil(pools, table): changes the pools first."""
    print(f"paged attention {dtype} B={B} H={H}/{hk} dh={dh} p={p} n={n} kv_len={kv_len} lens={lens} counts={counts} causal={causal} "
          f"take={take}", flush=True)
    real = [kv_len] * B if lens is None else [min(max(x, 0), kv_len) for x in lens]
    live = [n] * B if counts is None else [min(max(x, 0), n) for x in counts]
    pitch = -(-kv_len // p) + 1
    cache, table = _fill(dtype, B, hk, p, dh, real, pitch, seed, kscale)
    if spoil is not None:
        spoil(cache, table)
    if q is None:
        q = torch.randn((B, n, H, dh), generator=torch.Generator().manual_seed(seed)).to(DTYPES[dtype]).cuda()
    chosen = None
    if take:
        g = np.random.default_rng(seed + 7)
        pages = max(-(-kv_len // p), 1)
        chosen = np.full((B, n, hk, take), -1)
        for at in np.ndindex(B, n, hk):
            c = np.sort(g.permutation(pages)[:take])
            chosen[at][:len(c)] = c
    out, lse = _run(nova, cache, table, q, kv_len, lens, counts, causal, scale, chosen)
    pools = [_np(cache.k_pages), _np(cache.v_pages)]
    K, V = ([P.image_rows(pool, table[b], real[b]) for b in range(B)] for pool in pools)
    ref = P.attention(_np(q), K, V, dh ** -0.5 if scale is None else scale, live, causal, chosen, p)
    _compare(out, lse, ref, dtype, dh, kv_len)
    return out, lse


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("n,L,p", [(1, 1, 16), (1, 15, 16), (1, 16, 16), (1, 17, 16), (1, 33, 32), (1, 64, 64), (1, 129, 16), (1, 700, 32),
                                   (1, 3001, 256), (2, 5, 16), (7, 63, 64), (16, 65, 16), (17, 64, 32), (31, 200, 128), (33, 127, 16),
                                   (64, 640, 64), (127, 130, 32), (130, 259, 16), (300, 1030, 64)])
def test_lengths(nova, dtype, dh, causal, n, L, p):
    _check(nova, dtype, 2, 2, 2, dh, p, n, L, causal=causal)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("H,hk", [(1, 1), (6, 2), (8, 1), (12, 4), (32, 2), (40, 1)])
@pytest.mark.parametrize("n,L,p", [(1, 300, 16), (3, 77, 32), (50, 190, 64)])
def test_shared_key_heads(nova, dtype, dh, H, hk, n, L, p):
    _check(nova, dtype, 2, H, hk, dh, p, n, L, causal=True)
    _check(nova, dtype, 1, H, hk, dh, p, n, L, take=2, causal=n > 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
@pytest.mark.parametrize("take", [0, 3])
@pytest.mark.parametrize("n,kv_len", [(1, 40), (1, 2000), (9, 300), (40, 700), (200, 500), (1, 0), (150, 0)])
def test_images_with_their_own_lengths(nova, dtype, causal, take, n, kv_len):
    """No rows, one row, fewer rows than queries, counts past either bound (clamped), images without queries; NaN behind every
    length."""
    lens = [kv_len, 0, 1, kv_len // 2, kv_len + 9, -3]
    counts = [n, n, n + 5, 0, max(n - 1, 0), n]
    for dh in (64, 128):
        _check(nova, dtype, 6, 4, 2, dh, 32, n, kv_len, lens, counts, causal, take=take)
        _check(nova, dtype, 6, 4, 2, dh, 16, n, kv_len, lens, None, causal, take=take)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n,L,p", [(33, 2049, 16), (128, 2112, 64), (129, 2111, 32), (300, 2113, 256)])
def test_many_rows_over_many_tiles(nova, dtype, dh, n, L, p):
    _check(nova, dtype, 1, 2, 1, dh, p, n, L)
    _check(nova, dtype, 1, 2, 1, dh, p, n, L, causal=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("lens", [None, [700, 699, 140, 164, 141, 333, 650, 228, 700]])
def test_many_items(nova, dtype, lens):
    _check(nova, dtype, 9, 32, 32, 64, 32, 140, 700, lens, causal=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("scale", [0.0, -0.3, 3.0])
def test_scales(nova, dtype, dh, scale):
    for n, L, take in ((1, 100, 0), (40, 170, 0), (40, 170, 2)):
        _check(nova, dtype, 2, 4, 2, dh, 16, n, L, causal=n > 1, scale=scale, take=take)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
def test_wide_scores(nova, dtype, dh):
    """Keys whose scores are hundreds of nats apart: the reference moves, the sums stay."""
    for n, L in ((1, 900), (70, 1500)):
        _check(nova, dtype, 2, 2, 1, dh, 64, n, L, kscale=30.0, causal=n > 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n,L", [(3, 50), (20, 33), (140, 260), (140, 900)])
def test_what_a_query_does_not_see_has_no_part(nova, dtype, dh, n, L):
    """Keys and values of NaN and infinities in rows behind a query's own, and in pages that it has not chosen."""
    p = 16
    def spoil(cache, table):
        for b in range(2):
            for i, r in enumerate(range(L - n, L)):              # rows of the chunk: value or key of every other one
                if i % 2:
                    (cache.v_pages if i % 4 == 1 else cache.k_pages)[table[b, r // p], :, r % p, i % dh] = [float("nan"), float("inf"), -float("inf")][i % 3]
    real = [L, L]
    cache, table = _fill(dtype, 2, 2, p, dh, real, -(-L // p), 3)
    spoil(cache, table)
    q = torch.randn((2, n, 4, dh), generator=torch.Generator().manual_seed(2)).to(DTYPES[dtype]).cuda()
    pools = [_np(cache.k_pages), _np(cache.v_pages)]
    K, V = ([P.image_rows(pool, table[b], L) for b in range(2)] for pool in pools)
    out, lse = _run(nova, cache, table, q, L, causal=True)
    ref = P.attention(_np(q), K, V, dh ** -0.5, [n, n], True)
    good = np.isfinite(ref[0]).all((0, 2, 3))
    assert good[0] and not good.all()
    sub = lambda t: t[:, good]
    _compare(out[:, torch.from_numpy(good).cuda()], lse[:, torch.from_numpy(good).cuda()], [sub(t) for t in ref], dtype, dh, L)
    # pages of NaN that only some queries have chosen
    cache, table = _fill(dtype, 1, 2, p, dh, [L], -(-L // p), 4)
    pages = -(-L // p)
    cache.v_pages[int(table[0, 1])] = float("nan")
    cache.k_pages[int(table[0, 0]), 0, 3] = float("inf")
    chosen = np.full((1, n, 2, 2), -1)
    chosen[0, ::3, :, 0] = 1
    chosen[0, 1::3, :, 0] = 0
    chosen[0, :, :, 1] = pages - 1
    out, lse = _run(nova, cache, table, q[:1], L, chosen=chosen)
    pools = [_np(cache.k_pages), _np(cache.v_pages)]
    K, V = ([P.image_rows(pool, table[0], L)] for pool in pools)
    ref = P.attention(_np(q[:1]), K, V, dh ** -0.5, [n], False, chosen, p)
    good = np.zeros(n, dtype=bool)
    good[2::3] = True
    _compare(out[:, torch.from_numpy(good).cuda()], lse[:, torch.from_numpy(good).cuda()], [t[:, good] for t in ref], dtype, dh, L)
    assert torch.isnan(out[:, ::3]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_entries_that_are_no_pages(nova, dtype):
    """Rows of zeros, wherever the entry points."""
    B, H, hk, dh, p, n, L = 1, 4, 2, 64, 16, 5, 100
    cache, table = _fill(dtype, B, hk, p, dh, [L], 8, 5)
    table[0, 1], table[0, 3], table[0, 4] = -1, 2 ** 31 - 1, cache.k_pages.shape[0]
    q = torch.randn((B, n, H, dh), generator=torch.Generator().manual_seed(5)).to(DTYPES[dtype]).cuda()
    K, V = ([P.image_rows(_np(pool), table[0], L)] for pool in (cache.k_pages, cache.v_pages))
    _compare(*_run(nova, cache, table, q, L, causal=True), P.attention(_np(q), K, V, dh ** -0.5, [n], True), dtype, dh, L)
    none = np.full((1, 7), -1)
    out, lse = _run(nova, PagedCache.empty(0, hk, p, dh, DTYPES[dtype]), none, q, L)
    assert (out == 0).all() and np.allclose(_np(lse), np.log(L), atol=1e-6)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n", [1, 60])
def test_strides(nova, dtype, n):
    """Queries in the output of a joint projection, heads in front of rows, one query for all."""
    B, H, hk, dh, L = 2, 6, 2, 64, 150
    g = torch.Generator().manual_seed(9)
    joint = torch.randn((B, n, H + 2 * hk, dh), generator=g).to(DTYPES[dtype]).cuda()
    heads_first = torch.randn((H, B, n, dh), generator=g).to(DTYPES[dtype]).cuda().permute(1, 2, 0, 3)
    for q in (joint[:, :, :H], heads_first, joint[:1, :1, :1].expand(B, n, H, dh)):
        _check(nova, dtype, B, H, hk, dh, 32, n, L, causal=True, q=q)
        _check(nova, dtype, B, H, hk, dh, 32, n, L, take=2, q=q)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("p", [16, 64, 256])
@pytest.mark.parametrize("n,L,H,hk,take", [(1, 1, 2, 2, 1), (1, 2000, 8, 2, 7), (1, 5000, 4, 1, 40), (5, 900, 4, 4, 3), (33, 800, 6, 2, 9),
                                           (70, 1200, 1, 1, 2), (90, 3000, 2, 1, 33)])
def test_sparse(nova, dtype, dh, p, n, L, H, hk, take):
    _check(nova, dtype, 2, H, hk, dh, p, n, L, take=take)
    _check(nova, dtype, 2, H, hk, dh, p, n, L, take=take, causal=True, lens=[L, max(L - 40, n)])


def test_lists_in_any_order(nova):
    """Repeats, entries that are no pages of the image, any order; no entry at all."""
    B, n, H, hk, dh, p, L = 1, 12, 4, 2, 64, 16, 300
    g = np.random.default_rng(4)
    for dtype in ("f32", "bf16"):
        for n_ in (1, n):
            cache, table = _fill(dtype, B, hk, p, dh, [L], 20, 4)
            q = torch.randn((B, n_, H, dh), generator=torch.Generator().manual_seed(5)).to(DTYPES[dtype]).cuda()
            chosen = g.integers(0, 25, (B, n_, hk, 9))
            chosen[..., 3] = chosen[..., 2]
            chosen[..., 5] = [[-7, 2 ** 31 - 1][i % 2] for i in range(hk)]
            if n_ > 1:
                chosen[0, 3], chosen[0, 4] = -1, 900
            K, V = ([P.image_rows(_np(pool), table[0], L)] for pool in (cache.k_pages, cache.v_pages))
            real = np.where((chosen >= 0) & (chosen < -(-L // p)), chosen, -1)
            ref = P.attention(_np(q), K, V, dh ** -0.5, [n_], False, real, p)
            _compare(*_run(nova, cache, table, q, L, chosen=chosen), ref, dtype, dh, L)


def test_longest_lists(nova):
    """256 pages per query, 32 queries of one head: the largest union there is room for."""
    for dtype in ("f32", "bf16"):
        _check(nova, dtype, 1, 1, 1, 64, 16, 40, 9000, take=256)
        _check(nova, dtype, 1, 1, 1, 64, 16, 1, 9000, take=256)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_pools_past_32_bits(nova, dtype):
    """Pages from 2^31 elements on."""
    hk, p, dh, L, n = 8, 256, 128, 700, 3
    pages = 2 ** 31 // (hk * p * dh) + 40
    pools = [torch.zeros((pages, hk, p, dh), dtype=DTYPES[dtype], device="cuda") for _ in range(2)]
    table = np.array([[pages - 1, 5, pages - 7]])
    slots = np.array([[table[0, r // p] * p + r % p for r in range(L)]])
    g = torch.Generator().manual_seed(1)
    k, v = (torch.randn((1, L, hk, dh), generator=g).to(DTYPES[dtype]).cuda() for _ in range(2))
    cache = PagedCache(*pools)
    nova.paged_append(cache, k, v, _ints(slots))
    q = torch.randn((1, n, hk, dh), generator=g).to(DTYPES[dtype]).cuda()
    K, V = ([_np(t)[0].transpose(1, 0, 2)] for t in (k, v))
    ref = P.attention(_np(q), K, V, dh ** -0.5, [n], True)
    _compare(*_run(nova, cache, table, q, L, causal=True), ref, dtype, dh, L)
    means = torch.zeros((pages, hk, dh), dtype=torch.bfloat16, device="cuda")
    nova.paged_summarise(cache, _ints(table), means, L, L)
    want = [P.seven_bits(K[0][j, 2 * p:].sum(0) / (L - 2 * p)) for j in range(hk)]
    assert np.array_equal(_np(means[pages - 7]), np.array(want))


# ---- blocks of 128 rows, long lists, shared pages -------------------------------------------------------------------
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("H,hk,n,L,p", [(4, 2, 140, 2300, 16), (3, 1, 200, 2500, 64), (40, 20, 90, 600, 32)])
def test_what_a_query_does_not_see_in_blocks_of_128_rows(nova, dh, H, hk, n, L, p):
    """NaN and infinities among the keys and values of rows behind a query's own: blocks that end as NaN are gone over again."""
    B = 1 if L > 2048 else 4
    cache, table = _fill("bf16", B, hk, p, dh, [L] * B, -(-L // p), 3)
    for b in range(B):
        for r in range(L - n + n // 2, L, 3):
            pool = (cache.v_pages, cache.k_pages)[r % 2]
            pool[int(table[b, r // p]), r % hk, r % p, r % dh] = (float("nan"), float("inf"), -float("inf"))[r % 3]
    cache.v_pages[int(table[0, (L - n // 2) // p]), 0, (L - n // 2) % p, 5] = float("-inf")
    q = torch.randn((B, n, H, dh), generator=torch.Generator().manual_seed(2)).bfloat16().cuda()
    pools = [_np(cache.k_pages), _np(cache.v_pages)]
    K, V = ([P.image_rows(pool, table[b], L) for b in range(B)] for pool in pools)
    out, lse = _run(nova, cache, table, q, L, causal=True)
    ref = P.attention(_np(q), K, V, dh ** -0.5, [n] * B, True)
    good = np.isfinite(ref[0]).all((0, 2, 3))
    assert good[:n // 2].all() and not good.all()
    pick = torch.from_numpy(good).cuda()
    _compare(out[:, pick], lse[:, pick], [t[:, good] for t in ref], "bf16", dh, L)
    # an infinity or a NaN that is seen shows where it should
    bad = ~np.isfinite(ref[0])
    assert not np.isfinite(_np(out)[bad]).any()


@pytest.mark.parametrize("H,hk,n,L,p,take", [(16, 8, 260, 1100, 16, 20), (24, 8, 200, 1500, 64, 12), (40, 8, 130, 900, 32, 9), (130, 2, 70, 700, 16, 30),
                                             (8, 8, 2050, 640, 64, 2)])
@pytest.mark.parametrize("causal", [False, True])
def test_sparse_in_blocks_of_128_rows(nova, H, hk, n, L, p, take, causal):
    """Lists that overlap; heads that share a key head in threes and fives, so that a query's rows lie in two waves, or in two blocks."""
    B = max(1, 128 // (hk * -(-n * (H // hk) // 128)) + 1)
    L = max(L, n)
    _check(nova, "bf16", B, H, hk, 128, p, n, L, take=take, causal=causal, lens=None if B == 1 else [L - 13 * (b % 3) if L - 26 >= n else L for b in range(B)])


@pytest.mark.parametrize("G", [1, 3])
def test_chosen_pages_of_nan_in_blocks_of_128_rows(nova, G):
    """A page of NaN that only some queries have chosen.  The others' results are within the same bounds as without it: tiles with such
    a page are summed key by key, in another order (their logarithms are the same bits), and the bounds hold for any order."""
    B, hk, dh, p, n, L, take = 3, 16, 128, 16, 400 // G, 640, 12
    H = hk * G
    cache, table = _fill("bf16", B, hk, p, dh, [L] * B, 40, 8)
    q = torch.randn((B, n, H, dh), generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    g = np.random.default_rng(1)
    chosen = np.sort(np.stack([g.permutation(39)[:take] for _ in range(B * n * hk)]).reshape(B, n, hk, take) + 1, axis=-1)
    clean, clean_lse = _run(nova, cache, table, q, L, chosen=chosen)
    for b in range(B):
        cache.v_pages[int(table[b, 7]), :, 3] = float("nan")
    out, lse = _run(nova, cache, table, q, L, chosen=chosen)
    seen = torch.from_numpy((chosen == 7).any(-1).repeat(G, 2)).cuda()
    assert seen.any() and not seen.all()
    assert torch.isnan(out[seen]).all() and torch.equal(lse, clean_lse)
    K, V = ([P.image_rows(_np(pool), table[b], L) for b in range(B)] for pool in (cache.k_pages, cache.v_pages))
    ref = P.attention(_np(q), K, V, dh ** -0.5, [n] * B, False, chosen, p)
    t_out, _ = _bounds(ref, "bf16", dh, take * p)
    other = ~seen.cpu().numpy()
    for got in (out, clean):
        assert (np.abs(_np(got) - ref[0])[other] <= t_out[other]).all()


@pytest.mark.parametrize("H,hk,n,L,p,take", [(16, 8, 260, 1100, 16, 20), (24, 8, 200, 1500, 64, 12), (40, 8, 130, 900, 256, 2), (130, 2, 70, 700, 32, 15)])
@pytest.mark.parametrize("causal", [False, True])
def test_sparse_in_blocks_of_128_rows_of_64_channels(nova, H, hk, n, L, p, take, causal):
    B = max(1, 128 // (hk * -(-n * (H // hk) // 128)) + 1)
    _check(nova, "bf16", B, H, hk, 64, p, n, L, take=take, causal=causal, lens=None if B == 1 else [L - 13 * (b % 3) if L - 26 >= n else L for b in range(B)])


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("G,n", [(1, 300), (3, 100), (20, 15)])
def test_infinities_of_chosen_pages_in_blocks_of_128_rows(nova, dh, G, n):
    """Infinities of both signs and NaN among the values of pages that some queries have chosen, some of them behind a query's own row: an
    infinity shows with its sign, two of both signs and a NaN as NaN, and nothing of it in rows or channels that have none."""
    B, hk, p, L, take = 3, 16, 32, 640, 6
    cache, table = _fill("bf16", B, hk, p, dh, [L] * B, 20, 8)
    g = np.random.default_rng(4)
    chosen = np.stack([g.permutation(19)[:take] for _ in range(B * n * hk)]).reshape(B, n, hk, take)
    chosen[:, :, :, 0] = np.where(g.random((B, n, hk)) < 0.5, 19, chosen[:, :, :, 0])
    odd = (float("inf"), -float("inf"), float("nan"))
    for b in range(B):
        for i, (page, row) in enumerate([(2, 5), (2, 20), (7, 31), (11, 0), (19, 12), (19, 31), (18, 3)]):
            for c, kind in ((3, 0), (dh - 1, 1), (17, i % 2), (40, i % 3)):
                cache.v_pages[int(table[b, page]), i % hk:, row, c] = odd[kind]
    q = torch.randn((B, n, hk * G, dh), generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    out, lse = _run(nova, cache, table, q, L, chosen=chosen, causal=True)
    K, V = ([P.image_rows(_np(pool), table[b], L) for b in range(B)] for pool in (cache.k_pages, cache.v_pages))
    with np.errstate(invalid="ignore"):
        ref = P.attention(_np(q), K, V, dh ** -0.5, [n] * B, True, chosen, p)
    got = _np(out)
    assert (np.isnan(got) == np.isnan(ref[0])).all() and np.isnan(got).any()
    for sign in (np.inf, -np.inf):
        assert ((got == sign) == (ref[0] == sign)).all() and (got == sign).any()
    fine = np.isfinite(ref[0])
    ref = [np.where(np.isfinite(t), t, 0.0) for t in ref]
    t_out, t_lse = _bounds(ref, "bf16", dh, take * p)
    assert (np.abs(np.where(fine, got, 0.0) - ref[0]) <= t_out)[fine].all()


@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("scale", [0.0, -0.2, 4.0])
def test_scales_and_empty_images_of_chosen_pages_in_blocks_of_128_rows(nova, dh, scale):
    """Scores of either sign and far apart; images without rows, of one row, and without queries; keys that are no numbers in rows that
    some of the queries see, which leave the others' results alone."""
    B, G, hk, n, p, L, take = 5, 2, 8, 150, 16, 400, 7
    lens, counts = [L, 0, 1, L - 7, L], [n, n, n, 0, n - 31]
    cache, table = _fill("bf16", B, hk, p, dh, lens, 25, 8)
    g = np.random.default_rng(6)
    chosen = np.stack([g.permutation(25)[:take] for _ in range(B * n * hk)]).reshape(B, n, hk, take)
    q = torch.randn((B, n, hk * G, dh), generator=torch.Generator().manual_seed(5)).bfloat16().cuda()

    def reference():
        K, V = ([P.image_rows(_np(pool), table[b], lens[b]) for b in range(B)] for pool in (cache.k_pages, cache.v_pages))
        with np.errstate(invalid="ignore"):
            return P.attention(_np(q), K, V, scale, counts, True, chosen, p)

    kw = dict(lens=lens, counts=counts, causal=True, scale=scale, chosen=chosen)
    ref = reference()
    _compare(*_run(nova, cache, table, q, L, **kw), ref, "bf16", dh, take * p)
    for page, row, odd in ((3, 4, float("nan")), (24, 9, float("inf")), (20, 15, -float("inf"))):
        cache.k_pages[int(table[0, page]), :, row, 5] = odd
    out, lse = _run(nova, cache, table, q, L, **kw)
    fine = np.ones((B, n, hk * G), bool)
    see = np.repeat((chosen[0] == 3).any(-1) | ((chosen[0] == 24).any(-1) & (np.arange(n) + L - n >= 24 * p + 9)[:, None])
                    | ((chosen[0] == 20).any(-1) & (np.arange(n) + L - n >= 20 * p + 15)[:, None]), G, 1)
    fine[0] = ~see
    assert fine[0].any() and see.any()
    t_out, t_lse = _bounds(ref, "bf16", dh, take * p)
    assert (np.abs(_np(out) - ref[0]) <= t_out)[fine].all()
    empty = np.isneginf(ref[1])
    assert (np.isneginf(_np(lse)) == empty)[fine].all()
    assert (np.abs(np.where(empty, 0.0, _np(lse)) - np.where(empty, 0.0, ref[1])) <= t_lse)[fine & ~empty].all()
    assert np.isnan(_np(out)[0][np.repeat((chosen[0] == 3).any(-1), G, 1)]).all()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("hk,n,take", [(22, 96, 256), (1, 33, 256), (1, 1, 256)])
def test_longest_lists_of_the_longest_page_lists(nova, dtype, hk, n, take):
    """256 of 16384 pages for every query; the table names the same few pages over and over, as images with one beginning do."""
    p, dh, pages, L = 16, 64, 48, 16384 * 16 - 5
    g = np.random.default_rng(3)
    cache, _ = _fill(dtype, 1, hk, p, dh, [pages * p], pages, 3, spare=0)
    table = g.integers(0, pages, (1, 16384))
    q = torch.randn((1, n, hk, dh), generator=torch.Generator().manual_seed(5)).to(DTYPES[dtype]).cuda()
    chosen = np.sort(np.stack([g.permutation(16384)[:take] for _ in range(n * hk)]).reshape(1, n, hk, take), axis=-1)
    chosen[0, 0, 0, -1] = 16383
    out, lse = _run(nova, cache, table, q, L, chosen=chosen)
    pools = [_np(cache.k_pages), _np(cache.v_pages)]
    heads = [(0, 0), (n - 1, hk - 1), (n // 2, hk // 2)]
    for s, h in heads:                                           # the chosen pages, one after the other, as an image of their own
        K, V = ([P.image_rows(pool[:, h:h + 1], table[0, chosen[0, s, h]], take * p)] for pool in pools)
        rows = np.where(chosen[0, s, h][:, None] * p + np.arange(p) < L)
        K, V = ([x[0].reshape(1, take, p, dh)[:, rows[0], rows[1]]] for x in (K, V))
        ref = P.attention(_np(q)[:, s:s + 1, h:h + 1], K, V, dh ** -0.5, [1], False)
        _compare(out[:, s:s + 1, h:h + 1], lse[:, s:s + 1, h:h + 1], ref, dtype, dh, take * p)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("hk,n,L", [(32, 1, 200), (32, 1, 300), (32, 1, 777), (100, 1, 900), (130, 1, 1600), (64, 3, 500)])
def test_few_rows_whole_and_in_runs(nova, dtype, dh, hk, n, L):
    """One workgroup of eight waves per block, and runs that a second launch joins."""
    _check(nova, dtype, 1, hk, hk, dh, 16, n, L)
    _check(nova, dtype, 2, hk, hk // 2, dh, 64, n, L, lens=[L, max(L // 3, n)], causal=True)
    _check(nova, dtype, 1, hk, hk, dh, 16, n, L, take=5)


# ---- means and choices ----------------------------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("p", [16, 32, 64, 256])
@pytest.mark.parametrize("n,kv_len", [(1, 1), (1, 300), (40, 40), (33, 290), (700, 900), (0, 50), (1000, 900)])
def test_summarise(nova, dtype, dh, p, n, kv_len):
    B, hk = 4, 3
    lens, counts = [kv_len, kv_len // 2, 0, kv_len], [n, n, n, n // 2]
    print(f"paged summarise {dtype} dh={dh} p={p} n={n} kv_len={kv_len}", flush=True)
    for lv, cv in ((None, None), (lens, counts)):
        real, live = lv or [kv_len] * B, cv or [n] * B
        cache, table = _fill(dtype, B, hk, p, dh, real, -(-kv_len // p) + 1, n)
        if kv_len > 200:
            cache.k_pages[int(table[0, (kv_len - 1) // p]), 1, 0, 5] = float("inf")
            table[3, (kv_len - 1) // p] = -1
        means = torch.randn((cache.k_pages.shape[0], hk, dh), generator=torch.Generator().manual_seed(1)).bfloat16().cuda()
        want = P.summarise(_np(cache.k_pages), table, _np(means), real, live)
        nova.paged_summarise(cache, _ints(table), means, n, kv_len, n_per_row=_ints(cv), kv_len_per_row=_ints(lv))
        assert np.array_equal(_np(means), want, equal_nan=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_means_at_the_ends_of_the_range(nova, dtype):
    rows = torch.zeros((8, 1, 16, 64))
    rows[0, 0, :, 0] = 127.0
    rows[1, 0, :, 0] = 127.5
    rows[1, 0, :, 1] = 3.0                                       # halfway between two multiples
    rows[2] = 1e-39
    rows[3, 0, :, :2] = torch.tensor([3e38, -2e32])
    rows[4, 0, 0, 3] = -3.3e38
    rows[5, 0, 7, 9] = float("nan")
    rows[6] = -2.0 ** -100 * 50
    cache = PagedCache(rows.to(DTYPES[dtype]).cuda(), rows.to(DTYPES[dtype]).cuda())
    table = np.arange(8)[None]
    means = torch.full((8, 1, 64), 9.0, dtype=torch.bfloat16, device="cuda")
    nova.paged_summarise(cache, _ints(table), means, 128, 128)
    assert np.array_equal(_np(means), P.summarise(_np(cache.k_pages), table, _np(means), [128], [128]), equal_nan=True)


def _check_select(nova, dtype, B, H, hk, dh, p, n, kv_len, k, first=1, recent=1, causal=False, lens=None, counts=None, seed=1, coarse=False):
    print(f"paged select {dtype} B={B} H={H}/{hk} dh={dh} p={p} n={n} kv_len={kv_len} k={k} {first}/{recent} causal={causal} lens={lens}", flush=True)
    g = np.random.default_rng(seed)
    real = [kv_len] * B if lens is None else [min(max(x, 0), kv_len) for x in lens]
    live = [n] * B if counts is None else [min(max(x, 0), n) for x in counts]
    pitch = -(-kv_len // p) + 1
    pages = B * pitch + 2
    table = g.permutation(pages)[:B * pitch].reshape(B, pitch)
    x = g.integers(-1, 2, (pages, hk, dh)) if coarse else g.standard_normal((pages, hk, dh)) * np.exp(g.standard_normal((pages, hk, 1)))
    m = np.array([[P.seven_bits(x[i, j].astype(np.float64)) for j in range(hk)] for i in range(pages)])
    if kv_len > 500:
        m[table[0, 3]] = np.nan
        table[0, 5] = pages + 3
    means = torch.from_numpy(m).to(torch.bfloat16).cuda()
    assert np.array_equal(_np(means), m, equal_nan=True)
    q = torch.randn((B, n, H, dh), generator=torch.Generator().manual_seed(seed)).to(DTYPES[dtype])
    if n > 4:
        q[0, 2, 0, 5], q[0, 3], q[0, 4, -1, 1] = float("nan"), 0.0, float("-inf")
    q = q.cuda()
    chosen = torch.full((B, n, hk, k), -99, dtype=torch.int32, device="cuda")
    nova.paged_select(means, _ints(table), p, q, chosen, kv_len, first=first, recent=recent, causal=causal, n_per_row=_ints(counts),
                      kv_len_per_row=_ints(lens))
    want = P.select(_np(q), m, table, p, real, live, causal, first, recent, k)
    assert np.array_equal(chosen.cpu().numpy(), want), np.argwhere(chosen.cpu().numpy() != want)[:5]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("dh", [64, 128])
@pytest.mark.parametrize("n,kv_len,p,k", [(1, 1, 16, 2), (1, 17, 16, 2), (1, 2000, 16, 9), (1, 30000, 16, 64), (5, 700, 32, 6), (17, 1000, 16, 5),
                                          (40, 2500, 16, 256), (16, 5000, 256, 4), (33, 64, 64, 3)])
def test_select(nova, dtype, dh, n, kv_len, p, k):
    _check_select(nova, dtype, 2, 4, 2, dh, p, n, kv_len, k)
    _check_select(nova, dtype, 2, 3, 1, dh, p, n, kv_len, k, causal=True, lens=[max(kv_len - 20, 0), kv_len + 3])
    if n < 20:
        _check_select(nova, dtype, 1, 2, 2, dh, p, n, kv_len, k, first=0, recent=0)
        _check_select(nova, dtype, 1, 11, 1, dh, p, n, kv_len, k, first=k // 2, recent=k - k // 2)


@pytest.mark.parametrize("pages", [256, 257, 512, 513, 1024, 1025, 2048, 2049, 4096, 4097])
def test_select_among_any_number_of_pages(nova, pages):
    """A lane holds 4, 8, 16 or 32 keys; one wave, two or four choose for a query."""
    _check_select(nova, "bf16", 1, 2, 1, 64, 16, 3, pages * 16 - 7, 20, causal=True)
    _check_select(nova, "bf16", 1, 2, 2, 64, 16, 2, pages * 16, min(pages, 250), coarse=True)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("causal", [False, True])
def test_select_with_ties(nova, dtype, causal):
    """Means of -1, 0 and 1: many scores alike."""
    _check_select(nova, dtype, 2, 4, 4, 64, 16, 20, 1500, 12, causal=causal, coarse=True, lens=[1500, 33], counts=[20, 7])


def test_longest_page_lists(nova):
    """16384 pages of one image: as many as a query chooses from."""
    _check_select(nova, "bf16", 1, 2, 1, 64, 16, 2, 16384 * 16, 20)


def test_a_query_chooses_the_same_pages_alone(nova):
    """In chunks of any size, and with heads of any number."""
    B, n, H, hk, dh, p, L, k = 1, 37, 4, 2, 128, 16, 3000, 11
    g = torch.Generator().manual_seed(3)
    cache, table = _fill("bf16", B, hk, p, dh, [L], -(-L // p), 3)
    q = torch.randn((B, n, H, dh), generator=g).bfloat16().cuda()
    means = torch.zeros((cache.k_pages.shape[0], hk, dh), dtype=torch.bfloat16, device="cuda")
    nova.paged_summarise(cache, _ints(table), means, L, L)
    whole = torch.empty((B, n, hk, k), dtype=torch.int32, device="cuda")
    nova.paged_select(means, _ints(table), p, q, whole, L)
    for s in (0, 5, 36):
        one = torch.empty((B, 1, hk, k), dtype=torch.int32, device="cuda")
        nova.paged_select(means, _ints(table), p, q[:, s:s + 1], one, L)
        assert torch.equal(one, whole[:, s:s + 1])


# ---- together -------------------------------------------------------------------------------------------------------
class Server:
    """What a program keeps: a pool, page lists, lengths on the device; a step reserves, appends, summarises, chooses, attends."""

    def __init__(self, nova, dtype, B, H, hk, dh, p, pages, pitch, n, k):
        self.nova, self.B, self.H, self.n, self.p, self.most = nova, B, H, n, p, pitch * p
        self.cache = PagedCache.empty(pages, hk, p, dh, DTYPES[dtype])
        self.cache.k_pages.fill_(float("nan"))
        self.cache.v_pages.fill_(float("nan"))
        self.table = torch.full((B, pitch), -1, dtype=torch.int32, device="cuda")
        self.free = torch.arange(pages, dtype=torch.int32, device="cuda").flip(0).contiguous()
        self.height, self.lens = _ints([pages]), torch.zeros(B, dtype=torch.int32, device="cuda")
        self.count, self.keep = torch.zeros(B, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
        self.slots = torch.empty((B, n), dtype=torch.int32, device="cuda")
        self.means = torch.zeros((pages, hk, dh), dtype=torch.bfloat16, device="cuda")
        self.chosen = torch.empty((B, n, hk, k), dtype=torch.int32, device="cuda")
        mk = lambda *s: torch.empty(s, dtype=DTYPES[dtype], device="cuda")
        self.q, self.k, self.v, self.out, self.sparse = mk(B, n, H, dh), mk(B, n, hk, dh), mk(B, n, hk, dh), mk(B, n, H, dh), mk(B, n, H, dh)
        self.lse = torch.empty((B, n, H), device="cuda")
        bytes_ = max(nova.paged_attention_workspace_bytes(self.cache, B, H, n, self.most),
                     nova.paged_sparse_attention_workspace_bytes(self.cache, B, H, n, self.most, k), 16)
        self.ws = torch.full((bytes_,), 255, dtype=torch.uint8, device="cuda")

    def step(self):
        v, most = self.nova, self.most
        v.paged_reserve(self.table, self.p, self.n, most - self.n, self.free, self.height, self.lens, slots=self.slots,
                        kv_len_per_row=self.lens, n_per_row=self.count, keep_per_row=self.keep)
        v.paged_append(self.cache, self.k, self.v, self.slots)
        kw = dict(n_per_row=self.count, kv_len_per_row=self.lens)
        v.paged_attention(self.cache, self.table, self.q, self.out, self.ws, most, causal=True, lse=self.lse, **kw)
        v.paged_summarise(self.cache, self.table, self.means, self.n, most, **kw)
        v.paged_select(self.means, self.table, self.p, self.q, self.chosen, most, causal=True, **kw)
        v.paged_sparse_attention(self.cache, self.table, self.chosen, self.q, self.sparse, self.ws, most, causal=True, **kw)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("graph", [False, True])
def test_steps_of_a_program(nova, dtype, graph):
    """Images that grow, are cut back, end and are replaced, in a pool with little room; eagerly and as one captured graph that is
    replayed with other inputs, with the program's own work in between."""
    B, H, hk, dh, p, n, k = 3, 4, 2, 64, 16, 24, 4
    s = Server(nova, dtype, B, H, hk, dh, p, 40, 20, n, k)
    g = torch.Generator().manual_seed(1)
    rows = [[np.zeros((0, hk, dh))] * 2 for _ in range(B)]
    captured = None
    plan = [([0, 0, 0], [24, 5, 1]), ([99, 99, 99], [24, 1, 24]), ([30, 99, 99], [3, 0, 24]), ([99, 0, 99], [1, 17, 24]),
            ([99, 99, 0], [24, 24, 0]), ([99, 99, 99], [24, 24, 20]), ([0, 0, 0], [0, 2, 9])]
    if graph:
        s.step()                                                 # nothing comes: warms every path up
        torch.cuda.synchronize()
        captured = torch.cuda.CUDAGraph()
        with torch.cuda.graph(captured):
            s.step()
    for keep, come in plan:
        s.keep.copy_(_ints(keep))
        s.count.copy_(_ints(come))
        for t in (s.q, s.k, s.v):
            t.copy_(torch.randn(t.shape, generator=g))
        if captured is None:
            s.step()
        else:
            captured.replay()
        torch.cuda.synchronize()
        table, lens = s.table.cpu().numpy(), []
        for b in range(B):
            m = min(keep[b], len(rows[b][0]))
            rows[b] = [np.concatenate((r[:m], _np(t)[b, :come[b]])) for r, t in zip(rows[b], (s.k, s.v))]
            lens.append(len(rows[b][0]))
        assert s.lens.tolist() == lens
        held = [int(x) for b in range(B) for x in table[b, :-(-lens[b] // p)]]
        free = s.free[:s.height.item()].tolist()
        assert sorted(held + free) == list(range(40))            # every page has one owner
        K, V = ([rows[b][w].transpose(1, 0, 2) for b in range(B)] for w in range(2))
        for b in range(B):
            assert np.array_equal(P.image_rows(_np(s.cache.k_pages), table[b], lens[b]), K[b])
        ref = P.attention(_np(s.q), K, V, dh ** -0.5, come, True)
        _compare(s.out, s.lse, ref, dtype, dh, max(lens))
        chosen = P.select(_np(s.q), _np(s.means), table, p, lens, come, True, 1, 1, k)
        assert np.array_equal(s.chosen.cpu().numpy(), chosen)
        for b in range(B):
            for i in range(-(-lens[b] // p)):
                assert np.array_equal(_np(s.means[int(table[b, i])])[1], P.seven_bits(K[b][1, i * p:(i + 1) * p].mean(0)))
        ref = P.attention(_np(s.q), K, V, dh ** -0.5, come, True, chosen, p)
        t_out, _ = _bounds(ref, dtype, dh, max(lens))
        assert (np.abs(_np(s.sparse) - ref[0]) <= t_out).all()


def test_all_pages_chosen_is_dense(nova):
    """Every page chosen: what the dense call gives, to its tolerance."""
    B, n, H, hk, dh, p, L = 1, 20, 4, 2, 128, 64, 500
    cache, table = _fill("bf16", B, hk, p, dh, [L], 8, 6)
    q = torch.randn((B, n, H, dh), generator=torch.Generator().manual_seed(5)).bfloat16().cuda()
    chosen = np.broadcast_to(np.arange(8), (B, n, hk, 8))
    K, V = ([P.image_rows(_np(pool), table[0], L)] for pool in (cache.k_pages, cache.v_pages))
    _compare(*_run(nova, cache, table, q, L, causal=True, chosen=chosen), P.attention(_np(q), K, V, dh ** -0.5, [n], True), "bf16", dh, L)


def test_two_streams(nova):
    """Two calls at once, each on its stream with its workspace."""
    B, H, hk, dh, p, n, L = 2, 8, 2, 128, 16, 1, 6000
    cases = []
    for seed in (1, 2):
        cache, table = _fill("bf16", B, hk, p, dh, [L, L - 77], -(-L // p), seed)
        q = torch.randn((B, n, H, dh), generator=torch.Generator().manual_seed(seed)).bfloat16().cuda()
        need = nova.paged_attention_workspace_bytes(cache, B, H, n, L)
        cases.append((cache, _ints(table), q, torch.empty_like(q), torch.empty(max(need, 16), dtype=torch.uint8, device="cuda"), _ints([L, L - 77])))
    alone = []
    for cache, table, q, out, ws, lens in cases:
        nova.paged_attention(cache, table, q, out, ws, L, kv_len_per_row=lens)
        alone.append(out.clone())
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(5):
        for st, (cache, table, q, out, ws, lens) in zip(streams, cases):
            with torch.cuda.stream(st):
                out.fill_(float("nan"))
                nova.paged_attention(cache, table, q, out, ws, L, kv_len_per_row=lens)
    torch.cuda.synchronize()
    for (_, _, _, out, _, _), want in zip(cases, alone):
        assert torch.equal(out, want)
